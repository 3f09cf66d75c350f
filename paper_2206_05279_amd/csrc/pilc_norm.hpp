// Layer norm and its backward pass.
#pragma once

namespace pilc {

struct NormArgs {
    const void *x, *dy, *weight, *bias;
    void *y, *dx, *dweight, *dbias;
    float *mean, *rstd;
    const float *mean_in, *rstd_in;
    float *parts;  // [2][parts][width]
    uint64_t x_stride, y_stride, dx_stride;
    uint32_t rows, width, num_parts;
    float eps;
};

constexpr int kNormThreads = 256;

template <class T, class W>
__global__ __launch_bounds__(kNormThreads) void k_norm_forward(NormArgs a)
{
    constexpr int kWaves = kNormThreads / 64;
    __shared__ float room[kWaves];
    const W *weight = (const W *)a.weight, *bias = (const W *)a.bias;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.x_stride;
        T *y = (T *)a.y + row * a.y_stride;
        float sum = 0.0f;
        for (uint32_t j = threadIdx.x; j < a.width; j += kNormThreads) sum += widen(x[j]);
        const float mean = block_reduce<kWaves>(sum, Sum(), room) / (float)a.width;
        float square = 0.0f;
        for (uint32_t j = threadIdx.x; j < a.width; j += kNormThreads) {
            const float d = widen(x[j]) - mean;
            square += d * d;
        }
        const float rstd = 1.0f / sqrtf(block_reduce<kWaves>(square, Sum(), room) / (float)a.width + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for (uint32_t j = threadIdx.x; j < a.width; j += kNormThreads)
            y[j] = (T)((widen(x[j]) - mean) * rstd * (weight ? widen(weight[j]) : 1.0f) + (bias ? widen(bias[j]) : 0.0f));
        __syncthreads();
    }
}

template <class T, class W>
__global__ __launch_bounds__(kNormThreads) void k_norm_dx(NormArgs a)
{
    constexpr int kWaves = kNormThreads / 64;
    __shared__ float room[kWaves];
    const W *weight = (const W *)a.weight;
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.x_stride, *dy = (const T *)a.dy + row * a.y_stride;
        T *dx = (T *)a.dx + row * a.dx_stride;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float q_sum = 0.0f, qx_sum = 0.0f;
        for (uint32_t j = threadIdx.x; j < a.width; j += kNormThreads) {
            const float q = widen(dy[j]) * (weight ? widen(weight[j]) : 1.0f);
            q_sum += q;
            qx_sum += q * ((widen(x[j]) - mean) * rstd);
        }
        const float c1 = block_reduce<kWaves>(q_sum, Sum(), room) / (float)a.width;
        const float c2 = block_reduce<kWaves>(qx_sum, Sum(), room) / (float)a.width;
        for (uint32_t j = threadIdx.x; j < a.width; j += kNormThreads) {
            const float q = widen(dy[j]) * (weight ? widen(weight[j]) : 1.0f);
            dx[j] = (T)(rstd * (q - c1 - (widen(x[j]) - mean) * rstd * c2));
        }
    }
}

// Thread per column, the rows in num_parts runs; before dx, which may take dy's place.
template <class T>
__global__ __launch_bounds__(kNormThreads) void k_norm_parts(NormArgs a)
{
    const uint32_t j = blockIdx.x * kNormThreads + threadIdx.x;
    if (j >= a.width) return;
    float dw = 0.0f, db = 0.0f;
    for (uint32_t row = blockIdx.y; row < a.rows; row += a.num_parts) {
        const float d = widen(((const T *)a.dy)[row * a.y_stride + j]);
        db += d;
        dw += d * ((widen(((const T *)a.x)[row * a.x_stride + j]) - a.mean_in[row]) * a.rstd_in[row]);
    }
    a.parts[(size_t)blockIdx.y * a.width + j] = dw;
    a.parts[(size_t)(a.num_parts + blockIdx.y) * a.width + j] = db;
}

template <class W>
__global__ __launch_bounds__(kNormThreads) void k_norm_join(NormArgs a)
{
    const uint32_t j = blockIdx.x * kNormThreads + threadIdx.x;
    if (j >= a.width) return;
    float dw = 0.0f, db = 0.0f;
    for (uint32_t p = 0; p < a.num_parts; ++p) {
        dw += a.parts[(size_t)p * a.width + j];
        db += a.parts[(size_t)(a.num_parts + p) * a.width + j];
    }
    if (a.dweight) ((W *)a.dweight)[j] = (W)dw;
    if (a.dbias) ((W *)a.dbias)[j] = (W)db;
}

static uint32_t norm_parts(const pilc_norm_shape &) { return 64; }
static size_t norm_workspace(const pilc_norm_shape &s) { return std::max<size_t>(256, 2 * sizeof(float) * (size_t)norm_parts(s) * s.width); }

static bool norm_shape_ok(const pilc_norm_shape *s, bool backward)
{
    const uint64_t most = 1ull << 48;
    return s && s->width >= 1 && s->width <= 0x7FFFFFFFu && s->x_stride >= s->width && s->x_stride <= most && s->y_stride >= s->width &&
           s->y_stride <= most && (!backward || (s->dx_stride >= s->width && s->dx_stride <= most)) && s->dtype <= PILC_F16 &&
           (s->weight_type == s->dtype || s->weight_type == PILC_F32) && s->eps >= 0.0f && s->eps < kInf;
}

template <class Launch>
static int by_types(uint32_t type, uint32_t weight_type, Launch launch)
{
    return by_type(type, [&](auto *t) {
        if (weight_type == type)
            launch(t, t);
        else
            launch(t, (float *)nullptr);
    });
}

}  // namespace pilc

extern "C" {
using namespace pilc;

int pilc_norm_forward(const pilc_norm_shape *shape, const void *x_dev, const void *weight_dev, const void *bias_dev, void *y_dev,
                      float *mean_dev, float *rstd_dev, void *hip_stream)
{
    if (!norm_shape_ok(shape, false)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    const size_t bytes = value_bytes(shape->dtype), weight_bytes = value_bytes(shape->weight_type);
    if (!x_dev || !y_dev || !aligned_to(x_dev, bytes) || !aligned_to(y_dev, bytes) || !aligned_to(weight_dev, weight_bytes) ||
        !aligned_to(bias_dev, weight_bytes) || !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4) ||
        (x_dev == y_dev && shape->x_stride != shape->y_stride))
        return PILC_E_ARG;
    NormArgs a = {};
    a.x = x_dev, a.weight = weight_dev, a.bias = bias_dev, a.y = y_dev, a.mean = mean_dev, a.rstd = rstd_dev;
    a.x_stride = shape->x_stride, a.y_stride = shape->y_stride, a.rows = shape->rows, a.width = shape->width, a.eps = shape->eps;
    return by_types(shape->dtype, shape->weight_type, [&](auto *t, auto *w) {
        k_norm_forward<std::remove_pointer_t<decltype(t)>, std::remove_pointer_t<decltype(w)>>
            <<<row_blocks(a.rows), kNormThreads, 0, (hipStream_t)hip_stream>>>(a);
    });
}

int pilc_norm_workspace_size(const pilc_norm_shape *shape, size_t *workspace_bytes_host)
{
    if (!norm_shape_ok(shape, true) || !workspace_bytes_host) return PILC_E_ARG;
    *workspace_bytes_host = norm_workspace(*shape);
    return PILC_OK;
}

int pilc_norm_backward(const pilc_norm_shape *shape, const void *dy_dev, const void *x_dev, const void *weight_dev, const float *mean_dev,
                       const float *rstd_dev, void *dx_dev, void *dweight_dev, void *dbias_dev, void *workspace_dev,
                       size_t workspace_bytes, void *hip_stream)
{
    if (!norm_shape_ok(shape, true)) return PILC_E_ARG;
    if (!dx_dev && !dweight_dev && !dbias_dev) return PILC_E_ARG;
    const size_t bytes = value_bytes(shape->dtype), weight_bytes = value_bytes(shape->weight_type);
    if ((shape->rows && (!dy_dev || !x_dev || !mean_dev || !rstd_dev)) || !aligned_to(dy_dev, bytes) || !aligned_to(x_dev, bytes) ||
        !aligned_to(dx_dev, bytes) || !aligned_to(weight_dev, weight_bytes) || !aligned_to(dweight_dev, weight_bytes) ||
        !aligned_to(dbias_dev, weight_bytes) || !aligned_to(mean_dev, 4) || !aligned_to(rstd_dev, 4) || !workspace_dev ||
        !aligned_to(workspace_dev, 256) || (dx_dev && dx_dev == dy_dev && shape->dx_stride != shape->y_stride))
        return PILC_E_ARG;
    if (workspace_bytes < norm_workspace(*shape)) return PILC_E_WORKSPACE;
    NormArgs a = {};
    a.dy = dy_dev, a.x = x_dev, a.weight = weight_dev, a.mean_in = mean_dev, a.rstd_in = rstd_dev, a.dx = dx_dev, a.dweight = dweight_dev;
    a.dbias = dbias_dev, a.parts = (float *)workspace_dev, a.x_stride = shape->x_stride, a.y_stride = shape->y_stride;
    a.dx_stride = shape->dx_stride, a.rows = shape->rows, a.width = shape->width, a.num_parts = norm_parts(*shape);
    const hipStream_t stream = (hipStream_t)hip_stream;
    return by_types(shape->dtype, shape->weight_type, [&](auto *t, auto *w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        const uint32_t columns = (a.width + kNormThreads - 1) / kNormThreads;
        if (a.dweight || a.dbias) {
            k_norm_parts<T><<<dim3(columns, a.num_parts), kNormThreads, 0, stream>>>(a);
            k_norm_join<W><<<columns, kNormThreads, 0, stream>>>(a);
        }
        if (a.dx && a.rows) k_norm_dx<T, W><<<row_blocks(a.rows), kNormThreads, 0, stream>>>(a);
    });
}

}  // extern "C"
