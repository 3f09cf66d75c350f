// Log probabilities of symbols under rows of logits, with entropy and alternatives, and their gradient.
#pragma once

namespace pilc {

constexpr int kMaxTop = 32;
constexpr int kLogitsThreads = 256;

struct LogitsArgs {
    const void *x;
    const void *target;
    float *logp, *entropy, *lse;
    int32_t *top_sym;
    float *top_logp;
    const float *lse_in, *entropy_in, *up_logp, *up_entropy;
    void *grad;
    uint64_t stride, grad_stride;
    uint32_t rows, num_sym, top, target_type;
};

__device__ __forceinline__ int64_t target_of(const LogitsArgs &a, uint32_t row)
{
    return a.target_type == PILC_U8    ? (int64_t)((const uint8_t *)a.target)[row]
           : a.target_type == PILC_I32 ? (int64_t)((const int32_t *)a.target)[row]
                                       : ((const int64_t *)a.target)[row];
}

// Integers in the order of the values they are made of, and the lower symbol first among equals.
__device__ __forceinline__ uint64_t key_of(float x, uint32_t sym)
{
    const uint32_t b = __float_as_uint(x + 0.0f);  // no -0
    const uint32_t order = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)order << 32 | (0xFFFFFFFFu - sym);
}
__device__ __forceinline__ float value_of(uint64_t key)
{
    const uint32_t order = (uint32_t)(key >> 32);
    return __uint_as_float(order & 0x80000000u ? order & 0x7FFFFFFFu : ~order);
}

struct Law {
    float max, log_total, entropy;  // lse = max + log_total
};

// max, sum e^(x - max) and sum (x - max) e^(x - max) of a row as what is told of it.
__device__ __forceinline__ Law law_of(float max, float total, float inside)
{
    if (max == -kInf && total == 0.0f) return {-kInf, 0.0f, 0.0f};
    const float log_total = logf(total);
    if (!(log_total == log_total)) max = log_total;  // a NaN, or +inf less itself
    return {max, log_total, log_total - inside / total};
}

__device__ __forceinline__ float target_logp(const LogitsArgs &a, const Law &law, int64_t t, float at)
{
    if (t < 0) return 0.0f;
    if (t >= (int64_t)a.num_sym) return __builtin_nanf("");
    return law.max == -kInf ? -kInf : (at - law.max) - law.log_total;
}

template <class T>
__device__ void gradient_row(const T *x, T *grad, uint32_t num_sym, int64_t t, float lse, float entropy, float up, float up_entropy)
{
    const float a = t < 0 ? 0.0f : up, b = up_entropy;
    const bool zeros = (a == 0.0f && b == 0.0f) || lse == -kInf;
    const bool nothing = t >= (int64_t)num_sym;
    for (uint32_t j = threadIdx.x; j < num_sym; j += blockDim.x) {
        float d = 0.0f;
        if (!zeros) {
            const float lp = widen(x[j]) - lse;
            const float p = exp2_fast(lp * kLog2e);  // 0 below -88: what it is multiplied with need not go on falling
            d = -p * (a + b * (fmaxf(lp, -100.0f) + entropy));
            if ((int64_t)j == t) d += a;
            if (nothing) d = __builtin_nanf("");
        }
        grad[j] = (T)d;
    }
}

template <class T, bool kTrain>
__global__ __launch_bounds__(kLogitsThreads) void k_logprobs(LogitsArgs a)
{
    constexpr int kWaves = kLogitsThreads / 64;
    __shared__ float room[kWaves];
    __shared__ uint64_t key_room[kWaves];
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.stride;
        float max = -kInf;
        for (uint32_t j = threadIdx.x; j < a.num_sym; j += kLogitsThreads) max = fmaxf(max, widen(x[j]));
        max = block_reduce<kWaves>(max, Max(), room);
        const float from = max == -kInf ? 0.0f : max;
        float total = 0.0f, inside = 0.0f;
        for (uint32_t j = threadIdx.x; j < a.num_sym; j += kLogitsThreads) {
            const float z = widen(x[j]) - from, e = exp2_fast(z * kLog2e);
            total += e;
            inside += e * fmaxf(z, -3e38f);
        }
        total = block_reduce<kWaves>(total, Sum(), room);
        inside = block_reduce<kWaves>(inside, Sum(), room);
        const Law law = law_of(max, total, inside);
        const int64_t t = a.target ? target_of(a, row) : -1;
        if (threadIdx.x == 0) {
            const bool in = t >= 0 && t < (int64_t)a.num_sym;
            if (a.logp) a.logp[row] = target_logp(a, law, t, in ? widen(x[t]) : 0.0f);
            if (a.entropy) a.entropy[row] = law.entropy;
            if (a.lse) a.lse[row] = law.max + law.log_total;
        }
        if constexpr (kTrain) {
            __syncthreads();  // the gradient may lie where the logits are: the target's is read above
            gradient_row<T>(x, (T *)a.grad + row * a.grad_stride, a.num_sym, t, law.max + law.log_total, law.entropy, a.up_logp[row],
                            a.up_entropy ? a.up_entropy[row] : 0.0f);
        } else {
            uint64_t below = ~0ull;
            const bool none = !(law.max == law.max);  // NaN or +inf in the row
            for (uint32_t k = 0; k < a.top; ++k) {
                uint64_t best = 0;
                for (uint32_t j = threadIdx.x; j < a.num_sym; j += kLogitsThreads) {
                    const uint64_t key = key_of(widen(x[j]), j);
                    if (key < below && key > best) best = key;
                }
                below = block_reduce<kWaves>(best, Max(), key_room);
                if (threadIdx.x == 0) {
                    const float v = below ? value_of(below) : -kInf;
                    const size_t at = (size_t)row * a.top + k;
                    const bool there = !none && v > -kInf;
                    a.top_sym[at] = there ? (int32_t)(0xFFFFFFFFu - (uint32_t)below) : -1;
                    a.top_logp[at] = none ? __builtin_nanf("") : there ? (v - law.max) - law.log_total : -kInf;
                }
            }
        }
    }
}

template <class T>
__global__ __launch_bounds__(kLogitsThreads) void k_logprobs_grad(LogitsArgs a)
{
    for (uint32_t row = blockIdx.x; row < a.rows; row += gridDim.x)
        gradient_row<T>((const T *)a.x + row * a.stride, (T *)a.grad + row * a.grad_stride, a.num_sym, target_of(a, row), a.lse_in[row],
                        a.up_entropy ? a.entropy_in[row] : 0.0f, a.up_logp[row], a.up_entropy ? a.up_entropy[row] : 0.0f);
}

static size_t value_bytes(uint32_t type) { return type == PILC_F32 ? 4 : 2; }

static bool logits_shape_ok(const pilc_logits_shape *s)
{
    return s && s->num_sym >= 1 && s->num_sym <= 0x7FFFFFFFu && s->stride >= s->num_sym && s->stride <= (1ull << 48) && s->dtype <= PILC_F16 &&
           s->target_type <= PILC_I64 && s->top <= (uint32_t)kMaxTop;
}
static bool aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

static bool logits_in_ok(const pilc_logits_shape *s, const void *logits, const void *target)
{
    const size_t target_bytes = s->target_type == PILC_U8 ? 1 : s->target_type == PILC_I32 ? 4 : 8;
    return logits && aligned_to(logits, value_bytes(s->dtype)) && aligned_to(target, target_bytes);
}

static size_t logits_workspace(const pilc_logits_shape &s) { return 256; }

template <class Launch>
static void by_value_type(uint32_t type, Launch launch)
{
    switch (type) {
    case PILC_F32: launch((float *)nullptr); break;
    case PILC_BF16: launch((bf16_t *)nullptr); break;
    default: launch((f16_t *)nullptr); break;
    }
}
template <class Launch>
static int by_type(uint32_t type, Launch launch)
{
    by_value_type(type, launch);
    HIP_TRY(hipGetLastError());
    return PILC_OK;
}

static uint32_t row_blocks(uint32_t rows) { return std::min(rows, 1u << 20); }

}  // namespace pilc

extern "C" {
using namespace pilc;

int pilc_logprobs_workspace_size(const pilc_logits_shape *shape, size_t *workspace_bytes_host)
{
    if (!logits_shape_ok(shape) || !workspace_bytes_host) return PILC_E_ARG;
    *workspace_bytes_host = logits_workspace(*shape);
    return PILC_OK;
}

int pilc_logprobs(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev, float *logp_dev, float *entropy_dev,
                  float *lse_dev, int32_t *top_sym_dev, float *top_logp_dev, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!logits_shape_ok(shape)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    if (!logits_in_ok(shape, logits_dev, target_dev) || (logp_dev && !target_dev) || (shape->top && (!top_sym_dev || !top_logp_dev)) ||
        !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(lse_dev, 4) || !aligned_to(top_sym_dev, 4) ||
        !aligned_to(top_logp_dev, 4) || !workspace_dev || !aligned_to(workspace_dev, 256))
        return PILC_E_ARG;
    if (workspace_bytes < logits_workspace(*shape)) return PILC_E_WORKSPACE;
    LogitsArgs a = {};
    a.x = logits_dev, a.target = target_dev, a.logp = logp_dev, a.entropy = entropy_dev, a.lse = lse_dev, a.top_sym = top_sym_dev;
    a.top_logp = top_logp_dev, a.stride = shape->stride, a.rows = shape->rows, a.num_sym = shape->num_sym, a.top = shape->top;
    a.target_type = shape->target_type;
    return by_type(shape->dtype, [&](auto *t) {
        k_logprobs<std::remove_pointer_t<decltype(t)>, false><<<row_blocks(a.rows), kLogitsThreads, 0, (hipStream_t)hip_stream>>>(a);
    });
}

int pilc_logprobs_grad(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev, const float *lse_dev,
                       const float *entropy_dev, const float *up_logp_dev, const float *up_entropy_dev, void *grad_dev,
                       uint64_t grad_stride, void *hip_stream)
{
    if (!logits_shape_ok(shape) || grad_stride < shape->num_sym || grad_stride > (1ull << 48)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    if (!logits_in_ok(shape, logits_dev, target_dev) || !target_dev || !lse_dev || !up_logp_dev || (up_entropy_dev && !entropy_dev) ||
        !grad_dev || !aligned_to(grad_dev, value_bytes(shape->dtype)) || !aligned_to(lse_dev, 4) || !aligned_to(entropy_dev, 4) ||
        !aligned_to(up_logp_dev, 4) || !aligned_to(up_entropy_dev, 4) || (grad_dev == logits_dev && grad_stride != shape->stride))
        return PILC_E_ARG;
    LogitsArgs a = {};
    a.x = logits_dev, a.target = target_dev, a.lse_in = lse_dev, a.entropy_in = entropy_dev, a.up_logp = up_logp_dev;
    a.up_entropy = up_entropy_dev, a.grad = grad_dev, a.grad_stride = grad_stride, a.stride = shape->stride, a.rows = shape->rows;
    a.num_sym = shape->num_sym, a.target_type = shape->target_type;
    return by_type(shape->dtype, [&](auto *t) {
        k_logprobs_grad<std::remove_pointer_t<decltype(t)>><<<row_blocks(a.rows), kLogitsThreads, 0, (hipStream_t)hip_stream>>>(a);
    });
}

int pilc_logprobs_train(const pilc_logits_shape *shape, const void *logits_dev, const void *target_dev, const float *up_logp_dev,
                        const float *up_entropy_dev, float *logp_dev, float *entropy_dev, float *lse_dev, void *grad_dev,
                        uint64_t grad_stride, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    if (!logits_shape_ok(shape) || shape->top != 0 || grad_stride < shape->num_sym || grad_stride > (1ull << 48)) return PILC_E_ARG;
    if (shape->rows == 0) return PILC_OK;
    if (!logits_in_ok(shape, logits_dev, target_dev) || !target_dev || !up_logp_dev || !logp_dev || !grad_dev ||
        !aligned_to(grad_dev, value_bytes(shape->dtype)) || !aligned_to(up_logp_dev, 4) || !aligned_to(up_entropy_dev, 4) ||
        !aligned_to(logp_dev, 4) || !aligned_to(entropy_dev, 4) || !aligned_to(lse_dev, 4) || !workspace_dev ||
        !aligned_to(workspace_dev, 256) || (grad_dev == logits_dev && grad_stride != shape->stride))
        return PILC_E_ARG;
    if (workspace_bytes < logits_workspace(*shape)) return PILC_E_WORKSPACE;
    LogitsArgs a = {};
    a.x = logits_dev, a.target = target_dev, a.up_logp = up_logp_dev, a.up_entropy = up_entropy_dev, a.logp = logp_dev;
    a.entropy = entropy_dev, a.lse = lse_dev, a.grad = grad_dev, a.grad_stride = grad_stride, a.stride = shape->stride;
    a.rows = shape->rows, a.num_sym = shape->num_sym, a.target_type = shape->target_type;
    return by_type(shape->dtype, [&](auto *t) {
        k_logprobs<std::remove_pointer_t<decltype(t)>, true><<<row_blocks(a.rows), kLogitsThreads, 0, (hipStream_t)hip_stream>>>(a);
    });
}

}  // extern "C"
