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

constexpr int kNormThreads = 256, kNormLongThreads = 1024;
// Wavefronts a SIMD that the kernels' registers are kept down to, and that are launched: all at once, each going from row to row
// (forward with 4, 5 and 6 within 3 % of each other; backward, 32768 x 4096 bf16, with 2, 3 and 4: 154, 161 and 293 us, and
// 8192 x 4096 f32 with 2 and 3: 82 and 89, as more of them put down more parts and 4 leave too few registers).
constexpr int kNormForwardWaves = 5, kNormBackwardWaves = 2;

// Rows held in registers: kLanes lanes of a wavefront, or a whole workgroup of kLanes threads, hold kEach values of a
// row each, as packs of 16 bytes, and go from row to row with the weights in registers.  A pack that would reach over
// the row's end begins earlier: some values are then held twice, worked out twice to the same bits and stored twice,
// and left out of the row's sums the second time.
template <class T, class W, int kLanes, int kEach>
struct NormRow {
    static constexpr int kVec = 16 / sizeof(T), kPer = kEach / kVec;
    static constexpr bool kAhead = kLanes < 1024;  // the next row is asked for early; the largest workgroups lack the registers
    static constexpr bool kKeep = kEach <= 16;     // the weights stay in registers; the longest rows' come from the caches
    static constexpr int kThreads = kLanes > 256 ? kLanes : 256;
    static constexpr int kRows = kThreads / kLanes;  // that a workgroup has in hand
    static constexpr int kWaves = kLanes / 64;       // that share a row
    // of `most` wavefronts a SIMD, the whole workgroups' that fit
    static constexpr int waves(int most) { return kThreads == 1024 ? 4 : most * 256 / kThreads * kThreads / 256; }

    uint32_t width, lane, row_in_block;
    bool ragged;

    __device__ explicit NormRow(uint32_t w)
        : width(w), lane(threadIdx.x % kLanes), row_in_block(kRows > 1 ? threadIdx.x / kLanes : 0), ragged(w != (uint32_t)(kLanes * kEach))
    {
    }
    __device__ uint32_t place(int q) const { return (q * kLanes + lane) * kVec; }
    __device__ uint32_t column(int q) const { return min(place(q), width - kVec); }
    __device__ int twice(int q) const { return (int)min(place(q) - column(q), (uint32_t)kVec); }  // values at a pack's begin that another has

    __device__ void load(const T *p, Raw<T> (&out)[kPer]) const
    {
#pragma unroll
        for (int q = 0; q < kPer; ++q) out[q] = Raw<T>::load(p + column(q));
    }
    // weights as they lie in memory, `none` where there are none
    __device__ Pack<W, kVec> weights(const W *p, float none, int q) const
    {
        if (p) return *(const Pack<W, kVec> *)(p + column(q));
        Pack<W, kVec> t;
#pragma unroll
        for (int k = 0; k < kVec; ++k) t.v[k] = (W)none;
        return t;
    }
    __device__ void load_weights(const W *p, float none, Pack<W, kVec> (&out)[kPer]) const
    {
#pragma unroll
        for (int q = 0; q < kPer; ++q) out[q] = weights(p, none, q);
    }

    // The sum over a lane's values of f(pack, value)
    template <class V, class F>
    __device__ V own_sum(V sum, F f) const
    {
        if (!ragged) {
#pragma unroll
            for (int q = 0; q < kPer; ++q)
#pragma unroll
                for (int k = 0; k < kVec; ++k) f(sum, q, k);
        } else {
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                const int from = twice(q);
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    V with = sum;
                    f(with, q, k);
                    sum = k >= from ? with : sum;
                }
            }
        }
        return sum;
    }
    // Sums over the row of two numbers a lane.  `room` is used in turn: two halves, so that the workgroup meets
    // once a sum.
    __device__ float2 sum(float2 v, float2 *room, int half) const
    {
        constexpr int kWithin = kLanes < 64 ? kLanes : 64;
        v.x = lanes_reduce<kWithin>(v.x, Sum());
        v.y = lanes_reduce<kWithin>(v.y, Sum());
        if constexpr (kWaves > 1) {
            room += half * kWaves;
            if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
            __syncthreads();
            v = room[0];
#pragma unroll
            for (int w = 1; w < kWaves; ++w) v.x += room[w].x, v.y += room[w].y;
        }
        return v;
    }
    __device__ float sum(float v, float2 *room, int half) const { return sum(make_float2(v, 0.0f), room, half).x; }
};

// y = (x - mean) rstd w + b, the mean first and the deviations from it second, from the same registers.  Memory bounds it:
// 16384 x 8192 bf16 97 us (5.5 TB/s).
template <class T, class W, int kLanes, int kEach>
__global__ __launch_bounds__((NormRow<T, W, kLanes, kEach>::kThreads), (NormRow<T, W, kLanes, kEach>::waves(kNormForwardWaves))) void
k_norm_forward_rows(NormArgs a)
{
    using Row = NormRow<T, W, kLanes, kEach>;
    constexpr int kVec = Row::kVec, kPer = Row::kPer;
    __shared__ float2 room[2 * (Row::kWaves > 1 ? Row::kWaves : 1)];
    const Row r(a.width);
    const float per_value = 1.0f / (float)a.width;
    Pack<W, kVec> weight[kPer], bias[kPer];
    if (Row::kKeep) {
        r.load_weights((const W *)a.weight, 1.0f, weight);
        r.load_weights((const W *)a.bias, 0.0f, bias);
    }
    Raw<T> x[kPer], next[kPer];
    uint32_t row = blockIdx.x * Row::kRows + r.row_in_block;
    const uint32_t step = gridDim.x * Row::kRows, last = a.rows - 1;
    if (Row::kAhead) r.load((const T *)a.x + min(row, last) * a.x_stride, x);
    for (bool more = row < a.rows; more; more = next_row(row, step, last)) {
        if (Row::kAhead)
            r.load((const T *)a.x + (last - row > step ? row + step : last) * a.x_stride, next);
        else
            r.load((const T *)a.x + row * a.x_stride, x);
        const float own = r.own_sum(0.0f, [&](float &s, int q, int k) { s += x[q][k]; });
        const float mean = r.sum(own, room, 0) * per_value;
        const float square = r.own_sum(0.0f, [&](float &s, int q, int k) {
            const float d = x[q][k] - mean;
            s += d * d;
        });
        const float rstd = 1.0f / sqrtf(r.sum(square, room, 1) * per_value + a.eps);
        if (r.lane == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        T *y = (T *)a.y + row * a.y_stride;
#pragma unroll
        for (int q = 0; q < kPer; ++q) {
            if (!Row::kKeep) {
                weight[q] = r.weights((const W *)a.weight, 1.0f, q);
                bias[q] = r.weights((const W *)a.bias, 0.0f, q);
            }
            float out[kVec];
#pragma unroll
            for (int k = 0; k < kVec; ++k) out[k] = (x[q][k] - mean) * rstd * widen(weight[q].v[k]) + widen(bias[q].v[k]);
            Raw<T>::of(out).store(y + r.column(q));
            if (Row::kAhead) x[q] = next[q];
        }
    }
}

// dx row by row as above, and what the rows a workgroup meets add to the weights' gradients, in registers; at the end
// the workgroup's rows are added up and put down as one part.  The longest rows leave no room for that: k_norm_parts.
// Memory bounds it: 32768 x 4096 bf16 147 us and 5 for k_norm_join (5.6 TB/s with the parts).
template <class T, class W, int kLanes, int kEach>
__global__ __launch_bounds__((NormRow<T, W, kLanes, kEach>::kThreads), (NormRow<T, W, kLanes, kEach>::waves(kNormBackwardWaves))) void
k_norm_backward_rows(NormArgs a)
{
    using Row = NormRow<T, W, kLanes, kEach>;
    constexpr int kVec = Row::kVec, kPer = Row::kPer;
    __shared__ float2 room[2 * (Row::kWaves > 1 ? Row::kWaves : 1)];
    __shared__ float added[Row::kRows > 1 ? Row::kThreads * kEach : 1];
    const Row r(a.width);
    const float per_value = 1.0f / (float)a.width;
    Pack<W, kVec> weight[kPer];
    float dw[kPer][kVec] = {}, db[kPer][kVec] = {};
    if (Row::kKeep) r.load_weights((const W *)a.weight, 1.0f, weight);
    Raw<T> x[kPer], dy[kPer], next_x[kPer], next_dy[kPer];
    uint32_t row = blockIdx.x * Row::kRows + r.row_in_block;
    const uint32_t step = gridDim.x * Row::kRows, last = a.rows - 1;
    int half = 0;
    // a row's mean and rstd are asked for before its values: loads come back in order, and what was asked for late would
    // make the values of the next row be waited for with it
    float mean = 0.0f, rstd = 0.0f, next_mean = 0.0f, next_rstd = 0.0f;
    const auto fetch = [&](uint32_t of, float &m, float &s, Raw<T>(&to_x)[kPer], Raw<T>(&to_dy)[kPer]) {
        m = a.mean_in[of], s = a.rstd_in[of];
        r.load((const T *)a.x + of * a.x_stride, to_x);
        r.load((const T *)a.dy + of * a.y_stride, to_dy);
    };
    if (Row::kAhead) fetch(min(row, last), mean, rstd, x, dy);
    for (bool more = row < a.rows; more; more = next_row(row, step, last)) {
        if (Row::kAhead)
            fetch(last - row > step ? row + step : last, next_mean, next_rstd, next_x, next_dy);
        else
            fetch(row, mean, rstd, x, dy);
        if (!Row::kKeep) r.load_weights((const W *)a.weight, 1.0f, weight);
        float2 sums = r.own_sum(make_float2(0.0f, 0.0f), [&](float2 &s, int q, int k) {
            const float g = dy[q][k] * widen(weight[q].v[k]);
            s.x += g;
            s.y += g * ((x[q][k] - mean) * rstd);
        });
        if (Row::kKeep)
#pragma unroll
            for (int q = 0; q < kPer; ++q)
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    dw[q][k] += dy[q][k] * ((x[q][k] - mean) * rstd);
                    db[q][k] += dy[q][k];
                }
        if (a.dx) {
            sums = r.sum(sums, room, half);
            half ^= 1;
            const float c1 = sums.x * per_value, c2 = sums.y * per_value;
            T *dx = (T *)a.dx + row * a.dx_stride;
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                float out[kVec];
#pragma unroll
                for (int k = 0; k < kVec; ++k) out[k] = rstd * (dy[q][k] * widen(weight[q].v[k]) - c1 - (x[q][k] - mean) * rstd * c2);
                Raw<T>::of(out).store(dx + r.column(q));
            }
        }
        if (Row::kAhead) {
            mean = next_mean, rstd = next_rstd;
#pragma unroll
            for (int q = 0; q < kPer; ++q) x[q] = next_x[q], dy[q] = next_dy[q];
        }
    }
    if (!Row::kKeep || !a.parts) return;
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float *part = a.parts + ((size_t)which * gridDim.x + blockIdx.x) * a.width;
        float(&own)[kPer][kVec] = which ? db : dw;
        if constexpr (Row::kRows > 1) {
            // value v of lane l of row g at (g * kEach + v) * kLanes + l
            __syncthreads();
#pragma unroll
            for (int v = 0; v < kEach; ++v) added[(r.row_in_block * kEach + v) * kLanes + r.lane] = own[v / kVec][v % kVec];
            __syncthreads();
            for (uint32_t i = threadIdx.x; i < (uint32_t)(kEach * kLanes); i += Row::kThreads) {
                const uint32_t v = i / kLanes, l = i % kLanes, j = min((v / kVec * kLanes + l) * kVec, a.width - kVec) + v % kVec;
                float sum = 0.0f;
                for (int g = 0; g < Row::kRows; ++g) sum += added[g * kEach * kLanes + i];
                part[j] = sum;
            }
        } else {
#pragma unroll
            for (int q = 0; q < kPer; ++q) {
                Pack<float, kVec> out;
#pragma unroll
                for (int k = 0; k < kVec; ++k) out.v[k] = own[q][k];
                *(Pack<float, kVec> *)(part + r.column(q)) = out;
            }
        }
    }
}

// Rows shorter than eight values: a thread a row.
template <class T, class W>
__global__ __launch_bounds__(kNormThreads) void k_norm_forward_narrow(NormArgs a)
{
    const W *weight = (const W *)a.weight, *bias = (const W *)a.bias;
    for (uint64_t row = blockIdx.x * (uint64_t)kNormThreads + threadIdx.x; row < a.rows; row += gridDim.x * (uint64_t)kNormThreads) {
        const T *x = (const T *)a.x + row * a.x_stride;
        T *y = (T *)a.y + row * a.y_stride;
        float mean = 0.0f, square = 0.0f;
        for (uint32_t j = 0; j < a.width; ++j) mean += widen(x[j]);
        mean /= (float)a.width;
        for (uint32_t j = 0; j < a.width; ++j) {
            const float d = widen(x[j]) - mean;
            square += d * d;
        }
        const float rstd = 1.0f / sqrtf(square / (float)a.width + a.eps);
        if (a.mean) a.mean[row] = mean;
        if (a.rstd) a.rstd[row] = rstd;
        for (uint32_t j = 0; j < a.width; ++j)
            y[j] = (T)((widen(x[j]) - mean) * rstd * (weight ? widen(weight[j]) : 1.0f) + (bias ? widen(bias[j]) : 0.0f));
    }
}
template <class T, class W>
__global__ __launch_bounds__(kNormThreads) void k_norm_backward_narrow(NormArgs a)
{
    constexpr int kMost = 7, kWaves = kNormThreads / 64;
    __shared__ float room[kWaves];
    const W *weight = (const W *)a.weight;
    float dw[kMost] = {}, db[kMost] = {};
    for (uint64_t row = blockIdx.x * (uint64_t)kNormThreads + threadIdx.x; row < a.rows; row += gridDim.x * (uint64_t)kNormThreads) {
        const T *x = (const T *)a.x + row * a.x_stride, *dy = (const T *)a.dy + row * a.y_stride;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float q[kMost], xh[kMost], c1 = 0.0f, c2 = 0.0f;
#pragma unroll
        for (int j = 0; j < kMost; ++j) {
            q[j] = xh[j] = 0.0f;
            if (j < (int)a.width) {
                const float d = widen(dy[j]);
                q[j] = d * (weight ? widen(weight[j]) : 1.0f);
                xh[j] = (widen(x[j]) - mean) * rstd;
                dw[j] += d * xh[j];
                db[j] += d;
            }
            c1 += q[j];
            c2 += q[j] * xh[j];
        }
        c1 /= (float)a.width, c2 /= (float)a.width;
        if (a.dx)
#pragma unroll
            for (int j = 0; j < kMost; ++j)
                if (j < (int)a.width) ((T *)a.dx + row * a.dx_stride)[j] = (T)(rstd * (q[j] - c1 - xh[j] * c2));
    }
    if (!a.parts) return;
#pragma unroll
    for (int j = 0; j < kMost; ++j) {
        const float sw = block_reduce<kWaves>(dw[j], Sum(), room), sb = block_reduce<kWaves>(db[j], Sum(), room);
        if (threadIdx.x == 0 && j < (int)a.width) {
            a.parts[(size_t)blockIdx.x * a.width + j] = sw;
            a.parts[(size_t)(gridDim.x + blockIdx.x) * a.width + j] = sb;
        }
    }
}

// Rows too long for registers, over 32768 values: a workgroup goes through them two or three times and finds them in the caches
// after the first (8192 x 20000 bf16, while such rows came here, 539 us; 182 in registers).  Four packs a thread at a time, so
// that four loads are on their way: forward 4096 x 40000 bf16 247 us, with one at a time 531.
constexpr int kNormLongEach = 4;
constexpr uint32_t kNormLongStep = kNormLongThreads * kNormLongEach;
template <int kVec, class F>
__device__ __forceinline__ void for_packs(uint32_t width, F f)  // f(columns, how many of a pack's first values others have)
{
    for (uint32_t first = threadIdx.x * kVec; first < width; first += kNormLongStep * kVec) {
        uint32_t column[kNormLongEach];
        int twice[kNormLongEach];
#pragma unroll
        for (int q = 0; q < kNormLongEach; ++q) {
            const uint32_t place = first + q * kNormLongThreads * kVec;
            column[q] = min(place, width - kVec);  // the last one begins earlier: its first values have been gone through
            twice[q] = (int)min(place - column[q], (uint32_t)kVec);
        }
        f(column, twice);
    }
}
// What is written may be what is read: no value is gone through twice.
template <int kVec, class F>
__device__ __forceinline__ void for_whole_packs(uint32_t width, F f)  // f(count, column, valid)
{
    const uint32_t step = kNormLongStep * kVec;
    uint32_t begin = 0;
    for (; width - begin >= step; begin += step) f(std::integral_constant<int, kNormLongEach>(), begin + threadIdx.x * kVec, kVec);
    for (uint32_t place = begin + threadIdx.x * kVec; place < width; place += kNormLongThreads * kVec)
        f(std::integral_constant<int, 1>(), place, (int)min(width - place, (uint32_t)kVec));
}
template <int kVec, class T>
__device__ __forceinline__ Pack<T, kVec> pack_at(const T *p) { return *(const Pack<T, kVec> *)p; }

// No __restrict__, and what is stored twice is the same: y may be x.
template <class T, class W>
__global__ __launch_bounds__(kNormLongThreads) void k_norm_forward_long(NormArgs a)
{
    constexpr int kVec = 16 / sizeof(T);
    constexpr int kWaves = kNormLongThreads / 64;
    __shared__ float room[kWaves];
    const W *weight = (const W *)a.weight, *bias = (const W *)a.bias;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.x_stride;
        T *y = (T *)a.y + row * a.y_stride;
        float sum = 0.0f, square = 0.0f;
        for_packs<kVec>(a.width, [&](const auto &column, const auto &twice) {
            Pack<T, kVec> t[kNormLongEach];
#pragma unroll
            for (int q = 0; q < kNormLongEach; ++q) t[q] = pack_at<kVec>(x + column[q]);
#pragma unroll
            for (int q = 0; q < kNormLongEach; ++q)
#pragma unroll
                for (int k = 0; k < kVec; ++k) sum += k >= twice[q] ? widen(t[q].v[k]) : 0.0f;
        });
        const float mean = block_reduce<kWaves>(sum, Sum(), room) / (float)a.width;
        for_packs<kVec>(a.width, [&](const auto &column, const auto &twice) {
            Pack<T, kVec> t[kNormLongEach];
#pragma unroll
            for (int q = 0; q < kNormLongEach; ++q) t[q] = pack_at<kVec>(x + column[q]);
#pragma unroll
            for (int q = 0; q < kNormLongEach; ++q)
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const float d = k >= twice[q] ? widen(t[q].v[k]) - mean : 0.0f;
                    square += d * d;
                }
        });
        const float rstd = 1.0f / sqrtf(block_reduce<kWaves>(square, Sum(), room) / (float)a.width + a.eps);
        if (threadIdx.x == 0) {
            if (a.mean) a.mean[row] = mean;
            if (a.rstd) a.rstd[row] = rstd;
        }
        for_whole_packs<kVec>(a.width, [&](auto count, uint32_t place, int valid) {
            constexpr int kCount = decltype(count)::value;
            Pack<T, kVec> t[kCount];
            Pack<W, kVec> w[kCount], c[kCount];
#pragma unroll
            for (int q = 0; q < kCount; ++q) {
                const uint32_t at = place + q * kNormLongThreads * kVec;
                t[q] = load_pack<kVec>(x + at, valid);
                if (weight) w[q] = load_pack<kVec>(weight + at, valid);
                if (bias) c[q] = load_pack<kVec>(bias + at, valid);
            }
#pragma unroll
            for (int q = 0; q < kCount; ++q) {
#pragma unroll
                for (int k = 0; k < kVec; ++k)
                    t[q].v[k] = (T)((widen(t[q].v[k]) - mean) * rstd * (weight ? widen(w[q].v[k]) : 1.0f) + (bias ? widen(c[q].v[k]) : 0.0f));
                store_pack(y + place + q * kNormLongThreads * kVec, valid, t[q]);
            }
        });
        __syncthreads();
    }
}

template <class T, class W>
__global__ __launch_bounds__(kNormLongThreads) void k_norm_dx_long(NormArgs a)
{
    constexpr int kVec = 16 / sizeof(T);
    constexpr int kWaves = kNormLongThreads / 64;
    __shared__ float room[kWaves];
    const W *weight = (const W *)a.weight;
    for (uint64_t row = blockIdx.x; row < a.rows; row += gridDim.x) {
        const T *x = (const T *)a.x + row * a.x_stride, *dy = (const T *)a.dy + row * a.y_stride;
        T *dx = (T *)a.dx + row * a.dx_stride;
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
        float q_sum = 0.0f, qx_sum = 0.0f;
        for_packs<kVec>(a.width, [&](const auto &column, const auto &twice) {
            Pack<T, kVec> tx[kNormLongEach], td[kNormLongEach];
            Pack<W, kVec> w[kNormLongEach];
#pragma unroll
            for (int q = 0; q < kNormLongEach; ++q) {
                tx[q] = pack_at<kVec>(x + column[q]), td[q] = pack_at<kVec>(dy + column[q]);
                if (weight) w[q] = pack_at<kVec>(weight + column[q]);
            }
#pragma unroll
            for (int q = 0; q < kNormLongEach; ++q)
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const float g = k >= twice[q] ? widen(td[q].v[k]) * (weight ? widen(w[q].v[k]) : 1.0f) : 0.0f;
                    q_sum += g;
                    qx_sum += k >= twice[q] ? g * ((widen(tx[q].v[k]) - mean) * rstd) : 0.0f;
                }
        });
        const float c1 = block_reduce<kWaves>(q_sum, Sum(), room) / (float)a.width;
        const float c2 = block_reduce<kWaves>(qx_sum, Sum(), room) / (float)a.width;
        for_whole_packs<kVec>(a.width, [&](auto count, uint32_t place, int valid) {
            constexpr int kCount = decltype(count)::value;
            Pack<T, kVec> tx[kCount], td[kCount];
            Pack<W, kVec> w[kCount];
#pragma unroll
            for (int q = 0; q < kCount; ++q) {
                const uint32_t at = place + q * kNormLongThreads * kVec;
                tx[q] = load_pack<kVec>(x + at, valid), td[q] = load_pack<kVec>(dy + at, valid);
                if (weight) w[q] = load_pack<kVec>(weight + at, valid);
            }
#pragma unroll
            for (int q = 0; q < kCount; ++q) {
#pragma unroll
                for (int k = 0; k < kVec; ++k) {
                    const float g = widen(td[q].v[k]) * (weight ? widen(w[q].v[k]) : 1.0f);
                    td[q].v[k] = (T)(rstd * (g - c1 - (widen(tx[q].v[k]) - mean) * rstd * c2));
                }
                store_pack(dx + place + q * kNormLongThreads * kVec, valid, td[q]);
            }
        });
        __syncthreads();
    }
}

// A pack of columns a thread, the rows in num_parts runs; before dx, which may take dy's place.
template <class T>
__global__ __launch_bounds__(kNormThreads) void k_norm_parts(NormArgs a)
{
    constexpr int kVec = 16 / sizeof(T);
    const uint32_t place = (blockIdx.x * kNormThreads + threadIdx.x) * kVec;
    if (place >= a.width) return;
    const uint32_t column = min(place, a.width - kVec);
    float dw[kVec] = {}, db[kVec] = {};
#pragma unroll 4
    for (uint64_t row = blockIdx.y; row < a.rows; row += a.num_parts) {
        const auto tx = pack_at<kVec>((const T *)a.x + row * a.x_stride + column), td = pack_at<kVec>((const T *)a.dy + row * a.y_stride + column);
        const float mean = a.mean_in[row], rstd = a.rstd_in[row];
#pragma unroll
        for (int k = 0; k < kVec; ++k) {
            const float d = widen(td.v[k]);
            db[k] += d;
            dw[k] += d * ((widen(tx.v[k]) - mean) * rstd);
        }
    }
#pragma unroll
    for (int k = 0; k < kVec; ++k) {
        a.parts[(size_t)blockIdx.y * a.width + column + k] = dw[k];
        a.parts[(size_t)(a.num_parts + blockIdx.y) * a.width + column + k] = db[k];
    }
}

// The parts added up: 64 columns a workgroup at a time, each by sixteen threads that take every sixteenth part (512 parts of 4096
// columns, 17 MB: 5.4 us).
template <class W>
__global__ __launch_bounds__(1024) void k_norm_join(NormArgs a)
{
    __shared__ float room[16][64];
    const uint32_t column = threadIdx.x & 63, run = threadIdx.x >> 6;
    W *out = (W *)(blockIdx.y ? a.dbias : a.dweight);
    if (!out) return;
    for (uint32_t first = blockIdx.x * 64; first < a.width; first += gridDim.x * 64) {
        const uint32_t j = first + column;
        const float *part = a.parts + (size_t)blockIdx.y * a.num_parts * a.width + j;
        float sum = 0.0f;
        if (j < a.width) {
#pragma unroll 8
            for (uint32_t p = run; p < a.num_parts; p += 16) sum += part[(size_t)p * a.width];
        }
        room[run][column] = sum;
        __syncthreads();
        if (run == 0 && j < a.width) {
            for (int i = 1; i < 16; ++i) sum += room[i][column];
            out[j] = (W)sum;
        }
        __syncthreads();
    }
}

// Calls `go` with the lanes and values a lane that a row of `width` values goes into, or returns false where it is too long: the
// fewest that it fits, as lanes without values cost as much as others.  268 MB of bf16 in rows that just fit, forward and backward in
// us, with these lanes and the next ones: 64 values 105 149 and 259 387, 256 106 147 and 209 282, 1024 107 154 and 177 218,
// 2048 113 146 and 145 179, 4096 108 154 and 148 167, 8192 100 171 and 179 201, 16384 119 163 and 167 338, 32768 121 274 and, by
// the kernels for rows that no registers hold, 172 342.
template <class Go>
static bool norm_row(uint32_t width, Go go)
{
    using std::integral_constant;
    if (width < 8) return false;  // less than a pack
    const auto with = [&](auto lanes, auto each) {
        if (width > (uint32_t)(lanes.value * each.value)) return false;
        go(lanes, each);
        return true;
    };
    return with(integral_constant<int, 8>(), integral_constant<int, 8>()) || with(integral_constant<int, 32>(), integral_constant<int, 8>()) ||
           with(integral_constant<int, 64>(), integral_constant<int, 16>()) || with(integral_constant<int, 256>(), integral_constant<int, 8>()) ||
           with(integral_constant<int, 256>(), integral_constant<int, 16>()) || with(integral_constant<int, 512>(), integral_constant<int, 16>()) ||
           with(integral_constant<int, 1024>(), integral_constant<int, 16>()) || with(integral_constant<int, 1024>(), integral_constant<int, 32>());
}

// Parts of rows too long for kKeep (bf16, us of the backward pass with 32, 64, 128 and 256 of them: 8192 x 20000 466 376 363 381,
// 4096 x 40000 444 429 444 473, 500 x 20000 38 39 45 57, 64 x 200000 100 136 135 135).
constexpr uint32_t kNormLongParts = 64, kNormLongestKept = 16384;
static uint32_t narrow_blocks(uint32_t rows) { return std::min(div_up(rows, kNormThreads), 1u << 20); }
template <class Row>
static uint32_t norm_blocks(uint32_t rows, int most_waves)
{
    return std::min(div_up(rows, Row::kRows), compute_units() * (uint32_t)(Row::waves(most_waves) * 256 / Row::kThreads));
}
// Workgroups of the backward pass.  With weights' gradients each puts down a part, as much as two rows in 32 bits, so that few
// rows are shared out by four, once half the compute units have one (4096 columns bf16, us with a row and with four a workgroup:
// 16 rows 6.2 and 8.2, 256 rows 11.2 and 10.5, by two 9.4, 500 rows 17.9 and 12.7, 1000 rows 18.7 and 15.2).
template <class Row>
static uint32_t norm_backward_blocks(uint32_t rows, bool with_parts)
{
    const uint32_t blocks = div_up(rows, Row::kRows), most = norm_blocks<Row>(rows, kNormBackwardWaves);
    return with_parts ? std::min(most, std::max(compute_units() / 2, blocks / 4)) : most;
}
// The most parts of any of the ways below: rows too long for kKeep go by kNormLongParts, the others by workgroups that are all
// there at once, or with less than a pack a row by one a compute unit.
static uint32_t norm_most_parts(uint32_t rows, uint32_t width)
{
    const uint32_t most = width > kNormLongestKept ? kNormLongParts : std::max(kNormLongParts, (uint32_t)kNormBackwardWaves * compute_units());
    return std::max(1u, std::min(rows, most));
}
static size_t norm_workspace(const pilc_norm_shape &s)
{
    return std::max<size_t>(256, 2 * sizeof(float) * (size_t)norm_most_parts(s.rows, s.width) * s.width);
}

static bool norm_shape_ok(const pilc_norm_shape *s, bool backward)
{
    const uint64_t most = 1ull << 48;
    return s && s->width >= 1 && s->width <= 0x7FFFFFFFu && s->x_stride >= s->width && s->x_stride <= most && s->y_stride >= s->width &&
           s->y_stride <= most && (!backward || (s->dx_stride >= s->width && s->dx_stride <= most)) && s->dtype <= PILC_F16 &&
           (s->weight_type == s->dtype || s->weight_type == PILC_F32) && s->eps >= 0.0f && s->eps < kInf;
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
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        const bool done = norm_row(a.width, [&](auto lanes, auto each) {
            using Row = NormRow<T, W, decltype(lanes)::value, decltype(each)::value>;
            const uint32_t blocks = norm_blocks<Row>(a.rows, kNormForwardWaves);
            k_norm_forward_rows<T, W, decltype(lanes)::value, decltype(each)::value><<<blocks, Row::kThreads, 0, (hipStream_t)hip_stream>>>(a);
        });
        if (done) return;
        if (a.width < 8)
            k_norm_forward_narrow<T, W><<<narrow_blocks(a.rows), kNormThreads, 0, (hipStream_t)hip_stream>>>(a);
        else
            k_norm_forward_long<T, W><<<std::min(a.rows, 1u << 20), kNormLongThreads, 0, (hipStream_t)hip_stream>>>(a);
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
    a.dbias = dbias_dev, a.x_stride = shape->x_stride, a.y_stride = shape->y_stride, a.dx_stride = shape->dx_stride;
    a.rows = shape->rows, a.width = shape->width;
    if (dweight_dev || dbias_dev) a.parts = (float *)workspace_dev;
    const hipStream_t stream = (hipStream_t)hip_stream;
    return by_types(shape->dtype, shape->weight_type, [&](auto *t, auto *w) {
        using T = std::remove_pointer_t<decltype(t)>;
        using W = std::remove_pointer_t<decltype(w)>;
        const auto parts = [&](uint32_t most) {
            a.num_parts = std::min(a.rows, most);
            const uint32_t each = kNormThreads * 16 / sizeof(T);
            if (a.parts && a.rows)
                k_norm_parts<T><<<dim3((a.width + each - 1) / each, a.num_parts), kNormThreads, 0, stream>>>(a);  // before dx, which may take dy's place
        };
        if (a.width < 8) {
            a.num_parts = std::min(narrow_blocks(a.rows), compute_units());
            if (a.rows) k_norm_backward_narrow<T, W><<<a.num_parts, kNormThreads, 0, stream>>>(a);
        } else if (!norm_row(a.width, [&](auto lanes, auto each) {
                       using Row = NormRow<T, W, decltype(lanes)::value, decltype(each)::value>;
                       if (!Row::kKeep) parts(kNormLongParts);
                       const uint32_t blocks = norm_backward_blocks<Row>(a.rows, Row::kKeep && a.parts);
                       static_assert(Row::waves(kNormBackwardWaves) * 256 / Row::kThreads <= kNormBackwardWaves &&
                                     Row::kKeep == (Row::kThreads == 256 || decltype(lanes)::value * decltype(each)::value <= kNormLongestKept));
                       if (Row::kKeep) a.num_parts = blocks;
                       if (a.rows && (Row::kKeep || a.dx))
                           k_norm_backward_rows<T, W, decltype(lanes)::value, decltype(each)::value>
                               <<<blocks, Row::kThreads, 0, stream>>>(a);
                   })) {
            parts(kNormLongParts);
            if (a.dx && a.rows) k_norm_dx_long<T, W><<<std::min(a.rows, 1u << 20), kNormLongThreads, 0, stream>>>(a);
        }
        if (a.parts) k_norm_join<W><<<dim3(std::min((a.width + 63) / 64, 1u << 20), 2), 1024, 0, stream>>>(a);  // 2^30 threads at most
    });
}

}  // extern "C"
