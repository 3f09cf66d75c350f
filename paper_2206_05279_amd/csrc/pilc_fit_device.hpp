// Device helpers of the kernels that fit laws: values of three types handled in 32 bits, and reductions
// over a wavefront or a workgroup whose order is fixed.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pilc {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

// kCount of T as one access; the address is a multiple of its size, or of 16 bytes if that is less.
template <class T, int kCount>
struct alignas(sizeof(T) * kCount < 16 ? sizeof(T) * kCount : 16) Pack {
    T v[kCount];
};

template <class T>
__device__ __forceinline__ float widen(T v) { return (float)v; }

// `valid` of kCount values from p, 0 behind them.  whole: all are there and p is aligned for a Pack.
template <int kCount, class T>
__device__ __forceinline__ void load_pack(const T *p, bool whole, int valid, float (&out)[kCount])
{
    if (whole) {
        const Pack<T, kCount> t = *(const Pack<T, kCount> *)p;
#pragma unroll
        for (int k = 0; k < kCount; ++k) out[k] = widen(t.v[k]);
    } else {
#pragma unroll
        for (int k = 0; k < kCount; ++k) out[k] = k < valid ? widen(p[k]) : 0.0f;
    }
}
template <int kCount, class T>
__device__ __forceinline__ void store_pack(T *p, bool whole, int valid, const float (&in)[kCount])
{
    if (whole) {
        Pack<T, kCount> t;
#pragma unroll
        for (int k = 0; k < kCount; ++k) t.v[k] = (T)in[k];
        *(Pack<T, kCount> *)p = t;
    } else {
#pragma unroll
        for (int k = 0; k < kCount; ++k)
            if (k < valid) p[k] = (T)in[k];
    }
}

constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.44269504088896340736f;

// 2^x by the hardware's instruction, one unit in the last place off at most; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V v, Op op)
{
    for (int d = 32; d >= 1; d >>= 1) v = op(v, __shfl_xor(v, d, 64));
    return v;
}

// Over a workgroup of kWaves wavefronts; every thread gets the result.  `room` holds kWaves values; the
// workgroup meets before `room` is written and after, so that it can be used again at once.
template <int kWaves, class V, class Op>
__device__ __forceinline__ V block_reduce(V v, Op op, V *room)
{
    v = wave_reduce(v, op);
    if constexpr (kWaves > 1) {
        __syncthreads();
        if ((threadIdx.x & 63) == 0) room[threadIdx.x >> 6] = v;
        __syncthreads();
        v = room[0];
        for (int w = 1; w < kWaves; ++w) v = op(v, room[w]);
    }
    return v;
}

struct Max {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; }
};
struct Sum {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

}  // namespace pilc
