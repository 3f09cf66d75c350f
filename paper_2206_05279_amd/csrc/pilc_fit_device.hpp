// Device helpers of the kernels that fit laws: values of three types handled in 32 bits, and reductions
// over a wavefront or a workgroup whose order is fixed.
#pragma once
#include <hip/hip_runtime.h>

#include <cstdint>

namespace pilc {

typedef __bf16 bf16_t;
typedef _Float16 f16_t;

template <class T>
__device__ __forceinline__ float widen(T v) { return (float)v; }

// kCount of T as one access wherever they lie: this GPU's global memory takes accesses of 16 bytes at any address.
template <class T, int kCount>
struct __attribute__((packed, aligned(sizeof(T)))) Pack {
    T v[kCount];
};

// `valid` of kCount values from p, 0 behind them.
template <int kCount, class T>
__device__ __forceinline__ Pack<T, kCount> load_pack(const T *p, int valid)
{
    if (valid >= kCount) return *(const Pack<T, kCount> *)p;
    Pack<T, kCount> t;
#pragma unroll
    for (int k = 0; k < kCount; ++k) t.v[k] = k < valid ? p[k] : (T)0;
    return t;
}
template <int kCount, class T>
__device__ __forceinline__ void store_pack(T *p, int valid, const Pack<T, kCount> &t)
{
    if (valid >= kCount) {
        *(Pack<T, kCount> *)p = t;
    } else {
#pragma unroll
        for (int k = 0; k < kCount; ++k)
            if (k < valid) p[k] = t.v[k];
    }
}

constexpr float kInf = __builtin_inff();
constexpr float kLog2e = 1.44269504088896340736f;

// 2^x by the hardware's instruction, one unit in the last place off at most; results below 2^-126 are 0.
__device__ __forceinline__ float exp2_fast(float x) { return __builtin_amdgcn_exp2f(x); }

// Sixteen bytes of T as they lie in memory.  They stay four registers until they are looked into: taken apart where they
// are loaded, they would have to be waited for there.
typedef uint32_t u32x4_t __attribute__((ext_vector_type(4)));
template <class T>
struct Raw {
    static constexpr int kVec = 16 / sizeof(T);
    u32x4_t bits;

    __device__ static Raw load(const T *p)
    {
        struct __attribute__((packed, aligned(sizeof(T)))) At { u32x4_t v; };
        return {((const At *)p)->v};
    }
    __device__ void store(T *p) const
    {
        struct __attribute__((packed, aligned(sizeof(T)))) At { u32x4_t v; };
        ((At *)p)->v = bits;
    }
    // Nothing worked out from the values before is kept for after: widened, they would take twice the registers.
    __device__ void forget() { asm volatile("" : "+v"(bits)); }
    // -inf in place of the first `count` values
    __device__ void rule_out(int count)
    {
        if constexpr (sizeof(T) == 4) {
#pragma unroll
            for (int k = 0; k < 4; ++k) bits[k] = k < count ? 0xFF800000u : bits[k];
        } else {
            constexpr uint32_t kNone = __is_same(T, __bf16) ? 0xFF80u : 0xFC00u;
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const uint32_t low = (bits[i] & 0xFFFF0000u) | kNone;
                bits[i] = 2 * i + 1 < count ? kNone << 16 | kNone : 2 * i < count ? low : bits[i];
            }
        }
    }
    __device__ float operator[](int k) const { return widen(__builtin_bit_cast(Pack<T, kVec>, bits).v[k]); }
    // value k, for a k that is not known beforehand
    __device__ float at(uint32_t k) const
    {
        const uint32_t i = sizeof(T) == 4 ? k : k / 2;
        const uint32_t word = i == 0 ? bits[0] : i == 1 ? bits[1] : i == 2 ? bits[2] : bits[3];
        if constexpr (sizeof(T) == 4)
            return __uint_as_float(word);
        else
            return widen(__builtin_bit_cast(T, (uint16_t)(k & 1 ? word >> 16 : word)));
    }
    __device__ static Raw of(const float (&v)[kVec])
    {
        Pack<T, kVec> t;
#pragma unroll
        for (int k = 0; k < kVec; ++k) t.v[k] = (T)v[k];
        return {__builtin_bit_cast(u32x4_t, t)};
    }
};

// What a lane's partner has, the partner being 1, 2, 4, 8 lanes away within groups of 2, 4, 8, 16: the first two by
// their numbers, the others as mirror images, which is the same once the smaller groups are of one value.
template <int kDpp>
__device__ __forceinline__ float from_partner(float v)
{
    return __uint_as_float(__builtin_amdgcn_mov_dpp(__float_as_uint(v), kDpp, 15, 15, true));
}
template <int kDpp>
__device__ __forceinline__ uint32_t from_partner(uint32_t v)
{
    return __builtin_amdgcn_mov_dpp(v, kDpp, 15, 15, true);
}
__device__ __forceinline__ uint32_t bits_of(float v) { return __float_as_uint(v); }
__device__ __forceinline__ uint32_t bits_of(uint32_t v) { return v; }
__device__ __forceinline__ void from_bits(uint32_t b, float &v) { v = __uint_as_float(b); }
__device__ __forceinline__ void from_bits(uint32_t b, uint32_t &v) { v = b; }

// Over groups of kLanes neighbouring lanes, without LDS; every lane gets the result, the same bits in all.
template <int kLanes, class V, class Op>
__device__ __forceinline__ V lanes_reduce(V v, Op op)
{
    static_assert(kLanes >= 1 && kLanes <= 64 && (kLanes & (kLanes - 1)) == 0, "");
    if constexpr (kLanes >= 2) v = op(v, from_partner<0xB1>(v));   // quads 1 0 3 2
    if constexpr (kLanes >= 4) v = op(v, from_partner<0x4E>(v));   // quads 2 3 0 1
    if constexpr (kLanes >= 8) v = op(v, from_partner<0x141>(v));  // eights the other way round
    if constexpr (kLanes >= 16) v = op(v, from_partner<0x140>(v)); // sixteens the other way round
    if constexpr (kLanes >= 32) {
        const auto r = __builtin_amdgcn_permlane16_swap(bits_of(v), bits_of(v), false, false);
        V p, q;
        from_bits(r[0], p), from_bits(r[1], q);
        v = op(p, q);
    }
    if constexpr (kLanes >= 64) {
        const auto r = __builtin_amdgcn_permlane32_swap(bits_of(v), bits_of(v), false, false);
        V p, q;
        from_bits(r[0], p), from_bits(r[1], q);
        v = op(p, q);
    }
    return v;
}

// As lanes_reduce, in 64 bits.
template <int kDpp>
__device__ __forceinline__ double from_partner64(double v)
{
    const uint64_t b = __builtin_bit_cast(uint64_t, v);
    return __builtin_bit_cast(double, (uint64_t)from_partner<kDpp>((uint32_t)(b >> 32)) << 32 | from_partner<kDpp>((uint32_t)b));
}
template <int kLanes>
__device__ __forceinline__ double lanes_sum(double v)
{
    if constexpr (kLanes >= 2) v += from_partner64<0xB1>(v);
    if constexpr (kLanes >= 4) v += from_partner64<0x4E>(v);
    if constexpr (kLanes >= 8) v += from_partner64<0x141>(v);
    if constexpr (kLanes >= 16) v += from_partner64<0x140>(v);
    if constexpr (kLanes >= 32) v += __shfl_xor(v, 16, 64);
    if constexpr (kLanes >= 64) v += __shfl_xor(v, 32, 64);
    return v;
}

template <class V, class Op>
__device__ __forceinline__ V wave_reduce(V v, Op op)
{
    if constexpr (sizeof(V) == 4) {
        return lanes_reduce<64>(v, op);
    } else {
        for (int d = 32; d >= 1; d >>= 1) v = op(v, __shfl_xor(v, d, 64));
        return v;
    }
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

// One instruction, where the compiler would see to it first that no operand is a signalling NaN.
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float m;
    asm("v_max3_f32 %0, %1, %2, %3" : "=v"(m) : "v"(a), "v"(b), "v"(c));
    return m;
}
// What is not a number is passed over.
struct MaxFloat {
    __device__ __forceinline__ float operator()(float a, float b) const { return fmaxf(a, b); }
};
struct Max {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a > b ? a : b; }
};
struct Sum {
    template <class V>
    __device__ __forceinline__ V operator()(V a, V b) const { return a + b; }
};

}  // namespace pilc
