// AdamW over many tensors, states in 32 or 8 bits.
#pragma once

namespace pilc {

constexpr uint32_t kStateBlock = 256;  // values that share a scale

struct AdamwArgs {
    void *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    uint64_t count, first_block;  // blocks of 256 of the tensors before this one
    float keep, rate;             // 1 - lr decay, lr / (1 - beta1^t)
    float b1, b1_rest, b2, b2_rest, grad_scale, root_scale, eps;
    uint32_t dither;
};

struct Moments {
    float m, v;
};

// In this order and with every product rounded, so that the codes made of m and v are the same wherever
// they are computed.
__device__ __forceinline__ Moments move_moments(const AdamwArgs &a, Moments s, float g)
{
#pragma clang fp contract(off)
    g = g * a.grad_scale;
    const float m0 = s.m * a.b1, m1 = g * a.b1_rest, v0 = s.v * a.b2, v1 = g * g * a.b2_rest;
    return {m0 + m1, v0 + v1};
}

__device__ __forceinline__ float move_param(const AdamwArgs &a, float p, Moments s)
{
    return p * a.keep - a.rate * s.m / (sqrtf(s.v) * a.root_scale + a.eps);
}

template <bool kSigned>
struct Coding {
    static constexpr int kOctaves = kSigned ? 15 : 31;
    static constexpr uint32_t kBase = (127 - kOctaves) << 3;
    __device__ static float step() { return __uint_as_float((127 - kOctaves) << 23); }

    __device__ static uint32_t encode(float x, int exponent, uint32_t noise)
    {
#pragma clang fp contract(off)
        const float y = ldexpf(fabsf(x), 126 - exponent) + step();
        const uint32_t code = ((__float_as_uint(y) + (noise << 4) + 8) >> 20) - kBase;
        if constexpr (kSigned)
            return code | (x < 0.0f ? 128u : 0u);
        else
            return x > 0.0f && code == 0 ? 1u : code;
    }
    __device__ static float decode(uint32_t code, int exponent)
    {
#pragma clang fp contract(off)
        if (exponent == 255) return __builtin_nanf("");
        const uint32_t size = kSigned ? code & 127 : code;
        const float x = ldexpf(__uint_as_float((size + kBase) << 20) - step(), exponent - 126);
        return kSigned && code > 127 ? -x : x;
    }
};

__device__ __forceinline__ uint32_t hash_of(uint64_t number, uint32_t dither)
{
    uint32_t h = (uint32_t)number * 0x9E3779B9u + (uint32_t)(number >> 32) * 0x6A09E667u + dither * 0xBB67AE85u;
    h ^= h >> 16;
    h *= 0x3C6EF373u;
    h ^= h >> 15;
    h *= 0xA54FF53Bu;
    return h ^ (h >> 16);
}

template <class P, class G>
__global__ __launch_bounds__(256) void k_adamw(AdamwArgs a)
{
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < a.count; i += gridDim.x * 256ull) {
        float *m = (float *)a.m + i, *v = (float *)a.v + i;
        const Moments s = move_moments(a, {*m, *v}, widen(((const G *)a.grad)[i]));
        P *p = (P *)a.param + i;
        *p = (P)move_param(a, widen(*p), s);
        *m = s.m;
        *v = s.v;
    }
}

// A block of 256 values a workgroup at a time.
template <class P, class G>
__global__ __launch_bounds__(256) void k_adamw_bytes(AdamwArgs a)
{
    __shared__ int room[4];
    const uint64_t blocks = (a.count + kStateBlock - 1) / kStateBlock;
    for (uint64_t b = blockIdx.x; b < blocks; b += gridDim.x) {
        const uint64_t i = b * kStateBlock + threadIdx.x;
        const bool in = i < a.count;
        uint8_t *m = (uint8_t *)a.m + i, *v = (uint8_t *)a.v + i;
        Moments s = {0.0f, 0.0f};
        if (in) {
            s = {Coding<true>::decode(*m, a.m_scale[b]), Coding<false>::decode(*v, a.v_scale[b])};
            s = move_moments(a, s, widen(((const G *)a.grad)[i]));
            P *p = (P *)a.param + i;
            *p = (P)move_param(a, widen(*p), s);
        }
        const int em = max(1, block_reduce<4>((int)(__float_as_uint(s.m) >> 23 & 255), Max(), room));
        const int ev = max(1, block_reduce<4>((int)(__float_as_uint(s.v) >> 23 & 255), Max(), room));
        if (in) {
            const uint32_t h = hash_of((a.first_block + b) * kStateBlock + threadIdx.x, a.dither);
            *m = (uint8_t)Coding<true>::encode(s.m, em, h & 0xFFFF);
            *v = (uint8_t)Coding<false>::encode(s.v, ev, h >> 16);
        }
        if (threadIdx.x == 0) {
            a.m_scale[b] = (uint8_t)em;
            a.v_scale[b] = (uint8_t)ev;
        }
    }
}

template <bool kSigned>
__global__ __launch_bounds__(256) void k_adamw_values(const uint8_t *code, const uint8_t *scale, uint64_t count, float *values)
{
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < count; i += gridDim.x * 256ull)
        values[i] = Coding<kSigned>::decode(code[i], scale[i / kStateBlock]);
}

static bool adamw_ok(const pilc_adamw_params *h, const pilc_adamw_tensor *t, uint32_t num)
{
    const auto fine = [](double v) { return v >= 0.0 && v < (double)kInf; };
    if (!h || (num && !t) || !fine(h->lr) || !fine(h->eps) || !(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0) ||
        !std::isfinite(h->grad_scale) || h->step < 1 || h->param_type > PILC_F16 || h->grad_type > PILC_F16 ||
        (h->state_bits != 32 && h->state_bits != 8))
        return false;
    for (uint32_t k = 0; k < num; ++k) {
        const pilc_adamw_tensor &x = t[k];
        if (!std::isfinite(x.lr_mult) || !std::isfinite(x.decay)) return false;
        if (x.count == 0) continue;
        const size_t state = h->state_bits == 32 ? 4 : 1;
        if (!x.param || !x.grad || !x.m || !x.v || !aligned_to(x.param, value_bytes(h->param_type)) ||
            !aligned_to(x.grad, value_bytes(h->grad_type)) || !aligned_to(x.m, state) || !aligned_to(x.v, state) || x.count > (1ull << 48) ||
            (h->state_bits == 8 && (!x.m_scale || !x.v_scale)))
            return false;
    }
    return true;
}

}  // namespace pilc

extern "C" {
using namespace pilc;

int pilc_adamw_step(const pilc_adamw_params *params_host, const pilc_adamw_tensor *tensors_host, uint32_t num_tensors, void *hip_stream)
{
    if (!adamw_ok(params_host, tensors_host, num_tensors)) return PILC_E_ARG;
    const pilc_adamw_params &h = *params_host;
    AdamwArgs a = {};
    a.b1 = (float)h.beta1, a.b1_rest = (float)(1.0 - h.beta1), a.b2 = (float)h.beta2, a.b2_rest = (float)(1.0 - h.beta2);
    a.grad_scale = (float)h.grad_scale, a.eps = (float)h.eps, a.dither = h.dither;
    const double c1 = 1.0 - std::pow(h.beta1, (double)h.step), c2 = 1.0 - std::pow(h.beta2, (double)h.step);
    a.root_scale = (float)(1.0 / std::sqrt(c2));
    for (uint32_t k = 0; k < num_tensors; ++k) {
        const pilc_adamw_tensor &x = tensors_host[k];
        if (x.count == 0) continue;
        a.param = x.param, a.grad = x.grad, a.m = x.m, a.v = x.v, a.m_scale = x.m_scale, a.v_scale = x.v_scale, a.count = x.count;
        const double lr = h.lr * x.lr_mult;
        a.keep = (float)(1.0 - lr * x.decay), a.rate = (float)(lr / c1);
        const uint64_t blocks = (x.count + 255) / 256;
        const uint32_t grid = (uint32_t)std::min<uint64_t>(blocks, 1u << 20);
        const int rc = by_type(h.param_type, [&](auto *p) {
            by_type(h.grad_type, [&](auto *g) {
                using P = std::remove_pointer_t<decltype(p)>;
                using G = std::remove_pointer_t<decltype(g)>;
                if (h.state_bits == 32)
                    k_adamw<P, G><<<grid, 256, 0, (hipStream_t)hip_stream>>>(a);
                else
                    k_adamw_bytes<P, G><<<grid, 256, 0, (hipStream_t)hip_stream>>>(a);
            });
        });
        if (rc != PILC_OK) return rc;
        a.first_block += blocks;
    }
    return PILC_OK;
}

int pilc_adamw_values(const uint8_t *code_dev, const uint8_t *scale_dev, uint64_t count, int is_signed, float *values_dev, void *hip_stream)
{
    if (count == 0) return PILC_OK;
    if (!code_dev || !scale_dev || !values_dev || !aligned_to(values_dev, 4) || count > (1ull << 48)) return PILC_E_ARG;
    const uint32_t grid = (uint32_t)std::min<uint64_t>((count + 255) / 256, 1u << 20);
    if (is_signed)
        k_adamw_values<true><<<grid, 256, 0, (hipStream_t)hip_stream>>>(code_dev, scale_dev, count, values_dev);
    else
        k_adamw_values<false><<<grid, 256, 0, (hipStream_t)hip_stream>>>(code_dev, scale_dev, count, values_dev);
    HIP_TRY(hipGetLastError());
    return PILC_OK;
}

}  // extern "C"
