// AdamW over many tensors, states in 32 or 8 bits.
#pragma once

namespace pilc {

constexpr uint32_t kStateBlock = 256;  // values that share a scale

// What a launch works on goes to the kernel by value, so that nothing has to be copied to the GPU beforehand and
// nothing kept: up to 56 tensors, near 4 KB.
constexpr int kAdamwTensors = 56;

struct AdamwTensor {
    void *param;
    const void *grad;
    void *m, *v;
    uint8_t *m_scale, *v_scale;
    uint64_t count;
    float keep, rate;  // 1 - lr decay, lr / (1 - beta1^t)
};

struct AdamwArgs {
    AdamwTensor tensor[kAdamwTensors];
    uint32_t chunk_end[kAdamwTensors];  // chunks of the launch's tensors up to and with this one
    uint32_t block[kAdamwTensors];      // blocks of 256 of the launch's tensors before this one
    uint64_t first_block;               // and of those before the launch's
    float b1, b1_rest, b2, b2_rest, grad_scale, root_scale, eps;
    uint32_t dither, num;
};
static_assert(sizeof(AdamwArgs) <= 4096, "what a launch may carry");

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

// The weight's move needs no last bit: the root and the quotient are the hardware's, one unit off each.  Its root
// takes no denormal numbers, so small ones are brought up.
__device__ __forceinline__ float move_param(const AdamwArgs &a, const AdamwTensor &t, float p, Moments s)
{
    const bool small = s.v < 0x1p-96f;
    float root = __builtin_amdgcn_sqrtf(small ? s.v * 0x1p64f : s.v);
    root = small ? root * 0x1p-32f : root;
    return p * t.keep - t.rate * s.m * __builtin_amdgcn_rcpf(root * a.root_scale + a.eps);
}

// States in 8 bits.  Everything but the last rounding is exact: scales are powers of two, and where scaling a value
// would lose bits of it the constant that is added leaves nothing of those.
template <bool kSigned>
struct Coding {
    static constexpr int kOctaves = kSigned ? 15 : 31;
    static constexpr uint32_t kBase = (127 - kOctaves) << 3;

    // 2^(e-127) for decode, NaN for a block that is not finite
    __device__ static float scale_of(uint32_t e) { return __uint_as_float(e == 255 ? 0x7FC00000u : e == 0 ? 0x00400000u : e << 23); }
    // 2^(126-e) for encode
    __device__ static float inverse_of(uint32_t e) { return ldexpf(1.0f, 126 - (int)e); }

    // byte k of a word of codes
    __device__ static float decode(uint32_t word, int k, float scale)
    {
#pragma clang fp contract(off)
        const uint32_t size = word >> (8 * k) & (kSigned ? 127 : 255);
        // twice the number that is coded, less twice the constant
        const float x = (__uint_as_float((size + kBase + 8) << 20) - __uint_as_float((128 - kOctaves) << 23)) * scale;
        return kSigned ? __uint_as_float(__float_as_uint(x) ^ (word << (24 - 8 * k) & 0x80000000u)) : x;
    }
    __device__ static uint32_t encode(float x, float inverse, uint32_t noise)
    {
        const float y = __builtin_fmaf(fabsf(x), inverse, __uint_as_float((127 - kOctaves) << 23));
        const uint32_t code = (__float_as_uint(y) + (noise << 4) + (8u - (kBase << 20))) >> 20;
        if constexpr (kSigned)
            return code | (__float_as_uint(x) >> 24 & 128u);
        else
            return max(code, min(__float_as_uint(x), 1u));
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

// Which tensor a workgroup's chunk is of: every lane compares with one tensor's end, and how many ends lie before
// the chunk is counted over the wavefront.
__device__ __forceinline__ uint32_t tensor_of(const AdamwArgs &a, uint32_t chunk)
{
    const uint32_t lane = threadIdx.x & 63;
    const bool before = lane < a.num && a.chunk_end[lane < kAdamwTensors ? lane : 0] <= chunk;
    return (uint32_t)__builtin_popcountll(__ballot(before));
}

constexpr int kAdamwThreads = 256;
// Values a thread takes, and it takes no more: what would follow in a loop is on its way earlier in another workgroup (150
// million values f32 with states in 32 bits 787 us, in chunks of 4096 831; 300 million bf16 in 8 bits 564 and 632).
constexpr int kAdamwEach = 4, kAdamwBytesEach = 8;
constexpr uint32_t kAdamwChunk = kAdamwThreads * kAdamwEach, kAdamwBytesChunk = kAdamwThreads * kAdamwBytesEach;

// States in 32 bits.  28 bytes a value in f32 and 24 vector instructions: memory bounds it, at 5.3 TB/s (150 million
// values in 291 tensors).
template <class P, class G>
__global__ __launch_bounds__(kAdamwThreads) void k_adamw(AdamwArgs a)
{
    constexpr int kEach = kAdamwEach;
    const uint32_t k = __builtin_amdgcn_readfirstlane(tensor_of(a, blockIdx.x));
    const AdamwTensor &t = a.tensor[k];
    const uint64_t begin = (uint64_t)(blockIdx.x - (k ? a.chunk_end[k - 1] : 0)) * kAdamwChunk, i = begin + threadIdx.x * kEach;
    P *param = (P *)t.param + i;
    const G *grad = (const G *)t.grad + i;
    float *ms = (float *)t.m + i, *vs = (float *)t.v + i;
    const auto step = [&](int valid) {
        auto p = load_pack<kEach>(param, valid);
        const auto g = load_pack<kEach>(grad, valid);
        auto m = load_pack<kEach>(ms, valid), v = load_pack<kEach>(vs, valid);
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            const Moments s = move_moments(a, {m.v[j], v.v[j]}, widen(g.v[j]));
            p.v[j] = (P)move_param(a, t, widen(p.v[j]), s);
            m.v[j] = s.m, v.v[j] = s.v;
        }
        store_pack(param, valid, p);
        store_pack(ms, valid, m);
        store_pack(vs, valid, v);
    };
    if (t.count - begin >= kAdamwChunk)  // the same for all threads: their loads need not be told apart
        step(kEach);
    else if (i < t.count)
        step((int)min((uint64_t)kEach, t.count - i));
}

// `valid` codes, four a word; 0 behind them.
template <int kWords>
__device__ __forceinline__ void load_codes(const uint8_t *p, int valid, uint32_t (&out)[kWords])
{
    const auto t = load_pack<4 * kWords>(p, valid);
    __builtin_memcpy(out, &t, sizeof(out));
}
template <int kWords>
__device__ __forceinline__ void store_codes(uint8_t *p, int valid, const uint32_t (&in)[kWords])
{
    Pack<uint8_t, 4 * kWords> t;
    __builtin_memcpy(&t, in, sizeof(t));
    store_pack(p, valid, t);
}

// States in 8 bits: half a wavefront a block of 256, whose largest values it finds among its lanes.  10 bytes a value in
// bf16 and 67 vector instructions: the vector units are busy 90 % of the time, memory at 5.3 TB/s (300 million values: 564 us).
template <class P, class G>
__global__ __launch_bounds__(kAdamwThreads) void k_adamw_bytes(AdamwArgs a)
{
    constexpr int kEach = kAdamwBytesEach;
    const uint32_t k = __builtin_amdgcn_readfirstlane(tensor_of(a, blockIdx.x));
    const AdamwTensor &t = a.tensor[k];
    const uint64_t begin = (uint64_t)(blockIdx.x - (k ? a.chunk_end[k - 1] : 0)) * kAdamwBytesChunk, i = begin + threadIdx.x * kEach;
    P *param = (P *)t.param + i;
    uint8_t *ms = (uint8_t *)t.m + i, *vs = (uint8_t *)t.v + i, *m_scale = t.m_scale + i / kStateBlock, *v_scale = t.v_scale + i / kStateBlock;
    const G *grad = (const G *)t.grad + i;
    const auto step = [&](int valid) {
        auto p = load_pack<kEach>(param, valid);
        const auto g = load_pack<kEach>(grad, valid);
        uint32_t mc[kEach / 4], vc[kEach / 4];
        load_codes(ms, valid, mc);
        load_codes(vs, valid, vc);
        float m[kEach], v[kEach];
        const float m_unit = Coding<true>::scale_of(*m_scale), v_unit = Coding<false>::scale_of(*v_scale);
        uint32_t m_most = 0, v_most = 0;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            Moments s = {Coding<true>::decode(mc[j / 4], j & 3, m_unit), Coding<false>::decode(vc[j / 4], j & 3, v_unit)};
            s = move_moments(a, s, widen(g.v[j]));
            if (j >= valid) s = {0.0f, 0.0f};
            p.v[j] = (P)move_param(a, t, widen(p.v[j]), s);
            m[j] = s.m, v[j] = s.v;
            m_most = max(m_most, __float_as_uint(s.m) & 0x7FFFFFFFu);
            v_most = max(v_most, __float_as_uint(s.v));
        }
        store_pack(param, valid, p);
        m_most = lanes_reduce<32>(m_most, Max());
        v_most = lanes_reduce<32>(v_most, Max());
        const uint32_t em = max(1u, m_most >> 23), ev = max(1u, v_most >> 23 & 255);  // a NaN may have its sign set
        const float m_inverse = Coding<true>::inverse_of(em), v_inverse = Coding<false>::inverse_of(ev);
        const uint64_t number = (a.first_block + a.block[k]) * kStateBlock + i;
#pragma unroll
        for (int j = 0; j < kEach; ++j) {
            if (j % 4 == 0) mc[j / 4] = vc[j / 4] = 0;
            const uint32_t h = hash_of(number + j, a.dither);
            mc[j / 4] |= (Coding<true>::encode(m[j], m_inverse, h & 0xFFFF) & 255) << (8 * (j & 3));
            vc[j / 4] |= (Coding<false>::encode(v[j], v_inverse, h >> 16) & 255) << (8 * (j & 3));
        }
        store_codes(ms, valid, mc);
        store_codes(vs, valid, vc);
        if (i % kStateBlock == 0) *m_scale = (uint8_t)em, *v_scale = (uint8_t)ev;
    };
    if (t.count - begin >= kAdamwBytesChunk)  // the same for all threads: their loads need not be told apart
        step(kEach);
    else if (i / kStateBlock * kStateBlock < t.count)  // whole halves of wavefronts
        step(i < t.count ? (int)min((uint64_t)kEach, t.count - i) : 0);
}

// Eight values a thread, two times four, all codes asked for before the first value is written.  Memory bounds it, four bytes
// written for a byte read (300 million values with 4, 8, 12, 16 and 32 values a thread: signed 290, 238, 263, 266 and 262 us,
// unsigned 281, 245, 285, 270 and 262; 6.2 TB/s with 8).
constexpr int kValuesParts = 2;
constexpr uint32_t kValuesChunk = 256 * 4 * kValuesParts;
template <bool kSigned>
__global__ __launch_bounds__(256) void k_adamw_values(const uint8_t *__restrict__ code, const uint8_t *__restrict__ scale, uint64_t count,
                                                      float *__restrict__ values)
{
    for (uint64_t begin = (uint64_t)blockIdx.x * kValuesChunk; begin < count; begin += (uint64_t)gridDim.x * kValuesChunk) {
        if (count - begin >= kValuesChunk) {
            const uint64_t first = begin + threadIdx.x * 4;
            uint32_t c[kValuesParts][1], e[kValuesParts];
#pragma unroll
            for (int part = 0; part < kValuesParts; ++part) {
                load_codes(code + first + part * 1024, 4, c[part]);
                e[part] = scale[(first + part * 1024) / kStateBlock];  // of all four: 4 divides a block
            }
#pragma unroll
            for (int part = 0; part < kValuesParts; ++part) {
                const float unit = Coding<kSigned>::scale_of(e[part]);
                Pack<float, 4> x;
#pragma unroll
                for (int j = 0; j < 4; ++j) x.v[j] = Coding<kSigned>::decode(c[part][0], j, unit);
                *(Pack<float, 4> *)(values + first + part * 1024) = x;
            }
        } else {
            const uint64_t end = min(count, begin + kValuesChunk);
            for (uint64_t i = begin + threadIdx.x; i < end; i += 256)
                values[i] = Coding<kSigned>::decode(code[i], 0, Coding<kSigned>::scale_of(scale[i / kStateBlock]));
        }
    }
}

constexpr uint32_t kAdamwMostChunks = 1u << 20;  // a launch has fewer than 2^32 threads
static uint64_t ceil_div(uint64_t a, uint64_t b) { return (a + b - 1) / b; }

// c1 to be: 1 - beta1^step
static bool adamw_ok(const pilc_adamw_params *h, const pilc_adamw_tensor *t, uint32_t num, double &c1)
{
    constexpr double kMost = 3.4028234663852886e38;  // of 32 bits, in which the kernels have them
    const auto held = [](double v) { return v >= -kMost && v <= kMost; };
    const auto fine = [](double v) { return v >= 0.0 && v <= kMost; };
    if (!h || (num && !t) || !fine(h->lr) || !fine(h->eps) || !(h->beta1 >= 0.0 && h->beta1 < 1.0) || !(h->beta2 >= 0.0 && h->beta2 < 1.0) ||
        !held(h->grad_scale) || h->step < 1 || h->param_type > PILC_F16 || h->grad_type > PILC_F16 ||
        (h->state_bits != 32 && h->state_bits != 8))
        return false;
    c1 = 1.0 - std::pow(h->beta1, (double)h->step);
    const double most_lr = kMost * c1;
    for (uint32_t k = 0; k < num; ++k) {
        const pilc_adamw_tensor &x = t[k];
        const double lr = h->lr * x.lr_mult;
        if (!(std::fabs(lr) <= most_lr) || !held(1.0 - lr * x.decay)) return false;  // nor where a factor is not finite
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
    double c1;
    if (!adamw_ok(params_host, tensors_host, num_tensors, c1)) return PILC_E_ARG;
    const pilc_adamw_params &h = *params_host;
    AdamwArgs a = {};
    a.b1 = (float)h.beta1, a.b1_rest = (float)(1.0 - h.beta1), a.b2 = (float)h.beta2, a.b2_rest = (float)(1.0 - h.beta2);
    a.grad_scale = (float)h.grad_scale, a.dither = h.dither;
    a.eps = h.eps > 0.0 ? std::max((float)h.eps, 0x1p-126f) : 0.0f;  // the hardware's reciprocal of less is infinite
    const double c2 = 1.0 - std::pow(h.beta2, (double)h.step);
    a.root_scale = (float)(1.0 / std::sqrt(c2));
    uint64_t blocks = 0;
    const uint32_t chunk = h.state_bits == 32 ? kAdamwChunk : kAdamwBytesChunk;
    uint32_t chunks = 0;
    const auto launch = [&]() -> int {
        if (a.num == 0) return PILC_OK;
        const int rc = by_type(h.param_type, [&](auto *p) {
            by_value_type(h.grad_type, [&](auto *g) {
                using P = std::remove_pointer_t<decltype(p)>;
                using G = std::remove_pointer_t<decltype(g)>;
                if (h.state_bits == 32)
                    k_adamw<P, G><<<chunks, kAdamwThreads, 0, (hipStream_t)hip_stream>>>(a);
                else
                    k_adamw_bytes<P, G><<<chunks, kAdamwThreads, 0, (hipStream_t)hip_stream>>>(a);
            });
        });
        a.num = 0, chunks = 0, a.first_block = blocks;
        return rc;
    };
    for (uint32_t k = 0; k < num_tensors; ++k) {
        pilc_adamw_tensor x = tensors_host[k];
        const double lr = h.lr * x.lr_mult;
        while (x.count) {  // a tensor of more chunks than a launch has room for goes on in the next
            const uint64_t room = kAdamwMostChunks - chunks, wanted = ceil_div(x.count, chunk);
            const uint64_t here = std::min(room, wanted), count = here < wanted ? here * chunk : x.count;
            AdamwTensor &t = a.tensor[a.num];
            t = {x.param, x.grad, x.m, x.v, x.m_scale, x.v_scale, count, (float)(1.0 - lr * x.decay), (float)(lr / c1)};
            a.block[a.num] = (uint32_t)(blocks - a.first_block);
            chunks += (uint32_t)here, blocks += ceil_div(count, kStateBlock);
            a.chunk_end[a.num++] = chunks;
            x.count -= count;
            x.param = (char *)x.param + count * value_bytes(h.param_type);
            x.grad = (const char *)x.grad + count * value_bytes(h.grad_type);
            x.m = (char *)x.m + count * h.state_bits / 8, x.v = (char *)x.v + count * h.state_bits / 8;
            if (h.state_bits == 8) x.m_scale += count / kStateBlock, x.v_scale += count / kStateBlock;
            if (a.num == kAdamwTensors || chunks == kAdamwMostChunks)
                if (const int rc = launch(); rc != PILC_OK) return rc;
        }
    }
    return launch();
}

int pilc_adamw_values(const uint8_t *code_dev, const uint8_t *scale_dev, uint64_t count, int is_signed, float *values_dev, void *hip_stream)
{
    if (count == 0) return PILC_OK;
    if (!code_dev || !scale_dev || !values_dev || !aligned_to(values_dev, 4) || count > (1ull << 48)) return PILC_E_ARG;
    const uint32_t grid = (uint32_t)std::min<uint64_t>(ceil_div(count, kValuesChunk), 1u << 20);
    if (is_signed)
        k_adamw_values<true><<<grid, 256, 0, (hipStream_t)hip_stream>>>(code_dev, scale_dev, count, values_dev);
    else
        k_adamw_values<false><<<grid, 256, 0, (hipStream_t)hip_stream>>>(code_dev, scale_dev, count, values_dev);
    HIP_TRY(hipGetLastError());
    return PILC_OK;
}

}  // extern "C"
