// Product of two matrices in 8 bits under scales for blocks of 128, c = a b^T.
#pragma once

namespace pilc {

struct ProductArgs {
    Block8 a, b;  // [rows, depth], [cols, depth]
    void *c;
    float *part;  // with splits > 1: [splits][rows][cols]
    uint64_t c_stride;
    uint32_t rows, cols, depth, c_type;
    uint32_t blocks, splits, blocks_each;  // blocks of 128 along the depth; a split takes blocks_each of them
};

typedef int i32x8_t __attribute__((ext_vector_type(8)));
typedef float f32x4_t __attribute__((ext_vector_type(4)));
typedef __bf16 bf16x8_t __attribute__((ext_vector_type(8)));
typedef __bf16 bf16x2_t __attribute__((ext_vector_type(2)));

// The matrix unit's products of 8-bit values are exact, but before they are added to a sum of 32 bits eight of them are added
// up with 13 bits below the power of two of the largest (measured: 2^16 + 2^j loses all of 2^j from j = 2 on if they are of
// the same eight, and from j = -8 on if not).  What that costs against 64 bits, relative: 1.5e-5 for normally distributed values,
// 6e-5 where a few are a hundred times the others.  A c of 16 bits is rounded by 2^-9 or 2^-12, which is more; one
// of 32 bits is not, and its values are widened to bfloat16, which holds them under their scales, and multiplied at half the rate:
// 1e-8 to 9e-8.
enum Exactness { kGroups, kSingles };

// Sixteen codes from k on of a row, zeros behind its end.
__device__ __forceinline__ u32x4_t product_chunk(const uint8_t *row, uint32_t k, uint32_t depth)
{
    const int valid = (int)min(depth - min(k, depth), 16u);
    return __builtin_bit_cast(u32x4_t, load_pack<16>(row + (valid > 0 ? k : 0), valid));
}

__device__ __forceinline__ float scale_value(uint32_t byte) { return __uint_as_float(byte == 255 ? 0x7FC00000u : byte << 23); }

template <int kType>
__device__ __forceinline__ void widen8(const u32x4_t &codes, int half, float scale, bf16x8_t &to)
{
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const uint32_t w = codes[2 * half + i];
        bf16x2_t lo, hi;
        if constexpr (kType == PILC_E4M3) {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp8(w, scale, true);
        } else {
            lo = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, false);
            hi = __builtin_amdgcn_cvt_scalef32_pk_bf16_bf8(w, scale, true);
        }
        to[4 * i] = lo[0], to[4 * i + 1] = lo[1], to[4 * i + 2] = hi[0], to[4 * i + 3] = hi[1];
    }
}

__device__ __forceinline__ void product_store(const ProductArgs &p, uint32_t split, uint32_t row, uint32_t col, const f32x4_t &v)
{
    if (row >= p.rows) return;
    const int valid = (int)min(p.cols - min(col, p.cols), 4u);
    if (valid == 0) return;
    if (p.splits > 1) {
        store_pack<4>(p.part + ((uint64_t)split * p.rows + row) * p.cols + col, valid, Pack<float, 4>{v[0], v[1], v[2], v[3]});
    } else if (p.c_type == PILC_F32) {
        store_pack<4>((float *)p.c + (uint64_t)row * p.c_stride + col, valid, Pack<float, 4>{v[0], v[1], v[2], v[3]});
    } else if (p.c_type == PILC_BF16) {
        store_pack<4>((bf16_t *)p.c + (uint64_t)row * p.c_stride + col, valid, Pack<bf16_t, 4>{(bf16_t)v[0], (bf16_t)v[1], (bf16_t)v[2], (bf16_t)v[3]});
    } else {
        store_pack<4>((f16_t *)p.c + (uint64_t)row * p.c_stride + col, valid, Pack<f16_t, 4>{(f16_t)v[0], (f16_t)v[1], (f16_t)v[2], (f16_t)v[3]});
    }
}

// A tile of 128 x 128 of c a workgroup, a quarter a wavefront, a block of the depth at a time through LDS.
template <int kTypeA, int kTypeB, Exactness kExact>
__global__ __launch_bounds__(256) void k_product(ProductArgs p)
{
    constexpr int kTile = 128;
    __shared__ u32x4_t side_a[kTile * 8], side_b[kTile * 8];
    const uint32_t lane = threadIdx.x & 63, wave = threadIdx.x >> 6, r = lane & 15, g = lane >> 4;
    const uint32_t wave_row = (wave >> 1) * 64, wave_col = (wave & 1) * 64;
    const uint32_t across = div_up(p.cols, kTile), down = div_up(p.rows, kTile);
    const uint64_t items = (uint64_t)across * down * p.splits;
    for (uint64_t item = blockIdx.x; item < items; item += gridDim.x) {
    const uint32_t split = (uint32_t)(item % p.splits);
    const uint64_t tile = item / p.splits;
    const uint32_t row0 = (uint32_t)(tile / across) * kTile, col0 = (uint32_t)(tile % across) * kTile;
    f32x4_t sum[4][4] = {};
    const uint32_t first = split * p.blocks_each, last = min(p.blocks, first + p.blocks_each);
    for (uint32_t block = first; block < last; ++block) {
        __syncthreads();
#pragma unroll
        for (int i = 0; i < kTile * 8 / 256; ++i) {
            const uint32_t chunk = i * 256 + threadIdx.x, row = chunk / 8, c = chunk % 8, k = block * kBlock8 + c * 16;
            side_a[row * 8 + (c ^ (row & 7))] = product_chunk(p.a.code + (uint64_t)min(row0 + row, p.rows - 1) * p.a.stride, k, p.depth);
            side_b[row * 8 + (c ^ (row & 7))] = product_chunk(p.b.code + (uint64_t)min(col0 + row, p.cols - 1) * p.b.stride, k, p.depth);
        }
        uint32_t scale_a[4], scale_b[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const uint32_t row = min(row0 + wave_row + i * 16 + r, p.rows - 1), col = min(col0 + wave_col + i * 16 + r, p.cols - 1);
            scale_a[i] = p.a.scale[(uint64_t)(row >> p.a.shared_bits) * p.a.scale_stride + block];
            scale_b[i] = p.b.scale[(uint64_t)(col >> p.b.shared_bits) * p.b.scale_stride + block];
        }
        __syncthreads();
        const auto chunk_of = [&](const u32x4_t *side, uint32_t row, uint32_t c) { return side[row * 8 + (c ^ (row & 7))]; };
        if constexpr (kExact == kGroups) {
            i32x8_t b[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const u32x4_t lo = chunk_of(side_b, wave_col + j * 16 + r, 2 * g), hi = chunk_of(side_b, wave_col + j * 16 + r, 2 * g + 1);
                b[j] = i32x8_t{(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
            }
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const u32x4_t lo = chunk_of(side_a, wave_row + i * 16 + r, 2 * g), hi = chunk_of(side_a, wave_row + i * 16 + r, 2 * g + 1);
                const i32x8_t a = {(int)lo[0], (int)lo[1], (int)lo[2], (int)lo[3], (int)hi[0], (int)hi[1], (int)hi[2], (int)hi[3]};
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    sum[i][j] = __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(b[j], a, sum[i][j], kTypeB, kTypeA, 0, scale_b[j], 0, scale_a[i]);
            }
        } else {
#pragma unroll
            for (int part = 0; part < 4; ++part) {
                bf16x8_t b[4];
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    widen8<kTypeB>(chunk_of(side_b, wave_col + j * 16 + r, 2 * g + part / 2), part % 2, scale_value(scale_b[j]), b[j]);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    bf16x8_t a;
                    widen8<kTypeA>(chunk_of(side_a, wave_row + i * 16 + r, 2 * g + part / 2), part % 2, scale_value(scale_a[i]), a);
#pragma unroll
                    for (int j = 0; j < 4; ++j) sum[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a, sum[i][j], 0, 0, 0);
                }
            }
        }
    }
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) product_store(p, split, row0 + wave_row + i * 16 + r, col0 + wave_col + j * 16 + g * 4, sum[i][j]);
    }
}

// The splits added up.
__global__ __launch_bounds__(256) void k_product_join(ProductArgs p)
{
    const uint64_t count = (uint64_t)p.rows * p.cols;
    for (uint64_t i = blockIdx.x * 256ull + threadIdx.x; i < count; i += gridDim.x * 256ull) {
        float sum = 0.0f;
        for (uint32_t s = 0; s < p.splits; ++s) sum += p.part[s * count + i];
        const uint64_t row = i / p.cols, at = row * p.c_stride + (i - row * p.cols);
        if (p.c_type == PILC_F32)
            ((float *)p.c)[at] = sum;
        else if (p.c_type == PILC_BF16)
            ((bf16_t *)p.c)[at] = (bf16_t)sum;
        else
            ((f16_t *)p.c)[at] = (f16_t)sum;
    }
}

struct ProductPlan {
    uint32_t splits, blocks_each;
};
static ProductPlan product_plan(uint32_t rows, uint32_t cols, uint32_t depth)
{
    const uint64_t tiles = (uint64_t)div_up(rows, 128) * div_up(cols, 128);
    const uint32_t blocks = div_up(depth, kBlock8);
    uint32_t splits = 1;
    if (tiles < compute_units()) splits = std::max(1u, std::min(blocks / 4, (uint32_t)(2 * compute_units() / std::max<uint64_t>(tiles, 1))));
    const uint32_t each = std::max(1u, div_up(blocks, splits));
    return {std::max(1u, div_up(blocks, each)), each};
}

template <class Go>
static void by_types8(uint32_t a, uint32_t b, Go go)
{
    using std::integral_constant;
    const integral_constant<int, PILC_E4M3> e4m3;
    const integral_constant<int, PILC_E5M2> e5m2;
    if (a == PILC_E4M3)
        b == PILC_E4M3 ? go(e4m3, e4m3) : go(e4m3, e5m2);
    else
        b == PILC_E4M3 ? go(e5m2, e4m3) : go(e5m2, e5m2);
}

}  // namespace pilc

extern "C" {
using namespace pilc;

int pilc_block8_product_workspace_size(uint32_t rows, uint32_t cols, uint32_t depth, size_t *workspace_bytes_host)
{
    if (rows > kMostRows || cols > kMostRows || depth > kMostRows || !workspace_bytes_host) return PILC_E_ARG;
    const ProductPlan plan = product_plan(rows, cols, depth);
    *workspace_bytes_host = std::max<size_t>(256, plan.splits > 1 ? sizeof(float) * plan.splits * (size_t)rows * cols : 0);
    return PILC_OK;
}

int pilc_block8_product(uint32_t rows, uint32_t cols, uint32_t depth, const pilc_block8 *a, const pilc_block8 *b, void *c_dev, uint64_t c_stride,
                        uint32_t c_type, void *workspace_dev, size_t workspace_bytes, void *hip_stream)
{
    size_t needed = 0;
    if (pilc_block8_product_workspace_size(rows, cols, depth, &needed) != PILC_OK || !a || !b || !block8_ok(a, depth) || !block8_ok(b, depth) ||
        c_stride < cols || c_stride > (1ull << 48) || c_type > PILC_F16)
        return PILC_E_ARG;
    if (rows == 0 || cols == 0) return PILC_OK;
    if (!c_dev || !aligned_to(c_dev, value_bytes(c_type)) || (depth && (!a->code || !a->scale || !b->code || !b->scale)) || !workspace_dev ||
        !aligned_to(workspace_dev, 256))
        return PILC_E_ARG;
    if (workspace_bytes < needed) return PILC_E_WORKSPACE;
    const ProductPlan plan = product_plan(rows, cols, depth);
    ProductArgs p = {};
    p.a = block8_of(*a), p.b = block8_of(*b), p.c = c_dev, p.part = (float *)workspace_dev, p.c_stride = c_stride;
    p.rows = rows, p.cols = cols, p.depth = depth, p.c_type = c_type, p.blocks = div_up(depth, kBlock8);
    p.splits = plan.splits, p.blocks_each = plan.blocks_each;
    const hipStream_t stream = (hipStream_t)hip_stream;
    const uint32_t grid = (uint32_t)std::min<uint64_t>((uint64_t)div_up(cols, 128) * div_up(rows, 128) * plan.splits, 1u << 20);
    by_types8(a->type, b->type, [&](auto ta, auto tb) {
        if (c_type == PILC_F32 || rows <= 64)
            k_product<decltype(ta)::value, decltype(tb)::value, kSingles><<<grid, 256, 0, stream>>>(p);
        else
            k_product<decltype(ta)::value, decltype(tb)::value, kGroups><<<grid, 256, 0, stream>>>(p);
    });
    if (plan.splits > 1)
        k_product_join<<<(uint32_t)std::min<uint64_t>(((uint64_t)rows * cols + 255) / 256, 1u << 20), 256, 0, stream>>>(p);
    HIP_TRY(hipGetLastError());
    return PILC_OK;
}

}  // extern "C"
