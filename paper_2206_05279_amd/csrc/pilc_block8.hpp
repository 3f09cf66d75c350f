// Matrices into 8 bits under scales for blocks of 128, and back.
#pragma once

namespace pilc {

// A tile of 128 x 128 values in registers, eight rows of eight columns a thread: rows' or the tile's largest value gives the scales,
// codes are stored from there; the transposed codes go by LDS, so that both sides' stores are whole lines.  Bound by memory, and by a
// tile's one chain of loads, meetings and stores, which other workgroups' have to fill.
constexpr int kTileThreads = 256;

template <class T>
__global__ __launch_bounds__(kTileThreads) void k_block8_tiles(uint32_t rows, uint32_t width, const T *x, uint64_t x_stride, Block8 out, Block8 out_t)
{
    __shared__ uint32_t column_largest[16][kBlock8];
    __shared__ uint32_t tile_room[kTileThreads / 64];
    __shared__ uint64_t turned[kBlock8 * 16];
    const uint32_t across = threadIdx.x % 16, down = threadIdx.x / 16;
    const uint32_t tiles_across = div_up(width, kBlock8), tiles_down = div_up(rows, kBlock8);
    for (uint64_t tile = blockIdx.x; tile < (uint64_t)tiles_across * tiles_down; tile += gridDim.x) {
        const uint32_t tile_row = (uint32_t)(tile / tiles_across), tile_column = (uint32_t)(tile % tiles_across);
        const uint32_t row0 = tile_row * kBlock8 + down * 8, column0 = tile_column * kBlock8 + across * 8;
        const int valid = (int)min(width - min(column0, width), 8u);
        float v[8][8];
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            Pack<T, 8> p;
            if (row0 + i < rows && valid > 0)
                p = load_pack<8>(x + (uint64_t)(row0 + i) * x_stride + column0, valid);
            else
#pragma unroll
                for (int k = 0; k < 8; ++k) p.v[k] = (T)0;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[i][k] = widen(p.v[k]);
        }
        const bool by_tile = (out.code && out.shared_bits) || (out_t.code && out_t.shared_bits);
        uint32_t tile_largest = 0;
        if (by_tile) {
            uint32_t m = 0;
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int k = 0; k < 8; ++k) m = max(m, size_bits(v[i][k]));
            tile_largest = block_reduce<kTileThreads / 64>(m, Max(), tile_room);
        }
        if (out.code) {
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                uint32_t m = tile_largest;
                if (!out.shared_bits) {
                    m = 0;
#pragma unroll
                    for (int k = 0; k < 8; ++k) m = max(m, size_bits(v[i][k]));
                    m = lanes_reduce<16>(m, Max());
                }
                const uint32_t byte = scale_byte(m, out.type), row = row0 + i;
                const float f = scale_inverse(byte);
                Pack<uint8_t, 8> codes;
                const uint32_t lo = codes_of(v[i][0] * f, v[i][1] * f, v[i][2] * f, v[i][3] * f, out.type, byte);
                const uint32_t hi = codes_of(v[i][4] * f, v[i][5] * f, v[i][6] * f, v[i][7] * f, out.type, byte);
                codes = __builtin_bit_cast(decltype(codes), (uint64_t)hi << 32 | lo);
                if (row < rows) {
                    if (valid > 0) store_pack<8>(out.code + (uint64_t)row * out.stride + column0, valid, codes);
                    if (across == 0 && (!out.shared_bits || (i == 0 && down == 0)))
                        out.scale[(uint64_t)(row >> out.shared_bits) * out.scale_stride + tile_column] = (uint8_t)byte;
                }
            }
        }
        if (out_t.code) {
            if (!out_t.shared_bits) {
#pragma unroll
                for (int k = 0; k < 8; ++k) {
                    uint32_t m = 0;
#pragma unroll
                    for (int i = 0; i < 8; ++i) m = max(m, size_bits(v[i][k]));
                    column_largest[down][across * 8 + k] = m;
                }
                __syncthreads();
            }
#pragma unroll
            for (int k = 0; k < 8; ++k) {
                uint32_t m = tile_largest;
                if (!out_t.shared_bits) {
                    m = 0;
#pragma unroll
                    for (int d = 0; d < 16; ++d) m = max(m, column_largest[d][across * 8 + k]);
                }
                const uint32_t byte = scale_byte(m, out_t.type), column = column0 + k;
                const float f = scale_inverse(byte);
                const uint32_t lo = codes_of(v[0][k] * f, v[1][k] * f, v[2][k] * f, v[3][k] * f, out_t.type, byte);
                const uint32_t hi = codes_of(v[4][k] * f, v[5][k] * f, v[6][k] * f, v[7][k] * f, out_t.type, byte);
                turned[(across * 8 + k) * 16 + (down ^ across)] = (uint64_t)hi << 32 | lo;
                if (down == 0 && column < width && (!out_t.shared_bits || (k == 0 && across == 0)))
                    out_t.scale[(uint64_t)(column >> out_t.shared_bits) * out_t.scale_stride + tile_row] = (uint8_t)byte;
            }
            __syncthreads();
            // sixteen threads a row of the transposed tile
            const uint32_t first = tile_row * kBlock8 + across * 8;
            const int valid_t = (int)min(rows - min(first, rows), 8u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const uint32_t j = i * 16 + down, column = tile_column * kBlock8 + j;
                if (column < width && valid_t > 0)
                    store_pack<8>(out_t.code + (uint64_t)column * out_t.stride + first, valid_t,
                                  __builtin_bit_cast(Pack<uint8_t, 8>, turned[j * 16 + (across ^ (j / 8))]));
            }
            __syncthreads();
        }
    }
}

// Rows by themselves, where no transposed matrix is wanted and no scales are shared: sixteen lanes a block, four rows at a time.  In
// bfloat16, and by the tiles: 1021 x 50001 31 and 46 us, 16384 x 4096 36 and 46, 64 x 8192 5 and 6.
template <class T>
__global__ __launch_bounds__(256) void k_block8_rows(uint32_t rows, uint32_t width, const T *x, uint64_t x_stride, Block8 out)
{
    constexpr int kRows = 4;
    const uint32_t packs = div_up(width, kBlock8) * 16;
    const uint64_t items = (uint64_t)div_up(rows, kRows) * packs;  // whole blocks: lanes of a block go on together
    for (uint64_t item = blockIdx.x * 256ull + threadIdx.x; item < items; item += gridDim.x * 256ull) {
        const uint32_t group = (uint32_t)(items >> 32 ? item / packs : (uint32_t)item / packs), column = (uint32_t)(item - (uint64_t)group * packs) * 8;
        const int valid = (int)min(width - min(column, width), 8u);
        Pack<T, 8> p[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) p[i] = load_pack<8>(x + (uint64_t)min(group * kRows + i, rows - 1) * x_stride + (valid > 0 ? column : 0), valid);
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            float v[8];
            uint32_t m = 0;
#pragma unroll
            for (int k = 0; k < 8; ++k) v[k] = widen(p[i].v[k]), m = max(m, size_bits(v[k]));
            const uint32_t byte = scale_byte(lanes_reduce<16>(m, Max()), out.type), row = group * kRows + i;
            const float f = scale_inverse(byte);
            const uint32_t lo = codes_of(v[0] * f, v[1] * f, v[2] * f, v[3] * f, out.type, byte);
            const uint32_t hi = codes_of(v[4] * f, v[5] * f, v[6] * f, v[7] * f, out.type, byte);
            if (row < rows && valid > 0) {
                store_pack<8>(out.code + (uint64_t)row * out.stride + column, valid, __builtin_bit_cast(Pack<uint8_t, 8>, (uint64_t)hi << 32 | lo));
                if (column % kBlock8 == 0) out.scale[(uint64_t)row * out.scale_stride + column / kBlock8] = (uint8_t)byte;
            }
        }
    }
}

// Values back, eight a thread and row, so that lanes' stores of 16-bit values follow one another; two rows at a time.  Bound by memory.
template <class T>
__global__ __launch_bounds__(256) void k_block8_values(uint32_t rows, uint32_t width, Block8 in, T *out, uint64_t stride)
{
    constexpr int kRows = 2;
    const uint32_t packs = div_up(width, 8);
    const uint64_t items = (uint64_t)div_up(rows, kRows) * packs;
    for (uint64_t item = blockIdx.x * 256ull + threadIdx.x; item < items; item += gridDim.x * 256ull) {
        const uint32_t row = (uint32_t)(items >> 32 ? item / packs : (uint32_t)item / packs), column = (uint32_t)(item - (uint64_t)row * packs) * 8;
        const int valid = (int)min(width - column, 8u);
        Pack<uint8_t, 8> codes[kRows];
        uint32_t byte[kRows];
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint32_t r = min(row * kRows + i, rows - 1);
            byte[i] = in.scale[(uint64_t)(r >> in.shared_bits) * in.scale_stride + column / kBlock8];
            codes[i] = load_pack<8>(in.code + (uint64_t)r * in.stride + column, valid);
        }
#pragma unroll
        for (int i = 0; i < kRows; ++i) {
            const uint64_t both = __builtin_bit_cast(uint64_t, codes[i]);
            Pack<T, 8> t;
#pragma unroll
            for (int n = 0; n < 2; ++n) {
                float v[4];
                values_of((uint32_t)(both >> (32 * n)), in.type, byte[i], v);
#pragma unroll
                for (int k = 0; k < 4; ++k) t.v[4 * n + k] = (T)v[k];
            }
            if (row * kRows + i < rows) store_pack<8>(out + (uint64_t)(row * kRows + i) * stride + column, valid, t);
        }
    }
}

}  // namespace pilc

extern "C" {
using namespace pilc;

int pilc_block8_quantize(uint32_t rows, uint32_t width, const void *x_dev, uint64_t x_stride, uint32_t dtype, const pilc_block8 *out,
                         const pilc_block8 *out_t, void *hip_stream)
{
    if (rows > kMostRows || width > kMostRows || x_stride < width || x_stride > (1ull << 48) || dtype > PILC_F16 || (!out && !out_t) ||
        (out && !block8_ok(out, width)) || (out_t && !block8_ok(out_t, rows)))
        return PILC_E_ARG;
    if (rows == 0 || width == 0) return PILC_OK;
    if (!x_dev || !aligned_to(x_dev, value_bytes(dtype)) || (out && (!out->code || !out->scale)) || (out_t && (!out_t->code || !out_t->scale)))
        return PILC_E_ARG;
    const Block8 none = {}, o = out ? block8_of(*out) : none, t = out_t ? block8_of(*out_t) : none;
    return by_type(dtype, [&](auto *type) {
        using T = std::remove_pointer_t<decltype(type)>;
        if (!out_t && !o.shared_bits) {
            const uint64_t blocks = ((uint64_t)div_up(rows, 4) * div_up(width, kBlock8) * 16 + 255) / 256;
            k_block8_rows<T><<<(uint32_t)std::min<uint64_t>(blocks, 1u << 20), 256, 0, (hipStream_t)hip_stream>>>(rows, width, (const T *)x_dev, x_stride, o);
            return;
        }
        const uint64_t tiles = (uint64_t)div_up(rows, kBlock8) * div_up(width, kBlock8);
        k_block8_tiles<T><<<(uint32_t)std::min<uint64_t>(tiles, 1u << 20), kTileThreads, 0, (hipStream_t)hip_stream>>>(rows, width, (const T *)x_dev, x_stride, o, t);
    });
}

int pilc_block8_values(uint32_t rows, uint32_t width, const pilc_block8 *in, void *values_dev, uint64_t stride, uint32_t dtype, void *hip_stream)
{
    if (rows > kMostRows || width > kMostRows || !in || !block8_ok(in, width) || stride < width || stride > (1ull << 48) || dtype > PILC_F16)
        return PILC_E_ARG;
    if (rows == 0 || width == 0) return PILC_OK;
    if (!in->code || !in->scale || !values_dev || !aligned_to(values_dev, value_bytes(dtype))) return PILC_E_ARG;
    return by_type(dtype, [&](auto *type) {
        using T = std::remove_pointer_t<decltype(type)>;
        const uint64_t blocks = ((uint64_t)div_up(rows, 2) * div_up(width, 8) + 255) / 256;
        k_block8_values<T><<<(uint32_t)std::min<uint64_t>(blocks, 1u << 20), 256, 0, (hipStream_t)hip_stream>>>(rows, width, block8_of(*in), (T *)values_dev, stride);
    });
}

}  // extern "C"
