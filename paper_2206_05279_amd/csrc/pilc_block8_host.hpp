// Host checks of matrices in 8 bits.
#pragma once
#include "pilc_block8_device.hpp"
#include "pilc_fit_host.hpp"

namespace pilc {

inline bool block8_ok(const pilc_block8 *m, uint32_t width)
{
    const uint64_t most = 1ull << 48;
    return m->type <= PILC_E5M2 && (m->block_rows == 1 || m->block_rows == kBlock8) && m->stride >= width && m->stride <= most &&
           m->scale_stride >= div_up(width, kBlock8) && m->scale_stride <= most;
}
inline Block8 block8_of(const pilc_block8 &m)
{
    return {(uint8_t *)m.code, m.scale, m.stride, m.scale_stride, m.type, m.block_rows == 1 ? 0u : 7u};
}
constexpr uint32_t kMostRows = 0x7FFFFFFFu;

}  // namespace pilc
