// Host helpers of the operators that fit laws: types of values, alignment, and a launch for each type.
#pragma once
#include <algorithm>
#include <cmath>
#include <cstdint>
#include <type_traits>

#include "pilc_fit_device.hpp"
#include "pilc_host.hpp"
#include "pilc_row_rules.hpp"

namespace pilc {

inline size_t value_bytes(uint32_t type) { return type == PILC_F32 ? 4 : 2; }
inline bool aligned_to(const void *p, size_t bytes) { return ((uintptr_t)p & (bytes - 1)) == 0; }

template <class Launch>
inline void by_value_type(uint32_t type, Launch launch)
{
    switch (type) {
    case PILC_F32: launch((float *)nullptr); break;
    case PILC_BF16: launch((bf16_t *)nullptr); break;
    default: launch((f16_t *)nullptr); break;
    }
}
template <class Launch>
inline int by_type(uint32_t type, Launch launch)
{
    by_value_type(type, launch);
    HIP_TRY(hipGetLastError());
    return PILC_OK;
}

template <class Launch>
inline int by_types(uint32_t type, uint32_t weight_type, Launch launch)
{
    return by_type(type, [&](auto *t) {
        if (weight_type == type)
            launch(t, t);
        else
            launch(t, (float *)nullptr);
    });
}

}  // namespace pilc
