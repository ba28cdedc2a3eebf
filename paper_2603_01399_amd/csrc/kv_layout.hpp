// Where a key or value element lies in a block of 32 cached positions: the matrix-core operand order that attention.hpp explains.
#pragma once

#include "quasar_device.hpp"

namespace quasar {

constexpr int kHeadDim = 128;
constexpr int kKvBlock = 32;                 // positions per cache block
constexpr int kKvBlockBytes = 8192;          // 32 positions x 128 d x 2 B

__device__ __forceinline__ long long k_cache_index(int pos_in_block, int d) {
    const int sub = pos_in_block >> 4, p = pos_in_block & 15;
    return ((((long long)sub * 4 + (d >> 5)) * 4 + ((d & 31) >> 3)) * 16 + p) * 8 + (d & 7);
}
__device__ __forceinline__ long long v_cache_index(int pos_in_block, int d) {
    const int o = pos_in_block & 15;
    const int g4 = o >> 2, slot = (o & 3) + ((pos_in_block >> 4) << 2);
    return ((((long long)(d >> 4)) * 4 + g4) * 16 + (d & 15)) * 8 + slot;
}

}  // namespace quasar
