// What the kernels that write key / value cache codes share: which positions a lane carries, and how it stores them.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kKvTile = 1024;                  // channels per wave tile
constexpr int kKvLaneCodes = 16;               // codes per lane

// position of local code e of a lane inside the wave tile
template <int BITS>
__device__ __forceinline__ int kv_local_pos(int lane, int e) {
  if (BITS == 3) {
    // lanes 2g, 2g+1 share the 32-code group g: lane 2g carries codes 0..7, 24..27, 16..19,
    // lane 2g+1 codes 8..15, 28..31, 20..23 (so that each owns whole dwords of the group)
    const int role = lane & 1, gbase = (lane >> 1) * kGroup;
    if (e < 8) return gbase + role * 8 + e;
    if (e < 12) return gbase + 24 + role * 4 + (e - 8);
    return gbase + 16 + role * 4 + (e - 12);
  }
  return lane * kKvLaneCodes + e;
}

// Packs and stores a lane's 16 biased codes (code - qmin, one byte each, in D0..D3).  `p`: 8 and 4 bits, the lane's 16 or 8
// bytes; 3 bits, the 12 bytes of the group that lanes 2g and 2g + 1 share (both lanes call this).
template <int BITS>
__device__ __forceinline__ void kv_store_codes(uint8_t* p, int lane, bool ok, uint32_t D0, uint32_t D1, uint32_t D2, uint32_t D3) {
  if (BITS == 8) {
    const uint4 o = make_uint4(D0 ^ 0x80808080u, D1 ^ 0x80808080u, D2 ^ 0x80808080u, D3 ^ 0x80808080u);
    if (ok) *reinterpret_cast<uint4*>(p) = o;
  } else if (BITS == 4) {
    uint2 o;
    o.x = ((D0 << 4) | D1) ^ 0x88888888u;
    o.y = ((D2 << 4) | D3) ^ 0x88888888u;
    if (ok) *reinterpret_cast<uint2*>(p) = o;
  } else {
    const int role = lane & 1;
    const uint32_t w1 = ((D0 << 5) | (D1 << 2) | ((D2 >> 1) & 0x03030303u)) ^ 0x80808080u ^ 0x10101010u ^ 0x02020202u;
    const uint32_t mine = role ? (((D3 << 2) ^ 0x10101010u) | ((D2 & 0x01010101u) << 1))
                               : (((D3 << 5) ^ 0x80808080u) | (D2 & 0x01010101u));
    const uint32_t other = __shfl_xor(mine, 1, kWave);
    if (ok) {
      uint32_t* q = reinterpret_cast<uint32_t*>(p + role * 4);
      q[0] = w1;
      if (role) q[1] = mine | other;
    }
  }
}

}  // namespace rptq
