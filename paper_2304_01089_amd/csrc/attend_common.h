// What the kernels that score queries against cache codes on the int8 matrix cores share: exchanges between lanes, numbers in
// fixed point as digits, codes as operands.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

namespace rptq {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr int kTile = 64;                      // tokens of a wave's tile
constexpr int kRowHeads = 4;                   // queries per 16 rows of the matrix product

// ---- lane arithmetic ------------------------------------------------------------------------------------
template <int CTRL>
__device__ __forceinline__ uint32_t dpp_row(uint32_t v) {                // a permutation inside a row of 16 lanes
  return static_cast<uint32_t>(__builtin_amdgcn_mov_dpp(static_cast<int>(v), CTRL, 0xf, 0xf, true));
}
template <int CTRL>
__device__ __forceinline__ float dpp_row(float v) { return __uint_as_float(dpp_row<CTRL>(__float_as_uint(v))); }

__device__ __forceinline__ float row16_max(float v) {
  v = fmaxf(v, dpp_row<0xB1>(v));
  v = fmaxf(v, dpp_row<0x4E>(v));
  v = fmaxf(v, dpp_row<0x141>(v));
  return fmaxf(v, dpp_row<0x140>(v));
}
__device__ __forceinline__ float row16_add(float v) {
  v += dpp_row<0xB1>(v);
  v += dpp_row<0x4E>(v);
  v += dpp_row<0x141>(v);
  return v + dpp_row<0x140>(v);
}
__device__ __forceinline__ float wave_max(float v) {
  v = row16_max(v);
  auto row = [&](int lane) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(v), lane)); };
  return fmaxf(fmaxf(row(0), row(16)), fmaxf(row(32), row(48)));
}

template <int CTRL, int ROWS>
__device__ __forceinline__ int dpp_plus(int v) {
  return v + __builtin_amdgcn_update_dpp(0, v, CTRL, ROWS, 0xf, false);
}
__device__ __forceinline__ int wave_prefix(int v) {                      // inclusive
  v = dpp_plus<0x111, 0xf>(v);
  v = dpp_plus<0x112, 0xf>(v);
  v = dpp_plus<0x114, 0xf>(v);
  v = dpp_plus<0x118, 0xf>(v);
  v = dpp_plus<0x142, 0xa>(v);
  return dpp_plus<0x143, 0xc>(v);
}

// A lane's 64 bits in every lane.  (readlane gives a signed number: its lower half must not fill the upper with its sign.)
__device__ __forceinline__ uint64_t of_lane(uint32_t lo, uint32_t hi, int lane) {
  const uint32_t l = __builtin_amdgcn_readlane(lo, lane), h = __builtin_amdgcn_readlane(hi, lane);
  return static_cast<uint64_t>(h) << 32 | l;
}

// Four lanes' four bytes transposed: lane i's byte b becomes lane b's byte i.  (Two exchanges, of neighbours and of pairs.)
struct QuadSel {
  uint32_t s0, s1;
};
__device__ __forceinline__ QuadSel quad_sel(int lane) {
  return {lane & 1 ? 0x03070105u : 0x06020400u, lane & 2 ? 0x03020706u : 0x05040100u};
}
__device__ __forceinline__ uint32_t quad_transpose(uint32_t x, const QuadSel& s) {
  x = __builtin_amdgcn_perm(dpp_row<0xB1>(x), x, s.s0);
  return __builtin_amdgcn_perm(dpp_row<0x4E>(x), x, s.s1);
}

// A number of up to 31 bits as four signed digits to the base 256, lowest in the lowest byte.
__device__ __forceinline__ uint32_t digits(int v) { return (static_cast<uint32_t>(v) + 0x80808080u) ^ 0x80808080u; }

// The digits' sums, lowest first, as one fp32 number (the products of two digits' sums with the base are exact).
__device__ __forceinline__ float undigit(const v4i& c) {
  return fmaf(static_cast<float>(c[3] * 256 + c[2]), 65536.0f, static_cast<float>(c[1] * 256 + c[0]));
}

// 32 packed codes (of one token; or, after quad_transpose, byte b of four tokens) -> operand bytes code << kShift, codes 4e..4e+3 in w[e]
template <int BITS>
__device__ __forceinline__ void expand(const uint32_t (&x)[BITS], uint32_t (&w)[8]) {
  if constexpr (BITS == 8) {
#pragma unroll
    for (int e = 0; e < 8; ++e) w[e] = x[e];
  } else if constexpr (BITS == 4) {
#pragma unroll
    for (int u = 0; u < 4; ++u) {
      w[2 * u] = x[u] & 0xf0f0f0f0u;
      w[2 * u + 1] = (x[u] << 4) & 0xf0f0f0f0u;
    }
  } else {
#pragma unroll
    for (int u = 0; u < 3; ++u) {
      w[2 * u] = x[u] & 0xe0e0e0e0u;
      w[2 * u + 1] = (x[u] << 3) & 0xe0e0e0e0u;
    }
    w[6] = ((x[0] << 6) & 0xc0c0c0c0u) | ((x[2] << 5) & 0x20202020u);
    w[7] = ((x[1] << 6) & 0xc0c0c0c0u) | ((x[2] << 4) & 0x20202020u);
  }
}

}  // namespace rptq
