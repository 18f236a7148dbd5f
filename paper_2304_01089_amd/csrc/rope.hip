// Rotary positions: the pairs (a, b) of the first rotary_dim channels of every head turned by theta = position * frequency,
//   (a cos - b sin, b cos + a sin),   pairs (j, j + rotary_dim / 2) or (2 j, 2 j + 1),
// cosine and sine in 64 bits and rounded once to fp32, two products and a sum rounded to fp32 each, then once to the output's type.
//
// A workgroup takes a few rows: first their cosines and sines, one per thread, into LDS, then all heads of the rows, every thread
// a piece of up to 16 bytes (half style: two, W channels and their W partners).  The angles are thus computed once per row
// and group of heads and read from memory never.
// What bounds it: memory: 8192 rows of 80 heads of 128 take 69.9 us for 336 MB, 4.8 TB/s of as many bytes read as written (a copy reaches
// 5.15).  Few rows: the launch and two dependent loads, 2.4 us for one row, of which an empty launch is 1.8.
// Rows of a workgroup: 2 | 4 | 8 69.2 | 69.9 | 71.0 us here and 85.0 | 82.7 | 84.6 in front of the cache.  Not kept: two or four pieces a
// thread requested ahead (3 and 1 % more), non-temporal loads and stores (no change).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "rope_common.h"
#include "rptq_internal.h"

namespace rptq {

template <int W, bool HALF, typename TX, typename TY>
__global__ void __launch_bounds__(kRopeThreads) rope_kernel(RopeLaunch l) {
  __shared__ __align__(16) float turns[2 * kRopePairs];
  rope_rows<W, HALF, TX, TY>(l, blockIdx.x, turns);
}

template <int W, bool HALF>
static void launch_types(const RopeLaunch& l, hipStream_t st) {
  const bool xf = l.a.x_dtype == RPTQ_DTYPE_F32, yf = l.a.y_dtype == RPTQ_DTYPE_F32;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(l.groups), dim3(kRopeThreads), 0, st, l); };
  if (xf) yf ? go(rope_kernel<W, HALF, float, float>) : go(rope_kernel<W, HALF, float, __bf16>);
  else yf ? go(rope_kernel<W, HALF, __bf16, float>) : go(rope_kernel<W, HALF, __bf16, __bf16>);
}

int64_t plan_rope(const RopeArgs& a, int W, bool same, RopeLaunch* l) {
  const int half = a.rot / 2;
  l->turned = a.interleaved && W > 1 ? a.rot / W : half / W;
  l->units = l->turned + (same ? 0 : (a.hd - a.rot) / W);
  const RopeShares s = rope_shares(a.T, a.n_heads, half, l->units);
  l->rows = s.rows;
  l->heads = s.heads;
  l->head_groups = s.head_groups;
  return s.launch_rows;
}

void rope_part(const RopeArgs& a, int64_t first, int64_t rows, RopeLaunch* l) {
  const int x_size = a.x_dtype == RPTQ_DTYPE_F32 ? 4 : 2, y_size = a.y_dtype == RPTQ_DTYPE_F32 ? 4 : 2;
  l->a = a;
  l->a.x = static_cast<const uint8_t*>(a.x) + first * a.ld_x * x_size;
  l->a.y = static_cast<uint8_t*>(a.y) + first * a.ld_y * y_size;
  l->a.positions = a.positions + first;
  l->a.T = rows;
  l->groups = static_cast<int32_t>((rows + l->rows - 1) / l->rows * l->head_groups);
}

int32_t launch_rope(const RopeArgs& a, hipStream_t st) {
  const int32_t x_size = a.x_dtype == RPTQ_DTYPE_F32 ? 4 : 2, y_size = a.y_dtype == RPTQ_DTYPE_F32 ? 4 : 2;
  const bool same = a.x == a.y && a.ld_x == a.ld_y && a.x_dtype == a.y_dtype, halves = a.interleaved == 0;
  if (a.T == 0) return RPTQ_OK;
  // The widest piece (16 bytes of bf16) that strides, addresses and the ends of the rotated part allow.
  auto fits = [&](int w) {
    auto at = [&](const void* p, int size) { return reinterpret_cast<uintptr_t>(p) % std::min(w * size, 16) == 0; };
    return a.ld_x % w == 0 && a.ld_y % w == 0 && a.hd % w == 0 && (halves ? a.rot / 2 : a.rot) % w == 0 && at(a.x, x_size) && at(a.y, y_size);
  };
  int W = 8;
  while (W > 1 && !fits(W)) W /= 2;
  RopeLaunch l;
  const int64_t most = plan_rope(a, W, same, &l);
  for (int64_t first = 0; first < a.T; first += most) {
    rope_part(a, first, std::min(most, a.T - first), &l);
    if (W == 8) halves ? launch_types<8, true>(l, st) : launch_types<8, false>(l, st);
    else if (W == 4) halves ? launch_types<4, true>(l, st) : launch_types<4, false>(l, st);
    else if (W == 2) halves ? launch_types<2, true>(l, st) : launch_types<2, false>(l, st);
    else halves ? launch_types<1, true>(l, st) : launch_types<1, false>(l, st);
    RPTQ_HIP(hipGetLastError());
  }
  return RPTQ_OK;
}

}  // namespace rptq
