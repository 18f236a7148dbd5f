// The key / value cache in pages: new tokens in, as codes at given slots, and rows at given slots back out (Eq. 1 and the
// line under it, per position constants as in the dense cache).
//
// A page holds, for every 128 positions of the cluster order, one row of 16 * BITS bytes per token, so a token's codes lie
// in d / 128 pieces, page_size rows apart.  A wave owns 1024 consecutive channels (whole heads: a reorder index never leaves
// its head) of a row, eight such pieces, and moves them between channel and cluster order through a private piece of LDS; the
// constants of its 16 positions stay in a lane's registers over all rows of the wave.  Both tensors go in one launch.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "kv_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kLaneTab = kKvLaneCodes * 16 + 16;     // bytes of LDS per lane's 16 table records (padded: banks)

struct PagedLaunch {
  PagedTensor t[2];                                  // keys, values
  const int64_t* slots;
  int64_t T;
  PagedGeom g;
  int32_t segs;                                      // wave tiles per row
  int64_t rows_per_wave;
};

// Which tile, tensor and rows a wave has.
struct PagedShare {
  int base_ch, n_here;                               // first channel, channels (a multiple of 128)
  int64_t row, end;
  bool values;
};

__device__ __forceinline__ PagedShare paged_share(const PagedLaunch& a) {
  PagedShare s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned per = static_cast<unsigned>(a.segs) * 2;
  const unsigned which = blockIdx.x % per;
  s.values = which >= static_cast<unsigned>(a.segs);
  s.base_ch = static_cast<int>(which - (s.values ? a.segs : 0)) * kKvTile;
  s.n_here = min(a.g.d - s.base_ch, kKvTile);
  s.row = (static_cast<int64_t>(blockIdx.x / per) * 4 + wave) * a.rows_per_wave;
  s.end = min(s.row + a.rows_per_wave, a.T);
  return s;
}

// The workgroup's table records, in order, to LDS (a lane's own are 256 bytes apart from its neighbour's).
__device__ __forceinline__ void paged_table(const PagedTensor& t, const PagedShare& s, unsigned char* tab) {
  typedef unsigned u4v __attribute__((ext_vector_type(4)));
#pragma unroll
  for (int k = 0; k < kKvTile / 256; ++k) {
    const int i = k * 256 + static_cast<int>(threadIdx.x);
    *reinterpret_cast<u4v*>(tab + i * 16 + i / kKvLaneCodes * 16) =
        reinterpret_cast<const u4v*>(t.pos)[s.base_ch + (i < s.n_here ? i : 0)];
  }
}

// Bytes from the pages' start to this lane's piece of a row: 16 positions (3 bits: the group it shares with a neighbour).
template <int BITS>
__device__ __forceinline__ int64_t paged_row(const PagedGeom& g, int64_t slot, int block) {
  const int64_t page = slot >> g.page_shift, row = slot & ((INT64_C(1) << g.page_shift) - 1);
  return (((page * (g.d / kPageBlock) + block) << g.page_shift) + row) * (16 * BITS);
}

__device__ __forceinline__ bool paged_slot_ok(const PagedGeom& g, int64_t slot) {
  return slot >= 0 && slot < (g.n_pages << g.page_shift);
}

template <int BITS>
__global__ void __launch_bounds__(256) kv_quant_paged_kernel(PagedLaunch a) {
  constexpr int kQMin = -(1 << (BITS - 1));
  constexpr float kUMax = static_cast<float>((1 << BITS) - 1);
  __shared__ __align__(16) unsigned char tab[kWave * kLaneTab];
  __shared__ __align__(16) unsigned char lds[4][kKvTile * 2];
  const int lane = threadIdx.x & 63;
  unsigned char* my = lds[threadIdx.x >> 6];
  PagedShare s = paged_share(a);
  const PagedTensor& t = a.t[s.values];
  // (a lane's chunks of the row, clamped inside the tile; surplus data is never gathered)
  const int chunks = s.n_here / 8;
  const int ch0 = min(lane, chunks - 1), ch1 = min(64 + lane, chunks - 1);
  auto row_ptr = [&](int64_t r) {
    return reinterpret_cast<const uint4*>(t.x + min(r, a.T - 1) * t.ld + s.base_ch);
  };
  // (requested before the table, so that the two latencies run side by side)
  uint4 cur0 = row_ptr(s.row)[ch0], cur1 = row_ptr(s.row)[ch1];
  uint4 nxt0 = row_ptr(s.row + 1)[ch0], nxt1 = row_ptr(s.row + 1)[ch1];
  int64_t slot = a.slots[min(s.row, a.T - 1)], next_slot = a.slots[min(s.row + 1, a.T - 1)];
  paged_table(t, s, tab);
  __syncthreads();
  uint32_t src[kKvLaneCodes];
  float inv_s[kKvLaneCodes], zbf[kKvLaneCodes];
#pragma unroll
  for (int e = 0; e < kKvLaneCodes; ++e) {
    const int lp = kv_local_pos<BITS>(lane, e);
    const KvPos kp = *reinterpret_cast<const KvPos*>(tab + lp * 16 + lp / kKvLaneCodes * 16);
    src[e] = static_cast<uint32_t>(kp.src & (kKvTile - 1)) * 2u;
    inv_s[e] = kp.inv_s;
    zbf[e] = static_cast<float>(kp.z - kQMin);
  }
  const int block = s.base_ch / kPageBlock + (lane >> 3);             // this lane's 128 positions
  const int piece = BITS == 3 ? ((lane & 7) >> 1) * 12 : (lane & 7) * 2 * BITS;
  const bool lane_ok = lane * kKvLaneCodes < s.n_here;
  for (; s.row < s.end; ++s.row) {
    *reinterpret_cast<uint4*>(my + lane * 16) = cur0;
    *reinterpret_cast<uint4*>(my + (64 + lane) * 16) = cur1;
    cur0 = nxt0;
    cur1 = nxt1;
    nxt0 = row_ptr(s.row + 2)[ch0];
    nxt1 = row_ptr(s.row + 2)[ch1];
    wave_lds_fence();
    uint32_t D[4] = {0u, 0u, 0u, 0u};                // biased codes, one byte each
#pragma unroll
    for (int e = 0; e < kKvLaneCodes; ++e) {
      const uint32_t h = *reinterpret_cast<const uint16_t*>(my + src[e]);
      const float r = __fmul_rn(__uint_as_float(h << 16), inv_s[e]);
      float b = __fadd_rn(rintf(r), zbf[e]);         // round, then add the zero point (biased by -qmin)
      if (BITS < 8) b = fminf(b, kUMax);             // upper clamp; the conversion saturates at 0 and 255
      D[e / 4] = __builtin_amdgcn_cvt_pk_u8_f32(b, e & 3, D[e / 4]);
    }
    wave_lds_fence();
    const bool ok = lane_ok && paged_slot_ok(a.g, slot);
    kv_store_codes<BITS>(t.pages + paged_row<BITS>(a.g, ok ? slot : 0, block) + piece, lane, ok, D[0], D[1], D[2], D[3]);
    slot = next_slot;
    next_slot = a.slots[min(s.row + 2, a.T - 1)];
  }
}

// A lane expands 16 consecutive positions of a row, puts the values at their channels in LDS and stores two 16-byte pieces
// of the row in channel order (a wave writes 2 KiB contiguous).
template <int BITS>
__global__ void __launch_bounds__(256) kv_dequant_paged_kernel(PagedLaunch a) {
  constexpr int ND = BITS == 3 ? 3 : BITS / 2;       // dwords that hold a lane's 16 codes (3 bits: half of them)
  typedef unsigned u4v __attribute__((ext_vector_type(4)));
  __shared__ __align__(16) unsigned char tab[kWave * kLaneTab];
  __shared__ __align__(16) unsigned char lds[4][kKvTile * 2];
  const int lane = threadIdx.x & 63;
  unsigned char* my = lds[threadIdx.x >> 6];
  PagedShare s = paged_share(a);
  const PagedTensor& t = a.t[s.values];
  const int last_block = (s.base_ch + s.n_here) / kPageBlock - 1;
  const int block = min(s.base_ch / kPageBlock + (lane >> 3), last_block);
  const int piece = BITS == 3 ? ((lane & 7) >> 1) * 12 : (lane & 7) * 2 * BITS;
  auto slot_of = [&](int64_t r) { return a.slots[min(r, a.T - 1)]; };
  auto load = [&](int64_t slot, uint32_t (&w)[ND]) {
    const uint32_t* p = reinterpret_cast<const uint32_t*>(t.pages + paged_row<BITS>(a.g, paged_slot_ok(a.g, slot) ? slot : 0, block) + piece);
#pragma unroll
    for (int k = 0; k < ND; ++k) w[k] = p[k];
  };
  int64_t slot = slot_of(s.row), next_slot = slot_of(s.row + 1);
  uint32_t cur[ND], nxt[ND];
  load(slot, cur);
  load(next_slot, nxt);
  paged_table(t, s, tab);
  __syncthreads();
  uint32_t src[kKvLaneCodes];
  float sc[kKvLaneCodes], zf[kKvLaneCodes];
#pragma unroll
  for (int e = 0; e < kKvLaneCodes; ++e) {
    const KvPos kp = *reinterpret_cast<const KvPos*>(tab + lane * kLaneTab + e * 16);
    src[e] = static_cast<uint32_t>(kp.src & (kKvTile - 1)) * 2u;
    sc[e] = kp.s;
    zf[e] = static_cast<float>(kp.z);
  }
  const int chunks = s.n_here / 8;
  const bool lane_ok = lane * kKvLaneCodes < s.n_here;
  for (; s.row < s.end; ++s.row) {
    int q[kKvLaneCodes];
    if constexpr (BITS == 8) {
#pragma unroll
      for (int j = 0; j < 16; ++j) q[j] = static_cast<int>(cur[(j / 4) % ND] << (24 - 8 * (j & 3))) >> 24;
    } else if constexpr (BITS == 4) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        q[j] = static_cast<int>(cur[(j / 8) % ND] << ((j & 4 ? 28 : 24) - 8 * (j & 3))) >> 28;
    } else {
      // the upper half of a group: codes 16..23 are x2's own fields, 24..31 lie in the low bits of all three
      const uint32_t w3 = ((cur[0] << 6) & 0xc0c0c0c0u) | ((cur[2 % ND] << 5) & 0x20202020u) |
                          ((cur[1 % ND] << 3) & 0x18181818u) | ((cur[2 % ND] << 1) & 0x04040404u);
      const uint32_t v0 = lane & 1 ? cur[2 % ND] : cur[0], v1 = lane & 1 ? w3 : cur[1 % ND];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        q[j] = static_cast<int>((j < 8 ? v0 : v1) << ((j & 4 ? 27 : 24) - 8 * (j & 3))) >> 29;
    }
#pragma unroll
    for (int e = 0; e < kKvLaneCodes; ++e) {
      // s (x_q - z): the integer difference is exact in fp32, one rounded product, then bf16 (ties to even)
      const __bf16 h = static_cast<__bf16>(__fmul_rn(sc[e], static_cast<float>(q[e]) - zf[e]));
      if (lane_ok) *reinterpret_cast<__bf16*>(my + src[e]) = h;
    }
#pragma unroll
    for (int k = 0; k < ND; ++k) cur[k] = nxt[k];
    const int64_t after = slot_of(s.row + 2);
    load(after, nxt);
    wave_lds_fence();
    const u4v o0 = *reinterpret_cast<const u4v*>(my + lane * 16), o1 = *reinterpret_cast<const u4v*>(my + (64 + lane) * 16);
    wave_lds_fence();
    if (paged_slot_ok(a.g, slot)) {
      u4v* dst = reinterpret_cast<u4v*>(t.x + s.row * t.ld + s.base_ch);
      if (lane < chunks) dst[lane] = o0;
      if (64 + lane < chunks) dst[64 + lane] = o1;
    }
    slot = next_slot;
    next_slot = after;
  }
}

// Three workgroups of four waves per compute unit, and no more waves than rows.
static int32_t paged_launch(const PagedTensor& k, const PagedTensor& v, const int64_t* slots, int64_t T, const PagedGeom& g,
                            hipStream_t st, PagedLaunch* a, unsigned* grid) {
  int cus = 0;
  if (int32_t s = device_compute_units(st, &cus)) return s;
  const int segs = (g.d + kKvTile - 1) / kKvTile;
  const int64_t groups = std::max<int64_t>(1, static_cast<int64_t>(cus) * 3 / (2 * segs));
  const int64_t rows = std::max<int64_t>(1, (T + groups * 4 - 1) / (groups * 4));
  *a = PagedLaunch{{k, v}, slots, T, g, segs, rows};
  *grid = static_cast<unsigned>((T + rows * 4 - 1) / (rows * 4)) * 2 * segs;
  return RPTQ_OK;
}

int32_t launch_kv_quant_paged(const PagedTensor& k, const PagedTensor& v, const int64_t* slots, int64_t T,
                              const PagedGeom& g, int32_t bits, hipStream_t st) {
  if (T == 0) return RPTQ_OK;
  PagedLaunch a;
  unsigned grid = 0;
  if (int32_t s = paged_launch(k, v, slots, T, g, st, &a, &grid)) return s;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, st, a); };
  if (bits == 3) go(kv_quant_paged_kernel<3>);
  else if (bits == 4) go(kv_quant_paged_kernel<4>);
  else go(kv_quant_paged_kernel<8>);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

int32_t launch_kv_dequant_paged(const PagedTensor& k, const PagedTensor& v, const int64_t* slots, int64_t T,
                                const PagedGeom& g, int32_t bits, hipStream_t st) {
  if (T == 0) return RPTQ_OK;
  PagedLaunch a;
  unsigned grid = 0;
  if (int32_t s = paged_launch(k, v, slots, T, g, st, &a, &grid)) return s;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(grid), dim3(256), 0, st, a); };
  if (bits == 3) go(kv_dequant_paged_kernel<3>);
  else if (bits == 4) go(kv_dequant_paged_kernel<4>);
  else go(kv_dequant_paged_kernel<8>);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
