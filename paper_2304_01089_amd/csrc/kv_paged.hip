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
#include "kv_paged_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kRowsAhead = 8;                        // rows requested before those that are expanded (even, at most 64)
constexpr int64_t kKvStreamBytes = 128ll << 20;      // of values: beyond, past the last-level cache (as for the dense read-back)

template <int BITS>
__global__ void __launch_bounds__(256) kv_quant_paged_kernel(PagedLaunch a) {
  constexpr int kQMin = -(1 << (BITS - 1));
  constexpr float kUMax = static_cast<float>((1 << BITS) - 1);
  __shared__ __align__(16) unsigned char tab[kWave * kLaneTab];
  __shared__ __align__(16) unsigned char lds[4][kKvTile * 2];
  const int lane = threadIdx.x & 63;
  unsigned char* my = lds[threadIdx.x >> 6];
  const PagedShare s = paged_share(a, blockIdx.x);
  const PagedTensor& t = a.t[s.values];
  // (a lane's chunks of the row, clamped inside the tile; surplus data is never gathered)
  const int chunks = s.n_here / 8;
  const int ch0 = min(lane, chunks - 1), ch1 = min(64 + lane, chunks - 1);
  auto row_ptr = [&](int64_t r) {
    return reinterpret_cast<const uint4*>(t.x + min(r, a.T - 1) * t.ld + s.base_ch);
  };
  // (requested before the table, so that the two latencies run side by side)
  uint4 cur0 = row_ptr(s.row(0))[ch0], cur1 = row_ptr(s.row(0))[ch1];
  uint4 nxt0 = row_ptr(s.row(1))[ch0], nxt1 = row_ptr(s.row(1))[ch1];
  SlotWindow<BITS> win(a, s, lane);
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
  const bool lane_ok = lane * kKvLaneCodes < s.n_here;
  const int64_t lane_at = paged_lane<BITS>(a.g, s.base_ch / kPageBlock + (lane >> 3), lane);
  for (int i = 0; s.row(i) < a.T; ++i) {
    win.move_to(i, lane);
    const int64_t place = win.place(i);
    *reinterpret_cast<uint4*>(my + lane * 16) = cur0;
    *reinterpret_cast<uint4*>(my + (64 + lane) * 16) = cur1;
    cur0 = nxt0;
    cur1 = nxt1;
    nxt0 = row_ptr(s.row(i + 2))[ch0];
    nxt1 = row_ptr(s.row(i + 2))[ch1];
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
    kv_store_codes<BITS>(t.pages + max(place, INT64_C(0)) + lane_at, lane, lane_ok && place >= 0, D[0], D[1], D[2], D[3]);
  }
}

// A lane expands 16 consecutive positions of two rows at a time and puts the pairs of values at their channels in LDS, four
// bytes each; from there every lane takes eight channels apart into one 16-byte piece of either row (a wave writes 1 KiB
// contiguous).
template <int BITS, bool STREAM>
__global__ void __launch_bounds__(256) kv_dequant_paged_kernel(PagedLaunch a) {
  constexpr int ND = BITS == 3 ? 3 : BITS / 2;       // dwords that hold a lane's 16 codes (3 bits: half of them)
  constexpr int kDump = kKvTile * 4;                 // where lanes without positions write
  typedef unsigned u4v __attribute__((ext_vector_type(4)));
  typedef float f2 __attribute__((ext_vector_type(2)));
  typedef __bf16 b2 __attribute__((ext_vector_type(2)));
  __shared__ __align__(16) unsigned char tab[kWave * kLaneTab];
  __shared__ __align__(16) unsigned char lds[4][kKvTile * 4 + 16];
  const int lane = threadIdx.x & 63;
  unsigned char* my = lds[threadIdx.x >> 6];
  const PagedShare s = paged_share(a, blockIdx.x);
  const PagedTensor& t = a.t[s.values];
  const int last_block = (s.base_ch + s.n_here) / kPageBlock - 1;
  const int64_t lane_at = paged_lane<BITS>(a.g, min(s.base_ch / kPageBlock + (lane >> 3), last_block), lane);
  SlotWindow<BITS> win(a, s, lane);
  uint32_t buf[kRowsAhead][ND];
  auto load = [&](int i, uint32_t (&w)[ND]) {       // (where there is no slot: the first row of the pages, stored nowhere)
    const uint32_t* p = reinterpret_cast<const uint32_t*>(t.pages + max(win.place(i), INT64_C(0)) + lane_at);
#pragma unroll
    for (int k = 0; k < ND; ++k) w[k] = p[k];
  };
#pragma unroll
  for (int k = 0; k < kRowsAhead; ++k) load(k, buf[k]);
  paged_table(t, s, tab);
  __syncthreads();
  uint32_t dst_at[kKvLaneCodes];
  float sc[kKvLaneCodes], zf[kKvLaneCodes];
#pragma unroll
  for (int e = 0; e < kKvLaneCodes; ++e) {
    const KvPos kp = *reinterpret_cast<const KvPos*>(tab + lane * kLaneTab + e * 16);
    dst_at[e] = lane * kKvLaneCodes < s.n_here ? static_cast<uint32_t>(kp.src & (kKvTile - 1)) * 4u : kDump;
    sc[e] = kp.s;
    zf[e] = static_cast<float>(kp.z);
  }
  const int chunks = s.n_here / 8;
  auto expand = [&](const uint32_t (&w)[ND], int (&q)[kKvLaneCodes]) {
    if constexpr (BITS == 8) {
#pragma unroll
      for (int j = 0; j < 16; ++j) q[j] = static_cast<int>(w[(j / 4) % ND] << (24 - 8 * (j & 3))) >> 24;
    } else if constexpr (BITS == 4) {
#pragma unroll
      for (int j = 0; j < 16; ++j)
        q[j] = static_cast<int>(w[(j / 8) % ND] << ((j & 4 ? 28 : 24) - 8 * (j & 3))) >> 28;
    } else {
      // the upper half of a group: codes 16..23 are x2's own fields, 24..31 lie in the low bits of all three
      const uint32_t w3 = ((w[0] << 6) & 0xc0c0c0c0u) | ((w[2 % ND] << 5) & 0x20202020u) |
                          ((w[1 % ND] << 3) & 0x18181818u) | ((w[2 % ND] << 1) & 0x04040404u);
      const uint32_t v0 = lane & 1 ? w[2 % ND] : w[0], v1 = lane & 1 ? w3 : w[1 % ND];
#pragma unroll
      for (int j = 0; j < 16; ++j)
        q[j] = static_cast<int>((j < 8 ? v0 : v1) << ((j & 4 ? 27 : 24) - 8 * (j & 3))) >> 29;
    }
  };
  auto pair = [&](int i, uint32_t (&w0)[ND], uint32_t (&w1)[ND]) {
    int q0[kKvLaneCodes], q1[kKvLaneCodes];
    expand(w0, q0);
    expand(w1, q1);
    const bool there0 = win.place(i) >= 0, there1 = win.place(i + 1) >= 0 && s.row(i + 1) < a.T;
    load(i + kRowsAhead, w0);
    load(i + kRowsAhead + 1, w1);
#pragma unroll
    for (int e = 0; e < kKvLaneCodes; ++e) {
      // s (x_q - z): the integer difference is exact in fp32, one rounded product, then bf16 (ties to even)
      const f2 pr = {__fmul_rn(sc[e], static_cast<float>(q0[e]) - zf[e]), __fmul_rn(sc[e], static_cast<float>(q1[e]) - zf[e])};
      const b2 cv = __builtin_convertvector(pr, b2);
      *reinterpret_cast<uint32_t*>(my + dst_at[e]) = *reinterpret_cast<const uint32_t*>(&cv);
    }
    wave_lds_fence();
    u4v d[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) d[k] = *reinterpret_cast<const u4v*>(my + (k >> 1) * 2048 + lane * 32 + (k & 1) * 16);
    wave_lds_fence();
    auto put = [&](int64_t row, uint32_t sel) {
      u4v* dst = reinterpret_cast<u4v*>(t.x + row * t.ld + s.base_ch);
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const u4v& x = d[2 * k];
        const u4v& y = d[2 * k + 1];
        const u4v o = {__builtin_amdgcn_perm(x[1], x[0], sel), __builtin_amdgcn_perm(x[3], x[2], sel),
                       __builtin_amdgcn_perm(y[1], y[0], sel), __builtin_amdgcn_perm(y[3], y[2], sel)};
        if (k * 64 + lane >= chunks) continue;
        if (STREAM) __builtin_nontemporal_store(o, dst + k * 64 + lane);
        else dst[k * 64 + lane] = o;
      }
    };
    if (there0) put(s.row(i), 0x05040100u);
    if (there1) put(s.row(i + 1), 0x07060302u);
  };
  for (int i = 0; s.row(i) < a.T; i += kRowsAhead) {
    win.move_to(i, lane);
#pragma unroll
    for (int k = 0; k < kRowsAhead; k += 2)
      if (s.row(i + k) < a.T) pair(i + k, buf[k], buf[k + 1]);
  }
}

// Three workgroups of four waves per compute unit, and no more waves than rows.  What it was tried on, us: reading 16384 x 12288
// at 3 bits (memory: 186), one row at a time, its slot waited for, 2 rows ahead 328 (314 with non-temporal stores); slots 64 at
// a time, 4 rows ahead 237; four waves on neighbouring rows 232; in runs over all groups 219; two rows at a time, which halves
// the writes to LDS, 221, and 8 rows ahead 207 (4.6 TB/s; two, three, four workgroups per compute unit 209 | 207 | 210).  Writing
// 8192 x 5120 at 4 bits (memory: 41) by workgroups per compute unit two, three, four, six 49 | 46 | 47 | 52; runs of 4 | 8 | 16 rows 48 | 46 | 47.
int32_t paged_launch(const PagedTensor& k, const PagedTensor& v, const int64_t* slots, int64_t T, const PagedGeom& g,
                     hipStream_t st, PagedLaunch* a, unsigned* grid) {
  int cus = 0;
  if (int32_t s = device_compute_units(st, &cus)) return s;
  const int segs = (g.d + kKvTile - 1) / kKvTile;
  const int64_t most = std::max<int64_t>(1, static_cast<int64_t>(cus) * 3 / (2 * segs));
  const int64_t rows = (T + most * 4 - 1) / (most * 4);           // of a wave
  const int run_shift = rows >= 2 ? 1 : 0;
  const int64_t groups = std::min<int64_t>(most, (T + (4 << run_shift) - 1) / (4 << run_shift));
  *a = PagedLaunch{{k, v}, slots, T, g, segs, static_cast<int32_t>(groups), run_shift};
  *grid = static_cast<unsigned>(groups) * 2 * segs;
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
  const bool stream = T * g.d * 2 > kKvStreamBytes;
  if (bits == 3) stream ? go(kv_dequant_paged_kernel<3, true>) : go(kv_dequant_paged_kernel<3, false>);
  else if (bits == 4) stream ? go(kv_dequant_paged_kernel<4, true>) : go(kv_dequant_paged_kernel<4, false>);
  else stream ? go(kv_dequant_paged_kernel<8, true>) : go(kv_dequant_paged_kernel<8, false>);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
