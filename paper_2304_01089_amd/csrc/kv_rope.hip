// A serving step's queries, keys and values in one launch: queries rotated by their positions (rope.hip's workgroups), keys
// rotated in fp32 and quantized into the pages without having been bf16 in between, values quantized as by kv_paged.hip.
//
// Keys and values go as there: a wave has 1024 channels of a row, moves them to cluster order through a piece of LDS of its own,
// and has the constants of its 16 positions in registers.  A lane loads two pieces of eight channels that rotate together (half
// style: eight and their partners; interleaved: sixteen side by side), takes the eight cosines and sines from LDS, where the
// wave has put the row's, one pair per lane and once for the wave's heads, and writes fp32.
// What bounds it: memory, as without the rotation: 8192 tokens of 40 heads of 128, queries included, take 82.7 us for 378 MB at 4 bits,
// 4.6 TB/s.  One token: 3.9 us, a launch and a chain of dependent loads (slot and table, rows, positions); the host takes 4.8.
// (150 registers, three workgroups per compute unit; held to four it spills: 163 us.)
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "kv_common.h"
#include "kv_paged_common.h"
#include "rope_common.h"
#include "rptq_internal.h"

namespace rptq {

struct RopeQuantLaunch {
  PagedLaunch kv;
  RopeLaunch q;                                      // (the launch's last q.groups workgroups are the queries'; first 88.6 | last 82.7 us, 8192 x 40 x 128 at 4 bits)
  const int32_t* positions;
  const double* freqs;
  double amplitude;
  int32_t rot, hd_shift;
};

constexpr int kRowBytes = kKvTile * 4 + 1024;        // a wave's row in fp32, the cosines and sines of up to 128 pairs
constexpr int kRqLds = kWave * kLaneTab + 4 * kRowBytes;
static_assert(kRqLds >= 2 * kRopePairs * 4, "the queries' cosines lie there too");

template <int BITS, bool HALF>
__global__ void __launch_bounds__(256) rope_quant_paged_kernel(RopeQuantLaunch l) {
  constexpr int kQMin = -(1 << (BITS - 1));
  constexpr float kUMax = static_cast<float>((1 << BITS) - 1);
  __shared__ __align__(16) unsigned char smem[kRqLds];
  const unsigned first_q = gridDim.x - static_cast<unsigned>(l.q.groups);
  if (blockIdx.x >= first_q) {
    rope_rows<8, HALF, __bf16, __bf16>(l.q, blockIdx.x - first_q, reinterpret_cast<float*>(smem));
    return;
  }
  const PagedLaunch& a = l.kv;
  unsigned char* tab = smem;
  const int lane = threadIdx.x & 63;
  unsigned char* my = smem + kWave * kLaneTab + (threadIdx.x >> 6) * kRowBytes;
  const PagedShare s = paged_share(a, blockIdx.x);
  const PagedTensor& t = a.t[s.values];
  // the lane's two pieces of a row: the pair numbers of both are 8 i .. 8 i + 7
  const int per_head = 1 << (l.hd_shift - 4), i16 = lane & (per_head - 1), head_ch = (lane >> (l.hd_shift - 4)) << l.hd_shift;
  const bool turned = !s.values && i16 * 16 < l.rot;
  int at0 = head_ch + i16 * 16, at1 = at0 + 8;
  if (HALF && turned) at0 = head_ch + i16 * 8, at1 = at0 + l.rot / 2;
  const bool lane_ok = lane * kKvLaneCodes < s.n_here;         // (the tile's channels and its positions end at the same lane)
  const int from0 = lane_ok ? at0 : 0, from1 = lane_ok ? at1 : 0;
  auto row_ptr = [&](int64_t r) { return t.x + min(r, a.T - 1) * t.ld + s.base_ch; };
  auto load = [&](int64_t r, int at) { return *reinterpret_cast<const uint4*>(row_ptr(r) + at); };
  uint4 cur0 = load(s.row(0), from0), cur1 = load(s.row(0), from1);
  uint4 nxt0 = load(s.row(1), from0), nxt1 = load(s.row(1), from1);
  SlotWindow<BITS> win(a, s, lane);
  // positions of 64 of the wave's rows, a lane one of them, the next 64 requested ahead
  auto position_at = [&](int i) { return l.positions[min(s.row(i), a.T - 1)]; };
  int pos_here = position_at(lane), pos_next = position_at(64 + lane);
  const int half = l.rot / 2;
  const double f0 = l.freqs[min(lane, half - 1)], f1 = l.freqs[min(lane + 64, half - 1)];
  paged_table(t, s, tab);
  __syncthreads();
  uint32_t src[kKvLaneCodes];
  float inv_s[kKvLaneCodes], zbf[kKvLaneCodes];
#pragma unroll
  for (int e = 0; e < kKvLaneCodes; ++e) {
    const int lp = kv_local_pos<BITS>(lane, e);
    const KvPos kp = *reinterpret_cast<const KvPos*>(tab + lp * 16 + lp / kKvLaneCodes * 16);
    src[e] = static_cast<uint32_t>(kp.src & (kKvTile - 1)) * 4u;
    inv_s[e] = kp.inv_s;
    zbf[e] = static_cast<float>(kp.z - kQMin);
  }
  const int64_t lane_at = paged_lane<BITS>(a.g, s.base_ch / kPageBlock + (lane >> 3), lane);
  float* row = reinterpret_cast<float*>(my);
  float *cos_t = row + kKvTile, *sin_t = cos_t + 128;
  for (int i = 0; s.row(i) < a.T; ++i) {
    if (i - win.from >= 64) {
      pos_here = pos_next;
      pos_next = position_at(i + 64 + lane);
    }
    win.move_to(i, lane);
    const int64_t place = win.place(i);
    float p[8], q[8];
    const uint32_t w0[4] = {cur0.x, cur0.y, cur0.z, cur0.w}, w1[4] = {cur1.x, cur1.y, cur1.z, cur1.w};
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      p[2 * e] = bf16_lo(w0[e]);
      p[2 * e + 1] = bf16_hi(w0[e]);
      q[2 * e] = bf16_lo(w1[e]);
      q[2 * e + 1] = bf16_hi(w1[e]);
    }
    cur0 = nxt0;
    cur1 = nxt1;
    nxt0 = load(s.row(i + 2), from0);
    nxt1 = load(s.row(i + 2), from1);
    if (!s.values) {
      const double pos = static_cast<double>(__builtin_amdgcn_readlane(pos_here, i & 63));
      if (lane < half) {
        const float2 c = rope_turn(pos * f0, l.amplitude);
        cos_t[lane] = c.x;
        sin_t[lane] = c.y;
      }
      if (lane + 64 < half) {
        const float2 c = rope_turn(pos * f1, l.amplitude);
        cos_t[lane + 64] = c.x;
        sin_t[lane + 64] = c.y;
      }
      wave_lds_fence();
      if (turned) {
        float c[8], sn[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          c[e] = cos_t[i16 * 8 + e];
          sn[e] = sin_t[i16 * 8 + e];
        }
        if constexpr (HALF) {
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float u = rope_first(p[e], q[e], c[e], sn[e]);
            q[e] = rope_second(p[e], q[e], c[e], sn[e]);
            p[e] = u;
          }
        } else {
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float u = rope_first(p[2 * e], p[2 * e + 1], c[e], sn[e]);
            p[2 * e + 1] = rope_second(p[2 * e], p[2 * e + 1], c[e], sn[e]);
            p[2 * e] = u;
            const float v = rope_first(q[2 * e], q[2 * e + 1], c[e + 4], sn[e + 4]);
            q[2 * e + 1] = rope_second(q[2 * e], q[2 * e + 1], c[e + 4], sn[e + 4]);
            q[2 * e] = v;
          }
        }
      }
    }
#pragma unroll
    for (int e = 0; e < 8; e += 4) {
      *reinterpret_cast<float4*>(row + at0 + e) = make_float4(p[e], p[e + 1], p[e + 2], p[e + 3]);
      *reinterpret_cast<float4*>(row + at1 + e) = make_float4(q[e], q[e + 1], q[e + 2], q[e + 3]);
    }
    wave_lds_fence();
    uint32_t D[4] = {0u, 0u, 0u, 0u};                // biased codes, one byte each
#pragma unroll
    for (int e = 0; e < kKvLaneCodes; ++e) {
      const float r = __fmul_rn(*reinterpret_cast<const float*>(my + src[e]), inv_s[e]);
      float b = __fadd_rn(rintf(r), zbf[e]);         // round, then add the zero point (biased by -qmin)
      if (BITS < 8) b = fminf(b, kUMax);             // upper clamp; the conversion saturates at 0 and 255
      D[e / 4] = __builtin_amdgcn_cvt_pk_u8_f32(b, e & 3, D[e / 4]);
    }
    wave_lds_fence();
    kv_store_codes<BITS>(t.pages + max(place, INT64_C(0)) + lane_at, lane, lane_ok && place >= 0, D[0], D[1], D[2], D[3]);
  }
}

int32_t launch_rope_quant_paged(const RopeArgs* q, const RopeArgs& k, const PagedTensor& kt, const PagedTensor& vt, const int64_t* slots,
                                const PagedGeom& g, int32_t bits, hipStream_t st) {
  if (k.T == 0) return RPTQ_OK;
  RopeQuantLaunch l;
  l.q.groups = 0;
  l.amplitude = k.amplitude;
  l.freqs = k.freqs;
  l.rot = k.rot;
  l.hd_shift = __builtin_ctz(static_cast<unsigned>(k.hd));
  int64_t most = k.T;                                // (rows of a launch: keys and values need no more workgroups for more rows)
  if (q != nullptr) most = std::min(most, plan_rope(*q, 8, q->x == q->y && q->ld_x == q->ld_y, &l.q));
  for (int64_t first = 0; first < k.T; first += most) {
    const int64_t rows = std::min(most, k.T - first);
    PagedTensor kp = kt, vp = vt;
    kp.x += first * kt.ld;
    vp.x += first * vt.ld;
    unsigned grid = 0;
    if (int32_t s = paged_launch(kp, vp, slots + first, rows, g, st, &l.kv, &grid)) return s;
    if (q != nullptr) rope_part(*q, first, rows, &l.q);
    l.positions = k.positions + first;
    auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(l.q.groups + grid), dim3(256), 0, st, l); };
    const bool half = k.interleaved == 0;
    if (bits == 3) half ? go(rope_quant_paged_kernel<3, true>) : go(rope_quant_paged_kernel<3, false>);
    else if (bits == 4) half ? go(rope_quant_paged_kernel<4, true>) : go(rope_quant_paged_kernel<4, false>);
    else half ? go(rope_quant_paged_kernel<8, true>) : go(rope_quant_paged_kernel<8, false>);
    RPTQ_HIP(hipGetLastError());
  }
  return RPTQ_OK;
}

}  // namespace rptq
