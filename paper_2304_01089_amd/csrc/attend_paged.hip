// Attention of one new token per sequence over the paged cache, on the codes.  With q'_j = scale q[src_j] s^K_j,
//   a_t = sum_j q'_j k_tj - sum_j q'_j z^K_j,   out_j = s^V_j (sum_t p_t v_tj / sum_t p_t - z^V_j),   p_t = exp(a_t - max a):
// the zero points of the keys add one number to every score of a head, which the softmax does not see (only lse does), and
// those of the values come off the weighted mean.
//
// A workgroup takes one query head of one sequence through all of its tokens, 256 at a time, a token per thread for the
// scores and a channel per thread for the sums.
#include <hip/hip_runtime.h>

#include "device_common.h"
#include "pack_formats.h"
#include "rptq_internal.h"

namespace rptq {

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;

template <int BITS, bool F32>
__global__ void __launch_bounds__(256) attend_paged_kernel(AttendArgs a) {
  constexpr int GB = 4 * BITS;                         // bytes of 32 codes
  __shared__ float qs[256], p[256], red[8];
  __shared__ double redd[4];
  __shared__ int64_t vrow[256];
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int h = blockIdx.x % a.n_q, b = blockIdx.x / a.n_q;
  const int kvh = h / (a.n_q / a.n_kv);
  const int page_size = 1 << a.g.page_shift;
  const int len = static_cast<int>(min<int64_t>(max(a.lens[b], 0), static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift));
  auto sum_all = [&](float v) {
    for (int m = 32; m; m >>= 1) v += __shfl_xor(v, m, kWave);
    __syncthreads();
    if (lane == 0) red[wave] = v;
    __syncthreads();
    return red[0] + red[1] + red[2] + red[3];
  };
  auto max_all = [&](float v) {
    for (int m = 32; m; m >>= 1) v = fmaxf(v, __shfl_xor(v, m, kWave));
    __syncthreads();
    if (lane == 0) red[wave] = v;
    __syncthreads();
    return fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3]));
  };
  double zterm = 0.0;
  if (tid < a.hd) {
    const KvPos kp = a.k_pos[kvh * a.hd + tid];
    const float x = __uint_as_float(static_cast<uint32_t>(a.q[b * a.ld_q + h * a.hd + (kp.src & (a.hd - 1))]) << 16);
    qs[tid] = x * kp.s * (a.scale * kLog2e);
    zterm = static_cast<double>(qs[tid]) * kp.z;
  }
  for (int m = 32; m; m >>= 1) zterm += __shfl_xor(zterm, m, kWave);
  if (lane == 0) redd[wave] = zterm;
  __syncthreads();
  zterm = redd[0] + redd[1] + redd[2] + redd[3];
  float m_run = -1e30f, l_run = 0.0f, acc = 0.0f;
  const int block = kvh * a.hd / kPageBlock, first = kvh * a.hd % kPageBlock;
  auto row_at = [&](int page, int blk, int r) {
    return (((static_cast<int64_t>(page) * (a.g.d / kPageBlock) + blk) << a.g.page_shift) + r) * (16 * BITS);
  };
  for (int t0 = 0; t0 < len; t0 += 256) {
    const int t = t0 + tid;
    const int page = t < len ? a.page_table[b * a.ld_pt + (t >> a.g.page_shift)] : -1;
    const bool here = page >= 0 && page < a.g.n_pages;
    float score = -1e30f;
    if (here) {
      score = 0.0f;
      for (int j0 = 0; j0 < a.hd; j0 += 32) {
        const int at = first + j0;
        const uint8_t* src = a.k_pages + row_at(page, block + at / kPageBlock, t & (page_size - 1)) + at % kPageBlock / 32 * GB;
        uint32_t w[GB / 4];
        int c[32];
        for (int k = 0; k < GB / 4; ++k) w[k] = reinterpret_cast<const uint32_t*>(src)[k];
        decode_group<BITS>(w, c);
#pragma unroll
        for (int j = 0; j < 32; ++j) score = fmaf(qs[j0 + j], static_cast<float>(c[j]), score);
      }
    }
    const float m_new = fmaxf(m_run, max_all(score));
    const float e = here ? __builtin_amdgcn_exp2f(score - m_new) : 0.0f;
    const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
    l_run = l_run * alpha + sum_all(e);
    p[tid] = e;
    vrow[tid] = here ? row_at(page, block, t & (page_size - 1)) : -1;
    __syncthreads();
    if (tid < a.hd) {
      const int at = first + tid;
      const int64_t off = static_cast<int64_t>(at / kPageBlock) * (static_cast<int64_t>(page_size) * 16 * BITS) + at % kPageBlock / 32 * GB;
      acc *= alpha;
      for (int i = 0; i < 256; ++i) {
        if (vrow[i] < 0) continue;
        uint32_t w[GB / 4];
        int c[32];
        for (int k = 0; k < GB / 4; ++k) w[k] = reinterpret_cast<const uint32_t*>(a.v_pages + vrow[i] + off)[k];
        decode_group<BITS>(w, c);
        int mine = 0;
#pragma unroll
        for (int j = 0; j < 32; ++j) mine = (at & 31) == j ? c[j] : mine;
        acc = fmaf(p[i], static_cast<float>(mine), acc);
      }
    }
    m_run = m_new;
    __syncthreads();
  }
  if (tid < a.hd) {
    const KvPos vp = a.v_pos[kvh * a.hd + tid];
    const float y = l_run != 0.0f ? vp.s * (acc / l_run - static_cast<float>(vp.z)) : 0.0f;
    const int64_t at = b * a.ld_out + h * a.hd + (vp.src & (a.hd - 1));
    if (F32) static_cast<float*>(a.out)[at] = y;
    else static_cast<__bf16*>(a.out)[at] = static_cast<__bf16>(y);
  }
  if (a.lse && tid == 0)
    a.lse[static_cast<int64_t>(b) * a.n_q + h] = l_run != 0.0f ? kLn2 * static_cast<float>(m_run + log2f(l_run) - zterm) : -__builtin_huge_valf();
}

size_t attend_workspace_bytes(int32_t B, int32_t n_q, int32_t n_kv, int32_t hd) { return 16; }

int32_t launch_attend_paged(const AttendArgs& a, int32_t bits, int32_t out_dtype, hipStream_t st) {
  if (a.B == 0) return RPTQ_OK;
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(a.B) * a.n_q), dim3(256), 0, st, a); };
  const bool f32 = out_dtype == RPTQ_DTYPE_F32;
  if (bits == 3) f32 ? go(attend_paged_kernel<3, true>) : go(attend_paged_kernel<3, false>);
  else if (bits == 4) f32 ? go(attend_paged_kernel<4, true>) : go(attend_paged_kernel<4, false>);
  else f32 ? go(attend_paged_kernel<8, true>) : go(attend_paged_kernel<8, false>);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
