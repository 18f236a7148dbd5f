// What every token of the paged cache got of the attention of a sequence's last queries, added up per key/value head:
//   weight[b, h, t] += sum over queries i and query heads g of h:  exp(a_git - lse_gi),
// a as in the attention itself (q' = scale log2(e) q s, minus the keys' zero points), lse the logarithm of the sum that it left.
// The keys' codes are read once more, and no value.
//
// Scores come from the int8 matrix cores as there: a query head of a query is four rows of digits, four of them a row tile, 64
// tokens a wave's tile.  A row tile's four belong to one key/value head where it has three pairs (query, head) or more; two pairs
// share a tile with another head's two, single ones with three other heads' (heads under 128 wide).  A lane adds up its tokens'
// weights over the row tiles in fp32 in their order, the four rows' sums come together by two exchanges, and each weight is read and
// written by one lane: no order of adding depends on anything but the call.
// What bounds it: memory with few queries; with many, the vector instructions that make weights of digits' sums.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_common.h"
#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kTileTokens = 4 * kTile;         // of a workgroup's four waves
constexpr int kSeenWorkgroups = 2048;          // as many parts as make this many workgroups, where there are tokens for them

// Row tiles whose digits lie in LDS at one time; more go through the tokens several times.
__host__ __device__ constexpr int held_tiles(int blocks) { return blocks == 2 ? 8 : 16; }

struct WeightPlan {
  int32_t group;                               // rows of a tile that belong to one key/value head: 1, 2 or 4
  int32_t set_tiles, tiles;                    // row tiles of a set of heads (4 / group of them), and all
  int32_t parts;                               // workgroups that share a sequence's tokens
};

struct QueryRow {
  float scale, off;                            // score = digits' sum * scale - off, in units of log2
  int32_t end, unused;                         // tokens that it sees
};

template <int BITS, int NB>
__global__ void __launch_bounds__(256, 2) attend_weights_kernel(WeightArgs a, WeightPlan plan) {
  constexpr int kShift = BITS == 8 ? 0 : (BITS == 4 ? 4 : 5);
  constexpr int kRow = 16 * BITS;                          // bytes of a token's row in a block
  constexpr int P = NB * kPageBlock;                       // positions of the unit
  constexpr int kDigitRow = P + 16;                        // (16 more: other banks)
  constexpr int kHeld = held_tiles(NB);
  __shared__ __align__(16) unsigned char q_dig[kHeld * 16 * kDigitRow];
  __shared__ __align__(16) QueryRow rows[kHeld * kRowHeads];
  const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = blockIdx.x, unit = blockIdx.y, b = blockIdx.z;
  const int64_t room = min(static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift, a.capacity);
  const int len = static_cast<int>(min(static_cast<int64_t>(max(a.lens[b], 0)), room));
  if (part * kTileTokens >= len) return;

  const int share = a.n_q / a.n_kv, pairs = share * a.queries;
  const int unit_heads = P / a.hd;                         // key/value heads
  const int hd_shift = __builtin_ctz(a.hd), set_heads = kRowHeads / plan.group;
  const int group_shift = plan.group >> 1;                 // (log2 of 1, 2, 4)
  const KvPos* kt = a.k_pos + unit * P;
  KvPos kp[2 * NB];
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) kp[i] = kt[i * 64 + lane];

  // ---- a wave's tiles: every parts-th run of 256 tokens, 64 of them each -----------------------------------------
  const int32_t* pt = a.page_table + b * a.ld_pt;
  const int last_page = (len - 1) >> a.g.page_shift, block_rows = 1 << a.g.page_shift;
  auto token_of = [&](int k) { return (part + k * plan.parts) * kTileTokens + wave * kTile; };
  const int first_token = token_of(0), step = plan.parts * kTileTokens;
  const int my_tiles = first_token < len ? (len - first_token + step - 1) / step : 0;
  // lane 4 i + r's 16 tokens (r: lane & 3) of tile k: their page's number, or -1
  auto page_of = [&](int k) {
    const int t = token_of(k) + (lane & 3) * 16;
    const int id = pt[min(t >> a.g.page_shift, last_page)];
    return t < len && id >= 0 && id < a.g.n_pages ? id : -1;
  };
  const uint32_t k_off = n16 * kRow + g4 * (4 * BITS);
  const int block_bytes = block_rows * kRow;
  auto load_tile = [&](int k, int id, uint32_t (&x)[4][NB][BITS]) {
    typedef unsigned u3v __attribute__((ext_vector_type(3)));
    typedef unsigned u4v __attribute__((ext_vector_type(4)));
    const int t = (token_of(k) + (lane & 3) * 16) & (block_rows - 1);
    const uint64_t at = ((static_cast<uint64_t>(max(id, 0)) * (a.g.d / kPageBlock) + unit * NB) * block_rows + t) * kRow;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint64_t row = static_cast<uint64_t>(__builtin_amdgcn_readlane(static_cast<uint32_t>(at >> 32), r)) << 32 |
                           __builtin_amdgcn_readlane(static_cast<uint32_t>(at), r);
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.k_pages) + row, 0,
                                                                            (NB - 1) * block_bytes + 16 * kRow, 0x00020000);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (BITS == 3) {
          const u3v v = __builtin_amdgcn_raw_buffer_load_b96(rsrc, k_off, nb * block_bytes, 0);
#pragma unroll
          for (int e = 0; e < 3; ++e) x[r][nb][e] = v[e];
        } else {
#pragma unroll
          for (int h = 0; h < BITS / 4; ++h) {
            const u4v v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, k_off + 16 * h, nb * block_bytes, 0);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[r][nb][4 * h + e] = v[e];
          }
        }
      }
    }
  };

  for (int tile0 = 0; tile0 < plan.tiles; tile0 += kHeld) {
    const int tile1 = min(tile0 + kHeld, plan.tiles);
    uint32_t kr[4][NB][BITS];
    int id = my_tiles > 0 ? page_of(0) : -1;
    int next_id = my_tiles > 1 ? page_of(1) : -1;
    if (my_tiles > 0) load_tile(0, id, kr);
    if (tile0 > 0) __syncthreads();                        // (the digits before have been read)

    // ---- queries to digits: a wave takes every fourth row ----------------------------------------------------------
    for (int i = wave; i < (tile1 - tile0) * kRowHeads; i += 4) {
      const int tile = tile0 + i / kRowHeads, g = i & (kRowHeads - 1);
      const int set = tile / plan.set_tiles, in_set = tile - set * plan.set_tiles;
      const int head = set * set_heads + (g >> group_shift);                   // of the unit
      const int pair = in_set * plan.group + (g & (plan.group - 1));
      const bool there = head < unit_heads && pair < pairs;
      const int query = there ? pair / share : 0, q_head = (unit * unit_heads + (there ? head : 0)) * share + (there ? pair - query * share : 0);
      const int64_t q_row = static_cast<int64_t>(b) * a.queries + query;
      const uint16_t* q = a.q + q_row * a.ld_q + q_head * a.hd;
      float x[2 * NB], top = 0.0f;
      bool bad = false;
      double z = 0.0;
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j) {
        const int pos = j * 64 + lane;
        const bool own = there && (NB == 2 || pos >> hd_shift == head);
        const float v = __uint_as_float(static_cast<uint32_t>(q[kp[j].src & (a.hd - 1)]) << 16) * kp[j].s * (a.scale * kLog2e);
        x[j] = own ? v : 0.0f;
        top = fmaxf(top, fabsf(x[j]));
        bad = bad || !(fabsf(x[j]) < __builtin_huge_valf());
        z += static_cast<double>(x[j]) * kp[j].z;
      }
      top = wave_max(top);
      z = wave_sum(z);
      const int e = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;         // top < 2^e
#pragma unroll
      for (int j = 0; j < 2 * NB; ++j) {
        const uint32_t d = digits(static_cast<int>(rintf(ldexpf(x[j], 30 - e))));
#pragma unroll
        for (int by = 0; by < 4; ++by) q_dig[(i * 4 + by) * kDigitRow + j * 64 + lane] = static_cast<unsigned char>(d >> (8 * by));
      }
      QueryRow row;
      row.scale = __ballot(bad) != 0 ? __builtin_nanf("") : ldexpf(1.0f, e - 30 - kShift);
      const float lse = a.lse[q_row * a.n_q + q_head];
      row.off = static_cast<float>(z + static_cast<double>(lse) * 1.4426950408889634074);
      row.end = there ? len - (a.queries - 1 - query) : 0;
      row.unused = 0;
      if (lane == 0) rows[i] = row;
    }
    __syncthreads();

    for (int k = 0; k < my_tiles; ++k) {
      const int token = token_of(k);
      const uint64_t here = __ballot(id >= 0);             // (bit r: the tile's r-th 16 tokens)
      uint32_t kw[4][NB][8];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) expand<BITS>(kr[r][nb], kw[r][nb]);
      id = next_id;
      if (k + 1 < my_tiles) load_tile(k + 1, id, kr);
      next_id = k + 2 < my_tiles ? page_of(k + 2) : -1;
      // lane (row g4, token n16 of every 16): tokens of the r-th 16 that there are, before the row's own end
      int first_of[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) first_of[r] = here >> r & 1 ? token + r * 16 + n16 : 0x7fffffff;

      for (int tile = tile0; tile < tile1;) {
        const int set = tile / plan.set_tiles, set_end = min((set + 1) * plan.set_tiles, tile1);
        const bool first = tile == set * plan.set_tiles;
        // what this lane will write of the set: 4 / group of its tokens, of head `head`
        const int head = set * set_heads + (g4 >> group_shift);
        const int64_t at = (static_cast<int64_t>(b) * a.n_kv + unit * unit_heads + head) * a.capacity;
        const int r0 = (g4 & (plan.group - 1)) * set_heads;
        float old[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const int t = token + (r0 + j) * 16 + n16;
          old[j] = 0.0f;
          if (j < set_heads && head < unit_heads && t < len && !(first && t >= len - a.fresh)) old[j] = a.weights[at + t];
        }
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        for (; tile < set_end; ++tile) {
          const int i = tile - tile0;
          const QueryRow row = rows[i * kRowHeads + g4];
          v4i c[4];
#pragma unroll
          for (int r = 0; r < 4; ++r) c[r] = v4i{0, 0, 0, 0};
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < 2; ++s) {
              const v4i q = *reinterpret_cast<const v4i*>(q_dig + (i * 16 + n16) * kDigitRow + nb * kPageBlock + g4 * 32 + s * 16);
#pragma unroll
              for (int r = 0; r < 4; ++r) {
                const v4i w = {static_cast<int>(kw[r][nb][4 * s]), static_cast<int>(kw[r][nb][4 * s + 1]), static_cast<int>(kw[r][nb][4 * s + 2]),
                               static_cast<int>(kw[r][nb][4 * s + 3])};
                c[r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q, w, c[r], 0, 0, 0);
              }
            }
#pragma unroll
          for (int r = 0; r < 4; ++r) {
            const float p = __builtin_amdgcn_exp2f(fmaf(undigit(c[r]), row.scale, -row.off));
            sum[r] += first_of[r] < row.end ? p : 0.0f;
          }
        }
        if (plan.group >= 2) {
#pragma unroll
          for (int r = 0; r < 4; ++r) sum[r] += __shfl_xor(sum[r], 16, kWave);
        }
        if (plan.group == 4) {
#pragma unroll
          for (int r = 0; r < 4; ++r) sum[r] += __shfl_xor(sum[r], 32, kWave);
        }
        if (head < unit_heads) {
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const int r = r0 + j, t = token + r * 16 + n16;
            if (j >= set_heads || t >= len) continue;
            const float mine = r == 0 ? sum[0] : (r == 1 ? sum[1] : (r == 2 ? sum[2] : sum[3]));
            a.weights[at + t] = old[j] + mine;
            if (first && t >= len - a.fresh) a.token_positions[at + t] = a.positions ? a.positions[b] - (len - 1 - t) : t;
          }
        }
      }
    }
  }
}

int32_t launch_attend_weights(const WeightArgs& a, int32_t bits, hipStream_t st) {
  if (a.B == 0) return RPTQ_OK;
  const int P = a.hd > kPageBlock ? a.hd : kPageBlock, units = a.n_kv * a.hd / P, unit_heads = P / a.hd;
  const int pairs = a.n_q / a.n_kv * a.queries;
  WeightPlan p;
  p.group = pairs >= 3 ? 4 : pairs;
  p.set_tiles = (pairs + p.group - 1) / p.group;
  p.tiles = p.set_tiles * ((unit_heads + kRowHeads / p.group - 1) / (kRowHeads / p.group));
  const int64_t most = std::min<int64_t>(static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift, a.capacity);
  const int64_t runs = (most + kTileTokens - 1) / kTileTokens, each = static_cast<int64_t>(a.B) * units;
  p.parts = static_cast<int32_t>(std::min<int64_t>(runs, std::max<int64_t>(1, (kSeenWorkgroups + each - 1) / each)));
  auto go = [&](auto kern) { hipLaunchKernelGGL(kern, dim3(p.parts, units, a.B), dim3(256), 0, st, a, p); };
  if (a.hd > kPageBlock) {
    if (bits == 3) go(attend_weights_kernel<3, 2>);
    else if (bits == 4) go(attend_weights_kernel<4, 2>);
    else go(attend_weights_kernel<8, 2>);
  } else {
    if (bits == 3) go(attend_weights_kernel<3, 1>);
    else if (bits == 4) go(attend_weights_kernel<4, 1>);
    else go(attend_weights_kernel<8, 1>);
  }
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
