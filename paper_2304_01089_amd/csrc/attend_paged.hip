// Attention of one new token per sequence over the paged cache, on the codes.  With q'_j = scale log2(e) q[src_j] s^K_j,
//   a_t = sum_j q'_j k_tj - sum_j q'_j z^K_j,   out_j = s^V_j (sum_t p_t v_tj / sum_t p_t - z^V_j),   p_t = 2^(a_t - max a):
// the zero points of the keys add one number to every score of a head, which the softmax does not see (only lse does), and
// those of the values come off the weighted mean.
//
// Both sums run on the int8 matrix cores, whose products are exact.  A query's q' and a tile's weights p are written in fixed
// point, 31 bits below the head's largest |q'| and 30 below the tile's largest weight, as four signed digits to the base 256; a
// digit is a row of the matrix product, so four heads fill its 16 rows (one query head on a key/value head uses four of them: rows
// cost nothing here, the product is bound by the bytes of the cache).  Codes are the other operand as they are stored, one shift
// and one mask per four of them.  The digits' sums meet again in one lane.  What is rounded: q', once per factor and to its fixed
// point; a score, as its digits' sums become fp32 (the upper half of them and the whole, a half step each); the difference from
// the largest score and its 2^x (the hardware's, one step); a weight to its fixed point, downwards (a tile loses less than 2^-24 of its
// sum of weights); the weighted codes of a tile of 64 tokens like a score, then as they are scaled and added in fp32, as the sums of
// weights are.
//
// A workgroup takes a part of one sequence for the heads that read one block of 128 positions (two for heads 256 wide), a
// wave every fourth tile of 64 tokens: scores, weights and weighted codes of a tile stay in registers, its weights cross 1 KiB of
// LDS to become an operand, keys and values of the next tile are requested before they are needed.  How sequences are cut in parts
// follows their lengths, which the kernel reads: parts of equal length over the whole batch, as many as fill the chip.  Parts
// leave (max, sum, weighted codes), a second kernel joins them; sequences of one part are finished at once.
//
// What bounds it.  One row tile: memory, 16 x 8192 tokens of 96 x 128 at 3 bits 196 us, 6.2 TB/s; 32 x 4096 of 40 x 128 at 4
// bits (half as many on average) 62 us, 5.6 TB/s.  More row tiles: vector instructions, 339 a tile of 4-bit codes with one and
// 841 with four, of which 56 a row tile bring the digits' sums of 8 x 4 outputs together (16 x 8192 of 8 x 128, half as many on
// average, by query heads 32, 64, 128: 20, 24, 35 us; memory 14).  With 128 the part kernel takes 29: compute units hold waves
// for 24 of them, vector instructions issue two thirds of that time, two waves per SIMD that wait for memory or each other a
// third of theirs.  Few tokens: a chain of latencies, 7 us for 257 tokens (lengths and page numbers 1.0, keys, values and
// queries 1.2, a tile 0.9, the waves together and the stores 0.7, the launch the rest), and 4 more for the second launch.
// Tried: waves that take a row tile each and share the tokens (16 x 8192 of 64 on 8 27 -> 33 us: four times the loads), a wave
// by itself per short sequence (512 x 60 19 -> 13 us, but 32 x 1000 9 -> 24: a wave takes 1.1 us a tile).
#include <hip/hip_runtime.h>

#include <algorithm>

#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

typedef int v4i __attribute__((ext_vector_type(4)));

constexpr float kLog2e = 1.4426950408889634f;
constexpr float kLn2 = 0.6931471805599453f;
constexpr float kNone = -3.402823466e38f;      // below every score
constexpr int kTile = 64;                      // tokens of a wave's tile
// Into how many parts the tokens of a batch are cut, us of 4-bit codes.  Few: two workgroups per compute unit of 256 (one | two: 16 x
// 8192 of 32 on 8 x 128 22.8 | 19.4, 2 x 20000 of 40 x 128 47.9 | 45.6, 3500 of 96 x 128 at 3 bits 17.3 | 14.9; but 8000 of 32 on 8 9.2 | 10.2;
// two | four: 16 x 8192 20.2 | 21.9, 32768 of 32 on 8 16.4 | 17.8), if
// a part is then of kLongTiles tiles at most (32 | 64 | 128: 2 x 20000 of 40 x 128 47.6 | 45.6 | 45.7, 64 x 8000 of 32 on 8 58.2 |
// 57.5 | 61.9).  Else many, so that a long sequence does not end alone: 2048 with one row tile, half as many where a workgroup
// takes longer (1024 | 2048: 64 x 16000 of 8 x 128 102 | 95, but 256 x 4000 of 64 on 8 120 | 146), and parts of kShortTiles at least
// (4 | 16 | 64: 128 x 1000 of 64 on 8, tables for more, 47.9 | 29.5 | 29.4, 32 x 4096 of 40 x 128 65.2 | 65.4 | 70.6).
// (Counts for the 256 compute units of a whole device; on a part of one they are right, and not measured.)
constexpr int kFewWorkgroups = 512, kManyWorkgroups = 2048;
constexpr int kLongTiles = 64;
constexpr int kShortTiles = 16;
constexpr int kLeastTiles = 2;                 // of a part of a sequence that is cut (1 | 2 | 4: 7 x 1531 of 16 on 2 x 256 12.3 | 10.9 | 11.5, at 8 bits 12.5 | 12.3 | 14.0)
constexpr int kWholeTiles = 48;                // of a sequence that is never cut at most (one such among short ones keeps the others waiting)
constexpr int kMostTiles = 1 << 23;            // of a sequence
constexpr int kJoinWorkgroups = 2048;          // that join parts, about: more take several heads each (512 x 1500 of 64 on 8 x 128: 136 | 127 us)
// Bytes of keys and values that a call can reach: beyond the last-level cache's size they are read past it.  (By the pool and the tables:
// the lengths are not known here, so a short batch on a large pool is read past the cache too and loses what the small sizes below show.)
// us without | with, the same cache again and again: 36 MB 14.6 | 16.2, 100 MB 23.7 | 24.9, 250 MB 47.5 | 50.4, 350 MB 71.6 | 64.2, 1.2 GB
// 227 | 204 (5.9 TB/s).
constexpr int64_t kStreamBytes = 256ll << 20;
constexpr int kRowHeads = 4;                   // query heads per 16 rows of the matrix product

// Row tiles that a workgroup's registers hold: heads 256 wide take twice as many per row tile.
__host__ __device__ constexpr int most_row_tiles(int blocks) { return blocks == 2 ? 2 : 4; }

__host__ __device__ constexpr int row_tiles(int heads) { return (heads + kRowHeads - 1) / kRowHeads; }

// How a call is laid out; from sizes alone, so that the workspace's is known before the lengths are.
struct AttendPlan {
  int32_t units;                               // blocks of positions (heads 256 wide: pairs of blocks)
  int32_t unit_heads;                          // query heads that read a unit
  int32_t chunks, chunk_heads;                 // these heads in equal groups, each a workgroup's
  int32_t least;                               // tiles of a part at least
  bool join;                                   // whether a sequence may be cut
  double per_few, per_many;                    // 1 / parts, a little more, where the tokens of the batch are cut in few, and in many
  int32_t slots;                               // parts that there may be: one more per sequence, from rounding up
};

// row_tiles_of_one: a workgroup's at most.
static AttendPlan attend_plan(int32_t B, int32_t n_q, int32_t n_kv, int32_t hd, int64_t most_tokens, int row_tiles_of_one) {
  AttendPlan p;
  const int unit = hd > kPageBlock ? hd : kPageBlock;
  p.units = n_kv * hd / unit;
  p.unit_heads = n_q / p.units;
  const int most = kRowHeads * row_tiles_of_one;
  p.chunks = (p.unit_heads + most - 1) / most;
  p.chunk_heads = (p.unit_heads + p.chunks - 1) / p.chunks;
  const int each = p.units * p.chunks;
  auto parts = [&](int workgroups) { return std::max(1, (workgroups + each - 1) / each); };
  // (rounding up adds half a part per sequence)
  p.per_few = 1.0 / parts(kFewWorkgroups - static_cast<int>(std::min<int64_t>(static_cast<int64_t>(B) * each / 2, kFewWorkgroups - 1))) * (1.0 + 0x1p-50);
  const int weight = unit / kPageBlock * row_tiles(p.chunk_heads), many = parts(weight == 1 ? kManyWorkgroups : kManyWorkgroups / 2);
  p.per_many = 1.0 / many * (1.0 + 0x1p-50);
  // A sequence that cannot be longer than `whole` tiles is not cut, which saves the second launch (4 us, as long as a wave
  // takes for three tiles of one block and one row tile) and the search for a workgroup's part.  The more sequences there are,
  // the less cutting gives: cut | not, us, at 10, 20, 32, 48 tiles of 128 wide heads and 4 bits: 48 workgroups 8.3 9.1 9.6 10.3
  // | 6.9 9.3 12.5 17.1, 144: 9.8 10.7 13.7 15.0 | 7.0 9.3 13.9 18.4, 256: 10.5 13.8 15.8 18.4 | 7.1 11.0 14.4 19.4, 512:
  // 12.7 16.6 20.7 26.4 | 10.1 13.6 17.9 23.9; 16 heads on 2 256 wide at 8 bits, 144: 25.6 32.6 43.5 48.2 | 18.7 26.8 36.9 50.9.
  const int alone = std::max(4, 16 / weight);
  const int whole = std::max(alone, static_cast<int>(std::min<int64_t>(static_cast<int64_t>(B) * each / 6, kWholeTiles)));
  p.join = most_tokens > whole * kTile;
  p.least = p.join ? kLeastTiles : whole;
  // (a sequence is cut in no more parts than its pages hold)
  const int64_t per_seq = (most_tokens + p.least * kTile - 1) / (p.least * kTile);
  p.slots = static_cast<int32_t>(std::min<int64_t>(many + static_cast<int64_t>(B), B * per_seq));   // (not cut: B)
  return p;
}

// Workspace: [slots][n_q] {max, sum, the keys' zero-point term}, [slots][n_q][hd] weighted codes, [B] {slot of the second part, parts}.
struct PartHead {
  float m, l, zterm, unused;
};

size_t attend_workspace_bytes(int32_t B, int32_t n_q, int32_t n_kv, int32_t hd) {
  int64_t slots = 0;
  for (int rt = 1; rt <= most_row_tiles(hd > kPageBlock ? 2 : 1); ++rt)
    slots = std::max<int64_t>(slots, attend_plan(B, n_q, n_kv, hd, INT64_C(1) << 30, rt).slots);
  const size_t rows = static_cast<size_t>(slots) * n_q;
  return rows * sizeof(PartHead) + rows * hd * sizeof(float) + ((static_cast<size_t>(B) + 1) / 2) * 16;
}

struct PartBuffers {
  PartHead* heads;
  float* acc;
  int2* where;
};

__device__ __forceinline__ PartBuffers part_buffers(const AttendArgs& a, const AttendPlan& p) {
  const size_t rows = static_cast<size_t>(p.slots) * a.n_q;
  PartBuffers b;
  b.heads = static_cast<PartHead*>(a.workspace);
  b.acc = reinterpret_cast<float*>(b.heads + rows);
  b.where = reinterpret_cast<int2*>(b.acc + rows * a.hd);
  return b;
}

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

// ---- which tokens a workgroup takes ------------------------------------------------------------------------
struct Part {
  int b, len, index, count, first_tile, end_tile;
};

// Every workgroup adds up all lengths where sequences may be cut: B sequences of up to 300 tokens, half as many on average, 32 on 8 x 128,
// tables for 300 | 32768 tokens, us: 512 26 | 39, 2048 95 | 222, 8192 367 | 1814.  (Tables no wider than the sequences are not cut.)
// The part that slot number `slot` holds; false: none.  A sequence's first part is in the slot of its own number, the others,
// sequence after sequence, in those behind.  own_len: the length of sequence number `slot`; first_len: lane i's is that of sequence
// i (or the last's), where sequences may be cut.
__device__ __forceinline__ bool find_part(const AttendArgs& a, const AttendPlan& p, int first_len, int own_len, int slot, int lane, Part* out) {
  const int cap = a.pages_per_seq << a.g.page_shift;
  auto clamped = [&](int len) { return min(max(len, 0), cap); };
  auto len_of = [&](int i) { return i < a.B ? clamped(a.lens[min(i, a.B - 1)]) : 0; };
  auto tiles_of = [](int n) { return (n + kTile - 1) / kTile; };
  auto parts_of = [](int tiles, int n) {       // rounded up; (24 bits, which is all there is: a division by float)
    return ((static_cast<uint32_t>(tiles) + n - 1) & 0xffffffu) / (static_cast<uint32_t>(n) & 0xffffffu);
  };
  if (!p.join) {
    out->b = slot;
    out->len = __builtin_amdgcn_readfirstlane(clamped(own_len));
    out->index = out->first_tile = 0;
    out->count = 1;
    out->end_tile = tiles_of(out->len);
    return true;
  }
  const int len0 = lane < a.B ? clamped(first_len) : 0;
  double total;
  if (a.B <= 64) {
    total = __builtin_amdgcn_readlane(wave_prefix(tiles_of(len0)), 63);
  } else {
    total = tiles_of(len0);
#pragma unroll 8
    for (int i = 64; i < a.B; i += 64) total += tiles_of(len_of(i + lane));
    total = wave_sum(total);
  }
  // tiles of a part: all tiles over the number of parts, rounded up; no more than a sequence of 2^29 tokens has
  auto each_of = [&](double per) { return __builtin_amdgcn_readfirstlane(static_cast<int>(fmin((total - 1.0) * per, kMostTiles - 1.0))) + 1; };
  const int few = each_of(p.per_few), most = max(p.least, few <= kLongTiles ? few : max(kShortTiles, each_of(p.per_many)));
  if (slot < a.B) {
    out->b = slot;
    out->len = __builtin_amdgcn_readfirstlane(clamped(own_len));
    out->index = 0;
    out->count = max<int>(1, parts_of(tiles_of(out->len), most));
  } else {
    // (a sequence of t tiles has at most (t - 1) / most further parts)
    const int rank = slot - a.B;
    if (__builtin_amdgcn_readfirstlane(total <= (rank + 1.0) * most)) return false;
    int before = 0, next_len = len0;
    for (int base = 0;; base += 64) {
      if (base >= a.B) return false;
      const int len = next_len;
      if (base + 64 < a.B) next_len = len_of(base + 64 + lane);
      const int n = max<int>(1, parts_of(tiles_of(len), most)) - 1;
      const int upto = wave_prefix(n);
      const uint64_t hit = __ballot(rank >= before + upto - n && rank < before + upto);
      if (hit != 0) {
        const int l = __builtin_ctzll(hit);
        out->b = base + l;
        out->len = __builtin_amdgcn_readlane(len, l);
        out->count = __builtin_amdgcn_readlane(n, l) + 1;
        out->index = rank - before - __builtin_amdgcn_readlane(upto, l) + out->count;
        break;
      }
      before += __builtin_amdgcn_readlane(upto, 63);
    }
  }
  const int tiles = tiles_of(out->len), each = parts_of(tiles, out->count);
  out->first_tile = out->index * each;
  out->end_tile = min(out->first_tile + each, tiles);
  return true;
}

__device__ __forceinline__ void store_out(const AttendArgs& a, bool f32, int64_t at, float y) {
  if (f32) static_cast<float*>(a.out)[at] = y;
  else static_cast<__bf16*>(a.out)[at] = static_cast<__bf16>(y);
}

// What a head's (max, sum) and weighted codes give: no tokens, zeros.
__device__ __forceinline__ float finish(float acc, float l, const KvPos& v) {
  return l != 0.0f ? v.s * (acc / l - static_cast<float>(v.z)) : 0.0f;
}
__device__ __forceinline__ float finish_lse(float m, float l, float zterm) {
  return l != 0.0f ? kLn2 * ((m - zterm) + __log2f(l)) : -__builtin_huge_valf();
}

// Waves per SIMD that the registers are shared out for: what is fastest, with few spills or none.  (three with two row tiles at 8 bits,
// us: 16 x 8192 of 64 on 8 x 128 37 | 47, 128 x 1000 of 40 on 8 39 | 51; three row tiles at 4 bits two | three, within 4 % of each other)
__host__ __device__ constexpr int part_waves(int bits, int blocks, int tiles) {
  if (blocks == 2) return bits == 8 && tiles > 1 ? 1 : 2;
  if (bits == 8) return tiles == 1 ? 3 : 2;
  return tiles == 1 ? 4 : (tiles < 4 ? 3 : 2);
}

// ---- the parts ---------------------------------------------------------------------------------------------
// NB: blocks of a unit; RT: row tiles (of four heads); STREAM: codes past the last-level cache
template <int BITS, int NB, int RT, bool STREAM>
__global__ void __launch_bounds__(256, part_waves(BITS, NB, RT)) attend_part_kernel(AttendArgs a, AttendPlan plan, bool f32) {
  constexpr int kShift = BITS == 8 ? 0 : (BITS == 4 ? 4 : 5);
  constexpr int kRow = 16 * BITS;                          // bytes of a token's row in a block
  constexpr int P = NB * kPageBlock;                       // positions of the unit
  constexpr int kQBytes = RT * 16 * P, kPBytes = 4 * RT * 1024;
  __shared__ __align__(16) unsigned char smem[kQBytes + kPBytes];
  __shared__ float merge[RT][4][kRowHeads][P + 16];       // [..][block][code 4e..][lane of 16]; (the 16 more: other banks)
  __shared__ float h_scale[RT * kRowHeads], h_z[RT * kRowHeads];
  __shared__ float w_m[4][RT * kRowHeads], w_l[4][RT * kRowHeads];
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int n16 = lane & 15, g4 = lane >> 4;

  // (unit, slot); with chunks, (8 chunks x 8 slots, unit, slot / 8), so that the chunks of a unit's heads, which read the
  // same pages, run next to each other on one XCD (workgroups are dealt to the eight in turn)
  int unit = blockIdx.x, slot = blockIdx.y, chunk = 0;
  if (plan.chunks > 1) {
    unit = blockIdx.y;
    slot = static_cast<int>(blockIdx.z) * 8 + static_cast<int>(blockIdx.x & 7);
    chunk = static_cast<int>(blockIdx.x >> 3);
    if (slot >= plan.slots) return;
  }

  // (requested first: they depend on nothing, and the lengths are waited for first)
  const int own_len = a.lens[min(slot, a.B - 1)];
  int first_len = 0;
  if (plan.join) first_len = a.lens[min(lane, a.B - 1)];
  // (one argument of every 64 bytes of them, so that all are fetched at once and not one after the other)
  asm volatile("" ::"s"(a.q), "s"(a.v_pos), "s"(a.page_table), "s"(a.workspace), "s"(plan.per_few));
  __builtin_amdgcn_sched_barrier(0);
  // (a sequence's first part: its first pages' numbers as well, before the lengths are there to say which of them count)
  int early_page = 0;
  if (slot < a.B)
    early_page = a.page_table[slot * a.ld_pt + min(((wave + 4 * (lane >> 2)) * kTile + (lane & 3) * 16) >> a.g.page_shift, a.pages_per_seq - 1)];
  const KvPos* kt = a.k_pos + unit * P;
  KvPos kp[2 * NB];
#pragma unroll
  for (int i = 0; i < 2 * NB; ++i) kp[i] = kt[i * 64 + lane];
  const KvPos vp = a.v_pos[unit * P + tid % P];
  Part part;
  if (!find_part(a, plan, first_len, own_len, slot, lane, &part)) return;

  // ---- rows of this wave's tiles: lane 4k + i holds where its k-th tile's i-th 16 tokens lie, in bytes to the unit's first
  // block, and whether their page is there (else 0, the first page); sixteen tiles at a time, the next requested ahead ------
  const int32_t* pt = a.page_table + part.b * a.ld_pt;
  const int my_tiles = max(0, (part.end_tile - part.first_tile - wave + 3) >> 2);
  auto token_of = [&](int k) { return (part.first_tile + wave + 4 * k) * kTile; };
  const int last_page = max(part.len - 1, 0) >> a.g.page_shift;
  const int block_rows = 1 << a.g.page_shift;
  auto tokens_of = [&](int k) { return token_of(k + (lane >> 2)) + (lane & 3) * 16; };
  auto checked = [&](int k, int id) { return tokens_of(k) < part.len && id >= 0 && id < a.g.n_pages ? id : -1; };        // -1: none
  auto page_of = [&](int k) { return checked(k, pt[min(tokens_of(k) >> a.g.page_shift, last_page)]); };
  struct Rows {
    uint32_t lo, hi;
    uint64_t there;
  };
  auto rows_of = [&](int k, int id) {
    const int t = tokens_of(k) & (block_rows - 1);
    const uint64_t row = (static_cast<uint64_t>(max(id, 0)) * (a.g.d / kPageBlock) + unit * NB) * block_rows + t;
    return Rows{static_cast<uint32_t>(row * kRow), static_cast<uint32_t>(row * kRow >> 32), __ballot(id >= 0)};
  };
  const int first_page = part.index == 0 ? checked(0, early_page) : (my_tiles > 0 ? page_of(0) : -1);
  int next_page = my_tiles > 16 ? page_of(16) : -1;

  const int share = a.n_q / a.n_kv;
  const int first_head = chunk * plan.chunk_heads;
  const int heads = min(plan.chunk_heads, plan.unit_heads - first_head);       // of this workgroup
  const int q_head = unit * plan.unit_heads + first_head;                      // the first of them
  // whether a position belongs to the key/value head that head hh of the workgroup reads
  const int hd_shift = __builtin_ctz(a.hd);
  auto own = [&](int hh, int pos) {
    return NB == 2 || static_cast<unsigned>(first_head + hh - (pos >> hd_shift) * share) < static_cast<unsigned>(share);
  };
  // (the queries, before the tiles: loads come back in order)
  uint16_t q_raw[RT][2 * NB];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i)
      q_raw[rt][i] = a.q[part.b * a.ld_q + (q_head + min(rt * kRowHeads + wave, heads - 1)) * a.hd + (kp[i].src & (a.hd - 1))];

  // K and V of a tile: lane (token n16, group g4) of every 16 tokens' keys; lane (group n16 / 4, token 4 g4 + n16 % 4) of the values
  const uint32_t k_off = n16 * kRow + g4 * (4 * BITS);
  const uint32_t v_off = (4 * g4 + (n16 & 3)) * kRow + (n16 >> 2) * (4 * BITS);
  Rows rows_at = rows_of(0, first_page);
  // (buffer loads: a descriptor of the rows in scalar registers, a lane's offset in one register)
  constexpr int kAux = STREAM ? 2 : 0;                     // (2: non-temporal)
  uint32_t kr[4][NB][BITS], vr[4][NB][BITS];
  const int block_bytes = block_rows * kRow;
  auto load_tile = [&](int k, const uint8_t* pages, uint32_t off, uint32_t (&x)[4][NB][BITS]) {
    typedef unsigned u3v __attribute__((ext_vector_type(3)));
    typedef unsigned u4v __attribute__((ext_vector_type(4)));
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int at = (k & 15) * 4 + r;
      const uint64_t row = static_cast<uint64_t>(__builtin_amdgcn_readlane(rows_at.hi, at)) << 32 | __builtin_amdgcn_readlane(rows_at.lo, at);
      const __amdgpu_buffer_rsrc_t rows = __builtin_amdgcn_make_buffer_rsrc(
          const_cast<uint8_t*>(pages) + row, 0, (NB - 1) * block_bytes + 16 * kRow, 0x00020000);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (BITS == 3) {
          const u3v v = __builtin_amdgcn_raw_buffer_load_b96(rows, off, nb * block_bytes, kAux);
#pragma unroll
          for (int e = 0; e < 3; ++e) x[r][nb][e] = v[e];
        } else {
#pragma unroll
          for (int h = 0; h < BITS / 4; ++h) {
            const u4v v = __builtin_amdgcn_raw_buffer_load_b128(rows, off + 16 * h, nb * block_bytes, kAux);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[r][nb][4 * h + e] = v[e];
          }
        }
      }
    }
  };
  if (my_tiles > 0) {
    load_tile(0, a.k_pages, k_off, kr);
    load_tile(0, a.v_pages, v_off, vr);
  }

  // ---- queries to digits: wave w takes head w of every row tile (all of them side by side: each is a chain of reductions) ----
  unsigned char* q_dig = smem;
  float qx[RT][2 * NB], q_top[RT];
  bool q_bad[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int hh = rt * kRowHeads + wave;
    q_top[rt] = 0.0f;
    q_bad[rt] = false;
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
      const float x = __uint_as_float(static_cast<uint32_t>(q_raw[rt][i]) << 16) * kp[i].s * (a.scale * kLog2e);
      qx[rt][i] = hh < heads && own(hh, i * 64 + lane) ? x : 0.0f;
      q_top[rt] = fmaxf(q_top[rt], fabsf(qx[rt][i]));
      q_bad[rt] = q_bad[rt] || !(fabsf(qx[rt][i]) < __builtin_huge_valf());
    }
  }
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) q_top[rt] = wave_max(q_top[rt]);
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int hh = rt * kRowHeads + wave, e = q_top[rt] > 0.0f ? __builtin_amdgcn_frexp_expf(q_top[rt]) : 0;          // q_top < 2^e
#pragma unroll
    for (int i = 0; i < 2 * NB; ++i) {
      const uint32_t d = digits(static_cast<int>(rintf(ldexpf(qx[rt][i], 30 - e))));
#pragma unroll
      for (int b = 0; b < 4; ++b) q_dig[(hh * 4 + b) * P + i * 64 + lane] = static_cast<unsigned char>(d >> (8 * b));
    }
    h_scale[hh] = __ballot(q_bad[rt]) != 0 ? __builtin_nanf("") : ldexpf(1.0f, e - 30 - kShift);          // (every lane the same)
  }
  // (what the zero points of the keys add to a head's scores: lse alone sees it)
  if (a.lse && part.index == 0) {
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      double z = 0.0;
#pragma unroll
      for (int i = 0; i < 2 * NB; ++i) z += static_cast<double>(qx[rt][i]) * kp[i].z;
      z = wave_sum(z);
      if (lane == 0) h_z[rt * kRowHeads + wave] = static_cast<float>(z);
    }
  }
  __syncthreads();
  // One row tile's operands stay in registers, more are read again for every tile.
  auto q_operand = [&](int rt, int nb, int s) {
    return *reinterpret_cast<const v4i*>(q_dig + (rt * 16 + n16) * P + nb * kPageBlock + g4 * 32 + s * 16);
  };
  constexpr bool kHeld = RT * NB == 1;
  v4i held[2];
  float scale[RT];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) scale[rt] = h_scale[rt * kRowHeads + g4];
  if (kHeld) held[0] = q_operand(0, 0, 0), held[1] = q_operand(0, 0, 1);

  // ---- the tiles -----------------------------------------------------------------------------------------------
  unsigned char* p_buf = smem + kQBytes + wave * (RT * 1024);
  const QuadSel sel = quad_sel(lane);
  float m_run[RT], l_run[RT], acc[RT][NB][8];
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    m_run[rt] = kNone;
    l_run[rt] = 0.0f;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 8; ++e) acc[rt][nb][e] = 0.0f;
  }
  for (int k = 0; k < my_tiles; ++k) {
    // (a score's upper bound: below every score where there is no token.  Its weight is then 0 by itself, but for a tile
    // without any, whose sums are taken 0 times)
    float most[4];
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const int left = rows_at.there >> ((k & 15) * 4 + r) & 1 ? part.len - token_of(k) - r * 16 : 0;
      most[r] = n16 < left ? __builtin_huge_valf() : kNone;
    }
    const bool more = k + 1 < my_tiles;
    auto next_keys = [&] {                                 // (once the keys' registers are free)
      if (more && ((k + 1) & 15) == 0) {
        rows_at = rows_of(k + 1, next_page);
        next_page = k + 17 < my_tiles ? page_of(k + 17) : -1;
      }
      if (more) load_tile(k + 1, a.k_pages, k_off, kr);
    };
    auto operand = [](const uint32_t (&w)[8], int s) {
      return v4i{static_cast<int>(w[4 * s]), static_cast<int>(w[4 * s + 1]), static_cast<int>(w[4 * s + 2]), static_cast<int>(w[4 * s + 3])};
    };
    // One or two row tiles: their sums side by side, a block of codes expanded at a time.  More: the tile's codes stay
    // expanded and the row tiles go one after the other, which is fewer registers.
    constexpr bool kWide = NB == 1 && RT > 2;
    v4i c[kWide ? 1 : RT][4];
    uint32_t kw[kWide ? 4 : 1][8];
    if constexpr (kWide) {
#pragma unroll
      for (int r = 0; r < 4; ++r) expand<BITS>(kr[r][0], kw[r]);
      next_keys();
    } else {
#pragma unroll
      for (int r = 0; r < 4; ++r) {
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) c[rt][r] = v4i{0, 0, 0, 0};
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          expand<BITS>(kr[r][nb], kw[0]);
#pragma unroll
          for (int s = 0; s < 2; ++s)
#pragma unroll
            for (int rt = 0; rt < RT; ++rt)
              c[rt][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(kHeld ? held[s] : q_operand(rt, nb, s), operand(kw[0], s), c[rt][r], 0, 0, 0);
        }
      }
      next_keys();
    }

    // weights of the tile, relative to its largest, as digits: lane (head g4, token n16 of every 16) -> operand lane (row n16, tokens of g4)
    float alpha[RT], beta[RT];
    v4i pa[RT];
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) {
      if constexpr (kWide) {
        const v4i q0 = q_operand(rt, 0, 0), q1 = q_operand(rt, 0, 1);
#pragma unroll
        for (int r = 0; r < 4; ++r) {
          c[0][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q0, operand(kw[r], 0), v4i{0, 0, 0, 0}, 0, 0, 0);
          c[0][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(q1, operand(kw[r], 1), c[0][r], 0, 0, 0);
        }
      }
      float s[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) s[r] = fminf(undigit(c[kWide ? 0 : rt][r]) * scale[rt], most[r]);
      const float top = row16_max(fmaxf(fmaxf(s[0], s[1]), fmaxf(s[2], s[3])));
      const float m_new = fmaxf(m_run[rt], top);
      alpha[rt] = __builtin_amdgcn_exp2f(m_run[rt] - m_new);
      beta[rt] = top > kNone ? __builtin_amdgcn_exp2f(top - m_new) : 0.0f;
      float sum = 0.0f;
      v4i d;
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        // (2^30 is a factor of the weight and no term of its exponent, which next to 30 would be rounded to 2^-20)
        const float e = __builtin_amdgcn_exp2f(s[r] - top);
        sum += e;
        d[r] = static_cast<int>(quad_transpose(digits(static_cast<int>(e * 0x1p30f)), sel));
      }
      l_run[rt] = fmaf(l_run[rt], alpha[rt], sum * beta[rt]);
      m_run[rt] = m_new;
      *reinterpret_cast<v4i*>(p_buf + rt * 1024 + (g4 * 4 + (n16 & 3)) * 64 + (n16 >> 2) * 16) = d;
      if (kWide) __builtin_amdgcn_sched_barrier(0);       // (one row tile after the other: the scheduler would keep all their sums)
    }
    wave_lds_fence();
#pragma unroll
    for (int rt = 0; rt < RT; ++rt) pa[rt] = *reinterpret_cast<const v4i*>(p_buf + rt * 1024 + n16 * 64 + g4 * 16);
    wave_lds_fence();

#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      uint32_t w[4][8];
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        uint32_t t[BITS];
#pragma unroll
        for (int i = 0; i < BITS; ++i) t[i] = quad_transpose(vr[r][nb][i], sel);
        expand<BITS>(t, w[r]);
      }
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const v4i vb = {static_cast<int>(w[0][e]), static_cast<int>(w[1][e]), static_cast<int>(w[2][e]), static_cast<int>(w[3][e])};
#pragma unroll
        for (int rt = 0; rt < RT; ++rt) {
          const v4i o = __builtin_amdgcn_mfma_i32_16x16x64_i8(pa[rt], vb, v4i{0, 0, 0, 0}, 0, 0, 0);
          acc[rt][nb][e] = fmaf(acc[rt][nb][e], alpha[rt], undigit(o) * beta[rt]);
        }
        // (about eight products under way at a time: the scheduler would take registers for all of them)
        if (RT > 1 && (e + 1) % (8 / RT) == 0)
#pragma unroll
          for (int rt = 0; rt < RT; ++rt) asm volatile("" : "+v"(acc[rt][nb][e]), "+v"(pa[rt]));
      }
    }
    if (more) load_tile(k + 1, a.v_pages, v_off, vr);
  }

  // ---- the waves' sums together ------------------------------------------------------------------------------------
  // (first the largest scores, so that every wave scales its own sums once)
#pragma unroll
  for (int rt = 0; rt < RT; ++rt)
    if (n16 == 0) w_m[wave][rt * kRowHeads + g4] = m_run[rt];
  __syncthreads();
#pragma unroll
  for (int rt = 0; rt < RT; ++rt) {
    const int hh = rt * kRowHeads + g4;
    const float m = fmaxf(fmaxf(w_m[0][hh], w_m[1][hh]), fmaxf(w_m[2][hh], w_m[3][hh]));
    const float f = __builtin_amdgcn_exp2f(m_run[rt] - m), l = row16_add(l_run[rt]) * f;
    if (n16 == 0) w_l[wave][hh] = l;
    const float fs = f * (0x1p-30f / (1 << kShift));
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 8; ++e) merge[rt][wave][g4][nb * kPageBlock + e * 16 + n16] = acc[rt][nb][e] * fs;
  }
  const PartBuffers buf = part_buffers(a, plan);
  const bool whole = part.count == 1;
  if (part.index == (whole ? 0 : 1) && unit == 0 && chunk == 0 && tid == 0) buf.where[part.b] = make_int2(slot, part.count);
  __syncthreads();
  const int pos = tid % P, at = NB == 2 ? pos : pos & (a.hd - 1);
  const int from = (pos & ~(kPageBlock - 1)) + (pos >> 2 & 7) * 16 + (pos >> 5 & 3) * 4 + (pos & 3);
  auto sum_of = [&](int hh) {
    const int rt = hh / kRowHeads, g = hh % kRowHeads;
    return (merge[rt][0][g][from] + merge[rt][1][g][from]) + (merge[rt][2][g][from] + merge[rt][3][g][from]);
  };
  auto weight_of = [&](int hh) { return (w_l[0][hh] + w_l[1][hh]) + (w_l[2][hh] + w_l[3][hh]); };
  auto top_of = [&](int hh) { return fmaxf(fmaxf(w_m[0][hh], w_m[1][hh]), fmaxf(w_m[2][hh], w_m[3][hh])); };
  if (whole) {
#pragma unroll 2
    for (int hh = tid / P; hh < heads; hh += 256 / P) {
      const float y = finish(sum_of(hh), weight_of(hh), vp);
      if (!own(hh, pos)) continue;
      store_out(a, f32, part.b * a.ld_out + static_cast<int64_t>(q_head + hh) * a.hd + (vp.src & (a.hd - 1)), y);
    }
    if (a.lse && tid < heads)
      a.lse[static_cast<int64_t>(part.b) * a.n_q + q_head + tid] = finish_lse(top_of(tid), weight_of(tid), h_z[tid]);
  } else {
    const int64_t row = static_cast<int64_t>(slot) * a.n_q + q_head;
    float* dst = buf.acc + row * a.hd + at;
#pragma unroll 4
    for (int hh = tid / P; hh < heads; hh += 256 / P) {
      const float sum = sum_of(hh);
      if (own(hh, pos)) dst[hh * a.hd] = sum;
    }
    if (tid < heads) buf.heads[row + tid] = PartHead{top_of(tid), weight_of(tid), h_z[tid], 0.0f};
  }
}

// ---- the parts of a sequence together: a workgroup per (sequence, `each` query heads) ------------------------------
// A thread takes four channels of every (1024 / hd)-th part.
template <bool SEVERAL>
__global__ void __launch_bounds__(256) attend_join_kernel(AttendArgs a, AttendPlan plan, bool f32, int each) {
  __shared__ float weight[256], red[8];
  __shared__ __align__(16) float merge[256 * 4];
  typedef float f4 __attribute__((ext_vector_type(4)));
  const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6;
  const int b = blockIdx.y;
  const PartBuffers buf = part_buffers(a, plan);
  const int2 where = buf.where[b];
  if (where.y <= 1) return;
  int h = SEVERAL ? blockIdx.x * each : blockIdx.x;
  const int end = SEVERAL ? min(h + each, a.n_q) : 0;
  do {
    auto row_of = [&](int part) { return static_cast<int64_t>(part == 0 ? b : where.x + part - 1) * a.n_q + h; };
    const int per = a.hd / 4, c = tid % per, p0 = tid / per, step = 256 / per;
    const f4* src = reinterpret_cast<const f4*>(buf.acc) + c;
    // (what a join of up to 8 * step parts reads is requested before anything is waited for, the second half only where there are so
    // many; four | eight, us in a recorded graph: 32768 tokens of 32 on 8 x 128, 64 parts, 14.5 | 13.4, 16000 of 128 on 8 15.0 | 15.0,
    // 16 x 8192 of 32 on 8 19.5 | 19.7)
    constexpr int kAhead = 8;
    f4 first[kAhead];
    auto request = [&](int k) { first[k] = src[row_of(min(p0 + k * step, where.y - 1)) * per]; };
#pragma unroll
    for (int k = 0; k < kAhead / 2; ++k) request(k);
    if (where.y > kAhead / 2 * step) {
#pragma unroll
      for (int k = kAhead / 2; k < kAhead; ++k) request(k);
    }
    const KvPos vp = a.v_pos[h / (a.n_q / a.n_kv) * a.hd + min(tid, a.hd - 1)];
    float m = kNone, l = 0.0f;
    f4 acc = {0.0f, 0.0f, 0.0f, 0.0f};
    for (int base = 0; base < where.y; base += 256) {
      const int n = min(256, where.y - base);
      const PartHead ph = buf.heads[row_of(base + min(tid, n - 1))];
      __syncthreads();                                          // (the weights of the 256 before have been read)
      const float top = wave_max(ph.m);
      if (lane == 0) red[wave] = top;
      __syncthreads();
      const float m_new = fmaxf(m, fmaxf(fmaxf(red[0], red[1]), fmaxf(red[2], red[3])));
      const float alpha = __builtin_amdgcn_exp2f(m - m_new), f = __builtin_amdgcn_exp2f(ph.m - m_new);
      weight[tid] = f;
      l = fmaf(l, alpha, tid < n ? ph.l * f : 0.0f);
#pragma unroll
      for (int j = 0; j < 4; ++j) acc[j] *= alpha;
      m = m_new;
      __syncthreads();
      int i = p0;
      if (base == 0) {
#pragma unroll
        for (int k = 0; k < kAhead; ++k, i += step)
          if (i < n) {
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[j] = fmaf(first[k][j], weight[i], acc[j]);
          }
      }
#pragma unroll 8
      for (; i < n; i += step) {
        const f4 v = src[row_of(base + i) * per];
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[j] = fmaf(v[j], weight[i], acc[j]);
      }
    }
    l = row16_add(l);
    auto row = [&](int at) { return __uint_as_float(__builtin_amdgcn_readlane(__float_as_uint(l), at)); };
    l = (row(0) + row(16)) + (row(32) + row(48));
    if (lane == 0) red[4 + wave] = l;
    *reinterpret_cast<f4*>(merge + tid * 4) = acc;              // [part % step][channel]
    __syncthreads();
    l = (red[4] + red[5]) + (red[6] + red[7]);
    if (tid < a.hd) {
      float sum = 0.0f;
      for (int i = 0; i < step; ++i) sum += merge[i * a.hd + tid];
      store_out(a, f32, b * a.ld_out + h * a.hd + (vp.src & (a.hd - 1)), finish(sum, l, vp));
      if (a.lse && tid == 0) a.lse[static_cast<int64_t>(b) * a.n_q + h] = finish_lse(m, l, buf.heads[row_of(0)].zterm);
    }
    if (SEVERAL) __syncthreads();                               // (the next head's is another use of the shared memory)
  } while (SEVERAL && ++h < end);
}

template <int BITS, int NB, int RT>
static void launch_parts(const AttendArgs& a, const AttendPlan& p, bool f32, bool stream, hipStream_t st) {
  // (8 bits take a cache line by two loads, where streaming costs 7 %, and more row tiles may be parts of a unit's heads, whose
  // workgroups read the same pages: 4 %)
  constexpr bool kMay = BITS < 8 && NB * RT <= 2;
  const dim3 grid = p.chunks == 1 ? dim3(p.units, p.slots) : dim3(8 * p.chunks, p.units, (p.slots + 7) / 8);
  const auto kernel = kMay && stream ? attend_part_kernel<BITS, NB, RT, kMay> : attend_part_kernel<BITS, NB, RT, false>;
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, st, a, p, f32);
}

template <int BITS>
static void launch_bits(const AttendArgs& a, const AttendPlan& p, bool f32, bool stream, hipStream_t st) {
  const int tiles = row_tiles(p.chunk_heads);
  if (a.hd > kPageBlock) {
    if (tiles <= 1) launch_parts<BITS, 2, 1>(a, p, f32, stream, st);
    else launch_parts<BITS, 2, 2>(a, p, f32, stream, st);
  } else {
    if (tiles <= 1) launch_parts<BITS, 1, 1>(a, p, f32, stream, st);
    else if (tiles == 2) launch_parts<BITS, 1, 2>(a, p, f32, stream, st);
    else if (tiles == 3) launch_parts<BITS, 1, 3>(a, p, f32, stream, st);
    else launch_parts<BITS, 1, 4>(a, p, f32, stream, st);
  }
}

int32_t launch_attend_paged(const AttendArgs& a, int32_t bits, int32_t out_dtype, hipStream_t st) {
  if (a.B == 0) return RPTQ_OK;
  const bool f32 = out_dtype == RPTQ_DTYPE_F32;
  const int64_t most_tokens = static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift;
  // As few row tiles in a workgroup, and the heads that read a unit over as many workgroups, as the chip has room for if all
  // pages are full: four tiles for each of 1024 waves (two at 8 bits, where reading the pages again costs more), and no more than 1024
  // workgroups (512 of heads 256 wide) if every sequence is short.  us with most row tiles | with this: 9 x 3 tokens of 28 heads on 4 x 64
  // 8.1 | 4.7, 3 x 441 of 154 on 22 x 64 11.9 | 7.7, 2 x 13815 of 20 on 4 x 64 14.5 | 12.0, 16000 of 128 on 8 x 128 18.3 | 15.6, 7 x 1531 of
  // 16 on 2 x 256 at 8 bits 12.7 | 11.5; but beyond the room 16 x 8192 of 128 on 8 x 128 35 | 38, at 8 bits 44 | 54, 8 x 2000 of 64 on 8 at 8
  // bits 16.5 | 18.1, 32 x 15 of 144 on 48 x 32 8.4 | 8.7, 59 x 7 of 40 on 5 x 256 9.4 | 10.9.
  const int blocks = a.hd > kPageBlock ? 2 : 1;
  const int64_t tiles = (most_tokens + kTile - 1) / kTile * a.B, room = bits == 8 && blocks == 1 ? 2048 : 4096;
  AttendPlan p;
  for (int rt = 1; rt <= most_row_tiles(blocks); ++rt) {
    p = attend_plan(a.B, a.n_q, a.n_kv, a.hd, most_tokens, rt);
    const int64_t each = static_cast<int64_t>(p.units) * p.chunks;
    if (tiles * each <= room && a.B * each <= 1024 / blocks) break;
  }
  const int64_t pages = std::min<int64_t>(a.g.n_pages, static_cast<int64_t>(a.B) * a.pages_per_seq);
  const bool stream = pages * 2 * (static_cast<int64_t>(a.g.d) * bits / 8 << a.g.page_shift) > kStreamBytes;
  if (bits == 3) launch_bits<3>(a, p, f32, stream, st);
  else if (bits == 4) launch_bits<4>(a, p, f32, stream, st);
  else launch_bits<8>(a, p, f32, stream, st);
  RPTQ_HIP(hipGetLastError());
  if (!p.join) return RPTQ_OK;
  const int each = std::max(1, std::min(a.n_q, a.B * a.n_q / kJoinWorkgroups));
  const auto join = each > 1 ? attend_join_kernel<true> : attend_join_kernel<false>;
  hipLaunchKernelGGL(join, dim3((a.n_q + each - 1) / each, a.B), dim3(256), 0, st, a, p, f32, each);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
