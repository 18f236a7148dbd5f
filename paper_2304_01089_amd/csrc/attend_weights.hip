// What every token of the paged cache got of the attention of a sequence's last queries, added up per key/value head:
//   weight[b, h, t] += sum over queries i and query heads g of h:  exp(a_git - lse_gi),
// a as in the attention itself (q' = scale log2(e) q s, minus the keys' zero points), lse the logarithm of the sum that it left.
// The keys' codes are read once more, and no value.
//
// Scores come from the int8 matrix cores as there: a query head of a query is four rows of digits to the base 256, four of them a row
// tile, 64 tokens a wave's tile, 256 a workgroup's.  q' and the zero points' term are formed in 64 bits up to the fixed point of
// 30 bits below the head's largest |q'|; sums of digits are exact; a weight is rounded as its upper digits' sum becomes fp32 and
// meets lse, as the lower ones' comes to it, by 2^x and by the sum over pairs (6e-8 to 6e-7 of the weights in all, in long windows too: kPasses).
// A row tile's four belong to one key/value head where it has three pairs (query, head) or more; two pairs
// share a tile with another head's two, single ones with three other heads' (heads under 128 wide).  A lane adds up its tokens'
// weights over the row tiles in fp32 in their order, the four rows' sums come together by two exchanges, and each weight is read and
// written by one lane: no order of adding depends on anything but the call.
//
// Up to kFewTiles row tiles each wave makes one tile's digits itself: queries are requested with the first loads, in their own order,
// and gathered in LDS (from memory, behind the positions' records, took 1 x 257 tokens a quarter of a microsecond more).  More are made once
// by a launch of their own, into the workspace, instead of by each of a sequence's workgroups (a fifth off 5 x 8191 tokens, 32 queries).
// What bounds it: with few queries memory, and the start of every workgroup (length, page number, codes, one after the other, while
// its digits are made): 32 sequences of up to 4096 tokens, 40 heads of 128 at 4 bits take 43.7 us for 195 MB, 4.5 TB/s; one short
// sequence 5, of which a launch is 1.8.  With many queries waits: 5 x 8191 tokens, 32 on 8 heads, 32 queries take 23.4 us for 3.4 GFLOP, digits
// 4 of them.  Of the 19 of this kernel vector instructions (about seven and an exponential for a weight) fill 7 on every SIMD and matrix
// instructions 3.4 beside them; 1.4 waves are there on average, and wait for a third of their time: row tiles go through LDS in two passes,
// each with its digits, keys and weights requested anew behind a barrier, and a tile's operands are read from LDS as they are used.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attend_common.h"
#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kTileTokens = 4 * kTile;         // of a workgroup's four waves
// As many parts as make this many workgroups, where there are tokens for them (1024 | 2048 | 5000: 32 x 4096 of 40 heads 47.3 | 43.7 | 44.8 us,
// 16 x 8192 of 40 at 3 bits 72.5 | 63.2 | 63.0, 5 x 8191 of 32 on 8 with 32 queries 25.7 | 23.4 | 23.3, 16 x 4096 of 12 14.0 | 14.5 | 15.4, of 32 heads of
// 32 17.2 | 19.8 | 19.8).
constexpr int kSeenWorkgroups = 2048;

// Keys of larger caches, values included, are read past the last-level cache, at 3 and 4 bits (an ordinary | such a load: 32 x 4096 of 40
// heads 46.2 | 43.7 us, 16 x 8192 at 3 bits 67.2 | 63.2; a smaller cache, 16 x 4096 of 12, 14.5 | 15.7).
constexpr int64_t kStreamBytes = INT64_C(256) << 20;
constexpr int kFewTiles = 4;                   // row tiles of which each wave of a workgroup makes one
// Row tiles that a wave works on side by side (1 | 2 | 4: 5 x 8191, 32 queries, 25.1 | 23.4 | 35.3 us, 16 x 2048 of 32 heads of 32, 8 queries,
// 24.9 | 24.4 | 28.1, 8 x 4096 of 12 of 64, 16 queries, 8 bits, 16.0 | 18.5 | 18.4).
constexpr int kSide = 2;

// Row tiles whose digits lie in LDS at one time; more go through the tokens several times (16 | 32, and two workgroups per compute
// unit instead of three: 5 x 8191, 32 queries, 23.4 | 29.8 us).
__host__ __device__ constexpr int held_tiles(int blocks) { return blocks == 2 ? 8 : 16; }

// A token's weight is rounded to fp32 once for every time that its head's row tiles go through LDS.  In windows of more such passes (half a step
// each, 1.4e-6 at most) what that loses is kept in LDS and added at the end; a workgroup goes through all row tiles with so many token
// tiles of a wave before it turns to the next ones.  (Without | with it, 16384 queries alike, 32 heads on 4 of 32: off by 2.6e-5 | 1.5e-7,
// 48.7 | 52.5 ms; 32 on 8 of 128: 1.0e-5 | 1.7e-7, 5.45 | 5.77 ms.)
constexpr int kPasses = 24;
__host__ __device__ constexpr int carried_tiles(int heads) { return 8 / heads; }

struct WeightPlan {
  int32_t group;                               // rows of a tile that belong to one key/value head: 1, 2 or 4
  int32_t set_tiles, tiles;                    // row tiles of a set of heads (4 / group of them), and all
  int32_t parts;                               // workgroups that share a sequence's tokens
  int32_t share;                               // query heads on a key/value head
  double per_share, per_set;                   // 1 / share and 1 / set_tiles, a little more
};

// A weight: 2^(high * (digits 2, 3) - off + low * (digits 0, 1)) * rest.  The upper digits meet `off` first (what is left is small, and
// rounded as such); rest is 2 to what `off` lost as it became fp32 (with lse about 16, 10^-6 of every weight).
struct QueryRow {
  float low, high, off, rest;
};
struct TileRows {
  QueryRow row[kRowHeads];
  int32_t end[kRowHeads];                      // tokens that the query sees
};

typedef int i4v __attribute__((ext_vector_type(4)));

// Queries to digits: a wave makes row tile number `tile` of a unit's, 16 lanes a row, a lane eight positions of every block.
template <int BITS, int NB, int HEADS>
struct QueryDigits {
  static constexpr int kShift = BITS == 8 ? 0 : (BITS == 4 ? 4 : 5);
  static constexpr int P = NB * kPageBlock, kHd = P / HEADS;
  const WeightArgs& a;
  const WeightPlan& plan;
  static constexpr int kRaw = kHd * 2 + 16;                // bytes of a query in its own order, and 16 (banks)
  static constexpr int kScratch = kRowHeads * kRaw;        // of a wave
  int b, unit, group, g4, n16;
  i4v kp[NB][8];                                           // the lane's positions' records
  struct Query {
    int back;                                              // newer queries of the sequence; -1: no query
    bool own;                                              // whether the lane's positions are its head's
    float lse;
    i4v raw[NB];                                           // channels 8 n16 .. of every 128
  };
  // (in the queries' own order: nothing of it waits for the positions' records)
  __device__ __forceinline__ Query request(int tile) const {
    // (pairs and tiles are below 2^31, a quotient's fraction is a multiple of its divisor's inverse or 0: 2^-50 of it does not reach the next number)
    auto quotient = [](int n, double per) { return static_cast<int>(n * per); };
    Query r;
    const int set = HEADS == 1 ? 0 : quotient(tile, plan.per_set), in_set = tile - set * plan.set_tiles;
    const int head = set * (kRowHeads / group) + (g4 >> (group >> 1));         // of the unit
    const int pair = in_set * group + (g4 & (group - 1));
    const bool there = head < HEADS && pair < plan.share * a.queries;
    const int query = there ? quotient(pair, plan.per_share) : 0;
    const int q_head = (unit * HEADS + (there ? head : 0)) * plan.share + (there ? pair - query * plan.share : 0);
    const int64_t q_row = static_cast<int64_t>(b) * a.queries + query;
    const uint16_t* q = a.q + q_row * a.ld_q + q_head * kHd;
    r.lse = a.lse[q_row * a.n_q + q_head];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) r.raw[nb] = *reinterpret_cast<const i4v*>(q + nb * kPageBlock + (n16 & (kHd / 8 - 1)) * 8);
    r.back = there ? a.queries - 1 - query : -1;
    r.own = there && (NB == 2 || n16 * 8 / kHd == head);
    return r;
  }
  // scratch: kScratch bytes of LDS, `to` may be the same;  to: the tile's 16 rows, `stride` bytes apart
  __device__ __forceinline__ void make(const Query& now, int len, unsigned char* scratch, unsigned char* to, int stride, TileRows* rows) const {
    unsigned char* mine = scratch + g4 * kRaw;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) *reinterpret_cast<i4v*>(mine + nb * (2 * kPageBlock) + (n16 & (kHd / 8 - 1)) * 16) = now.raw[nb];
    wave_lds_fence();
    // (in 64 bits up to the fixed point: an error of 2^-24 of q' would be one of score / 2^24 in a score's logarithm, and zero points far
    // from the codes make scores large)
    const double to_log2 = static_cast<double>(a.scale) * 1.4426950408889634074;
    double x[NB][8], zterm = 0.0;
    float top = 0.0f;
    bool bad = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const double v = static_cast<double>(__uint_as_float(static_cast<uint32_t>(*reinterpret_cast<const uint16_t*>(mine + (kp[nb][e][0] & (kHd - 1)) * 2)) << 16)) * static_cast<double>(__int_as_float(kp[nb][e][2])) * to_log2;
        x[nb][e] = now.own ? v : 0.0;
        const float size = fabsf(static_cast<float>(x[nb][e]));
        top = fmaxf(top, size);
        bad = bad || !(size < __builtin_huge_valf());
        zterm = fma(x[nb][e], static_cast<double>(kp[nb][e][3]), zterm);
      }
    wave_lds_fence();                                      // (digits may take the queries' place)
    top = row16_max(top);
    zterm = row16_sum(zterm);
    const int ex = top > 0.0f ? __builtin_amdgcn_frexp_expf(top) : 0;          // top < 2^ex
    const double to_fixed = ldexp(1.0, 30 - ex);
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      uint32_t d[8], plane[4][2];
#pragma unroll
      for (int e = 0; e < 8; ++e) d[e] = digits(static_cast<int>(rint(x[nb][e] * to_fixed)));
#pragma unroll
      for (int f = 0; f < 2; ++f) {                        // (four numbers' bytes to four planes)
        const uint32_t l01 = __builtin_amdgcn_perm(d[4 * f + 1], d[4 * f], 0x05010400u), h01 = __builtin_amdgcn_perm(d[4 * f + 1], d[4 * f], 0x07030602u);
        const uint32_t l23 = __builtin_amdgcn_perm(d[4 * f + 3], d[4 * f + 2], 0x05010400u), h23 = __builtin_amdgcn_perm(d[4 * f + 3], d[4 * f + 2], 0x07030602u);
        plane[0][f] = __builtin_amdgcn_perm(l23, l01, 0x05040100u);
        plane[1][f] = __builtin_amdgcn_perm(l23, l01, 0x07060302u);
        plane[2][f] = __builtin_amdgcn_perm(h23, h01, 0x05040100u);
        plane[3][f] = __builtin_amdgcn_perm(h23, h01, 0x07060302u);
      }
#pragma unroll
      for (int by = 0; by < 4; ++by)
        *reinterpret_cast<uint2*>(to + (g4 * 4 + by) * stride + nb * kPageBlock + n16 * 8) = make_uint2(plane[by][0], plane[by][1]);
    }
    const float scale = (__ballot(bad) >> (g4 * 16) & 0xffffu) != 0 ? __builtin_nanf("") : ldexpf(1.0f, ex - 30 - kShift);
    const double off = zterm + static_cast<double>(now.lse) * 1.4426950408889634074;
    const float high = static_cast<float>(off);
    // (an lse that is not finite: what is lost of it is nothing)
    const float lost = fabsf(high) < __builtin_huge_valf() ? static_cast<float>(off - static_cast<double>(high)) : 0.0f;
    if (n16 == 0) {
      rows->row[g4] = QueryRow{scale, scale * 65536.0f, high, __builtin_amdgcn_exp2f(-lost)};
      rows->end[g4] = now.back < 0 ? 0 : len - now.back;
    }
  }
};

// Workspace, where there are more than kFewTiles row tiles: per (sequence, unit, tile) 16 rows of P digits and the TileRows.
template <int NB>
__host__ __device__ constexpr int made_bytes() { return NB * 16 * kPageBlock + static_cast<int>(sizeof(TileRows)); }

__device__ __forceinline__ int tokens_of(const WeightArgs& a, int length) {
  const int64_t room = min(static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift, a.capacity);
  return static_cast<int>(min(static_cast<int64_t>(max(length, 0)), room));
}

// A wave makes one tile's digits.
template <int BITS, int NB, int HEADS>
__global__ void __launch_bounds__(256) query_digits_kernel(WeightArgs a, WeightPlan plan) {
  const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
  const int tile = static_cast<int>(blockIdx.x) * 4 + __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), unit = blockIdx.y, b = blockIdx.z;
  using Maker = QueryDigits<BITS, NB, HEADS>;
  __shared__ __align__(16) unsigned char scratch[4 * Maker::kScratch];
  if (tile >= plan.tiles) return;
  Maker maker{a, plan, b, unit, HEADS == 1 ? 4 : plan.group, g4, n16, {}};
  const auto query = maker.request(tile);
#pragma unroll
  for (int nb = 0; nb < NB; ++nb)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      maker.kp[nb][e] = *reinterpret_cast<const i4v*>(a.k_pos + unit * maker.P + nb * kPageBlock + n16 * 8 + e);
  const int len = tokens_of(a, a.lens[b]);
  if (len == 0) return;
  unsigned char* to = static_cast<unsigned char*>(a.workspace) + ((static_cast<int64_t>(b) * gridDim.y + unit) * plan.tiles + tile) * made_bytes<NB>();
  maker.make(query, len, scratch + (threadIdx.x >> 6) * Maker::kScratch, to, maker.P, reinterpret_cast<TileRows*>(to + 16 * maker.P));
}

// NB: blocks of a unit; HEADS: key/value heads of a unit; MADE: the queries' digits are in the workspace; STREAM: keys are read past the
// last-level cache; CARRY: what sums lose is kept (in the kernel of all windows it cost registers, and spills in three of them).  Three waves per
// SIMD where their registers suffice, nearly (four instead: spills, or 23.4 -> 28.7 us); digits made, several heads: two (16 x 2048 of 32 heads
// of 32, 8 queries, 29.9 -> 24.4 us; 8 x 4096 of 12 of 64, 16 queries, 8 bits 20.1 -> 18.5), made here: three, with spills at heads of 32 (16 x 4096 of 32 at
// 4 bits 19.8, two 21.5; at 3 bits 17.6 | 21.3).
template <int BITS, int NB, int HEADS, bool MADE, bool STREAM, bool CARRY>
__global__ void __launch_bounds__(256, NB == 2 || BITS * HEADS >= (MADE ? 12 : 32) ? 2 : 3) attend_weights_kernel(WeightArgs a, WeightPlan plan) {
  constexpr int kRow = 16 * BITS;                          // bytes of a token's row in a block
  constexpr int P = NB * kPageBlock;                       // positions of the unit
  constexpr int kDigitRow = P + 16;                        // (16 more: other banks)
  constexpr int kHeld = MADE ? held_tiles(NB) : kFewTiles;
  __shared__ __align__(16) unsigned char q_dig[kHeld * 16 * kDigitRow];
  __shared__ __align__(16) TileRows rows[kHeld];
  __shared__ __align__(16) unsigned char table[MADE ? 16 : P / 8 * 144];         // eight positions' records, and 16 bytes (banks)
  constexpr int kCarried = carried_tiles(HEADS);
  __shared__ float lost[CARRY ? 4 * kCarried * HEADS * kTile : 1];               // [wave][token tile][slot][lane]
  const int lane = threadIdx.x & 63, n16 = lane & 15, g4 = lane >> 4;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const int part = blockIdx.x, unit = blockIdx.y, b = blockIdx.z;
  // (requested first, all at once: the length, the first two tiles' pages, the positions' records, the queries)
  const int length = a.lens[b];
  const int32_t* pt = a.page_table + b * a.ld_pt;
  auto token_of = [&](int k) { return (part + k * plan.parts) * kTileTokens + wave * kTile; };
  auto page_at = [&](int k) { return pt[min((token_of(k) + (lane & 3) * 16) >> a.g.page_shift, a.pages_per_seq - 1)]; };
  const int page0 = page_at(0), page1 = page_at(1);
  i4v record;
  if (!MADE) record = reinterpret_cast<const i4v*>(a.k_pos + unit * P)[threadIdx.x & (P - 1)];
  const int group = HEADS == 1 ? 4 : plan.group, group_shift = group >> 1;                 // (log2 of 1, 2, 4)
  using Maker = QueryDigits<BITS, NB, HEADS>;
  static_assert(Maker::kScratch <= 16 * kDigitRow, "a tile's queries take the place of its digits");
  Maker maker{a, plan, b, unit, group, g4, n16, {}};
  typename Maker::Query query;
  if (!MADE && wave < plan.tiles) query = maker.request(wave);
  const int len = tokens_of(a, length);
  if (part * kTileTokens >= len) return;

  const int share = plan.share, pairs = share * a.queries;
  const int set_heads = kRowHeads / group;
  const bool full_rows = pairs % group == 0;               // (no row without a query)

  // ---- a wave's tiles: every parts-th run of 256 tokens, 64 of them each -----------------------------------------
  const int block_rows = 1 << a.g.page_shift;
  const int first_token = token_of(0), step = plan.parts * kTileTokens;
  const int my_tiles = first_token < len ? (len - first_token + step - 1) / step : 0;
  // lane 4 i + r's 16 tokens (r: lane & 3) of tile k: their page's number, or -1
  auto page_of = [&](int k, int id) { return token_of(k) + (lane & 3) * 16 < len && id >= 0 && id < a.g.n_pages ? id : -1; };
  const uint32_t k_off = n16 * kRow + g4 * (4 * BITS);
  const int block_bytes = block_rows * kRow;
  constexpr int kAux = STREAM ? 2 : 0;                     // (2: non-temporal)
  uint32_t kr[4][NB][BITS];
  auto load_keys = [&](int k, int id) __attribute__((always_inline)) {
    typedef unsigned u3v __attribute__((ext_vector_type(3)));
    typedef unsigned u4v __attribute__((ext_vector_type(4)));
    const int t = (token_of(k) + (lane & 3) * 16) & (block_rows - 1);
    const uint64_t at = ((static_cast<uint64_t>(max(id, 0)) * (a.g.d / kPageBlock) + unit * NB) * block_rows + t) * kRow;
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const uint64_t row = of_lane(static_cast<uint32_t>(at), static_cast<uint32_t>(at >> 32), r);
      const __amdgpu_buffer_rsrc_t rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<uint8_t*>(a.k_pages) + row, 0,
                                                                            (NB - 1) * block_bytes + 16 * kRow, 0x00020000);
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        if constexpr (BITS == 3) {
          const u3v v = __builtin_amdgcn_raw_buffer_load_b96(rsrc, k_off, nb * block_bytes, kAux);
#pragma unroll
          for (int e = 0; e < 3; ++e) kr[r][nb][e] = v[e];
        } else {
#pragma unroll
          for (int h = 0; h < BITS / 4; ++h) {
            const u4v v = __builtin_amdgcn_raw_buffer_load_b128(rsrc, k_off + 16 * h, nb * block_bytes, kAux);
#pragma unroll
            for (int e = 0; e < 4; ++e) kr[r][nb][4 * h + e] = v[e];
          }
        }
      }
    }
  };
  // What this lane adds up of a tile, slot e: head e / set_heads * set_heads + g4 / group of the unit, token e % set_heads plus (g4 % group)
  // * set_heads times 16, plus n16, of the tile (every weight of the tile's 64 tokens and HEADS heads is one lane's).
  const int64_t first_at = (static_cast<int64_t>(b) * a.n_kv + unit * HEADS) * a.capacity;
  auto slot_head = [&](int e) { return e / set_heads * set_heads + (g4 >> group_shift); };
  auto slot_group = [&](int e) { return (g4 & (group - 1)) * set_heads + (e & (set_heads - 1)); };       // of 16 tokens
  auto slot_token = [&](int k, int e) { return token_of(k) + slot_group(e) * 16 + n16; };
  float old[HEADS], old_next[HEADS];
  auto load_old = [&](int k) __attribute__((always_inline)) {      // (behind the end: the last token's, not used)
#pragma unroll
    for (int e = 0; e < HEADS; ++e) old_next[e] = a.weights[first_at + slot_head(e) * a.capacity + min(slot_token(k, e), len - 1)];
  };

  // (CARRY: the wave's tiles from `reached` on, kCarried of them, and round again with the next ones; the first wave has the most)
  const int most_tiles = CARRY ? (len - part * kTileTokens + step - 1) / step : 0;
  int reached = 0;
  for (int tile0 = 0; tile0 < plan.tiles; tile0 += kHeld) {
    const int tile1 = min(tile0 + kHeld, plan.tiles);
    const int k0 = CARRY ? reached : 0, k1 = CARRY ? min(k0 + kCarried, my_tiles) : my_tiles;
    int id = page_of(k0, CARRY ? page_at(k0) : page0), next_page = CARRY ? page_at(k0 + 1) : page1;
    if (k0 < k1) {
      load_old(k0);
      load_keys(k0, id);
    }
    if constexpr (MADE) {
      // 16 bytes of a row at a time, rows P apart there and kDigitRow apart here
      constexpr int kPieces = made_bytes<NB>() / 16;
      const i4v* from = reinterpret_cast<const i4v*>(static_cast<const unsigned char*>(a.workspace) +
                                                         ((static_cast<int64_t>(b) * gridDim.y + unit) * plan.tiles + tile0) * made_bytes<NB>());
      constexpr int kEach = (kHeld * kPieces + 255) / 256;
      const int pieces = (tile1 - tile0) * kPieces;
      i4v v[kEach];
#pragma unroll
      for (int k = 0; k < kEach; ++k) v[k] = from[min(k * 256 + static_cast<int>(threadIdx.x), pieces - 1)];
      if (tile0 > 0 || k0 > 0) __syncthreads();            // (the digits before have been read)
#pragma unroll
      for (int k = 0; k < kEach; ++k) {
        const int i = k * 256 + static_cast<int>(threadIdx.x);
        const int tile = i / kPieces, at = i - tile * kPieces, row = at / (P / 16);
        unsigned char* to = row < 16 ? q_dig + (tile * 16 + row) * kDigitRow + (at & (P / 16 - 1)) * 16
                                     : reinterpret_cast<unsigned char*>(rows + tile) + (at - P) * 16;
        if (i < pieces) *reinterpret_cast<i4v*>(to) = v[k];
      }
    } else {
      *reinterpret_cast<i4v*>(table + (threadIdx.x & (P - 1)) * 16 + (threadIdx.x & (P - 1)) / 8 * 16) = record;
      __syncthreads();
      if (wave < tile1) {
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
#pragma unroll
          for (int e = 0; e < 8; ++e) maker.kp[nb][e] = *reinterpret_cast<const i4v*>(table + (nb * 16 + n16) * 144 + e * 16);
        unsigned char* to = q_dig + wave * 16 * kDigitRow;
        maker.make(query, len, to, to, kDigitRow, rows + wave);
      }
    }
    __syncthreads();

    for (int k = k0; k < k1; ++k) {
      const int token = token_of(k);
      const uint64_t here = __ballot(id >= 0);             // (bit r: the tile's r-th 16 tokens)
      uint32_t kw[4][NB][8];
#pragma unroll
      for (int r = 0; r < 4; ++r)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) expand<BITS>(kr[r][nb], kw[r][nb]);
#pragma unroll
      for (int e = 0; e < HEADS; ++e) old[e] = old_next[e];
      // (the next tile's: weights first, loads come back in order)
      if (k + 1 < k1) {
        id = page_of(k + 1, next_page);
        if (k + 2 < k1) next_page = page_at(k + 2);
        load_old(k + 1);
        load_keys(k + 1, id);
      }
      // lane (row g4, token n16 of every 16): tokens of the r-th 16 that there are
      int token_r[4];
#pragma unroll
      for (int r = 0; r < 4; ++r) token_r[r] = here >> r & 1 ? token + r * 16 + n16 : 0x7fffffff;

      const bool whole = (here & 15) == 15 && token + kTile <= len - (a.queries - 1) && full_rows;
      // Adds the weights of row tiles from .. to - 1 to `sum`, kSide of them side by side where their digits were made before.
      auto add_up = [&](int from, int to, float (&sum)[4], auto&& seen) __attribute__((always_inline)) {
        struct Operands {
          QueryRow row;
          v4i q[NB][2];
        };
        auto fetch = [&](int i) __attribute__((always_inline)) {
          Operands o;
          o.row = rows[i].row[g4];
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < 2; ++s)
              o.q[nb][s] = *reinterpret_cast<const v4i*>(q_dig + (i * 16 + n16) * kDigitRow + nb * kPageBlock + g4 * 32 + s * 16);
          return o;
        };
        // (the products of two row tiles side by side: with two waves per SIMD each is a chain of latencies)
        auto some = [&](auto count, int i) __attribute__((always_inline)) {
          constexpr int N = decltype(count)::value;
          Operands o[N];
          v4i c[N][4];
#pragma unroll
          for (int n = 0; n < N; ++n) {
            o[n] = fetch(i + n);
#pragma unroll
            for (int r = 0; r < 4; ++r) c[n][r] = v4i{0, 0, 0, 0};
          }
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
#pragma unroll
            for (int s = 0; s < 2; ++s)
#pragma unroll
              for (int n = 0; n < N; ++n)
#pragma unroll
                for (int r = 0; r < 4; ++r) {
                  const v4i w = {static_cast<int>(kw[r][nb][4 * s]), static_cast<int>(kw[r][nb][4 * s + 1]), static_cast<int>(kw[r][nb][4 * s + 2]),
                                 static_cast<int>(kw[r][nb][4 * s + 3])};
                  c[n][r] = __builtin_amdgcn_mfma_i32_16x16x64_i8(o[n].q[nb][s], w, c[n][r], 0, 0, 0);
                }
#pragma unroll
          for (int n = 0; n < N; ++n)
#pragma unroll
            for (int r = 0; r < 4; ++r) {
              const float high = fmaf(static_cast<float>(c[n][r][3] * 256 + c[n][r][2]), o[n].row.high, -o[n].row.off);
              const float p = __builtin_amdgcn_exp2f(fmaf(static_cast<float>(c[n][r][1] * 256 + c[n][r][0]), o[n].row.low, high));
              sum[r] = fmaf(seen(p, r, i + n), o[n].row.rest, sum[r]);
            }
        };
        int i = from;
        if constexpr (MADE)
          for (; i + kSide <= to; i += kSide) some(std::integral_constant<int, kSide>{}, i);
        for (; i < to; ++i) some(std::integral_constant<int, 1>{}, i);
      };

      float got[HEADS];
#pragma unroll
      for (int e = 0; e < HEADS; ++e) got[e] = 0.0f;
#pragma unroll
      for (int e0 = 0; e0 < HEADS; ++e0) {                 // (slots of a set begin at a multiple of set_heads)
        if (HEADS > 1 && (e0 & (set_heads - 1)) != 0) continue;
        const int set = HEADS == 1 ? 0 : e0 / set_heads;
        const int from = max(set * plan.set_tiles, tile0) - tile0, to = min((set + 1) * plan.set_tiles, tile1) - tile0;
        float sum[4] = {0.0f, 0.0f, 0.0f, 0.0f};
        if (whole) add_up(from, to, sum, [&](float p, int, int) { return p; });
        else add_up(from, to, sum, [&](float p, int r, int i) { return token_r[r] < rows[i].end[g4] ? p : 0.0f; });
        // the rows of a head together
        if (HEADS == 1 || group >= 2) {
#pragma unroll
          for (int r = 0; r < 4; ++r) sum[r] += __shfl_xor(sum[r], 16, kWave);
        }
        if (HEADS == 1 || group == 4) {
#pragma unroll
          for (int r = 0; r < 4; ++r) sum[r] += __shfl_xor(sum[r], 32, kWave);
        }
#pragma unroll
        for (int j = 0; j < HEADS; ++j) {
          if (j < e0 || (HEADS > 1 && j >= e0 + set_heads)) continue;
          const int r = slot_group(j);
          got[j] = r == 0 ? sum[0] : (r == 1 ? sum[1] : (r == 2 ? sum[2] : sum[3]));
        }
      }
      // (a head's first row tiles set what starts here, later ones add to it)
#pragma unroll
      for (int e = 0; e < HEADS; ++e) {
        const int t = slot_token(k, e), set = HEADS == 1 ? 0 : e / set_heads;
        const int64_t at = first_at + slot_head(e) * a.capacity + t;
        const bool first = set * plan.set_tiles >= tile0, any = first ? set * plan.set_tiles < tile1 : (set + 1) * plan.set_tiles > tile0;
        const bool starts = first && t >= len - a.fresh;
        if (!any || t >= len) continue;
        const float before = starts ? 0.0f : old[e];
        float sum = before + got[e];
        if constexpr (CARRY) {
          // (what the sum of two loses is a number of fp32 itself)
          float* mine = lost + ((wave * kCarried + (k - k0)) * HEADS + e) * kTile + lane;
          const float second = sum - before;
          float all = fabsf(sum) < __builtin_huge_valf() ? (before - (sum - second)) + (got[e] - second) : 0.0f;
          if (!first) all += *mine;
          if ((set + 1) * plan.set_tiles <= tile1) sum += all;
          else *mine = all;
        }
        a.weights[at] = sum;
        if (starts) a.token_positions[at] = a.positions ? a.positions[b] - (len - 1 - t) : t;
      }
    }
    if (CARRY && tile1 == plan.tiles && k0 + kCarried < most_tiles) {
      reached = k0 + kCarried;
      tile0 = -kHeld;
    }
  }
}

static WeightPlan weight_plan(int32_t queries, int32_t n_q, int32_t n_kv, int32_t hd) {
  const int heads = hd > kPageBlock ? 1 : kPageBlock / hd;
  WeightPlan p;
  p.share = n_q / n_kv;
  const int pairs = p.share * queries;
  p.group = std::max(pairs >= 3 ? 4 : pairs, kRowHeads / heads);         // (not less than gives every lane a weight to write)
  p.set_tiles = (pairs + p.group - 1) / p.group;
  p.per_share = 1.0 / p.share * (1.0 + 0x1p-50);
  p.per_set = 1.0 / p.set_tiles * (1.0 + 0x1p-50);
  p.tiles = p.set_tiles * (heads / (kRowHeads / p.group));
  p.parts = 0;
  return p;
}

size_t attend_weights_workspace_bytes(int32_t B, int32_t queries, int32_t n_q, int32_t n_kv, int32_t hd) {
  const WeightPlan p = weight_plan(queries, n_q, n_kv, hd);
  if (p.tiles <= kFewTiles) return 0;
  const int64_t units = n_kv * hd / std::max(hd, kPageBlock);
  return static_cast<size_t>(B * units * p.tiles) * (hd > kPageBlock ? made_bytes<2>() : made_bytes<1>());
}

int32_t launch_attend_weights(const WeightArgs& a, int32_t bits, hipStream_t st) {
  if (a.B == 0) return RPTQ_OK;
  const int P = a.hd > kPageBlock ? a.hd : kPageBlock, units = a.n_kv * a.hd / P, heads = P / a.hd;
  WeightPlan p = weight_plan(a.queries, a.n_q, a.n_kv, a.hd);
  const int64_t most = std::min<int64_t>(static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift, a.capacity);
  const int64_t runs = (most + kTileTokens - 1) / kTileTokens, each = static_cast<int64_t>(a.B) * units;
  p.parts = static_cast<int32_t>(std::min<int64_t>(runs, std::max<int64_t>(1, (kSeenWorkgroups + each - 1) / each)));
  const dim3 grid(p.parts, units, a.B), makers((p.tiles + 3) / 4, units, a.B);
  const int64_t pages = std::min<int64_t>(a.g.n_pages, static_cast<int64_t>(a.B) * a.pages_per_seq);
  const bool stream = pages * 2 * (static_cast<int64_t>(a.g.d) * bits / 8 << a.g.page_shift) > kStreamBytes;
  const bool carry = p.set_tiles > kPasses * held_tiles(P / kPageBlock);
  auto go = [&](auto digits, auto made, auto carried, auto alone, auto streamed) {
    if (p.tiles > kFewTiles) {
      hipLaunchKernelGGL(digits, makers, dim3(256), 0, st, a, p);
      hipLaunchKernelGGL(carry ? carried : made, grid, dim3(256), 0, st, a, p);
    } else {
      hipLaunchKernelGGL(stream ? streamed : alone, grid, dim3(256), 0, st, a, p);
    }
  };
#define RPTQ_GO(BITS, NB, HEADS) \
  go(query_digits_kernel<BITS, NB, HEADS>, attend_weights_kernel<BITS, NB, HEADS, true, false, false>,                  \
     attend_weights_kernel<BITS, NB, HEADS, true, false, true>, attend_weights_kernel<BITS, NB, HEADS, false, false, false>, \
     attend_weights_kernel<BITS, NB, HEADS, false, BITS < 8, false>)
#define RPTQ_BY_BITS(NB, HEADS)                 \
  do {                                          \
    if (bits == 3) RPTQ_GO(3, NB, HEADS);       \
    else if (bits == 4) RPTQ_GO(4, NB, HEADS);  \
    else RPTQ_GO(8, NB, HEADS);                 \
  } while (0)
  if (a.hd > kPageBlock) RPTQ_BY_BITS(2, 1);
  else if (heads == 1) RPTQ_BY_BITS(1, 1);
  else if (heads == 2) RPTQ_BY_BITS(1, 2);
  else RPTQ_BY_BITS(1, 4);
#undef RPTQ_BY_BITS
#undef RPTQ_GO
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
