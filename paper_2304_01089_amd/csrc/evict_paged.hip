// Eviction from the paged cache: every key/value head of a sequence longer than its budget keeps `budget` tokens - the first, the
// newest, then the heaviest, ties to the lowest index - and the kept tokens behind the budget move, in their order, into the
// holes that the others leave before it.  A move is a row of codes of keys and one of values and the token's record; what lies
// before the budget and is kept stays where it is, so a step that evicts one token moves one.  (Attention does not depend on
// the order of the tokens; a token's position is in its record.)
//
// One workgroup per (sequence, head) finds the threshold: a token's key is its weight's bits in an order of whole numbers, and the
// budget-th largest key is found from the top, twelve bits, ten and ten: the workgroup counts its keys in bins in LDS, sums them in 64
// groups, and every wave finds by itself the group and in it the bin where the sum from the top reaches the budget.  A bin of up to 64
// keys ends the search: they are compared with each other.  Where only one token leaves - a step of a batch at its budget - the
// smallest key is found by maxima over lanes and waves and no threshold (32 x 2049 tokens of 8 heads 9.6 -> 5.4 us).  A wave has a run
// of consecutive tokens, so the order among equal keys and the places in the lists of holes and movers are counts of votes.
// Few moves are done by the same workgroup, many by a second launch over the whole chip.
// What bounds it: a chain of short steps, each of one to three thousand cycles and most of them across the workgroup's waves: 7
// sequences of 1531 tokens, 2 heads of 256, budget 700 take 10.3 us (moves 6300 of 18500 cycles, keys and bins 2400, the search
// 3400).  Long sequences: one compute unit's LDS and instructions per head: 4 of 32768 tokens, 8 heads, budget 4096 take 36.4 us, 28 in
// the first kernel (of 45000 cycles of a head in the middle 11000 are keys and bins, 7000 the later looks, 18000 votes and lists), 7.8 in the moves.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <type_traits>

#include "attend_common.h"
#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kFirstBins = 4096, kLaterBins = 1024;              // of twelve and of ten bits of a key
// Keys stay in registers up to eight of a lane, with eight waves up to 4096 tokens (four | eight up to 2048: 7 x 1531 11.2 | 10.3 us) and
// sixteen up to 8192; they lie in LDS up to 32 of a lane (32768 tokens); longer sequences' are made anew from their records.
constexpr int kFewItems = 8;
constexpr int kLdsItems = 32;
// Movers of an item, up to which a lane writes them down by itself (always | up to 8 | 16 | 32: 4 x 32768 39.2 | 36.6 | 36.4 | 36.4 us, 16 x 10000 to
// 4096, 8 heads, 54.9 | 49.8 | 50.7 | 53.9).
constexpr int kFewMovers = 16;
constexpr int kHeldPages = 1024;               // page numbers of a sequence that are kept at hand
constexpr int kFewMoves = 2048;                // of a head at most where the workgroup that finds them does them (512 | 2048: 16 x 4000 to 2000, 8 heads, 19.1 | 17.1 us)
constexpr int kMoveChunks = 1024;              // workgroups of a head there at most
constexpr uint32_t kSafe = 0xffffffffu, kNanKey = 0xfffffffeu;

typedef unsigned Bytes16 __attribute__((ext_vector_type(4)));
typedef unsigned Bytes8 __attribute__((ext_vector_type(2)));

struct EvictPlan {
  int32_t most;                                // moves of a head at most
  int32_t vec;                                 // bytes moved at a time: 4, 8 or 16
  int32_t units;                               // of them in a head's row
  bool few;
};

__device__ __forceinline__ int evict_room(const EvictArgs& a) {
  return static_cast<int>(min(static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift, a.capacity));
}

// Workspace: [B * n_kv] moves, a multiple of four of them, then [B * n_kv][2][most] tokens they go to and come from.
__host__ __device__ constexpr int64_t list_start(int64_t heads) { return (heads + 3) / 4 * 4; }

template <int THREADS, typename T>
__device__ __forceinline__ void copy(T* to, const T* from, int n) {
#pragma unroll 8
  for (int t = threadIdx.x; t < n; t += THREADS) to[t] = from[t];
}

// Records number 0 .. end - 1 of the lists.
template <int THREADS>
__device__ __forceinline__ void move_records(const EvictArgs& a, int64_t base, const int32_t* to, const int32_t* from, int end) {
  for (int i = THREADS - 1 - static_cast<int>(threadIdx.x); i < end; i += 4 * THREADS) {
    float w[4];
    int32_t p[4], t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = min(i + k * THREADS, end - 1), f = from[j];
      t[k] = to[j];
      w[k] = a.weights[base + f];
      p[k] = a.positions[base + f];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      if (i + k * THREADS >= end) continue;
      a.weights_out[base + t[k]] = w[k];
      a.positions_out[base + t[k]] = p[k];
    }
  }
}

// Rows number first, first + step, ... of the lists: the thread's `which`-th of 2 units pieces.  page_of: a page's number.  MANY: eight rows
// at a time (eight | sixteen: 7 x 1531 10.3 | 12.0 us, whose last rows are moved several times).
template <bool MANY, typename V, typename P, typename L>
__device__ __forceinline__ void move_pieces(const EvictArgs& a, int units, int h, P&& page_of, L to, L from, int first, int end, int step,
                                            int which) {
  const int row_bytes = 16 * a.bits, head_bytes = a.hd * a.bits / 8;
  const bool values = which >= units;
  const int off = (which - (values ? units : 0)) * static_cast<int>(sizeof(V));       // of the head's row
  // heads over 128 wide: the row lies in several blocks; others share one
  const int64_t place = static_cast<int64_t>(h) * head_bytes + off;
  const int block = static_cast<int>(place / row_bytes), in_row = static_cast<int>(place - static_cast<int64_t>(block) * row_bytes);
  const int shift = a.g.page_shift, block_bytes = row_bytes << shift;            // (below 2^20)
  const uint64_t pages = reinterpret_cast<uint64_t>(values ? a.v_pages : a.k_pages) + static_cast<uint64_t>(block * block_bytes + in_row);
  const uint32_t page_bytes = static_cast<uint32_t>(a.g.d / kPageBlock * block_bytes);
  auto at = [&](int t) __attribute__((always_inline)) {        // (one wide product and one narrow one: addresses are what a row costs)
    const uint64_t page = pages + static_cast<uint64_t>(static_cast<uint32_t>(page_of(t >> shift))) * page_bytes;
    return reinterpret_cast<V*>(page + __umul24(t & ((1 << shift) - 1), row_bytes));
  };
  // (N at a time; the last row several times, if need be: the same bytes)
  auto some = [&](auto count, int i) __attribute__((always_inline)) {
    constexpr int N = decltype(count)::value;
    V x[N];
    V* y[N];
#pragma unroll
    for (int k = 0; k < N; ++k) {
      const int j = min(i + k * step, end - 1);
      x[k] = *at(from[j]);
      y[k] = at(to[j]);
    }
#pragma unroll
    for (int k = 0; k < N; ++k) *y[k] = x[k];
  };
  int i = first;
  if constexpr (MANY)
    for (; i + 4 * step < end; i += 8 * step) some(std::integral_constant<int, 8>{}, i);
  for (; i < end; i += 4 * step) some(std::integral_constant<int, 4>{}, i);
}

template <int THREADS, bool MANY, typename P, typename L>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const EvictPlan& p, int h, P&& page_of, L to, L from, int moves, int begin) {
  const int each = 2 * p.units, rows = THREADS / each, row = static_cast<int>(threadIdx.x) / each, which = static_cast<int>(threadIdx.x) - row * each;
  if (row >= rows) return;
  if (p.vec == 16) move_pieces<MANY, Bytes16>(a, p.units, h, page_of, to, from, begin + row, moves, rows, which);
  else if (p.vec == 8) move_pieces<MANY, Bytes8>(a, p.units, h, page_of, to, from, begin + row, moves, rows, which);
  else move_pieces<MANY, uint32_t>(a, p.units, h, page_of, to, from, begin + row, moves, rows, which);
}

// A list of one token.
struct One {
  int token;
  __device__ __forceinline__ int operator[](int) const { return token; }
};

// The wave's largest, in every lane.
template <int CTRL, int ROWS>
__device__ __forceinline__ uint32_t dpp_larger(uint32_t v) {
  return max(v, static_cast<uint32_t>(__builtin_amdgcn_update_dpp(0, static_cast<int>(v), CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ uint32_t wave_largest(uint32_t v) {
  v = dpp_larger<0x111, 0xf>(v);
  v = dpp_larger<0x112, 0xf>(v);
  v = dpp_larger<0x114, 0xf>(v);
  v = dpp_larger<0x118, 0xf>(v);
  v = dpp_larger<0x142, 0xa>(v);
  v = dpp_larger<0x143, 0xc>(v);
  return __builtin_amdgcn_readlane(v, 63);
}
__device__ __forceinline__ int wave_largest_int(int v) {
  return static_cast<int>(wave_largest(static_cast<uint32_t>(v) ^ 0x80000000u) ^ 0x80000000u);
}

// Over the 16 lanes of a row.
__device__ __forceinline__ int row16_add_int(int v) {
  v += static_cast<int>(dpp_row<0xB1>(static_cast<uint32_t>(v)));
  v += static_cast<int>(dpp_row<0x4E>(static_cast<uint32_t>(v)));
  v += static_cast<int>(dpp_row<0x141>(static_cast<uint32_t>(v)));
  return v + static_cast<int>(dpp_row<0x140>(static_cast<uint32_t>(v)));
}

enum class Keys { registers, lds, made };      // where a token's key is when it is looked at again; made: from its record

// WAVES: of the workgroup
template <int WAVES, Keys KEYS>
__global__ void __launch_bounds__(WAVES * 64) evict_select_kernel(EvictArgs a, EvictPlan plan) {
  constexpr int kRun = KEYS == Keys::registers ? kFewItems : 16;             // of its items a lane works on so many together (8 | 16 | 32: 4 x 32768 37.6 | 36.4 | 38.0 us)
  constexpr int kThreads = WAVES * 64, kKeys = KEYS == Keys::lds ? kThreads * kLdsItems : 1;
  constexpr int kAllBins = kFirstBins + 2 * kLaterBins;
  __shared__ __align__(16) int32_t bins[kAllBins];             // (later the lists of a few moves)
  __shared__ uint32_t key_lds[kKeys];
  __shared__ int32_t ids[kHeldPages];
  __shared__ int32_t groups[3][64];                            // of a sixty-fourth of the bins each
  __shared__ int32_t sums[3][2][16];
  __shared__ uint32_t some[64];                                // keys of a bin that holds few
  __shared__ uint32_t some_over[64];                           // those above, those not below
  __shared__ int32_t some_count;
  static_assert(2 * kFewMoves <= kAllBins, "the lists take the bins' place");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int n = min(max(a.lens[b], 0), evict_room(a));
  const int64_t base = static_cast<int64_t>(blockIdx.x) * a.capacity;
  const float* weights = a.weights + base;
  const int32_t* positions = a.positions + base;
  float* weights_out = a.weights_out + base;
  int32_t* positions_out = a.positions_out + base;
  const bool w_apart = weights_out != weights, p_apart = positions_out != positions;
  int32_t* workspace = static_cast<int32_t*>(a.workspace);
  auto leave = [&] {                                           // the sequence as it is
    if (h == 0 && tid == 0) a.lens_out[b] = n;
    if (!plan.few && tid == 0) workspace[blockIdx.x] = 0;
    if (w_apart) copy<kThreads>(weights_out, weights, n);
    if (p_apart) copy<kThreads>(positions_out, positions, n);
  };
  if (n <= a.budget) {
    leave();
    return;
  }

  // a wave's tokens: `items` times 64 consecutive ones, several items at a time (a run)
  const int items = ((n + WAVES - 1) / WAVES + 63) >> 6, start = wave * items * 64;
  const int end = min(start + items * 64, n);
  float w[kRun];
  int32_t pos[kRun];
  // (buffer loads: an item is 256 bytes from the last, which is part of the instruction, and what lies beyond the sequence reads as 0)
  const uint32_t record_bytes = 4u * static_cast<uint32_t>(n);       // (up to 2^31)
  const __amdgpu_buffer_rsrc_t w_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<float*>(weights), 0, record_bytes, 0x00020000);
  const __amdgpu_buffer_rsrc_t p_rsrc = __builtin_amdgcn_make_buffer_rsrc(const_cast<int32_t*>(positions), 0, record_bytes, 0x00020000);
  // (both loads of an item together: all positions first measured 0.4 us more for 32 x 2049)
  auto read = [&](int first) __attribute__((always_inline)) {
    const uint32_t at = static_cast<uint32_t>(start + first * 64 + lane) * 4u;
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      pos[i] = static_cast<int32_t>(__builtin_amdgcn_raw_buffer_load_b32(p_rsrc, at + i * 256, 0, 0));
      w[i] = __uint_as_float(__builtin_amdgcn_raw_buffer_load_b32(w_rsrc, at + i * 256, 0, 0));
    }
  };
  read(0);
  // the sequence's pages; one that is not there: it stays as it is
  const int32_t* pt = a.page_table + b * a.ld_pt;
  const int pages = ((n - 1) >> a.g.page_shift) + 1;
  bool gone = false;
  for (int p = tid; p < pages; p += kThreads) {
    const int id = pt[p];
    gone = gone || id < 0 || id >= a.g.n_pages;
    if (p < kHeldPages) ids[p] = id;
  }
  for (int i = tid; i < kAllBins / 4; i += kThreads) reinterpret_cast<int4*>(bins)[i] = make_int4(0, 0, 0, 0);
  if (tid < 64) some_over[tid] = 0;
  if (tid == 0) some_count = 0;
  int newest = INT32_MIN;
  if (a.recent > 0) {
    for (int first = 0; first < items; first += kRun) {
      if (first > 0) read(first);
      if (start + (first + kRun) * 64 <= end) {                // (uniform: all of the run's tokens are there)
#pragma unroll
        for (int i = 0; i < kRun; ++i) newest = max(newest, pos[i]);
      } else {
#pragma unroll
        for (int i = 0; i < kRun; ++i)
          if (start + (first + i) * 64 + lane < end) newest = max(newest, pos[i]);
      }
    }
    newest = wave_largest_int(newest);
  }
  const bool wave_gone = __ballot(gone) != 0;
  if (lane == 0) sums[0][0][wave] = newest, sums[0][1][wave] = wave_gone;
  __syncthreads();
  if (__ballot(sums[0][1][lane & (WAVES - 1)] != 0) != 0) {
    leave();
    return;
  }
  if (a.recent > 0) newest = wave_largest_int(sums[0][0][lane & (WAVES - 1)]);

  // The run's keys from its records: 0 where no token of the wave's is.  (A weight's is at least 0x007fffff, minus infinity's.)
  uint32_t keys[kRun];
  auto make_keys = [&](int first) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      keys[i] = 0;
      if (first + i >= items) continue;
      const uint32_t k = w[i] == w[i] ? float_key(w[i] + 0.0f) : kNanKey;      // (minus zero is zero)
      // (newest - position is no negative number and may have 32 bits)
      const bool safe = pos[i] < a.first || static_cast<uint32_t>(newest) - static_cast<uint32_t>(pos[i]) < static_cast<uint32_t>(a.recent);
      keys[i] = safe ? kSafe : k;
    }
    if (start + (first + kRun) * 64 > end) {
#pragma unroll
      for (int i = 0; i < kRun; ++i)
        if (start + (first + i) * 64 + lane >= end) keys[i] = 0;
    }
  };
  // Calls f(first) for every run, its keys at hand.
  auto each_run = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (KEYS == Keys::registers) {
      f(0);
    } else {
#pragma unroll 1
      for (int first = 0; first < items; first += kRun) {
        if constexpr (KEYS == Keys::lds) {
#pragma unroll
          for (int i = 0; i < kRun; ++i) keys[i] = first + i < items ? key_lds[(wave * kLdsItems + first + i) * 64 + lane] : 0u;
        } else {
          read(first);
          make_keys(first);
        }
        f(first);
      }
    }
  };
  auto count = [&](int32_t* mine, uint32_t k, int shift, uint32_t size) __attribute__((always_inline)) { atomicAdd(&mine[k >> shift & (size - 1)], 1); };
  // Every key once: to where it will be looked at again, and counted by its first twelve bits - or, where only one token leaves,
  // compared with the smallest so far.  Records go to their place (where a token leaves, the one that comes is written later).
  const bool one = n - a.budget == 1;
  uint32_t least = ~0u;                                        // the lane's smallest key, and the last token that has it
  int leaves = -1;
#pragma unroll 1
  for (int first = 0; first < items; first += kRun) {
    if (KEYS == Keys::made ? items > kRun : KEYS == Keys::lds) read(first);
    make_keys(first);
#pragma unroll
    for (int i = 0; i < kRun; ++i) {
      if (first + i >= items) continue;
      if (one) {
        const bool less = keys[i] != 0 && keys[i] <= least;
        least = less ? keys[i] : least;
        leaves = less ? start + (first + i) * 64 + lane : leaves;
        continue;
      }
      if (KEYS == Keys::lds) key_lds[(wave * kLdsItems + first + i) * 64 + lane] = keys[i];
      if (keys[i] != 0) count(bins, keys[i], 20, kFirstBins);
    }
    if ((w_apart || p_apart) && start + first * 64 < a.budget) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const int t = start + (first + i) * 64 + lane;
        if (t >= min(end, a.budget)) continue;
        if (w_apart) weights_out[t] = w[i];
        if (p_apart) positions_out[t] = pos[i];
      }
    }
    if (KEYS == Keys::registers) break;
  }

  if (one) {
    // The smallest key leaves, of equal ones the last token's; the sequence's last token comes into its place.
    const uint32_t mine = ~wave_largest(~least);
    const int last = wave_largest_int(least == mine ? leaves : -1);
    if (lane == 0) sums[1][0][wave] = static_cast<int32_t>(mine), sums[1][1][wave] = last;
    __syncthreads();
    const uint32_t of_wave = static_cast<uint32_t>(sums[1][0][lane & (WAVES - 1)]);
    const int hole = wave_largest_int(of_wave == ~wave_largest(~of_wave) ? sums[1][1][lane & (WAVES - 1)] : -1);
    if (hole < a.budget) {
      const One to{hole}, from{a.budget};
      if (pages <= kHeldPages) move_rows<kThreads, false>(a, plan, h, [&](int page) { return ids[page]; }, to, from, 1, 0);
      else move_rows<kThreads, false>(a, plan, h, [&](int page) { return pt[page]; }, to, from, 1, 0);
      if (tid == kThreads - 1) {
        const float weight = weights[a.budget];
        const int32_t position = positions[a.budget];
        weights_out[hole] = weight;
        positions_out[hole] = position;
      }
    }
    if (!plan.few && tid == 0) workspace[blockIdx.x] = 0;
    if (h == 0 && tid == 0) a.lens_out[b] = a.budget;
    return;
  }

  // ---- the budget-th largest key, from the top: twelve bits, ten and ten ----------------------------------------------
  // All waves count into the same bins and sum them in 64 groups; then every wave finds by itself the group, and in it the bin, where
  // the sum from the top reaches what is needed.
  uint32_t key = 0;                                            // the bits that are known
  int need = a.budget;                                         // that many keys of those that begin with them
  int like = 0;                                                // ... of so many
#pragma unroll 1
  for (int which = 0;; ++which) {
    const int shift = which == 0 ? 20 : (which == 1 ? 10 : 0), size = which == 0 ? kFirstBins : kLaterBins, of_group = size / 64;
    int32_t* mine = bins + (which == 0 ? 0 : (which == 1 ? kFirstBins : kFirstBins + kLaterBins));
    __syncthreads();
    // (WAVES neighbours sum the bins of a group)
    int part = 0;
    if (which == 0) {
#pragma unroll
      for (int i = 0; i < kFirstBins / kThreads; ++i) part += mine[tid * (kFirstBins / kThreads) + i];
    } else {
#pragma unroll
      for (int i = 0; i < kLaterBins / kThreads; ++i) part += mine[tid * (kLaterBins / kThreads) + i];
    }
    part += static_cast<int>(dpp_row<0xB1>(static_cast<uint32_t>(part)));
    part += static_cast<int>(dpp_row<0x4E>(static_cast<uint32_t>(part)));
    if (WAVES > 4) part += static_cast<int>(dpp_row<0x141>(static_cast<uint32_t>(part)));
    if (WAVES > 8) part += static_cast<int>(dpp_row<0x140>(static_cast<uint32_t>(part)));
    if ((lane & (WAVES - 1)) == 0) groups[which][tid / WAVES] = part;
    __syncthreads();
    const int sum = groups[which][63 - lane];
    const int upto = wave_prefix(sum);
    const int l = __builtin_ctzll(__ballot(upto >= need));     // (there is one: as many keys as are needed are in the bins)
    const int over = __builtin_amdgcn_readlane(upto - sum, l);
    const int top = size - 1 - of_group * l, c = lane < of_group ? mine[top - lane] : 0;
    const int upto2 = over + wave_prefix(c);
    const int m = __builtin_ctzll(__ballot(upto2 >= need));
    like = __builtin_amdgcn_readlane(c, m);
    key |= static_cast<uint32_t>(top - m) << shift;
    need -= __builtin_amdgcn_readlane(upto2, m) - like;
    if (like == need || which == 2) break;
    if (like <= 64) {
      // Few: they are written side by side, and each is compared with all, the waves sharing them.
      each_run([&](int first) __attribute__((always_inline)) {
#pragma unroll
        for (int i = 0; i < kRun; ++i)
          if (first + i < items && keys[i] != 0 && (keys[i] ^ key) >> shift == 0) some[atomicAdd(&some_count, 1) & 63] = keys[i];
      });
      __syncthreads();
      const uint32_t v = some[min(lane, like - 1)];
      uint32_t above = 0;                                      // those above in the lower half, those not below in the upper
      for (int j = wave; j < like; j += WAVES) {
        const uint32_t other = some[j];
        above += (other > v ? 1u : 0u) + (other >= v ? 0x10000u : 0u);
      }
      if (above != 0) atomicAdd(&some_over[lane], above);
      __syncthreads();
      above = some_over[lane];
      const int gt = above & 0xffff, ge = above >> 16;
      const int at = __builtin_ctzll(__ballot(gt < need && ge >= need));       // (there is one)
      key = __builtin_amdgcn_readlane(v, at);
      need -= __builtin_amdgcn_readlane(gt, at);
      like = __builtin_amdgcn_readlane(ge - gt, at);
      break;
    }
    int32_t* later = bins + (which == 0 ? kFirstBins : kFirstBins + kLaterBins);
    each_run([&](int first) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kRun; ++i)
        if (first + i < items && keys[i] != 0 && (keys[i] ^ key) >> shift == 0) count(later, keys[i], which == 0 ? 10 : 0, kLaterBins);
    });
  }
  const bool exact = like == need;                             // all keys that begin with `key`, else the first `need` that equal it

  // ---- who stays -----------------------------------------------------------------------------------------------------
  // lanes 16 j .. 16 j + 15: the j-th number of every wave; row j of `all` and `before` has its sums over all waves and over those
  // before this one
  struct Sums {
    int all, before;
  };
  auto over_waves = [&](int which, int c0, int c1) __attribute__((always_inline)) {
    if (lane < 2) sums[which][lane][wave] = lane == 0 ? c0 : c1;
    __syncthreads();
    const int of = lane & 15, v = of < WAVES && lane < 32 ? sums[which][lane >> 4][of] : 0;
    return Sums{row16_add_int(v), row16_add_int(of < wave ? v : 0)};
  };
  auto rank_in = [](uint64_t votes) { return static_cast<int>(__builtin_amdgcn_mbcnt_hi(votes >> 32, __builtin_amdgcn_mbcnt_lo(votes, 0))); };
  int ties = 0;                                                // equal keys of the waves before
  if (!exact) {
    int same = 0;
    each_run([&](int) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) same += __builtin_popcountll(__ballot(keys[i] == key));
    });
    ties = __builtin_amdgcn_readlane(over_waves(1, same, 0).before, 0);
  }
  // Calls f(token of lane 0, votes: who of the item's tokens lies before the budget, who is kept) for the wave's items.
  auto each_item = [&](auto&& f) __attribute__((always_inline)) {
    int r = ties;
    each_run([&](int first) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < kRun; ++i) {
        const int t0 = start + (first + i) * 64, in_front = a.budget - t0;
        if (t0 >= end) continue;
        const uint64_t front = in_front >= 64 ? ~0ull : (in_front > 0 ? (1ull << in_front) - 1 : 0ull);
        uint64_t kept = __ballot(keys[i] >= key);
        if (!exact) {
          const uint64_t same = __ballot(keys[i] == key);
          if (same != 0) {
            kept = __ballot(keys[i] > key || (keys[i] == key && r + rank_in(same) < need));
            r += __builtin_popcountll(same);
          }
        }
        f(t0, front, kept);
      }
    });
  };
  int holes = 0, movers = 0;
  uint32_t votes_lo = 0, votes_hi = 0;                         // (lane i: who of item i's tokens is kept)
  each_item([&](int t0, uint64_t front, uint64_t kept) __attribute__((always_inline)) {
    holes += __builtin_popcountll(front & ~kept);
    movers += __builtin_popcountll(kept & ~front);
    if (KEYS == Keys::lds) {
      const bool mine = lane == (t0 - start) >> 6;
      votes_lo = mine ? static_cast<uint32_t>(kept) : votes_lo;
      votes_hi = mine ? static_cast<uint32_t>(kept >> 32) : votes_hi;
    }
  });
  const int any = holes + movers;
  const Sums s = over_waves(2, holes, movers);
  holes = __builtin_amdgcn_readlane(s.before, 0);
  movers = __builtin_amdgcn_readlane(s.before, 16);
  // (as many holes as movers)
  const int moves = min(min(__builtin_amdgcn_readlane(s.all, 0), __builtin_amdgcn_readlane(s.all, 16)), plan.most);
  auto write_lists = [&](int32_t* to, int32_t* from) __attribute__((always_inline)) {
    if constexpr (KEYS == Keys::lds) {
      // Lane i has item i's votes and writes its tokens down one after the other; an item with many - holes, the newest - is written down by
      // all lanes.
      static_assert(kLdsItems <= 64, "a lane has one item");
      auto write_down = [&](uint64_t who, int before, int32_t* list) __attribute__((always_inline)) {
        const int many = __builtin_popcountll(who);
        int r = before + wave_prefix(many) - many;
        for (uint64_t full = __ballot(many > kFewMovers); full != 0; full &= full - 1) {
          const int item = __builtin_ctzll(full);
          const uint64_t votes = of_lane(static_cast<uint32_t>(who), static_cast<uint32_t>(who >> 32), item);
          const int place = __builtin_amdgcn_readlane(r, item) + rank_in(votes);
          if (__builtin_amdgcn_inverse_ballot_w64(votes) && place < moves) list[place] = start + item * 64 + lane;
          if (lane == item) who = 0;
        }
        while (__ballot(who != 0) != 0) {
          if (who != 0) {
            if (r < moves) list[r] = start + lane * 64 + __builtin_ctzll(who);
            ++r;
            who &= who - 1;
          }
        }
      };
      const int in_front = a.budget - (start + lane * 64);
      const uint64_t front = in_front >= 64 ? ~0ull : (in_front > 0 ? (1ull << in_front) - 1 : 0ull);
      const uint64_t kept = static_cast<uint64_t>(votes_hi) << 32 | votes_lo;
      write_down(kept & ~front, movers, from);
      if (start < a.budget) write_down(lane < items ? front & ~kept : 0ull, holes, to);
      return;
    }
    each_item([&](int t0, uint64_t front, uint64_t kept) __attribute__((always_inline)) {
      const uint64_t go = front & ~kept, come = kept & ~front;
      if (go != 0) {
        const int r = holes + rank_in(go);
        if (__builtin_amdgcn_inverse_ballot_w64(go) && r < moves) to[r] = t0 + lane;
        holes += __builtin_popcountll(go);
      }
      if (come != 0) {
        const int r = movers + rank_in(come);
        if (__builtin_amdgcn_inverse_ballot_w64(come) && r < moves) from[r] = t0 + lane;
        movers += __builtin_popcountll(come);
      }
    });
  };
  if (plan.few) {
    if (any > 0) write_lists(bins, bins + kFewMoves);
    __syncthreads();
    // (records by the last threads, rows by the first: few of both go side by side)
    if (pages <= kHeldPages) move_rows<kThreads, true>(a, plan, h, [&](int page) { return ids[page]; }, bins, bins + kFewMoves, moves, 0);
    else move_rows<kThreads, true>(a, plan, h, [&](int page) { return pt[page]; }, bins, bins + kFewMoves, moves, 0);
    move_records<kThreads>(a, base, bins, bins + kFewMoves, moves);
  } else {
    int32_t* to = workspace + list_start(static_cast<int64_t>(a.B) * a.n_kv) + static_cast<int64_t>(blockIdx.x) * 2 * plan.most;
    if (any > 0) write_lists(to, to + plan.most);
    __syncthreads();
    if (tid == 0) workspace[blockIdx.x] = moves;
    move_records<kThreads>(a, base, to, to + plan.most, moves);
  }
  if (h == 0 && tid == 0) a.lens_out[b] = a.budget;
}

// A workgroup: the rows that its 256 threads move four each of at a time, about (the grid has room for `most` moves of a head).
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a, EvictPlan plan) {
  const int32_t* workspace = static_cast<const int32_t*>(a.workspace);
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int32_t* to = workspace + list_start(static_cast<int64_t>(a.B) * a.n_kv) + static_cast<int64_t>(blockIdx.x) * 2 * plan.most;
  const int32_t* pt = a.page_table + b * a.ld_pt;
  const int moves = workspace[blockIdx.x], rows = 4 * (256 / (2 * plan.units));
  for (int begin = blockIdx.y * rows; begin < moves; begin += gridDim.y * rows)
    move_rows<256, false>(a, plan, h, [&](int page) { return pt[page]; }, to, to + plan.most, min(begin + rows, moves), begin);
}

static int64_t most_moves(int64_t capacity, int64_t budget) { return std::max<int64_t>(0, std::min(budget, capacity - budget)); }

size_t evict_workspace_bytes(int32_t B, int32_t n_kv, int64_t capacity, int32_t budget) {
  const int64_t heads = static_cast<int64_t>(B) * n_kv, most = most_moves(capacity, budget);
  return static_cast<size_t>(list_start(heads) + (most > kFewMoves ? 2 * most * heads : 0)) * 4;
}

int32_t launch_evict_paged(const EvictArgs& a, hipStream_t st) {
  if (a.B == 0) return RPTQ_OK;
  const int64_t room = std::min<int64_t>(static_cast<int64_t>(a.pages_per_seq) << a.g.page_shift, a.capacity);
  const int head_bytes = a.hd * a.bits / 8;
  EvictPlan p;
  p.most = static_cast<int32_t>(most_moves(room, a.budget));
  p.vec = head_bytes % 16 == 0 ? 16 : (head_bytes % 8 == 0 ? 8 : 4);
  p.units = head_bytes / p.vec;
  p.few = p.most <= kFewMoves;
  const int64_t heads = static_cast<int64_t>(a.B) * a.n_kv;
  auto go = [&](auto kern, int waves) { hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(heads)), dim3(waves * 64), 0, st, a, p); };
  if (room <= 8 * 64 * kFewItems) go(evict_select_kernel<8, Keys::registers>, 8);
  else if (room <= 16 * 64 * kFewItems) go(evict_select_kernel<16, Keys::registers>, 16);
  else if (room <= 16 * 64 * kLdsItems) go(evict_select_kernel<16, Keys::lds>, 16);
  else go(evict_select_kernel<16, Keys::made>, 16);
  RPTQ_HIP(hipGetLastError());
  if (p.few) return RPTQ_OK;
  const int rows = 4 * (256 / (2 * p.units)), chunks = std::min((p.most + rows - 1) / rows, kMoveChunks);
  hipLaunchKernelGGL(evict_move_kernel, dim3(static_cast<unsigned>(heads), chunks), dim3(256), 0, st, a, p);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
