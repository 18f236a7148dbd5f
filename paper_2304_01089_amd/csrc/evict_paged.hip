// Eviction from the paged cache: every key/value head of a sequence longer than its budget keeps `budget` tokens - the first, the
// newest, then the heaviest, ties to the lowest index - and the kept tokens behind the budget move, in their order, into the
// holes that the others leave before it.  A move is a row of codes of keys and one of values and the token's record; what lies
// before the budget and is kept stays where it is, so a step that evicts one token moves one.  (Attention does not depend on
// the order of the tokens; a token's position is in its record.)
//
// One workgroup per (sequence, head) finds the threshold: a token's key is its weight's bits in an order of whole numbers, and the
// budget-th largest key is found two bits at a time, every wave counting its tokens' keys that reach the three candidates by votes;
// a count that hits the budget ends it.  A wave has a run of consecutive tokens, so the order among equal keys and the
// places in the lists of holes and movers are counts of votes, too.  Keys stay in registers up to 32 per lane.
// Few moves are done by the same workgroup, many by a second launch over the whole chip.
// What bounds it: a chain of short steps, some of them across the workgroup's waves; long prompts: memory.
#include <hip/hip_runtime.h>

#include <algorithm>

#include "attend_common.h"
#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kBins = 2048;                    // of eleven bits of a key
constexpr int kHeldPages = 1024;               // page numbers of a sequence that are kept at hand
constexpr int kFewMoves = 2048;                // of a head at most where the workgroup that finds them does them
constexpr int kMoveChunks = 1024;              // workgroups of a head there at most
constexpr uint32_t kSafe = 0xffffffffu, kNanKey = 0xfffffffeu;

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

// Rows number first, first + step, ... of the lists: the thread's `which`-th of 2 units pieces.  page_of: a page's number.
template <typename V, typename P>
__device__ __forceinline__ void move_pieces(const EvictArgs& a, int units, int h, P&& page_of, const int32_t* to, const int32_t* from, int first, int end,
                                            int step, int which) {
  const int row_bytes = 16 * a.bits, head_bytes = a.hd * a.bits / 8;
  const bool values = which >= units;
  const int off = (which - (values ? units : 0)) * static_cast<int>(sizeof(V));       // of the head's row
  // heads over 128 wide: the row lies in several blocks; others share one
  const int64_t place = static_cast<int64_t>(h) * head_bytes + off;
  const int block = static_cast<int>(place / row_bytes), in_row = static_cast<int>(place - static_cast<int64_t>(block) * row_bytes);
  uint8_t* pages = (values ? a.v_pages : a.k_pages) + in_row;
  const int blocks = a.g.d / kPageBlock, shift = a.g.page_shift;
  auto at = [&](int t) __attribute__((always_inline)) {
    const int64_t row = ((static_cast<int64_t>(page_of(t >> shift)) * blocks + block) << shift) + (t & ((1 << shift) - 1));
    return reinterpret_cast<V*>(pages + row * row_bytes);
  };
  for (int i = first; i < end; i += 4 * step) {
    const int i1 = min(i + step, end - 1), i2 = min(i + 2 * step, end - 1), i3 = min(i + 3 * step, end - 1);
    const V x0 = *at(from[i]), x1 = *at(from[i1]), x2 = *at(from[i2]), x3 = *at(from[i3]);
    V *y0 = at(to[i]), *y1 = at(to[i1]), *y2 = at(to[i2]), *y3 = at(to[i3]);
    *y0 = x0;                                                  // (the last row several times, if need be: the same bytes)
    *y1 = x1;
    *y2 = x2;
    *y3 = x3;
  }
}

template <int THREADS, typename P>
__device__ __forceinline__ void move_rows(const EvictArgs& a, const EvictPlan& p, int h, P&& page_of, const int32_t* to, const int32_t* from, int moves,
                                          int begin) {
  const int each = 2 * p.units, rows = THREADS / each, row = static_cast<int>(threadIdx.x) / each, which = static_cast<int>(threadIdx.x) - row * each;
  if (row >= rows) return;
  if (p.vec == 16) move_pieces<uint4>(a, p.units, h, page_of, to, from, begin + row, moves, rows, which);
  else if (p.vec == 8) move_pieces<uint2>(a, p.units, h, page_of, to, from, begin + row, moves, rows, which);
  else move_pieces<uint32_t>(a, p.units, h, page_of, to, from, begin + row, moves, rows, which);
}

__device__ __forceinline__ int wave_max_int(int v) {
#pragma unroll
  for (int s = 32; s > 0; s >>= 1) v = max(v, __shfl_xor(v, s, kWave));
  return v;
}

// Over the 16 lanes of a row.
__device__ __forceinline__ int row16_add_int(int v) {
  v += static_cast<int>(dpp_row<0xB1>(static_cast<uint32_t>(v)));
  v += static_cast<int>(dpp_row<0x4E>(static_cast<uint32_t>(v)));
  v += static_cast<int>(dpp_row<0x141>(static_cast<uint32_t>(v)));
  return v + static_cast<int>(dpp_row<0x140>(static_cast<uint32_t>(v)));
}

// WAVES: of the workgroup; ITEMS: keys of a lane that stay in registers; LONG: a wave's tokens are more than 64 of those, whose keys are
// made again whenever they are looked at
template <int WAVES, int ITEMS, bool LONG>
__global__ void __launch_bounds__(WAVES * 64) evict_select_kernel(EvictArgs a, EvictPlan plan) {
  constexpr int kThreads = WAVES * 64;
  __shared__ __align__(16) int32_t bins[3 * kBins];            // (later the lists of a few moves)
  __shared__ int32_t ids[kHeldPages];
  __shared__ int32_t groups[3][64];                            // of 32 bins each
  __shared__ int32_t sums[3][4][16];
  static_assert(2 * kFewMoves <= 3 * kBins, "the lists take the bins' place");
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int n = min(max(a.lens[b], 0), evict_room(a));
  const int64_t base = static_cast<int64_t>(blockIdx.x) * a.capacity;
  const float* weights = a.weights + base;
  const int32_t* positions = a.positions + base;
  float* weights_out = a.weights_out + base;
  int32_t* positions_out = a.positions_out + base;
  int32_t* workspace = static_cast<int32_t*>(a.workspace);
  auto leave = [&] {                                           // the sequence as it is
    if (h == 0 && tid == 0) a.lens_out[b] = n;
    if (!plan.few && tid == 0) workspace[blockIdx.x] = 0;
    if (weights_out != weights) copy<kThreads>(weights_out, weights, n);
    if (positions_out != positions) copy<kThreads>(positions_out, positions, n);
  };
  if (n <= a.budget) {
    leave();
    return;
  }

  // a wave's tokens: `items` times 64 consecutive ones
  const int items = ((n + WAVES - 1) / WAVES + 63) >> 6, start = wave * items * 64;
  float w[ITEMS];
  int32_t pos[ITEMS];
  auto read = [&](int first) __attribute__((always_inline)) {  // (beyond the end: the last token)
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      if (first + i >= items) continue;
      const int t = min(start + (first + i) * 64 + lane, n - 1);
      w[i] = weights[t];
      pos[i] = positions[t];
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
  for (int i = tid; i < 3 * kBins / 4; i += kThreads) reinterpret_cast<int4*>(bins)[i] = make_int4(0, 0, 0, 0);
  int newest = INT32_MIN;
  if (a.recent > 0) {
    for (int first = 0; first < items; first += ITEMS) {
      if (LONG && first > 0) read(first);
#pragma unroll
      for (int i = 0; i < ITEMS; ++i)
        if (first + i < items) newest = max(newest, pos[i]);
    }
    if (LONG) read(0);
    newest = wave_max_int(newest);
  }
  const bool wave_gone = __ballot(gone) != 0;
  if (lane == 0) sums[0][0][wave] = newest, sums[0][1][wave] = wave_gone;
  __syncthreads();
  if (__ballot(sums[0][1][lane & (WAVES - 1)] != 0) != 0) {
    leave();
    return;
  }
  if (h == 0 && tid == 0) a.lens_out[b] = a.budget;
  if (a.recent > 0) newest = wave_max_int(sums[0][0][lane & (WAVES - 1)]);
  const int64_t young = static_cast<int64_t>(newest) - a.recent;       // positions beyond are safe
  uint32_t keys[ITEMS];                                        // (of a token that there is not: 0.  A weight's is at least 0x007fffff, minus infinity's)
  auto make_keys = [&](int first) __attribute__((always_inline)) {
#pragma unroll
    for (int i = 0; i < ITEMS; ++i) {
      keys[i] = 0;
      if (first + i >= items) continue;
      uint32_t k = w[i] == w[i] ? float_key(w[i] + 0.0f) : kNanKey;    // (minus zero is zero)
      if (pos[i] < a.first || (a.recent > 0 && pos[i] > young)) k = kSafe;
      keys[i] = start + (first + i) * 64 + lane < n ? k : 0;
    }
  };
  if (!LONG) make_keys(0);
  // calls f(first) with the records and keys of items first .. first + ITEMS - 1 at hand
  auto each_run = [&](auto&& f) __attribute__((always_inline)) {
    if constexpr (LONG) {
      for (int first = 0; first < items; first += ITEMS) {
        read(first);
        make_keys(first);
        f(first);
      }
    } else {
      f(0);
    }
  };

  // ---- the budget-th largest key, eleven bits at a time (the last time ten) from the top ----------------------------
  // All waves count into the same bins and sum them in groups of 32; then every wave finds by itself the group, and in it the bin,
  // where the sum from the top reaches what is needed.
  uint32_t key = 0;                                            // the bits that are known
  int need = a.budget;                                         // that many keys of those that begin with them
  bool exact = false;                                          // ... which are all of them
  auto look = [&](int which, int shift, int size) __attribute__((always_inline)) {
    int32_t* mine = bins + which * kBins;
    each_run([&](int first) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const uint32_t k = keys[i];
        if (first + i < items && k != 0 && (which == 0 || (k ^ key) >> shift < static_cast<uint32_t>(size)))
          atomicAdd(&mine[k >> shift & (size - 1)], 1);
      }
    });
    __syncthreads();
    // (a lane sums its few bins, neighbours the 32 of a group)
    constexpr int kEach = kBins / kThreads;
    int part = 0;
#pragma unroll
    for (int i = 0; i < kEach; ++i) part += mine[tid * kEach + i];
    part += static_cast<int>(dpp_row<0xB1>(static_cast<uint32_t>(part)));
    part += static_cast<int>(dpp_row<0x4E>(static_cast<uint32_t>(part)));
    if (kEach < 8) part += static_cast<int>(dpp_row<0x141>(static_cast<uint32_t>(part)));
    if (kEach < 4) part += static_cast<int>(dpp_row<0x140>(static_cast<uint32_t>(part)));
    if ((lane & (32 / kEach - 1)) == 0) groups[which][tid / (32 / kEach)] = part;
    __syncthreads();
    const int sum = groups[which][63 - lane];
    const int upto = wave_prefix(sum);
    const int l = __builtin_ctzll(__ballot(upto >= need));     // (there is one: as many keys as are needed are in the bins)
    const int over = __builtin_amdgcn_readlane(upto - sum, l);
    const int bin = kBins - 1 - 32 * l - (lane & 31), c = lane < 32 ? mine[bin] : 0;
    const int upto2 = over + wave_prefix(c);
    const int m = __builtin_ctzll(__ballot(upto2 >= need));
    const int count = __builtin_amdgcn_readlane(c, m);
    key |= static_cast<uint32_t>(kBins - 1 - 32 * l - m) << shift;
    need -= __builtin_amdgcn_readlane(upto2, m) - count;
    exact = count == need;
  };
  look(0, 21, kBins);
  if (!exact) look(1, 10, kBins);
  if (!exact) look(2, 0, kBins / 2);

  // ---- who stays: bit i of a lane's word for its item number first + i ----------------------------------------------
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
  const uint64_t below = (1ull << lane) - 1;
  int rank = 0;                                                // of equal keys before the run
  if (!exact) {                                                // (key is the whole key, of which the first `need` are kept)
    int same = 0;
    each_run([&](int first) __attribute__((always_inline)) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) same += __builtin_popcountll(__ballot(keys[i] == key));
    });
    rank = __builtin_amdgcn_readlane(over_waves(1, same, 0).before, 0);
  }
  auto kept = [&](int first) __attribute__((always_inline)) {
    uint32_t mask = 0;
    if (exact) {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) mask |= static_cast<uint32_t>(keys[i] >= key) << i;
    } else {
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        bool keep = keys[i] > key;
        const uint64_t same = __ballot(keys[i] == key);
        if (same != 0) {
          keep = keep || (keys[i] == key && rank + __builtin_popcountll(same & below) < need);
          rank += __builtin_popcountll(same);
        }
        mask |= static_cast<uint32_t>(keep) << i;
      }
    }
    return mask;
  };
  // the items of the run whose tokens lie before the budget
  auto before = [&](int first) {
    const int c = min((a.budget - (start + first * 64 + lane) + 63) >> 6, min(items - first, ITEMS));
    return c >= 32 ? 0xffffffffu : (1u << max(c, 0)) - 1;
  };
  const int rank0 = rank;
  int holes = 0, movers = 0;
  uint32_t stay = 0;                                           // (not LONG: the lane's one word)
  each_run([&](int first) __attribute__((always_inline)) {
    stay = kept(first);
    holes += __builtin_popcount(before(first) & ~stay);
    movers += __builtin_popcount(stay & ~before(first));
  });
  const int holes_here = __builtin_amdgcn_readlane(wave_prefix(holes), 63), movers_here = __builtin_amdgcn_readlane(wave_prefix(movers), 63);
  const Sums s = over_waves(2, holes_here, movers_here);
  holes = __builtin_amdgcn_readlane(s.before, 0);
  movers = __builtin_amdgcn_readlane(s.before, 16);
  // (as many holes as movers)
  const int moves = min(min(__builtin_amdgcn_readlane(s.all, 0), __builtin_amdgcn_readlane(s.all, 16)), plan.most);
  int32_t* list = workspace + list_start(static_cast<int64_t>(a.B) * a.n_kv) + static_cast<int64_t>(blockIdx.x) * 2 * plan.most;
  int32_t* to = plan.few ? bins : list;
  int32_t* from = plan.few ? bins + kFewMoves : list + plan.most;
  rank = rank0;
  const bool apart = weights_out != weights, pos_apart = positions_out != positions;
  if (holes_here + movers_here > 0 || apart || pos_apart)
    each_run([&](int first) __attribute__((always_inline)) {
      if (LONG) stay = kept(first);
      const uint32_t front = before(first);
      const uint32_t go = front & ~stay, come = stay & ~front;
      if (holes_here > 0)
        for (int i = 0; i < ITEMS && first + i < items; ++i) {
          const uint64_t votes = __ballot(go >> i & 1);
          const int r = holes + __builtin_popcountll(votes & below);
          if ((go >> i & 1) && r < moves) to[r] = start + (first + i) * 64 + lane;
          holes += __builtin_popcountll(votes);
        }
      if (movers_here > 0)
        for (int i = 0; i < ITEMS && first + i < items; ++i) {
          const uint64_t votes = __ballot(come >> i & 1);
          const int r = movers + __builtin_popcountll(votes & below);
          if ((come >> i & 1) && r < moves) from[r] = start + (first + i) * 64 + lane;
          movers += __builtin_popcountll(votes);
        }
      // the records of those that stay where they are
#pragma unroll
      for (int i = 0; i < ITEMS; ++i) {
        const int t = start + (first + i) * 64 + lane;
        if (!(front & stay & 1u << i)) continue;
        if (apart) weights_out[t] = w[i];
        if (pos_apart) positions_out[t] = pos[i];
      }
    });
  __syncthreads();
  // (records by the last threads, rows by the first: few of both go side by side)
  move_records<kThreads>(a, base, to, from, moves);
  if (!plan.few) {
    if (tid == 0) workspace[blockIdx.x] = moves;
  } else if (pages <= kHeldPages) {
    move_rows<kThreads>(a, plan, h, [&](int page) { return ids[page]; }, to, from, moves, 0);
  } else {
    move_rows<kThreads>(a, plan, h, [&](int page) { return pt[page]; }, to, from, moves, 0);
  }
}

// A workgroup: the rows that its 256 threads move four each of at a time, about (the grid has room for `most` moves of a head).
__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a, EvictPlan plan) {
  const int32_t* workspace = static_cast<const int32_t*>(a.workspace);
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int32_t* to = workspace + list_start(static_cast<int64_t>(a.B) * a.n_kv) + static_cast<int64_t>(blockIdx.x) * 2 * plan.most;
  const int32_t* pt = a.page_table + b * a.ld_pt;
  const int moves = workspace[blockIdx.x], rows = 4 * (256 / (2 * plan.units));
  for (int begin = blockIdx.y * rows; begin < moves; begin += gridDim.y * rows)
    move_rows<256>(a, plan, h, [&](int page) { return pt[page]; }, to, to + plan.most, min(begin + rows, moves), begin);
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
  if (room <= 4 * 64 * 8) go(evict_select_kernel<4, 8, false>, 4);
  else if (room <= 16 * 64 * 8) go(evict_select_kernel<16, 8, false>, 16);
  else if (room <= 16 * 64 * 32) go(evict_select_kernel<16, 32, false>, 16);
  else go(evict_select_kernel<16, 32, true>, 16);
  RPTQ_HIP(hipGetLastError());
  if (p.few) return RPTQ_OK;
  const int rows = 4 * (256 / (2 * p.units)), chunks = std::min((p.most + rows - 1) / rows, kMoveChunks);
  hipLaunchKernelGGL(evict_move_kernel, dim3(static_cast<unsigned>(heads), chunks), dim3(256), 0, st, a, p);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
