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

#include "device_common.h"
#include "rptq_internal.h"

namespace rptq {

constexpr int kItems = 32;                     // keys of a lane that stay in registers
constexpr int kFewMoves = 2048;                // of a head at most where the workgroup that finds them does them
constexpr int kMoveRows = 64;                  // of a workgroup of the second launch at a time
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

// Rows number first, first + step, ... of the list, by threads of `row_threads` = 2 units each.
template <typename V>
__device__ __forceinline__ void move_rows(const EvictArgs& a, int units, int b, int h, const int32_t* to, const int32_t* from, int first, int end, int step,
                                          int which) {
  const int row_bytes = 16 * a.bits, head_bytes = a.hd * a.bits / 8;
  const bool values = which >= units;
  const int off = (which - (values ? units : 0)) * static_cast<int>(sizeof(V));       // of the head's row
  // heads over 128 wide: the row lies in several blocks; others share one
  const int64_t place = static_cast<int64_t>(h) * head_bytes + off;
  const int block = static_cast<int>(place / row_bytes), in_row = static_cast<int>(place - static_cast<int64_t>(block) * row_bytes);
  uint8_t* pages = values ? a.v_pages : a.k_pages;
  const int32_t* pt = a.page_table + b * a.ld_pt;
  auto at = [&](int t) {
    const int64_t page = pt[t >> a.g.page_shift];
    const int64_t row = ((page * (a.g.d / kPageBlock) + block) << a.g.page_shift) + (t & ((1 << a.g.page_shift) - 1));
    return reinterpret_cast<V*>(pages + row * row_bytes + in_row);
  };
  for (int i = first; i < end; i += 4 * step) {
    V x[4];
    int t[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const int j = min(i + k * step, end - 1);
      x[k] = *at(from[j]);
      t[k] = to[j];
    }
#pragma unroll
    for (int k = 0; k < 4; ++k)
      if (i + k * step < end) *at(t[k]) = x[k];
  }
}

__device__ __forceinline__ void move_rows(const EvictArgs& a, const EvictPlan& p, int b, int h, const int32_t* to, const int32_t* from, int begin, int end,
                                          int threads) {
  const int each = 2 * p.units, rows = threads / each, row = threadIdx.x / each, which = threadIdx.x - row * each;
  if (row >= rows) return;
  if (p.vec == 16) move_rows<uint4>(a, p.units, b, h, to, from, begin + row, end, rows, which);
  else if (p.vec == 8) move_rows<uint2>(a, p.units, b, h, to, from, begin + row, end, rows, which);
  else move_rows<uint32_t>(a, p.units, b, h, to, from, begin + row, end, rows, which);
}

__device__ __forceinline__ int dpp_row_sum(int v) {            // over the 16 lanes of a row
  v += __builtin_amdgcn_update_dpp(0, v, 0xB1, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x4E, 0xf, 0xf, false);
  v += __builtin_amdgcn_update_dpp(0, v, 0x141, 0xf, 0xf, false);
  return v + __builtin_amdgcn_update_dpp(0, v, 0x140, 0xf, 0xf, false);
}

// WAVES: of the workgroup; REG: keys in registers (up to WAVES * 64 * kItems tokens)
template <int WAVES, bool REG>
__global__ void __launch_bounds__(WAVES * 64) evict_select_kernel(EvictArgs a, EvictPlan plan) {
  __shared__ int32_t counts[2][4][16];
  __shared__ int32_t few_lists[2][kFewMoves];
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

  int gone = 0;                                                // (a page that is not there: the sequence stays as it is)
  if (n > a.budget) {
    const int32_t* pt = a.page_table + b * a.ld_pt;
    for (int p = tid; p <= (n - 1) >> a.g.page_shift; p += WAVES * 64) gone |= pt[p] < 0 || pt[p] >= a.g.n_pages;
  }
  gone = __syncthreads_or(gone);
  const bool cut = n > a.budget && !gone;
  const int left = cut ? a.budget : n;
  if (h == 0 && tid == 0) a.lens_out[b] = left;
  if (!cut) {
    if (!plan.few && tid == 0) workspace[blockIdx.x] = 0;
    if (weights_out != weights)
      for (int t = tid; t < n; t += WAVES * 64) weights_out[t] = weights[t];
    if (positions_out != positions)
      for (int t = tid; t < n; t += WAVES * 64) positions_out[t] = positions[t];
    return;
  }

  // a wave's tokens: `items` times 64 consecutive ones
  const int items = ((n + WAVES - 1) / WAVES + 63) >> 6, start = wave * items * 64;
  auto token = [&](int i) { return start + i * 64 + lane; };
  int newest = INT32_MIN;
  if (a.recent > 0) {
    for (int i = 0; i < items; ++i)
      if (token(i) < n) newest = max(newest, positions[token(i)]);
#pragma unroll
    for (int s = 32; s > 0; s >>= 1) newest = max(newest, __shfl_xor(newest, s, kWave));
    if (lane == 0) counts[0][0][wave] = newest;
    __syncthreads();
    newest = counts[0][0][lane % WAVES];
#pragma unroll
    for (int s = WAVES / 2; s > 0; s >>= 1) newest = max(newest, __shfl_xor(newest, s, kWave));
    __syncthreads();
  }
  const int64_t young = static_cast<int64_t>(newest) - a.recent;       // positions beyond are safe
  // 0: no token.  (A weight's key is at least 0x007fffff, minus infinity's.)
  auto make_key = [&](int i) -> uint32_t {
    const int t = token(i);
    if (t >= n) return 0u;
    const float w = weights[t];
    const int pos = positions[t];
    if (pos < a.first || (a.recent > 0 && pos > young)) return kSafe;
    if (w != w) return kNanKey;
    return float_key(w + 0.0f);                                // (minus zero is zero)
  };
  uint32_t held[REG ? kItems : 1];
  if constexpr (REG) {
#pragma unroll
    for (int i = 0; i < kItems; ++i) held[i] = i < items ? make_key(i) : 0u;
  }
  // calls f(i, key) for the wave's items in order
  auto each_key = [&](auto&& f) {
    if constexpr (REG) {
#pragma unroll
      for (int i = 0; i < kItems; ++i)
        if (i < items) f(i, held[i]);
    } else {
      for (int i = 0; i < items; ++i) f(i, make_key(i));
    }
  };
  // sums over the waves of up to four numbers, and over the waves before this one of the same
  int turn = 0;
  struct Sums {
    int all[4], before[4];
  };
  auto over_waves = [&](int c0, int c1, int c2, int c3) {
    if (lane < 4) counts[turn][lane][wave] = lane == 0 ? c0 : (lane == 1 ? c1 : (lane == 2 ? c2 : c3));
    __syncthreads();
    const int w = lane & 15, v = w < WAVES ? counts[turn][lane >> 4][w] : 0;
    const int all = dpp_row_sum(v), before = dpp_row_sum(w < wave ? v : 0);
    Sums s;
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      s.all[j] = __builtin_amdgcn_readlane(all, j * 16);
      s.before[j] = __builtin_amdgcn_readlane(before, j * 16);
    }
    turn ^= 1;                                                 // (the next call's barrier lies between this call's reads and the use after next)
    return s;
  };

  uint32_t key = 0;                                            // at least `budget` keys reach it
  bool exact = false;
  for (int bit = 30; bit >= 0 && !exact; bit -= 2) {
    const uint32_t k1 = key | 1u << bit, k2 = key | 2u << bit, k3 = key | 3u << bit;
    int c1 = 0, c2 = 0, c3 = 0;
    each_key([&](int, uint32_t k) {
      c1 += __builtin_popcountll(__ballot(k >= k1));
      c2 += __builtin_popcountll(__ballot(k >= k2));
      c3 += __builtin_popcountll(__ballot(k >= k3));
    });
    const Sums s = over_waves(c1, c2, c3, 0);
    const int reach = s.all[2] >= a.budget ? 2 : (s.all[1] >= a.budget ? 1 : (s.all[0] >= a.budget ? 0 : -1));
    if (reach >= 0) {
      key = reach == 2 ? k3 : (reach == 1 ? k2 : k1);
      exact = (reach == 2 ? s.all[2] : (reach == 1 ? s.all[1] : s.all[0])) == a.budget;
    }
  }
  // of the keys that equal it, the first so many are kept
  int ties = 0, tie_rank = 0;
  if (!exact) {
    int over = 0, same = 0;
    each_key([&](int, uint32_t k) {
      over += __builtin_popcountll(__ballot(k > key));
      same += __builtin_popcountll(__ballot(k == key));
    });
    const Sums s = over_waves(over, same, 0, 0);
    ties = a.budget - s.all[0];
    tie_rank = s.before[1];
  }
  const uint64_t below = (1ull << lane) - 1;
  // calls f(i, votes for kept) for the wave's items in order
  auto each_kept = [&](auto&& f) {
    int rank = tie_rank;
    each_key([&](int i, uint32_t k) {
      bool keep = exact ? k >= key : k > key;
      if (!exact) {
        const uint64_t same = __ballot(k == key);
        keep = keep || (k == key && rank + __builtin_popcountll(same & below) < ties);
        rank += __builtin_popcountll(same);
      }
      f(i, __ballot(keep));
    });
  };
  int holes = 0, movers = 0;
  auto hole_votes = [&](int i, uint64_t kept) { return __ballot(token(i) < a.budget && !(kept >> lane & 1)); };
  auto mover_votes = [&](int i, uint64_t kept) { return __ballot(token(i) >= a.budget && (kept >> lane & 1)); };
  each_kept([&](int i, uint64_t kept) {
    holes += __builtin_popcountll(hole_votes(i, kept));
    movers += __builtin_popcountll(mover_votes(i, kept));
  });
  const Sums s = over_waves(holes, movers, 0, 0);
  const int moves = min(s.all[0], plan.most);                  // (as many holes as movers)
  int32_t* list = workspace + list_start(static_cast<int64_t>(a.B) * a.n_kv) + static_cast<int64_t>(blockIdx.x) * 2 * plan.most;
  int32_t* to = plan.few ? few_lists[0] : list;
  int32_t* from = plan.few ? few_lists[1] : list + plan.most;
  holes = s.before[0], movers = s.before[1];
  each_kept([&](int i, uint64_t kept) {
    const uint64_t hv = hole_votes(i, kept), mv = mover_votes(i, kept);
    const int hr = holes + __builtin_popcountll(hv & below), mr = movers + __builtin_popcountll(mv & below);
    if ((hv >> lane & 1) && hr < moves) to[hr] = token(i);
    if ((mv >> lane & 1) && mr < moves) from[mr] = token(i);
    if ((kept >> lane & 1) && token(i) < a.budget) {           // (those that stay)
      const int t = token(i);
      if (weights_out != weights) weights_out[t] = weights[t];
      if (positions_out != positions) positions_out[t] = positions[t];
    }
    holes += __builtin_popcountll(hv);
    movers += __builtin_popcountll(mv);
  });
  __syncthreads();
  for (int i = tid; i < moves; i += WAVES * 64) {
    weights_out[to[i]] = weights[from[i]];
    positions_out[to[i]] = positions[from[i]];
  }
  if (plan.few) move_rows(a, plan, b, h, to, from, 0, moves, WAVES * 64);
  else if (tid == 0) workspace[blockIdx.x] = moves;
}

__global__ void __launch_bounds__(256) evict_move_kernel(EvictArgs a, EvictPlan plan) {
  const int32_t* workspace = static_cast<const int32_t*>(a.workspace);
  const int moves = workspace[blockIdx.x];
  const int b = blockIdx.x / a.n_kv, h = blockIdx.x - b * a.n_kv;
  const int32_t* to = workspace + list_start(static_cast<int64_t>(a.B) * a.n_kv) + static_cast<int64_t>(blockIdx.x) * 2 * plan.most;
  for (int begin = blockIdx.y * kMoveRows; begin < moves; begin += gridDim.y * kMoveRows)
    move_rows(a, plan, b, h, to, to + plan.most, begin, min(begin + kMoveRows, moves), 256);
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
  if (room <= 4 * 64 * kItems) go(evict_select_kernel<4, true>, 4);
  else if (room <= 16 * 64 * kItems) go(evict_select_kernel<16, true>, 16);
  else go(evict_select_kernel<16, false>, 16);
  RPTQ_HIP(hipGetLastError());
  if (p.few) return RPTQ_OK;
  const int chunks = std::min((p.most + kMoveRows - 1) / kMoveRows, kMoveChunks);
  hipLaunchKernelGGL(evict_move_kernel, dim3(static_cast<unsigned>(heads), chunks), dim3(256), 0, st, a, p);
  RPTQ_HIP(hipGetLastError());
  return RPTQ_OK;
}

}  // namespace rptq
