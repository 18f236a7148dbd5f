// What the kernels that move rows between tensors and the cache's pages share: which rows and channels a wave has, its table
// records, and where its rows lie.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

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
  int32_t groups;                                    // of workgroups that share the rows
  int32_t run_shift;                                 // log2 of the rows that a wave takes of every run of rows
};

// A launch of `grid` workgroups of four waves (kv_paged.hip).
int32_t paged_launch(const PagedTensor& k, const PagedTensor& v, const int64_t* slots, int64_t T, const PagedGeom& g,
                     hipStream_t st, PagedLaunch* a, unsigned* grid);

// Which tile, tensor and rows a wave has.  Rows go round the groups in runs of eight, two of each of the workgroup's
// waves: the rows of a run are neighbours in a page as a rule, so that a workgroup moves whole cache lines of codes, and the
// runs under way at one time are neighbours in x.
struct PagedShare {
  int base_ch, n_here;                               // first channel, channels (a multiple of 128)
  bool values;
  int64_t first;                                     // the wave's first row
  int64_t stride;                                    // rows from run to run
  int32_t run_shift;
  __device__ __forceinline__ int64_t row(int i) const {
    return first + (i >> run_shift) * stride + 4 * (i & ((1 << run_shift) - 1));
  }
};

__device__ __forceinline__ PagedShare paged_share(const PagedLaunch& a, unsigned group) {
  PagedShare s;
  const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
  const unsigned per = static_cast<unsigned>(a.segs) * 2;
  const unsigned which = group % per;
  s.values = which >= static_cast<unsigned>(a.segs);
  s.base_ch = static_cast<int>(which - (s.values ? a.segs : 0)) * kKvTile;
  s.n_here = min(a.g.d - s.base_ch, kKvTile);
  s.run_shift = a.run_shift;
  s.first = (static_cast<int64_t>(group / per) << (2 + a.run_shift)) + wave;
  s.stride = static_cast<int64_t>(a.groups) << (2 + a.run_shift);
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

// Where a wave's rows lie: a lane holds the place of one of 64 in its page's first block, in bytes from the pages' start, or
// -1.  The next 64 are requested while these are worked on: a row's slot is never waited for on its own.
template <int BITS>
struct SlotWindow {
  int64_t here, next;
  int from;
  const PagedLaunch& a;
  const PagedShare& s;
  __device__ __forceinline__ int64_t at(int i) const {
    const int64_t slot = a.slots[min(s.row(i), a.T - 1)];
    const int64_t page = slot >> a.g.page_shift, r = slot & ((INT64_C(1) << a.g.page_shift) - 1);
    const bool ok = slot >= 0 && slot < (a.g.n_pages << a.g.page_shift);
    return ok ? ((page * (a.g.d / kPageBlock) << a.g.page_shift) + r) * (16 * BITS) : -1;
  }
  __device__ __forceinline__ SlotWindow(const PagedLaunch& launch, const PagedShare& share, int lane) : from(0), a(launch), s(share) {
    here = at(lane);
    next = s.row(64) < a.T ? at(64 + lane) : -1;
  }
  // (i: the number of one of the wave's rows, uniform, at most 127 more than `from`)
  __device__ __forceinline__ int64_t place(int i) const {
    const int64_t v = i - from < 64 ? here : next;
    const uint32_t lo = __builtin_amdgcn_readlane(static_cast<uint32_t>(v), i & 63);
    const uint32_t hi = __builtin_amdgcn_readlane(static_cast<uint32_t>(v >> 32), i & 63);
    return static_cast<int64_t>(static_cast<uint64_t>(hi) << 32 | lo);
  }
  __device__ __forceinline__ void move_to(int i, int lane) {
    if (i - from < 64) return;
    from += 64;
    here = next;
    next = s.row(from + 64) < a.T ? at(from + 64 + lane) : -1;
  }
};

// Bytes from a row's place to this lane's 16 positions of it (3 bits: to the group that it shares with a neighbour).
template <int BITS>
__device__ __forceinline__ int64_t paged_lane(const PagedGeom& g, int block, int lane) {
  return (static_cast<int64_t>(block) << g.page_shift) * (16 * BITS) + (BITS == 3 ? ((lane & 7) >> 1) * 12 : (lane & 7) * 2 * BITS);
}

}  // namespace rptq
