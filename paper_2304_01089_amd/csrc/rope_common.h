// What the kernels that rotate queries and keys by their positions share: the angle's cosine and sine, and a pair's rotation.
#pragma once
#include <hip/hip_runtime.h>
#include <stdint.h>

#include "launch_rules.h"
#include "rptq_internal.h"

namespace rptq {

struct RopeLaunch {
  RopeArgs a;
  int32_t rows, heads;                         // of a workgroup
  int32_t head_groups, groups;                 // workgroups per `rows` rows, and of this launch
  int32_t turned, units;                       // pieces of a head's rotated channels, and all that are moved
};
// The launch of all rows but for their number; how many rows one launch takes.  W: channels of a piece.
int64_t plan_rope(const RopeArgs& a, int W, bool same, RopeLaunch* l);         // (rope.hip)
// Rows first .. first + rows - 1 of `a` into *l.
void rope_part(const RopeArgs& a, int64_t first, int64_t rows, RopeLaunch* l);

// (cos, sin) of an angle, times `amplitude`, rounded once to fp32.  In 64 bits: at position 10^6 the angle of the fastest pair has
// 20 bits in front of the point, of which fp32 would leave four behind it.  k = round(2 theta / pi); theta - k pi / 2 by two fused
// products with pi / 2 in two pieces (the first is exact); Taylor's series of sine and cosine to the 15th and 16th power, whose next
// terms are below 2^-53 of the result for |r| <= pi / 4.  What is rounded to fp32 is thus within 2^-51 or so of the exact value, or 2^-62 of
// the amplitude (pi / 2's next piece, next to a zero of a far angle), and the fp32 number is the nearest one but for one angle in 2^27 or so.
// This holds up to angles of 2^47 (65536 a position at position 2^31), where k is up to 0.02 off and |r| up to 0.81.  Beyond 2^48 k's own
// rounding leaves ever larger r, and the series soon no cosine: larger angles, and what is no number, become NaN.
__device__ __forceinline__ float2 rope_turn(double theta, double amplitude) {
  const double k = rint(theta * 0.63661977236758134308);
  double r = fma(-k, 1.57079632679489661923, theta);
  r = fma(-k, 6.12323399573676588613e-17, r);
  const double z = r * r;
  double s = -1.0 / 1307674368000.0;                       // 1 / 15!
  s = fma(s, z, 1.0 / 6227020800.0);
  s = fma(s, z, -1.0 / 39916800.0);
  s = fma(s, z, 1.0 / 362880.0);
  s = fma(s, z, -1.0 / 5040.0);
  s = fma(s, z, 1.0 / 120.0);
  s = fma(s, z, -1.0 / 6.0);
  s = fma(s * z, r, r);
  double c = 1.0 / 20922789888000.0;                       // 1 / 16!
  c = fma(c, z, -1.0 / 87178291200.0);
  c = fma(c, z, 1.0 / 479001600.0);
  c = fma(c, z, -1.0 / 3628800.0);
  c = fma(c, z, 1.0 / 40320.0);
  c = fma(c, z, -1.0 / 720.0);
  c = fma(c, z, 1.0 / 24.0);
  c = fma(c, z, -0.5);
  c = fma(c, z, 1.0);
  const int quarter = static_cast<int>(fma(-4.0, floor(k * 0.25), k));
  const double a = quarter & 1 ? s : c, b = quarter & 1 ? c : s;
  const double cos_t = quarter == 1 || quarter == 2 ? -a : a, sin_t = quarter >= 2 ? -b : b;
  const double size = fabs(theta) <= 0x1p47 ? amplitude : __builtin_nan("");
  return make_float2(static_cast<float>(cos_t * size), static_cast<float>(sin_t * size));
}

// (a, b) turned: two products and their sum, each rounded (the order that decides a code).
__device__ __forceinline__ float rope_first(float a, float b, float c, float s) { return __fsub_rn(__fmul_rn(a, c), __fmul_rn(b, s)); }
__device__ __forceinline__ float rope_second(float a, float b, float c, float s) { return __fadd_rn(__fmul_rn(b, c), __fmul_rn(a, s)); }

// n / d for n < 2^16 and m = ceil(2^32 / d): the error n (m d - 2^32) / (d 2^32) is below 1 / d for d <= 2^16.
struct Divisor {
  uint32_t d, m;
};
__device__ __forceinline__ Divisor divisor(uint32_t d) { return {d, 0xffffffffu / d + 1}; }
__device__ __forceinline__ uint32_t quotient(uint32_t n, const Divisor& v) { return v.d == 1 ? n : __umulhi(n, v.m); }

// W elements as fp32.
template <int W>
struct Piece {
  float v[W];
};
template <int W>
__device__ __forceinline__ Piece<W> load_piece(const __bf16* p) {
  typedef __bf16 vec __attribute__((ext_vector_type(W)));
  const vec x = *reinterpret_cast<const vec*>(p);
  Piece<W> o;
#pragma unroll
  for (int i = 0; i < W; ++i) o.v[i] = static_cast<float>(x[i]);
  return o;
}
template <int W>
__device__ __forceinline__ Piece<W> load_piece(const float* p) {
  constexpr int N = W < 4 ? W : 4;
  typedef float vec __attribute__((ext_vector_type(N)));
  Piece<W> o;
#pragma unroll
  for (int k = 0; k < W / N; ++k) {
    const vec x = reinterpret_cast<const vec*>(p)[k];
#pragma unroll
    for (int i = 0; i < N; ++i) o.v[k * N + i] = x[i];
  }
  return o;
}
template <int W>
__device__ __forceinline__ void store_piece(__bf16* p, const Piece<W>& x) {
  typedef __bf16 vec __attribute__((ext_vector_type(W)));
  vec o;
#pragma unroll
  for (int i = 0; i < W; ++i) o[i] = static_cast<__bf16>(x.v[i]);
  *reinterpret_cast<vec*>(p) = o;
}
template <int W>
__device__ __forceinline__ void store_piece(float* p, const Piece<W>& x) {
  constexpr int N = W < 4 ? W : 4;
  typedef float vec __attribute__((ext_vector_type(N)));
#pragma unroll
  for (int k = 0; k < W / N; ++k) {
    vec o;
#pragma unroll
    for (int i = 0; i < N; ++i) o[i] = x.v[k * N + i];
    reinterpret_cast<vec*>(p)[k] = o;
  }
}

// Workgroup number `group`'s rows and heads.  turns: 2 kRopePairs of LDS.  A piece is W channels (half style: and their W partners);
// interleaved pairs at addresses that are none of two channels go pair by pair (W = 1).
template <int W, bool HALF, typename TX, typename TY>
__device__ __forceinline__ void rope_rows(const RopeLaunch& l, unsigned group, float* turns) {
  const RopeArgs& a = l.a;
  float *cos_t = turns, *sin_t = turns + kRopePairs;
  const int half = a.rot / 2;
  const unsigned row_group = group / static_cast<unsigned>(l.head_groups);
  const int head_group = static_cast<int>(group - row_group * l.head_groups);
  const int64_t first_row = static_cast<int64_t>(row_group) * l.rows;
  const int rows = static_cast<int>(min(static_cast<int64_t>(l.rows), a.T - first_row));
  const int first_head = head_group * l.heads, heads = min(l.heads, a.n_heads - first_head);
  const Divisor by_half = divisor(half), by_units = divisor(l.units), by_heads = divisor(heads);
  for (int i = threadIdx.x; i < rows * half; i += kRopeThreads) {
    const int r = quotient(i, by_half), j = i - r * half;
    const float2 t = rope_turn(static_cast<double>(a.positions[first_row + r]) * a.freqs[j], a.amplitude);
    cos_t[i] = t.x;
    sin_t[i] = t.y;
  }
  __syncthreads();
  const int n = rows * heads * l.units;
  for (int i = threadIdx.x; i < n; i += kRopeThreads) {
    const int rest = quotient(i, by_units), unit = i - rest * l.units;
    const int r = quotient(rest, by_heads), h = first_head + rest - r * heads;
    const TX* x = static_cast<const TX*>(a.x) + (first_row + r) * a.ld_x + h * a.hd;
    TY* y = static_cast<TY*>(a.y) + (first_row + r) * a.ld_y + h * a.hd;
    const float *cs = cos_t + r * half, *sn = sin_t + r * half;
    if (unit >= l.turned) {                    // (not rotated: only where y is another tensor)
      const int at = a.rot + (unit - l.turned) * W;
      store_piece<W>(y + at, load_piece<W>(x + at));
    } else if constexpr (HALF) {
      const int at = unit * W;
      const Piece<W> p = load_piece<W>(x + at), q = load_piece<W>(x + half + at);
      Piece<W> u, v;
#pragma unroll
      for (int e = 0; e < W; ++e) {
        u.v[e] = rope_first(p.v[e], q.v[e], cs[at + e], sn[at + e]);
        v.v[e] = rope_second(p.v[e], q.v[e], cs[at + e], sn[at + e]);
      }
      store_piece<W>(y + at, u);
      store_piece<W>(y + half + at, v);
    } else if constexpr (W == 1) {
      const float p = static_cast<float>(x[2 * unit]), q = static_cast<float>(x[2 * unit + 1]);
      y[2 * unit] = static_cast<TY>(rope_first(p, q, cs[unit], sn[unit]));
      y[2 * unit + 1] = static_cast<TY>(rope_second(p, q, cs[unit], sn[unit]));
    } else {
      const int at = unit * W;
      const Piece<W> p = load_piece<W>(x + at);
      Piece<W> u;
#pragma unroll
      for (int e = 0; e < W / 2; ++e) {
        u.v[2 * e] = rope_first(p.v[2 * e], p.v[2 * e + 1], cs[at / 2 + e], sn[at / 2 + e]);
        u.v[2 * e + 1] = rope_second(p.v[2 * e], p.v[2 * e + 1], cs[at / 2 + e], sn[at / 2 + e]);
      }
      store_piece<W>(y + at, u);
    }
  }
}

}  // namespace rptq
