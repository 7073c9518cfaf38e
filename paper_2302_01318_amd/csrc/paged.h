// Device-side helpers of the paged cache's kernels: the rows and positions of
// a call's sequences, and rotary angles.
#pragma once
#include "common.h"
#include "launch.h"

namespace sps {

constexpr int kErrBadPage = 16;   // SPS_DEV_BAD_PAGE

// Eight elements at any element-aligned address: callers' row strides and
// base pointers are their own.
typedef __bf16 bf16x8u __attribute__((ext_vector_type(8), aligned(2)));
typedef __bf16 bf16x4u __attribute__((ext_vector_type(4), aligned(2)));
typedef float f32x8u __attribute__((ext_vector_type(8), aligned(4)));
typedef float f32x4u __attribute__((ext_vector_type(4), aligned(4)));
__device__ __forceinline__ Frag<bf16> load_frag_any(const bf16* p) {
  Frag<bf16> f; f.v = *reinterpret_cast<const bf16x8u*>(p); return f;
}
__device__ __forceinline__ Frag<float> load_frag_any(const float* p) {
  Frag<float> f; f.v = *reinterpret_cast<const f32x8u*>(p); return f;
}
__device__ __forceinline__ void store8_any(bf16* p, f32x8 v) {
  *reinterpret_cast<bf16x8u*>(p) = __builtin_convertvector(v, bf16x8u);
}
__device__ __forceinline__ void store8_any(float* p, f32x8 v) { *reinterpret_cast<f32x8u*>(p) = v; }
__device__ __forceinline__ void store4_any(bf16* p, f32x4 v) {
  *reinterpret_cast<bf16x4u*>(p) = __builtin_convertvector(v, bf16x4u);
}
__device__ __forceinline__ void store4_any(float* p, f32x4 v) { *reinterpret_cast<f32x4u*>(p) = v; }

// Rows r0 .. r0 + n - 1 of the call belong to sequence b, the first at
// position p0 (kept inside +-2^24, far past any capacity). `bad`: its starts
// break the rules of sps.h; what is taken then stays inside the rows.
struct SeqRows {
  int r0, n, p0;
  bool bad;
};
__device__ __forceinline__ SeqRows seq_rows(const PagedView& c, const PagedRows& r, int b) {
  SeqRows s;
  const long p = static_cast<long>(c.lengths[b]) + r.pos_offset;
  s.p0 = static_cast<int>(p < -(1L << 24) ? -(1L << 24) : p > (1L << 24) ? (1L << 24) : p);
  s.bad = false;
  if (!r.starts) {
    s.r0 = b * r.max_tokens;
    s.n = r.max_tokens;
    return s;
  }
  const int a = r.starts[b], e = r.starts[b + 1];
  s.r0 = min(max(a, 0), r.rows);
  s.n = min(max(e, s.r0), r.rows) - s.r0;
  s.bad = a < 0 || e < a || e > r.rows || s.n > r.max_tokens;
  s.n = min(s.n, r.max_tokens);
  return s;
}

// (cos, sin) of pair i's angle at position pos, times the amplitude. The
// angle is formed in fp64 and in turns: whole and quarter turns are taken off
// exactly, and what is left, |x| <= pi / 4, goes into the Taylor polynomials
// (first terms left out: x^11 / 11! < 2e-9 and x^12 / 12! < 2e-10).
__device__ __forceinline__ double rope_turns(const RopeArgs& r, int i) {
  double f = exp2(r.step * i) * 0.15915494309189533577;
  if (r.by_parts) {
    const double g = fmin(fmax((r.original * f - r.low) * r.inv_span, 0.0), 1.0);
    f *= g + (1.0 - g) * r.inv_factor;
  } else {
    f *= r.inv_factor;
  }
  return f;
}
__device__ __forceinline__ float2 rope_cs(double turns, int pos, float amp) {
  double t = turns * pos;
  t -= rint(t);
  const double k = rint(t * 4.0);
  const float x = static_cast<float>((t - 0.25 * k) * 6.283185307179586477);
  const float z = x * x;
  const float s = x + x * z * (-1.f / 6 + z * (1.f / 120 + z * (-1.f / 5040 + z * (1.f / 362880))));
  const float c = 1.f + z * (-0.5f + z * (1.f / 24 + z * (-1.f / 720 + z * (1.f / 40320 - z * (1.f / 3628800)))));
  const int n = static_cast<int>(k) & 3;           // quarter turns
  const float cs = n & 1 ? s : c, sn = n & 1 ? c : s;
  return make_float2(amp * (n == 1 || n == 2 ? -cs : cs), amp * (n >= 2 ? -sn : sn));
}

}  // namespace sps
