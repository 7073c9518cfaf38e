// Rotary positions on given heads (sps_rope), and the paged cache's append
// (sps_paged_append), which rotates keys on their way into their pages and the
// queries beside them.
#include <cmath>

#include "paged.h"

namespace sps {

RopeArgs rope_args(const sps_rope_spec& s) {
  RopeArgs r{};
  r.rot = s.rot_dim;
  r.interleaved = s.layout == SPS_ROPE_INTERLEAVED;
  r.amp = s.amplitude;
  r.step = -2.0 / s.rot_dim * std::log2(static_cast<double>(s.base));
  r.inv_factor = 1.0 / s.factor;
  r.by_parts = s.original_len > 0;
  if (r.by_parts) {
    r.original = s.original_len;
    r.low = s.low_turns;
    r.inv_span = 1.0 / (static_cast<double>(s.high_turns) - s.low_turns);
  }
  return r;
}

// Elements of pair i of a head.
__device__ __forceinline__ int pair_a(const RopeArgs& r, int i) { return r.interleaved ? 2 * i : i; }
__device__ __forceinline__ int pair_b(const RopeArgs& r, int i) { return r.interleaved ? 2 * i + 1 : i + r.rot / 2; }

// Heads h of one row: x[h][:] -> out[h][:], cs the row's (cos, sin) table.
template <typename T>
__device__ void rotate_row(const T* x, const RopeArgs& r, const float2* cs, int heads, int DH, float sign, T* out) {
  const int np = r.rot / 2, rest = DH - r.rot, units = np + rest;
  for (int e = threadIdx.x; e < heads * units; e += blockDim.x) {
    const int h = e / units, u = e % units;
    const size_t base = static_cast<size_t>(h) * DH;
    if (u < np) {
      const int ia = pair_a(r, u), ib = pair_b(r, u);
      const float a = to_f32(x[base + ia]), b = to_f32(x[base + ib]);
      const float2 t = cs[u];
      const float sn = sign * t.y;
      out[base + ia] = from_f32<T>(a * t.x - b * sn);
      out[base + ib] = from_f32<T>(a * sn + b * t.x);
    } else {
      out[base + r.rot + u - np] = x[base + r.rot + u - np];
    }
  }
}

template <typename T>
__global__ __launch_bounds__(256) void rope_kernel(const T* x, int64_t ldx, const int32_t* __restrict__ positions,
                                                   RopeArgs r, int heads, int DH, float sign, T* out, int64_t ldo) {
  __shared__ float2 cs[kMaxRopeDim / 2];
  const int row = blockIdx.x, i = threadIdx.x;
  if (i < r.rot / 2) cs[i] = rope_cs(rope_turns(r, i), positions[row], r.amp);
  __syncthreads();
  rotate_row(x + row * ldx, r, cs, heads, DH, sign, out + row * ldo);
}

hipError_t launch_rope(int dtype, const void* x, int64_t ldx, const int32_t* positions, const RopeArgs& r, int rows,
                       int heads, int DH, bool backward, void* out, int64_t ldo, hipStream_t st) {
  const float sign = backward ? -1.f : 1.f;
  if (dtype == 1)
    hipLaunchKernelGGL(rope_kernel<bf16>, dim3(rows), dim3(256), 0, st, static_cast<const bf16*>(x), ldx, positions, r,
                       heads, DH, sign, static_cast<bf16*>(out), ldo);
  else
    hipLaunchKernelGGL(rope_kernel<float>, dim3(rows), dim3(256), 0, st, static_cast<const float*>(x), ldx, positions,
                       r, heads, DH, sign, static_cast<float*>(out), ldo);
  return hipGetLastError();
}

// One work-group per new token.
template <typename T>
__global__ __launch_bounds__(256) void paged_append_kernel(PagedView c, PagedRows r, const T* __restrict__ k,
                                                           int64_t ldk, const T* __restrict__ v, int64_t ldv,
                                                           bool rotate, RopeArgs ra, const T* q, int64_t ldq, T* qo,
                                                           int64_t ldqo, int* err) {
  __shared__ float2 cs[64];
  __shared__ T head[128];
  __shared__ int owner;
  const int row = blockIdx.x;
  if (threadIdx.x == 0) owner = c.B;
  __syncthreads();
  for (int b = threadIdx.x; b < c.B; b += blockDim.x) {
    const SeqRows s = seq_rows(c, r, b);
    if (s.bad && row == 0) atomicOr(err, kErrCapacity);
    if (row >= s.r0 && row < s.r0 + s.n) atomicMin(&owner, b);
  }
  __syncthreads();
  const int b = owner;
  if (b == c.B) return;                            // no sequence's row
  const SeqRows s = seq_rows(c, r, b);
  const int pos = s.p0 + row - s.r0;
  const int i = threadIdx.x;
  if (rotate && i < ra.rot / 2) cs[i] = rope_cs(rope_turns(ra, i), pos, ra.amp);
  if (!rotate) ra.rot = 0;
  __syncthreads();
  if (q) rotate_row(q + row * ldq, ra, cs, c.H * c.G, c.DH, 1.f, qo + row * ldqo);
  if (pos < 0 || pos >= c.max_pages << c.page_log2) {
    if (threadIdx.x == 0) atomicOr(err, kErrCapacity);
    return;
  }
  const int page = c.table[static_cast<size_t>(b) * c.max_pages + (pos >> c.page_log2)];
  if (page < 0 || page >= c.n_pages) {
    if (threadIdx.x == 0) atomicOr(err, kErrBadPage);
    return;
  }
  const int in = pos & ((1 << c.page_log2) - 1);
  const size_t area = static_cast<size_t>(c.DH) << c.page_log2;
  for (int h = 0; h < c.H; ++h) {
    const size_t base = (static_cast<size_t>(page) * c.H + h) * area;
    rotate_row(k + row * ldk + h * c.DH, ra, cs, 1, c.DH, 1.f, head);
    __syncthreads();
    if (i < c.DH) {
      static_cast<T*>(c.k)[base + k_offset(in, i, c.DH)] = head[i];
      static_cast<T*>(c.v)[base + v_offset(in, i, c.DH)] = v[row * ldv + h * c.DH + i];
    }
    __syncthreads();
  }
}

hipError_t launch_paged_append(int dtype, const PagedView& c, const PagedRows& r, const void* k, int64_t ldk,
                               const void* v, int64_t ldv, const RopeArgs* rope, const void* q, int64_t ldq, void* qo,
                               int64_t ldqo, int* err, hipStream_t st) {
  const RopeArgs ra = rope ? *rope : RopeArgs{};
  if (dtype == 1)
    hipLaunchKernelGGL(paged_append_kernel<bf16>, dim3(r.rows), dim3(256), 0, st, c, r, static_cast<const bf16*>(k), ldk,
                       static_cast<const bf16*>(v), ldv, rope != nullptr, ra, static_cast<const bf16*>(q), ldq,
                       static_cast<bf16*>(qo), ldqo, err);
  else
    hipLaunchKernelGGL(paged_append_kernel<float>, dim3(r.rows), dim3(256), 0, st, c, r, static_cast<const float*>(k),
                       ldk, static_cast<const float*>(v), ldv, rope != nullptr, ra, static_cast<const float*>(q), ldq,
                       static_cast<float*>(qo), ldqo, err);
  return hipGetLastError();
}

}  // namespace sps
