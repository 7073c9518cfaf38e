// Rotary positions on given heads (sps_rope), and the paged cache's append
// (sps_paged_append), which rotates keys on their way into their pages and the
// queries beside them. Both move every element once and are bound by that; a
// work-group computes the cosines and sines of its rows once, in LDS, and its
// heads share them. Measured: rope of 8192 x 64 x 128 bf16 54 us, 5.0 TB/s read
// and written (a plain copy reaches 5.1); append of five chunks, 5189 tokens
// with 32 heads on 8, 33 us against 25 at that rate; of single tokens both are a
// launch (3.6 us, and 7 with the 64 sequences' search for their blocks).
#include <algorithm>
#include <cmath>

#include "paged.h"

namespace sps {

RopeArgs rope_args(const sps_rope_spec* s, int DH) {
  RopeArgs r{};
  if (!s) {
    r.whole = DH % 8 == 0;
    return r;
  }
  r.rot = s->rot_dim;
  r.interleaved = s->layout == SPS_ROPE_INTERLEAVED;
  r.whole = DH % 8 == 0 && s->rot_dim % (r.interleaved ? 8 : 16) == 0;
  r.amp = s->amplitude;
  r.step = -2.0 / s->rot_dim * std::log2(static_cast<double>(s->base));
  r.inv_factor = 1.0 / s->factor;
  r.by_parts = s->original_len > 0;
  if (r.by_parts) {
    r.original = s->original_len;
    r.low = s->low_turns;
    r.inv_span = 1.0 / (static_cast<double>(s->high_turns) - s->low_turns);
  }
  return r;
}

// cs[row][pair] of `rows` rows at positions pos(row). A thread keeps to one
// pair where they divide the work-group, whose frequency it forms once.
template <typename P>
__device__ __forceinline__ void fill_cs(const RopeArgs& r, int rows, P pos, float2* cs) {
  const int np = r.rot / 2;
  if (np == 0) return;
  const int n = rows * np;
  int last = -1;
  double turns = 0.0;
  for (int e = threadIdx.x; e < n; e += blockDim.x) {
    const int row = static_cast<int>(static_cast<uint32_t>(e) / static_cast<uint32_t>(np)), i = e - row * np;
    if (i != last) turns = rope_turns(r, i);
    last = i;
    cs[e] = rope_cs(turns, pos(row), r.amp);
  }
}

// `rows` rows of `heads` heads rotated (sign -1: the transpose), x -> out,
// which may be x: a thread reads both halves of its pairs before it writes them.
// kBatch: the runs of a thread whose loads go out before the first is needed (a
// full card of work-groups hides them by itself: rope of 8192 x 64 x 128 54 us
// with 1, 58 with 4; append, with its LDS, 40 and 35).
template <int kBatch, typename T>
__device__ __forceinline__ void rotate_rows(const T* x, int64_t ldx, int rows, int heads, int DH, const RopeArgs& r,
                                            const float2* cs, float sign, T* out, int64_t ldo) {
  const int np = r.rot / 2;
  if (r.whole) {
    // Runs of 8 elements: in the half layout a run and its partners half the
    // rotated dims on, then the runs that are passed through.
    const int pairs = r.interleaved ? r.rot / 8 : np / 8;          // rotating units of a head
    const int units = pairs + (DH - r.rot) / 8;
    const int u = threadIdx.x % static_cast<uint32_t>(units), h0 = threadIdx.x / static_cast<uint32_t>(units);
    const int per = static_cast<int>(blockDim.x / static_cast<uint32_t>(units)), n = rows * heads;
    if (h0 >= per) return;
    const float inv = 1.f / heads;
    const bool half = u < pairs && !r.interleaved;
    const int d = u < pairs ? u * 8 : r.rot + (u - pairs) * 8;
    for (int i0 = h0; i0 < n; i0 += per * kBatch) {
      Frag<T> a[kBatch], b[kBatch];
      int rows_at[kBatch];
      int64_t at[kBatch];
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        const int i = i0 + j * per;
        if (i >= n) break;
        const int row = static_cast<int>((i + 0.5f) * inv), h = i - row * heads;   // i < 2^17: exact
        rows_at[j] = row;
        at[j] = row * ldo + h * DH;
        const T* src = x + row * ldx + h * DH;
        a[j] = load_frag_any(src + d);
        if (half) b[j] = load_frag_any(src + np + d);
      }
#pragma unroll
      for (int j = 0; j < kBatch; ++j) {
        if (i0 + j * per >= n) break;
        T* dst = out + at[j];
        if (u >= pairs) {
          store8_any(dst + d, __builtin_convertvector(a[j].v, f32x8));
          continue;
        }
        const f32x8 xa = __builtin_convertvector(a[j].v, f32x8);
        f32x8 y;
        if (half) {
          const f32x8 xb = __builtin_convertvector(b[j].v, f32x8);
          const float2* t = cs + rows_at[j] * np + d;
          f32x8 z;
#pragma unroll
          for (int e = 0; e < 8; ++e) {
            const float2 w = t[e];
            const float sn = sign * w.y;
            y[e] = xa[e] * w.x - xb[e] * sn;
            z[e] = xa[e] * sn + xb[e] * w.x;
          }
          store8_any(dst + np + d, z);
        } else {
          const float2* t = cs + rows_at[j] * np + d / 2;
#pragma unroll
          for (int e = 0; e < 4; ++e) {
            const float2 w = t[e];
            const float sn = sign * w.y;
            y[2 * e] = xa[2 * e] * w.x - xa[2 * e + 1] * sn;
            y[2 * e + 1] = xa[2 * e] * sn + xa[2 * e + 1] * w.x;
          }
        }
        store8_any(dst + d, y);
      }
    }
    return;
  }
  const int units = np + DH - r.rot;
  for (int i = threadIdx.x; i < rows * heads * units; i += blockDim.x) {
    const int rh = static_cast<int>(static_cast<uint32_t>(i) / static_cast<uint32_t>(units)), u = i - rh * units;
    const int row = static_cast<int>(static_cast<uint32_t>(rh) / static_cast<uint32_t>(heads)), h = rh - row * heads;
    const T* src = x + row * ldx + h * DH;
    T* dst = out + row * ldo + h * DH;
    if (u < np) {
      const int ia = r.interleaved ? 2 * u : u, ib = r.interleaved ? 2 * u + 1 : u + np;
      const float a = to_f32(src[ia]), b = to_f32(src[ib]);
      const float2 w = cs[row * np + u];
      const float sn = sign * w.y;
      dst[ia] = from_f32<T>(a * w.x - b * sn);
      dst[ib] = from_f32<T>(a * sn + b * w.x);
    } else {
      dst[r.rot + u - np] = src[r.rot + u - np];
    }
  }
}

// Grid (row groups, head groups).
template <typename T>
__global__ __launch_bounds__(256) void rope_kernel(const T* x, int64_t ldx, const int32_t* __restrict__ positions,
                                                   RopeArgs r, int rows, int group, int heads, int head_group, int DH,
                                                   float sign, T* out, int64_t ldo) {
  extern __shared__ float4 smem[];
  float2* cs = reinterpret_cast<float2*>(smem);
  const int row0 = blockIdx.x * group, n = min(group, rows - row0);
  const int h0 = blockIdx.y * head_group, nh = min(head_group, heads - h0);
  fill_cs(r, n, [&](int row) { return positions[row0 + row]; }, cs);
  __syncthreads();
  rotate_rows<1>(x + row0 * ldx + h0 * DH, ldx, n, nh, DH, r, cs, sign, out + row0 * ldo + h0 * DH, ldo);
}

hipError_t launch_rope(int dtype, const void* x, int64_t ldx, const int32_t* positions, const RopeArgs& r, int rows,
                       int heads, int DH, bool backward, void* out, int64_t ldo, hipStream_t st) {
  const float sign = backward ? -1.f : 1.f;
  // Rows per work-group: four once that leaves four work-groups per CU. Few
  // rows: the heads over several work-groups, 32 (2^14 elements or so) each.
  const int group = rows >= 16 * kCUs ? 4 : rows >= 8 * kCUs ? 2 : 1;
  const int head_group = rows >= 4 * kCUs ? heads : std::min(heads, 32);
  const dim3 grid((rows + group - 1) / group, (heads + head_group - 1) / head_group);
  const size_t lds = static_cast<size_t>(group) * (r.rot / 2) * sizeof(float2);
  if (dtype == 1)
    hipLaunchKernelGGL(rope_kernel<bf16>, grid, dim3(256), lds, st, static_cast<const bf16*>(x), ldx, positions, r, rows,
                       group, heads, head_group, DH, sign, static_cast<bf16*>(out), ldo);
  else
    hipLaunchKernelGGL(rope_kernel<float>, grid, dim3(256), lds, st, static_cast<const float*>(x), ldx, positions, r,
                       rows, group, heads, head_group, DH, sign, static_cast<float*>(out), ldo);
  return hipGetLastError();
}

// One work-group per (32-position block of a sequence's new tokens, KV head):
// its keys rotated into LDS, the queries of its heads rotated in passing, its
// values copied over the keys once these are out, and both written in the tiles' order: a 16-byte run
// of keys is 8 dims of a position, one of values 8 positions of a dim (whole
// ones where the tokens cover them, else element by element). One LDS tile for
// both leaves room for six work-groups a CU in bf16 (1368 of them for 5189
// tokens 32.9 us, 35.5 with a tile each and four a CU).
template <typename T>
__global__ __launch_bounds__(256, sizeof(T) == 2 ? 6 : 4) void paged_append_kernel(PagedView c, PagedRows r, const T* __restrict__ k,
                                                           int64_t ldk, const T* __restrict__ v, int64_t ldv,
                                                           RopeArgs ra, const T* q, int64_t ldq, T* qo, int64_t ldqo,
                                                           int* err) {
  constexpr int kPad = 8;                          // elements behind a row, against bank conflicts
  __shared__ __align__(16) float2 cs[32 * 64];
  __shared__ __align__(16) T tile[32 * (128 + kPad)];   // keys, then values
  int* words = reinterpret_cast<int*>(cs);         // blocks of every sequence, before the cosines
  const int lane = threadIdx.x & 63, h = blockIdx.y;
  auto blocks_of = [&](int b) {
    const SeqRows s = seq_rows(c, r, b);
    if (s.bad && blockIdx.x == 0 && h == 0) atomicOr(err, kErrCapacity);
    return s.n > 0 ? ((s.p0 + s.n - 1) >> 5) - (s.p0 >> 5) + 1 : 0;
  };
  if (c.B > 64) {
    for (int b = threadIdx.x; b < c.B; b += blockDim.x) words[b] = blocks_of(b);
    __syncthreads();
  }
  int b = -1, blk = 0, before = 0;
  for (int b0 = 0; b0 < c.B; b0 += 64) {
    const int mine = b0 + lane >= c.B ? 0 : c.B > 64 ? words[b0 + lane] : blocks_of(lane);
    const int incl = static_cast<int>(wave_incl_scan_u64(static_cast<uint64_t>(mine))) + before;
    const uint64_t hit = __ballot(static_cast<int>(blockIdx.x) < incl);
    if (hit) {
      const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      b = b0 + src;
      blk = static_cast<int>(blockIdx.x) - (__builtin_amdgcn_readlane(incl, src) - __builtin_amdgcn_readlane(mine, src));
      break;
    }
    before = __builtin_amdgcn_readlane(incl, 63);
  }
  if (b < 0) return;                               // past the last block; alike in every wave
  const SeqRows s = seq_rows(c, r, b);
  // Tokens j0 .. j1 - 1 of the sequence, at places w0 .. of the block from pos0 on.
  const int pos0 = ((s.p0 >> 5) + blk) * 32;
  const int j0 = max(0, pos0 - s.p0), j1 = min(s.n, pos0 + 32 - s.p0), n = j1 - j0, w0 = s.p0 + j0 - pos0;
  const int row0 = s.r0 + j0, DH = c.DH, ld = DH + kPad;
  // The block's page; -1: not written.
  int page = -1;
  if (pos0 < 0 || pos0 >= c.max_pages << c.page_log2) {
    if (threadIdx.x == 0) atomicOr(err, kErrCapacity);
  } else {
    page = c.table[static_cast<size_t>(b) * c.max_pages + (pos0 >> c.page_log2)];
    if (page < 0 || page >= c.n_pages) {
      if (threadIdx.x == 0) atomicOr(err, kErrBadPage);
      page = -1;
    }
  }
  const int runs = DH / 8;                         // 8 or 16: at most two a thread in 32 rows
  Frag<T> vr[2];
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = threadIdx.x + j * 256, row = i / static_cast<uint32_t>(runs), d = (i - row * runs) * 8;
    if (i < n * runs) vr[j] = load_frag_any(v + (row0 + row) * ldv + h * DH + d);
  }
  if (c.B > 64) __syncthreads();                   // `words` have been read
  fill_cs(ra, n, [&](int row) { return s.p0 + j0 + row; }, cs);
  __syncthreads();
  if (page >= 0) rotate_rows<4>(k + row0 * ldk + h * DH, ldk, n, 1, DH, ra, cs, 1.f, tile, ld);
  __syncthreads();
  if (q)
    rotate_rows<4>(q + row0 * ldq + h * c.G * DH, ldq, n, c.G, DH, ra, cs, 1.f, qo + row0 * ldqo + h * c.G * DH, ldqo);
  if (page < 0) return;
  const size_t area = static_cast<size_t>(DH) << c.page_log2;
  const int in = pos0 & ((1 << c.page_log2) - 1);
  const size_t base = (static_cast<size_t>(page) * c.H + h) * area + static_cast<size_t>(in) * DH;
  T* kd = static_cast<T*>(c.k) + base;
  T* vd = static_cast<T*>(c.v) + base;
  // Keys: run i is place (i / 16 / runs) * 16 + i % 16 of the block, dims 8 (i / 16 % runs) on.
  for (int i = threadIdx.x; i < 32 * runs; i += blockDim.x) {
    const int w = (i >= 16 * runs ? 16 : 0) + (i & 15), g = (i >> 4) & (runs - 1);
    if (w >= w0 && w < w0 + n)
      *reinterpret_cast<Frag<T>*>(kd + i * 8) = *reinterpret_cast<const Frag<T>*>(tile + (w - w0) * ld + g * 8);
  }
  __syncthreads();                                 // the keys have been read
#pragma unroll
  for (int j = 0; j < 2; ++j) {
    const int i = threadIdx.x + j * 256, row = i / static_cast<uint32_t>(runs), d = (i - row * runs) * 8;
    if (i < n * runs) *reinterpret_cast<Frag<T>*>(tile + row * ld + d) = vr[j];
  }
  __syncthreads();
  // Values: run i is dim (i / 64) * 16 + i % 16, places 4 g + e and 16 + 4 g + e with g = i / 16 % 4.
  for (int i = threadIdx.x; i < 4 * DH; i += blockDim.x) {
    const int d = (i >> 6) * 16 + (i & 15), g = (i >> 4) & 3;
    Frag<T> f;
    bool whole = true;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const int w = (e >> 2) * 16 + g * 4 + (e & 3) - w0;
      const bool there = w >= 0 && w < n;
      whole &= there;
      f.v[e] = tile[(there ? w : 0) * ld + d];
    }
    if (whole) {
      *reinterpret_cast<Frag<T>*>(vd + i * 8) = f;
    } else {
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int w = (e >> 2) * 16 + g * 4 + (e & 3) - w0;
        if (w >= 0 && w < n) vd[i * 8 + e] = f.v[e];
      }
    }
  }
}

hipError_t launch_paged_append(int dtype, const PagedView& c, const PagedRows& r, const void* k, int64_t ldk,
                               const void* v, int64_t ldv, const RopeArgs& rope, const void* q, int64_t ldq, void* qo,
                               int64_t ldqo, int* err, hipStream_t st) {
  // n tokens touch at most (n + 30) / 32 + 1 blocks.
  const long seqs = std::min(c.B, r.rows);
  const long blocks = std::min(seqs * ((r.max_tokens + 30L) / 32 + 1), (r.rows + 30 * seqs) / 32 + seqs);
  const dim3 grid(static_cast<unsigned>(blocks), c.H);
  if (dtype == 1)
    hipLaunchKernelGGL(paged_append_kernel<bf16>, grid, dim3(256), 0, st, c, r, static_cast<const bf16*>(k), ldk,
                       static_cast<const bf16*>(v), ldv, rope, static_cast<const bf16*>(q), ldq,
                       static_cast<bf16*>(qo), ldqo, err);
  else
    hipLaunchKernelGGL(paged_append_kernel<float>, grid, dim3(256), 0, st, c, r, static_cast<const float*>(k), ldk,
                       static_cast<const float*>(v), ldv, rope, static_cast<const float*>(q), ldq,
                       static_cast<float*>(qo), ldqo, err);
  return hipGetLastError();
}

}  // namespace sps
