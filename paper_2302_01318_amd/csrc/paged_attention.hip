// Attention of a batch's new tokens over the pages of their sequences
// (sps_paged_attention). With G query heads per KV head, the query rows of one
// (sequence, KV head) are its tokens x G; a work item is a tile of 16 QT of
// them against a range of 32-position blocks, which its four waves take in
// turn. Per block S^T = K Q^T with MFMA (A = key tile, B = Q^T), an online
// softmax on the S^T registers, and O^T += V^T P^T (A = value tile, B = the
// softmax tile as the score MFMA leaves it, which the value tiles' position
// order is made for): both tiles go from the page straight into registers, a
// KiB per wave and load. The waves' (O, max, sum) meet in LDS; ranges of one
// tile meet in a second launch.
#include "paged.h"

namespace sps {

// Where an item, or a (tile, KV head) with several ranges, belongs.
struct Place {
  int b, tile, range, ranges, kvh;
  int per;                 // blocks per range
  long slot;               // of the tile's first range (ranges > 1)
};

// The tiles and blocks of every sequence of the call, per sequence in LDS,
// and from them the place of item (join: of the (tile, KV head) pair) number
// `idx`. Every work-group of both launches computes the same plan from the
// same lengths. Returns false past the last one.
__device__ __forceinline__ bool find_place(const PagedView& c, const PagedRows& r, int window, int tile_rows,
                                           int target, bool join, long idx, int* s_tiles, int* s_blocks, int* err,
                                           Place* out) {
  const int lane = threadIdx.x & 63;
  const int cap = c.max_pages << c.page_log2;
  for (int b = threadIdx.x; b < c.B; b += blockDim.x) {
    const SeqRows s = seq_rows(c, r, b);
    if (s.bad && idx == 0 && err) atomicOr(err, kErrCapacity);
    const int end = min(max(s.p0 + s.n, 0), cap);
    const int lo = window ? min(max(s.p0 - window + 1, 0), end) : 0;
    s_tiles[b] = (s.n * c.G + tile_rows - 1) / tile_rows;
    s_blocks[b] = (end + 31) / 32 - lo / 32;
  }
  __syncthreads();
  uint64_t all = 0;
  for (int b0 = 0; b0 < c.B; b0 += 64)
    all += wave_sum_u64(b0 + lane < c.B ? static_cast<uint64_t>(s_tiles[b0 + lane]) * s_blocks[b0 + lane] : 0);
  const int per = max(kPagedMinBlocks, static_cast<int>(ceil(static_cast<double>(all) * c.H / target)));
  const int h = static_cast<int>(idx % c.H);
  const uint32_t want = static_cast<uint32_t>(idx / c.H);
  uint64_t before = 0;                             // (items or joins) << 32 | slots, per KV head
  for (int b0 = 0; b0 < c.B; b0 += 64) {
    const int b = b0 + lane;
    const uint32_t tiles = b < c.B ? s_tiles[b] : 0;
    const uint32_t ranges = b < c.B ? max(1, (s_blocks[b] + per - 1) / per) : 1;
    const uint32_t slots = ranges > 1 ? tiles * ranges : 0;
    const uint32_t mine = join ? (ranges > 1 ? tiles : 0) : tiles * ranges;
    const uint64_t incl = wave_incl_scan_u64(static_cast<uint64_t>(mine) << 32 | slots) + before;
    const uint64_t hit = __ballot(want < static_cast<uint32_t>(incl >> 32));
    if (hit) {
      const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
      const uint64_t inc = readlane_u64(incl, src);
      const int m = __builtin_amdgcn_readlane(static_cast<int>(mine), src);
      const int sl = __builtin_amdgcn_readlane(static_cast<int>(slots), src);
      const int nr = __builtin_amdgcn_readlane(static_cast<int>(ranges), src);
      const int at = static_cast<int>(want - (static_cast<uint32_t>(inc >> 32) - m));
      out->b = b0 + src;
      out->ranges = nr;
      out->tile = join ? at : at / nr;
      out->range = join ? 0 : at % nr;
      out->kvh = h;
      out->per = per;
      const uint32_t slot0 = static_cast<uint32_t>(inc) - sl;
      out->slot = (static_cast<long>(slot0) + static_cast<long>(out->tile) * nr) * c.H + h;   // ranges H apart
      return true;
    }
    before = readlane_u64(incl, 63);
  }
  return false;
}

template <typename T> __device__ __forceinline__ bool nonfinite(T x);
template <> __device__ __forceinline__ bool nonfinite<bf16>(bf16 x) {
  return (__builtin_bit_cast(unsigned short, x) & 0x7f80) == 0x7f80;
}
template <> __device__ __forceinline__ bool nonfinite<float>(float x) {
  return (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) == 0x7f800000u;
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// Scores of one block for one query tile with the positions a row does not see
// at -Inf. vis collects, per lane, which of its eight positions its row sees.
template <typename T, int DH>
__device__ __forceinline__ void block_scores(const Frag<T> (&kf)[2][DH / 32], const Frag<T> (&qf)[DH / 32], int pos0,
                                             int qpos, int window, int end, bool masked, int grp, f32x4 (&s)[2],
                                             uint32_t* vis) {
#pragma unroll
  for (int pt = 0; pt < 2; ++pt) {
    s[pt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt) s[pt] = mma8(s[pt], kf[pt][dt], qf[dt]);
  }
  *vis = 0xff;
  if (masked) {
    *vis = 0;
    const int lo = window ? qpos - window : -1;
#pragma unroll
    for (int pt = 0; pt < 2; ++pt)
#pragma unroll
      for (int r = 0; r < 4; ++r) {
        const int pos = pos0 + pt * 16 + grp * 4 + r;
        const bool seen = pos <= qpos && pos > lo && pos < end;
        s[pt][r] = seen ? s[pt][r] : -INFINITY;
        *vis |= seen ? 1u << (pt * 4 + r) : 0;
      }
  }
}

// Online softmax step on one tile's scores: the weights as a hi + lo pair of
// bf16 values (p = hi + lo to 2^-16 relative; the second product costs nothing
// where the loads of K and V are what takes the time), or fp32.
template <typename T, int DH>
__device__ __forceinline__ void softmax_step(const f32x4 (&s)[2], float c_log2, float& m_run, float& l_run,
                                             f32x4 (&o)[DH / 16], Frag<T>& hi, Frag<T>& lo) {
  float mx = -INFINITY;
#pragma unroll
  for (int pt = 0; pt < 2; ++pt)
#pragma unroll
    for (int r = 0; r < 4; ++r) mx = fmaxf(mx, s[pt][r]);
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const float m_new = fmaxf(m_run, mx);
  const float m_use = m_new == -INFINITY ? 0.f : m_new;
  const float alpha = fast_exp2((m_run - m_use) * c_log2);
  float ps = 0.f;
#pragma unroll
  for (int pt = 0; pt < 2; ++pt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      const float pv = fast_exp2((s[pt][r] - m_use) * c_log2);
      const T h = from_f32<T>(pv);
      hi.v[pt * 4 + r] = h;
      lo.v[pt * 4 + r] = from_f32<T>(pv - to_f32(h));
      ps += pv;
    }
  l_run = l_run * alpha + ps;
  m_run = m_new;
#pragma unroll
  for (int dt = 0; dt < DH / 16; ++dt) o[dt] *= alpha;
}

// Values that are not finite, in a block with positions that not every row of
// the tile sees: 0 x Inf would carry them into rows that do not see them. They
// are taken out of the tile, and put into the rows that do see them by
// counting, per row and dim, visible +Inf, -Inf and NaN with products of ones.
template <typename T, int DH, int QT>
__device__ __forceinline__ void infinite_values(Frag<T> (&vf)[DH / 16], const uint32_t (&vis)[QT], f32x4 (&o)[QT][DH / 16]) {
  float inf = INFINITY;
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {
#pragma unroll
    for (int dt = 0; dt < DH / 16; ++dt) {
      Frag<T> one;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float x = to_f32(vf[dt].v[e]);
        const bool is = kind == 0 ? x == INFINITY : kind == 1 ? x == -INFINITY : x != x;
        one.v[e] = from_f32<T>(is ? 1.f : 0.f);
      }
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        Frag<T> see;
#pragma unroll
        for (int e = 0; e < 8; ++e) see.v[e] = from_f32<T>(vis[qt] >> e & 1 ? 1.f : 0.f);
        const f32x4 n = mma8(f32x4{0.f, 0.f, 0.f, 0.f}, one, see);
#pragma unroll
        for (int r = 0; r < 4; ++r)
          if (n[r] > 0.f) o[qt][dt][r] += kind == 0 ? inf : kind == 1 ? -inf : NAN;
      }
    }
  }
#pragma unroll
  for (int dt = 0; dt < DH / 16; ++dt)
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (nonfinite(vf[dt].v[e])) vf[dt].v[e] = from_f32<T>(0.f);
}

template <typename T, int DH, int QT>
__global__ __launch_bounds__(256) void paged_attn_kernel(PagedView c, PagedRows r, int target,
                                                         const T* __restrict__ q, int64_t ldq, float scale, int window,
                                                         T* __restrict__ out, int64_t ldo, float* __restrict__ lse,
                                                         float* __restrict__ part_o, float2* __restrict__ part_ml,
                                                         int* err) {
  constexpr int TR = 16 * QT, ND = DH / 16;
  // The plan's words per sequence, then two waves' (O, max, sum).
  constexpr int kMergeF4 = 2 * QT * ND * 64, kPlanF4 = 2 * kMaxPagedB / 4;
  __shared__ f32x4 sm[kMergeF4 > kPlanF4 ? kMergeF4 : kPlanF4];
  __shared__ float2 sml[2 * QT * 64];
  int* s_tiles = reinterpret_cast<int*>(sm);
  Place pl;
  if (!find_place(c, r, window, TR, target, false, blockIdx.x, s_tiles, s_tiles + kMaxPagedB, err, &pl)) return;
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  const int r16 = lane & 15, grp = lane >> 4;
  const SeqRows s = seq_rows(c, r, pl.b);
  const int cap = c.max_pages << c.page_log2;
  const int nrows = s.n * c.G, row0 = pl.tile * TR;
  // Positions of the tile's first and last token, and what they see.
  const int first = s.p0 + row0 / c.G, last = s.p0 + (min(row0 + TR, nrows) - 1) / c.G;
  const int end = min(max(last + 1, 0), cap);
  const int lo = window ? min(max(first - window + 1, 0), end) : 0;
  const int base = (window ? min(max(s.p0 - window + 1, 0), min(max(s.p0 + s.n, 0), cap)) : 0) / 32;
  const int blk0 = max(base + pl.range * pl.per, lo / 32), blk1 = min(base + (pl.range + 1) * pl.per, (end + 31) / 32);
  const float c_log2 = scale * 1.4426950408889634f;

  Frag<T> qf[QT][DH / 32];
  int qpos[QT], tok[QT], head[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int row = row0 + qt * 16 + r16;
    const bool valid = row < nrows;
    const int t = valid ? row / c.G : 0;
    tok[qt] = s.r0 + t;
    head[qt] = pl.kvh * c.G + (valid ? row - t * c.G : 0);
    qpos[qt] = valid ? s.p0 + t : -1;
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt)
      qf[qt][dt] = valid ? load_frag_any(q + tok[qt] * ldq + head[qt] * DH + dt * 32 + grp * 8) : Frag<T>::zero();
  }
  float m_run[QT], l_run[QT];
  f32x4 o[QT][ND];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    m_run[qt] = -INFINITY;
    l_run[qt] = 0.f;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};
  }

  // This wave's blocks are blk0 + wave + 4 i; the pages of 64 of them at a time.
  const int32_t* tab = c.table + static_cast<size_t>(pl.b) * c.max_pages;
  const size_t area = static_cast<size_t>(DH) << c.page_log2;
  const int nb = blk1 > blk0 + wave ? (blk1 - blk0 - wave + 3) / 4 : 0;
  for (int i0 = 0; i0 < nb; i0 += 64) {
    int id = -1;
    if (i0 + lane < nb) {
      id = tab[(blk0 + wave + 4 * (i0 + lane)) >> (c.page_log2 - 5)];
      if (id < 0 || id >= c.n_pages) {
        atomicOr(err, kErrBadPage);
        id = -1;
      }
    }
    const int n = min(64, nb - i0);
    for (int i = 0; i < n; ++i) {
      const int page = __builtin_amdgcn_readlane(id, i);
      if (page < 0) continue;
      const int blk = blk0 + wave + 4 * (i0 + i), pos0 = blk * 32;
      const size_t off = (static_cast<size_t>(page) * c.H + pl.kvh) * area +
                         static_cast<size_t>(pos0 & ((1 << c.page_log2) - 1)) * DH + lane * 8;
      const T* kp = static_cast<const T*>(c.k) + off;
      const T* vp = static_cast<const T*>(c.v) + off;
      Frag<T> kf[2][DH / 32], vf[ND];
#pragma unroll
      for (int pt = 0; pt < 2; ++pt)
#pragma unroll
        for (int dt = 0; dt < DH / 32; ++dt) kf[pt][dt] = load_frag(kp + (pt * (DH / 32) + dt) * 512);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) vf[dt] = load_frag(vp + dt * 512);
      const bool masked = pos0 + 31 > first || pos0 + 31 >= end || (window && pos0 <= last - window);
      if (pos0 + 32 > end) {
        // Positions no row of the tile sees hold anything, and 0 x NaN is not 0.
#pragma unroll
        for (int e = 0; e < 8; ++e)
          if (pos0 + (e < 4 ? grp * 4 + e : 16 + grp * 4 + e - 4) >= end) {
#pragma unroll
            for (int dt = 0; dt < ND; ++dt) vf[dt].v[e] = from_f32<T>(0.f);
          }
      }
      f32x4 sc[QT][2];
      uint32_t vis[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
        block_scores<T, DH>(kf, qf[qt], pos0, qpos[qt], window, end, masked, grp, sc[qt], &vis[qt]);
      Frag<T> hi[QT], lw[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt)
        softmax_step<T, DH>(sc[qt], c_log2, m_run[qt], l_run[qt], o[qt], hi[qt], lw[qt]);
      if (masked) {
        bool odd = false;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
#pragma unroll
          for (int e = 0; e < 8; ++e) odd |= nonfinite(vf[dt].v[e]);
        if (__ballot(odd)) infinite_values<T, DH, QT>(vf, vis, o);
      }
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) {
          o[qt][dt] = mma8(o[qt][dt], vf[dt], hi[qt]);
          if (sizeof(T) == 2) o[qt][dt] = mma8(o[qt][dt], vf[dt], lw[qt]);
        }
    }
  }

  // Waves 2, 3 into 0, 1, then 1 into 0.
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    l_run[qt] += __shfl_xor(l_run[qt], 16);
    l_run[qt] += __shfl_xor(l_run[qt], 32);
  }
  __syncthreads();                                 // the plan's words have been read
#pragma unroll
  for (int half = 2; half; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        sml[((wave - half) * QT + qt) * 64 + lane] = make_float2(m_run[qt], l_run[qt]);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) sm[(((wave - half) * QT + qt) * ND + dt) * 64 + lane] = o[qt][dt];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const float2 ml = sml[(wave * QT + qt) * 64 + lane];
        const float m = fmaxf(m_run[qt], ml.x), mu = m == -INFINITY ? 0.f : m;
        const float a = fast_exp2((m_run[qt] - mu) * c_log2), b = fast_exp2((ml.x - mu) * c_log2);
        m_run[qt] = m;
        l_run[qt] = a * l_run[qt] + b * ml.y;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[qt][dt] = a * o[qt][dt] + b * sm[((wave * QT + qt) * ND + dt) * 64 + lane];
      }
    }
    __syncthreads();
  }
  if (wave) return;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int row = row0 + qt * 16 + r16;
    if (row >= nrows) continue;
    if (pl.ranges > 1) {
      const size_t at = (pl.slot + static_cast<long>(pl.range) * c.H) * TR + qt * 16 + r16;
      if (grp == 0) part_ml[at] = make_float2(m_run[qt], l_run[qt]);
#pragma unroll
      for (int dt = 0; dt < ND; ++dt)
        *reinterpret_cast<f32x4*>(part_o + at * DH + dt * 16 + grp * 4) = o[qt][dt];
    } else {
      // A sum of zero: no visible position, or none with weight.
      const float inv = l_run[qt] == 0.f ? 0.f : 1.f / l_run[qt];
      T* dst = out + tok[qt] * ldo + head[qt] * DH + grp * 4;
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) store4_any(dst + dt * 16, l_run[qt] == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[qt][dt] * inv);
      if (lse && grp == 0)
        lse[static_cast<size_t>(tok[qt]) * c.H * c.G + head[qt]] =
            l_run[qt] == 0.f ? -INFINITY : m_run[qt] * scale + logf(l_run[qt]);
    }
  }
}

// The ranges of a tile's rows joined: one wave per row.
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedView c, PagedRows r, int target, int tile_rows,
                                                         float scale, int window, const float* __restrict__ part_o,
                                                         const float2* __restrict__ part_ml, T* __restrict__ out,
                                                         int64_t ldo, float* __restrict__ lse) {
  __shared__ int words[2 * kMaxPagedB];
  Place pl;
  if (!find_place(c, r, window, tile_rows, target, true, blockIdx.x, words, words + kMaxPagedB, nullptr, &pl)) return;
  const SeqRows s = seq_rows(c, r, pl.b);
  const int lane = threadIdx.x & 63, in = blockIdx.y * 4 + (threadIdx.x >> 6);
  const int row = pl.tile * tile_rows + in;
  if (row >= s.n * c.G) return;
  const float c_log2 = scale * 1.4426950408889634f;
  const float2* ml = part_ml + pl.slot * tile_rows + in;
  const float* po = part_o + (pl.slot * tile_rows + in) * DH + lane * (DH / 64);
  const size_t step = static_cast<size_t>(c.H) * tile_rows;      // from range to range
  float m = -INFINITY;
  for (int i = lane; i < pl.ranges; i += 64) m = fmaxf(m, ml[i * step].x);
  m = wave_max(m);
  float l = 0.f, acc[DH / 64] = {};
  if (m != -INFINITY) {
#pragma unroll 8
    for (int i = 0; i < pl.ranges; ++i) {
      const float2 x = ml[i * step];
      if (x.x == -INFINITY) continue;
      const float w = fast_exp2((x.x - m) * c_log2);
      l += w * x.y;
#pragma unroll
      for (int d = 0; d < DH / 64; ++d) acc[d] += w * po[i * step * DH + d];
    }
  }
  const int t = row / c.G, tok = s.r0 + t, head = pl.kvh * c.G + row - t * c.G;
#pragma unroll
  for (int d = 0; d < DH / 64; ++d)
    out[tok * ldo + head * DH + lane * (DH / 64) + d] = from_f32<T>(l == 0.f ? 0.f : acc[d] / l);
  if (lse && lane == 0)
    lse[static_cast<size_t>(tok) * c.H * c.G + head] = l == 0.f ? -INFINITY : m * scale + logf(l);
}

template <typename T, int DH>
static hipError_t attn_t(const PagedView& c, const PagedRows& r, const PagedPlan& p, const void* q, int64_t ldq,
                         float scale, int window, void* out, int64_t ldo, float* lse, float* part_o, float2* part_ml,
                         int* err, hipStream_t st) {
  auto kern = p.qt == 1 ? paged_attn_kernel<T, DH, 1> : paged_attn_kernel<T, DH, 2>;
  hipLaunchKernelGGL(kern, dim3(static_cast<unsigned>(p.items)), dim3(256), 0, st, c, r, p.target,
                     static_cast<const T*>(q), ldq, scale, window, static_cast<T*>(out), ldo, lse, part_o, part_ml, err);
  hipError_t e = hipGetLastError();
  if (e != hipSuccess || p.joins == 0) return e;
  hipLaunchKernelGGL((paged_join_kernel<T, DH>), dim3(static_cast<unsigned>(p.joins), 4 * p.qt), dim3(256), 0, st, c, r,
                     p.target, 16 * p.qt, scale, window, part_o, part_ml, static_cast<T*>(out), ldo, lse);
  return hipGetLastError();
}

hipError_t launch_paged_attention(int dtype, const PagedView& c, const PagedRows& r, const PagedPlan& p, const void* q,
                                  int64_t ldq, float scale, int window, void* out, int64_t ldo, float* lse,
                                  float* part_o, float2* part_ml, int* err, hipStream_t st) {
  if (dtype == 1)
    return c.DH == 128 ? attn_t<bf16, 128>(c, r, p, q, ldq, scale, window, out, ldo, lse, part_o, part_ml, err, st)
                       : attn_t<bf16, 64>(c, r, p, q, ldq, scale, window, out, ldo, lse, part_o, part_ml, err, st);
  return c.DH == 128 ? attn_t<float, 128>(c, r, p, q, ldq, scale, window, out, ldo, lse, part_o, part_ml, err, st)
                     : attn_t<float, 64>(c, r, p, q, ldq, scale, window, out, ldo, lse, part_o, part_ml, err, st);
}

}  // namespace sps
