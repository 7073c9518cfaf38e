// Attention of a batch's new tokens over the pages of their sequences
// (sps_paged_attention). With G query heads per KV head, the query rows of one
// (sequence, KV head) are its tokens x G; a work item is a tile of them against
// a range of 32-position blocks. Per block S^T = K Q^T with MFMA (A = key tile,
// B = Q^T), an online softmax on the S^T registers, and O^T += V^T P^T (A =
// value tile, B = the softmax tile as the score MFMA leaves it, which the value
// tiles' position order is made for). Two classes of sequences:
//  - few rows (a token, or a speculative chunk, per sequence): the keys and
//    values are read once for all of a KV head's rows and their bytes bound it.
//    The four waves take blocks in turn, page tiles go straight into registers,
//    and their (O, reference, sum) meet in LDS. Many rows (17 to 48) share the
//    read in two or three tiles; in the other class, whose tiles would be mostly
//    empty, they took 178 us where this one then took 126 (16 sequences x 5
//    tokens, the third line below).
//  - many rows (prompts): the matrix units bound it. Waves take different rows
//    against blocks that all share through LDS.
// Where the items of whole sequences would leave CUs idle, ranges of the
// positions are items of their own, joined by a second launch. Their length is
// chosen on the device from the lengths as they are, so that a captured call
// follows them: by pricing up to 64 lengths for up to 64 sequences (whose items
// are few enough for the rounds over the card to matter), by an even share of
// all blocks for more.
// Measured, bf16, head_dim 128, with the second launch (reads of ~7 TB/s and
// 1258 TFLOP/s in a large product are this card's rates):
//   1 token at position 2048, 32 heads on 32                   14 us (launches)
//   16 x 5 tokens at 4.5 to 8 thousand, 64 heads on 8          92 us, 4.8 TB/s
//   4 x 1 tokens at 105 to 126 thousand, 32 heads on 8        284 us, 6.6 TB/s
//   a prompt of 8192 tokens, 32 heads on 8                    540 us, 1.02 PFLOP/s (574 on another card)
//   1297 tokens of 27 sequences (three of 264 to 665), 64
//     heads on 8, over windows of 4096 positions              293 us
// fp32: 2 x 5 tokens at 64 to 79 positions 7 us, a launch.
#include <algorithm>

#include "paged.h"

namespace sps {

// A value that is the same in every lane, in a scalar register.
__device__ __forceinline__ int uniform(int x) { return __builtin_amdgcn_readfirstlane(x); }
__device__ __forceinline__ const char* uniform(const char* p) {
  const uint64_t x = reinterpret_cast<uint64_t>(p);
  const uint32_t lo = uniform(static_cast<int>(x)), hi = uniform(static_cast<int>(x >> 32));
  return reinterpret_cast<const char*>(static_cast<uint64_t>(hi) << 32 | lo);
}
__device__ __forceinline__ SeqRows uniform(SeqRows s) {
  s.r0 = uniform(s.r0);
  s.n = uniform(s.n);
  s.p0 = uniform(s.p0);
  return s;
}

// Where an item belongs.
struct Place {
  SeqRows s;
  int b, tile, range, ranges, kvh;
  int per;                 // blocks per range
  long slot;               // of the tile's first range (ranges > 1); the others follow H apart
};

// Sequences with more than `above` and up to `limit` query rows, in tiles of
// `tile` (plan.h). What an item costs beside its blocks, in blocks: own, and
// where it is one of several ranges split more for its partials.
struct Class {
  int tile, target, above, limit, own, split;
  int items, slots;        // the grid's, the workspace's
};

// What the second launch has to join: entry i of the slots' descriptors, if i
// is a tile's first slot (ranges > 1).
struct Join {
  int r0, rows, tile, kvh, ranges;
};

// A sequence's tiles in the class, and the blocks that its rows see.
__device__ __forceinline__ int2 tiles_blocks(const PagedView& c, const Class& k, const SeqRows& s, int window) {
  const int cap = c.max_pages << c.page_log2;
  const int end = min(max(s.p0 + s.n, 0), cap);
  const int lo = window ? min(max(s.p0 - window + 1, 0), end) : 0;
  const int rows = s.n * c.G;
  return make_int2(rows > k.above && rows <= k.limit ? static_cast<int>((rows + k.tile - 1u) / k.tile) : 0,
                   (end + 31) / 32 - lo / 32);
}

// The smallest of 64 lanes' values, with DPP moves (lanes without a source keep theirs).
template <int CTRL, int ROWS>
__device__ __forceinline__ float dpp_min(float v) {
  const int x = __builtin_bit_cast(int, v);
  return fminf(v, __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(x, x, CTRL, ROWS, 0xf, false)));
}
__device__ __forceinline__ float wave_min_dpp(float v) {
  v = dpp_min<0x111, 0xf>(v);   // row_shr:1 .. 8, then across the rows of 16: lane 63 has it
  v = dpp_min<0x112, 0xf>(v);
  v = dpp_min<0x114, 0xf>(v);
  v = dpp_min<0x118, 0xf>(v);
  v = dpp_min<0x142, 0xa>(v);
  v = dpp_min<0x143, 0xc>(v);
  return __builtin_bit_cast(float, __builtin_amdgcn_readlane(__builtin_bit_cast(int, v), 63));
}

// How the positions are split: the first `whole` tiles (of the sequences in
// order) not at all, the others in ranges of `per` blocks.
struct Split {
  int whole, per;
};

// The split of up to 64 sequences' tiles and blocks (one a lane), priced in the
// time of a block: lane r - 1 has r ranges of the longest, over the rounds that
// the items take on the card's `target` slots, or where sizes or rounds are
// uneven over the work per slot and most of an item until the last one ends
// (work-groups go faster as others end). Where the tiles fill a round by
// themselves the upper 32 lanes leave whole rounds unsplit and split what is
// left (64 heads on 8, chunks of 1100 tokens at position 12000: 665 us with all
// tiles alike, 469 so; 2300 at 8000 764 and 715). Joining costs kJoinBlocks.
// Every lane takes the cheapest.
constexpr int kJoinBlocks = 3;
__device__ __forceinline__ Split choose_split(const PagedView& c, const Class& k, int tiles, int blocks) {
  const int lane = threadIdx.x & 63;
  int most = 0, all = 0;
  for (int b = 0; b < c.B; ++b) {
    most = max(most, __builtin_amdgcn_readlane(blocks, b));
    all += __builtin_amdgcn_readlane(tiles, b);
  }
  const float slots = static_cast<float>(k.target);
  const int rounds = static_cast<int>(static_cast<float>(all) * c.H / slots);
  const bool rest = rounds && lane >= 32;
  const int whole = rest ? rounds * k.target / c.H : 0, parts = rest ? lane - 30 : lane + 1;
  const int per = max(kPagedMinBlocks, static_cast<int>((most + parts - 1u) / static_cast<uint32_t>(parts)));
  const float inv = 1.f / per;
  int items = 0, before = 0;
  float work = 0.f;
  for (int b = 0; b < c.B; ++b) {
    const int t = __builtin_amdgcn_readlane(tiles, b), n = __builtin_amdgcn_readlane(blocks, b);
    const int left = min(max(before + t - whole, 0), t);
    before += t;
    // (n + per - 1) / per, exactly: n < 2^17, so that half a unit outweighs the rounding.
    items += left * max(static_cast<int>((static_cast<float>(n + per - 1) + 0.5f) * inv), 1);
    work += static_cast<float>(left) * n;
  }
  const bool split = parts > 1 && per < most;
  const float own = static_cast<float>(k.own + (split ? k.split : 0));
  const float n = static_cast<float>(items) * c.H;
  const float each = min(per, most) + own;
  float cost = n > 0.f ? fminf(ceilf(n / slots) * each, (work * c.H + n * own) / fminf(n, slots) + 0.75f * each) : 0.f;
  if (split) cost += kJoinBlocks;
  if (rest) cost += rounds * static_cast<float>(most + k.own);
  if (lane && n > (rest ? 1 : kPagedMostItems) * slots) cost = INFINITY;   // the grid's and the workspace's bound
  const uint64_t cheapest = __ballot(cost == wave_min_dpp(cost));
  if (!cheapest) return Split{0, kPagedMinBlocks};
  const int src = __ffsll(static_cast<unsigned long long>(cheapest)) - 1;
  return Split{__builtin_amdgcn_readlane(whole, src), __builtin_amdgcn_readlane(per, src)};
}

// One step of the search for item `want` (of H KV heads each): `tiles` and
// `blocks` of 64 sequences, one a lane, the first `whole` of a lane's tiles
// unsplit; *before: (items << 32 | slots) of the sequences before them. The lane
// that has it, or -1.
__device__ __forceinline__ int find_lane(int tiles, int blocks, int whole, int per, int want, int kvh, int H,
                                         uint64_t* before, Place* out) {
  const uint32_t ranges = max(1u, (blocks + per - 1u) / per), cut = (tiles - whole) * ranges;
  const uint32_t slots = ranges > 1 ? cut : 0, mine = whole + cut;
  const uint64_t incl = wave_incl_scan_u64(static_cast<uint64_t>(mine) << 32 | slots) + *before;
  const uint64_t hit = __ballot(want < static_cast<int>(incl >> 32));
  *before = readlane_u64(incl, 63);
  if (!hit) return -1;
  const int src = __ffsll(static_cast<unsigned long long>(hit)) - 1;
  const uint64_t inc = readlane_u64(incl, src);
  const int at = want - (static_cast<int>(inc >> 32) - __builtin_amdgcn_readlane(static_cast<int>(mine), src));
  const int first = __builtin_amdgcn_readlane(whole, src);
  out->kvh = kvh;
  if (at < first) {
    out->ranges = 1;
    out->tile = at;
    out->range = 0;
    out->per = 1 << 20;                            // all blocks
    out->slot = 0;
    return src;
  }
  out->ranges = __builtin_amdgcn_readlane(static_cast<int>(ranges), src);
  const int tile = uniform(static_cast<int>(static_cast<uint32_t>(at - first) / static_cast<uint32_t>(out->ranges)));
  out->tile = first + tile;
  out->range = at - first - tile * out->ranges;
  out->per = per;
  const uint32_t slot0 = static_cast<uint32_t>(inc) - __builtin_amdgcn_readlane(static_cast<int>(slots), src);
  out->slot = (static_cast<long>(slot0) + static_cast<long>(tile) * out->ranges) * H + kvh;
  return src;
}

// The place of item number idx; false past the last. Every work-group
// computes the same plan from the same lengths; the first one leaves the number
// of slots in *count. `words`: LDS for 2 kMaxPagedB ints, free again after the next barrier.
__device__ __forceinline__ bool find_place(const PagedView& c, const PagedRows& r, int window, const Class& k, int idx,
                                           int* words, int* count, int* err, Place* out) {
  const int lane = threadIdx.x & 63;
  const int want = uniform(static_cast<int>(static_cast<uint32_t>(idx) / static_cast<uint32_t>(c.H)));
  const int kvh = idx - want * c.H;
  uint64_t before = 0;
  bool found = false;
  if (c.B <= kMaxFew) {
    // A sequence a lane, in registers.
    SeqRows s{};
    if (lane < c.B) s = seq_rows(c, r, lane);
    if (idx == 0 && s.bad) atomicOr(err, kErrCapacity);
    const int2 tb = lane < c.B ? tiles_blocks(c, k, s, window) : make_int2(0, 0);
    const Split sp = choose_split(c, k, tb.x, tb.x ? tb.y : 0);
    int whole = 0;
    if (sp.whole) {
      const int end = static_cast<int>(wave_incl_scan_u64(static_cast<uint64_t>(tb.x)));
      whole = tb.x - min(max(end - sp.whole, 0), tb.x);
    }
    const int src = find_lane(tb.x, tb.y, whole, sp.per, want, kvh, c.H, &before, out);
    if (src >= 0) {
      out->b = src;
      out->s.r0 = __builtin_amdgcn_readlane(s.r0, src);
      out->s.n = __builtin_amdgcn_readlane(s.n, src);
      out->s.p0 = __builtin_amdgcn_readlane(s.p0, src);
      found = true;
    }
  } else {
    // More sequences fill the card by themselves: about `target` items and one per tile.
    int *s_tiles = words, *s_blocks = words + kMaxPagedB;
    for (int b = threadIdx.x; b < c.B; b += blockDim.x) {
      const SeqRows s = seq_rows(c, r, b);
      if (idx == 0 && s.bad) atomicOr(err, kErrCapacity);
      const int2 tb = tiles_blocks(c, k, s, window);
      s_tiles[b] = tb.x;
      s_blocks[b] = tb.y;
    }
    __syncthreads();
    uint64_t all = 0;
    for (int b0 = 0; b0 < c.B; b0 += 64)
      all += wave_sum_u64(b0 + lane < c.B ? static_cast<uint64_t>(s_tiles[b0 + lane]) * s_blocks[b0 + lane] : 0);
    const int per = uniform(max(kPagedMinBlocks, static_cast<int>(ceil(static_cast<double>(all) * c.H / k.target))));
    for (int b0 = 0; b0 < c.B && (!found || idx == 0); b0 += 64) {
      Place here;
      const int b = b0 + lane;
      const int src = find_lane(b < c.B ? s_tiles[b] : 0, b < c.B ? s_blocks[b] : 0, 0, per, want, kvh, c.H,
                                &before, &here);
      if (src < 0 || found) continue;
      *out = here;
      out->b = uniform(b0 + src);
      out->s = uniform(seq_rows(c, r, out->b));
      found = true;
    }
  }
  // More items than the grid has (only starts that break the rules): not every
  // slot's descriptor is written, so that nothing is joined.
  if (idx == 0 && threadIdx.x == 0)
    *count = static_cast<int64_t>(before >> 32) * c.H <= k.items ? static_cast<int>(static_cast<uint32_t>(before)) * c.H : 0;
  return found;
}

// A tile's first range leaves what the second launch needs, the others that
// there is nothing. False: no slot for this item (only starts that break the
// rules claim more rows than there are, and with them more slots).
__device__ __forceinline__ bool leave_join(const PagedView& c, const Class& k, const Place& pl, Join* joins) {
  if (pl.ranges == 1) return true;
  const long slot = pl.slot + static_cast<long>(pl.range) * c.H, last = pl.slot + static_cast<long>(pl.ranges - 1) * c.H;
  if (slot >= k.slots) return false;
  if (threadIdx.x == 0)
    joins[slot] = Join{pl.s.r0, pl.s.n * c.G, pl.tile, pl.kvh, pl.range == 0 && last < k.slots ? pl.ranges : 0};
  return true;
}

template <typename T> __device__ __forceinline__ bool nonfinite(T x);  // Inf or NaN
template <> __device__ __forceinline__ bool nonfinite<bf16>(bf16 x) {
  return (__builtin_bit_cast(unsigned short, x) & 0x7f80) == 0x7f80;
}
template <> __device__ __forceinline__ bool nonfinite<float>(float x) {
  return (__builtin_bit_cast(uint32_t, x) & 0x7f800000u) == 0x7f800000u;
}

__device__ __forceinline__ float fast_exp2(float x) { return __builtin_amdgcn_exp2f(x); }

// What a row sees of a block, in places of this lane's (place k: position pos0 +
// 4 grp + k, of the block's 16-position tiles k = 16 pt + r): lo < k <= hi.
struct Seen {
  int lo, hi;
};
__device__ __forceinline__ Seen seen_of(int pos0, int qpos, int window, int end, int grp) {
  const int at = pos0 + grp * 4;
  return Seen{window ? qpos - window - at : -1 - at, min(qpos, end - 1) - at};
}
// The scores of a block at places that the row does not see go to -Inf.
__device__ __forceinline__ void mask_scores(const Seen& v, bool windowed, f32x4 (&s)[2]) {
#pragma unroll
  for (int pt = 0; pt < 2; ++pt)
#pragma unroll
    for (int r = 0; r < 4; ++r) s[pt][r] = pt * 16 + r <= v.hi ? s[pt][r] : -INFINITY;
  if (!windowed) return;
#pragma unroll
  for (int pt = 0; pt < 2; ++pt)
#pragma unroll
    for (int r = 0; r < 4; ++r) s[pt][r] = pt * 16 + r > v.lo ? s[pt][r] : -INFINITY;
}

// Online softmax of one query row, spread over the four lanes with its column.
// The reference `off` that is taken off the scaled scores (in units of log2)
// follows the running maximum only once that is kLag above it: weights are at
// most 2^kLag instead of 1, which fp32 sums and bf16 weights hold as precisely,
// and the accumulators are rescaled a few times per row instead of in nearly
// every block. Each lane sums its own positions' weights.
constexpr float kLag = 8.f;
struct RowSoftmax {
  float off = 0.f;
  float lim = -INFINITY;   // kLag once there is a reference
  float sum = 0.f;
  __device__ float ref() const { return lim == -INFINITY ? -INFINITY : off; }
};
// Scores of NP tiles of 16 positions scaled and without the reference;
// returns the largest of the lane's.
template <int NP>
__device__ __forceinline__ float scale_scores(f32x4 (&s)[NP], float c_log2, const RowSoftmax& w) {
  float mx = -INFINITY;
#pragma unroll
  for (int pt = 0; pt < NP; ++pt) {
#pragma unroll
    for (int r = 0; r < 4; ++r) s[pt][r] = fmaf(s[pt][r], c_log2, -w.off);
    mx = fmaxf(fmaxf(fmaxf(fmaxf(mx, s[pt][0]), s[pt][1]), s[pt][2]), s[pt][3]);
  }
  return mx;
}
// The first reference: nothing is summed yet, so nothing else changes.
template <int NP>
__device__ __forceinline__ void first_reference(f32x4 (&s)[NP], float mx, RowSoftmax& w) {
  mx = fmaxf(mx, __shfl_xor(mx, 16));
  mx = fmaxf(mx, __shfl_xor(mx, 32));
  const bool some = mx > -INFINITY;
  w.off = some ? mx : 0.f;
  w.lim = some ? kLag : -INFINITY;
#pragma unroll
  for (int pt = 0; pt < NP; ++pt)
#pragma unroll
    for (int r = 0; r < 4; ++r) s[pt][r] -= w.off;
}
// scale_scores with a new reference where one is due; all QT rows of the lane
// together, so that one branch skips the rescaling.
template <int QT, int NP, int ND>
__device__ __forceinline__ void softmax_scale(f32x4 (&s)[QT][NP], float c_log2, RowSoftmax (&w)[QT], f32x4 (&o)[QT][ND]) {
  float mx[QT];
  bool up = false;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    mx[qt] = scale_scores(s[qt], c_log2, w[qt]);
    up |= mx[qt] > w[qt].lim;
  }
  if (!__ballot(up)) return;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    float m = fmaxf(mx[qt], __shfl_xor(mx[qt], 16));
    m = fmaxf(m, __shfl_xor(m, 32));
    const bool mine = m > w[qt].lim;               // alike in the four lanes of a row
    // Nothing summed yet: 0.
    const float alpha = !mine ? 1.f : w[qt].lim == -INFINITY ? 0.f : fast_exp2(-m);
    m = mine ? m : 0.f;
    w[qt].off += m;
    w[qt].lim = mine ? kLag : w[qt].lim;
    w[qt].sum *= alpha;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[qt][dt] *= alpha;
#pragma unroll
    for (int pt = 0; pt < NP; ++pt)
#pragma unroll
      for (int r = 0; r < 4; ++r) s[qt][pt][r] -= m;
  }
}
template <int NP>
__device__ __forceinline__ void softmax_weights(f32x4 (&s)[NP], RowSoftmax& w) {
#pragma unroll
  for (int pt = 0; pt < NP; ++pt)
#pragma unroll
    for (int r = 0; r < 4; ++r) {
      s[pt][r] = fast_exp2(s[pt][r]);
      w.sum += s[pt][r];
    }
}

// The values of positions past the last one, which may hold anything, cleared:
// n fragments of a block, `left` positions of which are to be kept.
template <typename T, int N>
__device__ __forceinline__ void clear_past(Frag<T> (&vf)[N], int left, int grp) {
  constexpr int kWords = 8 * sizeof(T) / 4, kPer = 4 / sizeof(T);   // 32-bit words of a fragment, elements of a word
  typedef uint32_t words __attribute__((ext_vector_type(kWords)));
  words keep;
#pragma unroll
  for (int i = 0; i < kWords; ++i) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < kPer; ++e) {
      const int x = i * kPer + e;
      m |= (x >> 2) * 16 + (x & 3) < left - grp * 4 ? (kPer == 1 ? ~0u : 0xffffu << (16 * e)) : 0;
    }
    keep[i] = m;
  }
#pragma unroll
  for (int j = 0; j < N; ++j)
    vf[j].v = __builtin_bit_cast(decltype(vf[j].v), __builtin_bit_cast(words, vf[j].v) & keep);
}

// Values of a block in which some row of the tile does not see some position:
// 0 x Inf would carry a value that is not finite into the rows that do not see
// it. Such values are taken out of the fragment, and put into the rows that see
// them by counting, per row and dim, visible +Inf, -Inf and NaN with products
// of ones.
template <typename T, int QT, int ND>
__device__ __forceinline__ void clean_values(Frag<T>& vf, int pos0, const int (&qpos)[QT], int window, int end, int grp,
                                             f32x4 (&o)[QT][ND], int dt) {
#pragma unroll 1
  for (int kind = 0; kind < 3; ++kind) {
    const float what = kind == 0 ? INFINITY : kind == 1 ? -INFINITY : NAN;
    Frag<T> one;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
      const float x = to_f32(vf.v[e]);
      one.v[e] = from_f32<T>((kind == 2 ? x != x : x == what) ? 1.f : 0.f);
    }
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      Frag<T> see;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const int pos = pos0 + (e >> 2) * 16 + grp * 4 + (e & 3);
        see.v[e] = from_f32<T>(pos <= qpos[qt] && (!window || pos > qpos[qt] - window) && pos < end ? 1.f : 0.f);
      }
      const f32x4 n = mma8(f32x4{0.f, 0.f, 0.f, 0.f}, one, see);
#pragma unroll
      for (int r = 0; r < 4; ++r)
        if (n[r] > 0.f) o[qt][dt][r] += what;
    }
  }
#pragma unroll
  for (int e = 0; e < 8; ++e)
    if (nonfinite(vf.v[e])) vf.v[e] = from_f32<T>(0.f);
}

// Row `in` of a tile, of its dims 16 dt .. 16 (dt + N) - 1 the runs 4 grp .. + 3 of
// 16: the output, or a partial if the tile has more ranges.
template <typename T, int DH, int N>
__device__ __forceinline__ void write_row(const PagedView& c, const Class& k, const Place& pl, int in, int tok, int head,
                                          int grp, int dt, float ref, float l, const f32x4 (&o)[N], T* out, int64_t ldo,
                                          float* lse, float* part_o, float2* part_ml) {
  const bool first = grp == 0 && dt == 0;
  if (pl.ranges > 1) {
    const size_t at = (pl.slot + static_cast<long>(pl.range) * c.H) * k.tile + in;
    if (first) part_ml[at] = make_float2(ref, l);
#pragma unroll
    for (int d = 0; d < N; ++d) *reinterpret_cast<f32x4*>(part_o + at * DH + (dt + d) * 16 + grp * 4) = o[d];
    return;
  }
  // A sum of zero: no visible position, or none with weight.
  const float inv = 1.f / l;
  T* dst = out + tok * ldo + head * DH + dt * 16 + grp * 4;
#pragma unroll
  for (int d = 0; d < N; ++d) store4_any(dst + d * 16, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : o[d] * inv);
  if (lse && first)
    lse[static_cast<size_t>(tok) * c.H * c.G + head] = l == 0.f ? -INFINITY : 0.69314718f * ref + logf(l);
}

// LDS of a work-group whose sequences have up to QT tiles.
template <typename T, int DH, int QT>
struct FewLds {
  // The plan's words per sequence, then two waves' (O, reference, sum), or with one tile all four's.
  static constexpr int kF4 = (QT > 2 ? 2 * QT : 4) * (DH / 16) * 64, kPlanF4 = 2 * kMaxPagedB / 4;
  f32x4 o[kF4 > kPlanF4 ? kF4 : kPlanF4];
  float2 ml[(QT > 2 ? 2 * QT : 4) * 64];
  Frag<T> q[QT > 1 || sizeof(T) == 4 ? QT * (DH / 32) * 64 : 1];
};

// An item of QT tiles. Reads of pages bypass the caches' retention (each is read
// once: 285 us so, 321 without, for the 4 x 1 tokens at 105 thousand positions and more).
template <typename T, int DH, int QT, typename Lds>
__device__ __forceinline__ void few_item(const PagedView& c, const Class& k, const Place& pl, const T* __restrict__ q,
                                         int64_t ldq, float scale, int window, T* __restrict__ out, int64_t ldo,
                                         float* __restrict__ lse, float* __restrict__ part_o,
                                         float2* __restrict__ part_ml, int* err, Lds& lds) {
  constexpr int ND = DH / 16;
  f32x4* sm = lds.o;
  float2* sml = lds.ml;
  Frag<T>* sq = lds.q;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int r16 = lane & 15, grp = lane >> 4;
  const SeqRows& s = pl.s;
  const int cap = c.max_pages << c.page_log2;
  const int nrows = s.n * c.G;
  // Positions of the first and last token, and what they see.
  const int first = s.p0, last = s.p0 + s.n - 1;
  const int end = min(max(last + 1, 0), cap);
  const int lo = window ? min(max(first - window + 1, 0), end) : 0;
  const int base = (window ? min(max(s.p0 - window + 1, 0), min(max(s.p0 + s.n, 0), cap)) : 0) / 32;
  const int blk0 = max(base + pl.range * pl.per, lo / 32), blk1 = min(base + (pl.range + 1) * pl.per, (end + 31) / 32);
  const float c_log2 = scale * 1.4426950408889634f;

  // The queries' fragments, in registers or (kStaged: more than a 16-row tile,
  // or fp32) in LDS, where all waves read them: two waves per SIMD need the room.
  constexpr bool kStaged = QT > 1 || sizeof(T) == 4;
  Frag<T> qf[kStaged ? 1 : DH / 32];
  // Token of row qt * 16 + r16 (-1: none): 64 rows at most, the quotient is exact.
  const float inv_g = 1.f / c.G;
  int in16 = r16;
  auto token = [&](int qt) {
    const int row = qt * 16 + in16;
    return row < nrows ? static_cast<int>((row + 0.5f) * inv_g) : -1;
  };
  auto position = [&](int qt) {
    const int t = token(qt);
    return t < 0 ? -1 : s.p0 + t;
  };
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int row = qt * 16 + r16, t = max(token(qt), 0);
    const bool valid = row < nrows;
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt) {
      const T* src = q + (s.r0 + t) * ldq + (pl.kvh * c.G + row - t * c.G) * DH + dt * 32 + grp * 8;
      if (!kStaged)
        qf[dt] = valid ? load_frag_any(src) : Frag<T>::zero();
      else if ((qt * (DH / 32) + dt) % 4 == wave)
        sq[(qt * (DH / 32) + dt) * 64 + lane] = valid ? load_frag_any(src) : Frag<T>::zero();
    }
  }
  auto query = [&](int qt, int dt) { return kStaged ? sq[(qt * (DH / 32) + dt) * 64 + lane] : qf[kStaged ? 0 : dt]; };
  RowSoftmax w[QT];
  f32x4 o[QT][ND];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};

  // This wave's blocks are blk0 + wave + 4 i; the pages of 64 of them at a
  // time. The next block's keys are asked for once the scores are done with
  // this one's, its values once the products are: one block's registers keep
  // the loads going.
  const int32_t* tab = c.table + static_cast<size_t>(pl.b) * c.max_pages;
  const size_t area = static_cast<size_t>(DH) << c.page_log2;
  const int in_page = (1 << c.page_log2) - 1;
  const int nb = blk1 > blk0 + wave ? (blk1 - blk0 - wave + 3) / 4 : 0;
  int id = -1, id0 = 0;                            // the pages of blocks id0 .. id0 + 63, one a lane
  auto pages = [&](int i0) {
    id0 = i0;
    id = -1;
    if (i0 + lane < nb) {
      id = tab[(blk0 + wave + 4 * (i0 + lane)) >> (c.page_log2 - 5)];
      if (id < 0 || id >= c.n_pages) {
        atomicOr(err, kErrBadPage);
        id = -1;
      }
    }
  };
  // The first block from i on whose page is good (nb: none), and its place.
  size_t off = 0;
  auto seek = [&](int i) {
    for (; i < nb; ++i) {
      if (i - id0 >= 64) pages(i);
      const int page = __builtin_amdgcn_readlane(id, i - id0);
      if (page < 0) continue;
      off = (static_cast<size_t>(page) * c.H + pl.kvh) * area +
            static_cast<size_t>((blk0 + wave + 4 * i) * 32 & in_page) * DH + lane * 8;
      break;
    }
    return i;
  };
  Frag<T> kf[2][DH / 32], vf[ND];
  auto load_keys = [&] {
    const T* kp = static_cast<const T*>(c.k) + off;
#pragma unroll
    for (int pt = 0; pt < 2; ++pt)
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt) kf[pt][dt] = load_frag_stream(kp + (pt * (DH / 32) + dt) * 512);
  };
  auto load_values = [&] {
    const T* vp = static_cast<const T*>(c.v) + off;
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) vf[dt] = load_frag_stream(vp + dt * 512);
  };
  pages(0);
  __syncthreads();                                 // the staged queries; the plan's words have been read
  int i = seek(0);
  if (i < nb) {
    load_keys();
    load_values();
  }
  auto scores = [&](f32x4 (&sc)[QT][2]) {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      sc[qt][0] = sc[qt][1] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt) {
        const Frag<T> qd = query(qt, dt);
#pragma unroll
        for (int pt = 0; pt < 2; ++pt) sc[qt][pt] = mma8(sc[qt][pt], kf[pt][dt], qd);
      }
    }
  };
  auto products = [&](f32x4 (&sc)[QT][2]) {
#pragma unroll
    for (int qt = 0; qt < QT; ++qt) {
      softmax_weights(sc[qt], w[qt]);
      // The weights in bf16 as hi + lo, p to 2^-16 relative: the second product
      // costs nothing where the loads are what takes the time.
      constexpr bool kLow = sizeof(T) == 2;
      Frag<T> hi, lw;
#pragma unroll
      for (int e = 0; e < 8; ++e) {
        const float p = sc[qt][e >> 2][e & 3];
        hi.v[e] = from_f32<T>(p);
        if (kLow) lw.v[e] = from_f32<T>(p - to_f32(hi.v[e]));
      }
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) {
        o[qt][dt] = mma8(o[qt][dt], vf[dt], hi);
        if (kLow) o[qt][dt] = mma8(o[qt][dt], vf[dt], lw);
      }
    }
  };
  bool fresh = true;                               // no reference yet
  while (i < nb) {
    f32x4 sc[QT][2];
    // Blocks that every row sees all of and that need no new reference: nothing
    // but products on the accumulators.
    while (true) {
      const int pos0 = (blk0 + wave + 4 * i) * 32;
      if (pos0 + 31 > min(first, end - 1) || (window && pos0 <= last - window)) break;
      scores(sc);
      bool up = false;
      float mx[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        mx[qt] = scale_scores(sc[qt], c_log2, w[qt]);
        up |= mx[qt] > w[qt].lim;
      }
      if (fresh) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) first_reference(sc[qt], mx[qt], w[qt]);
        fresh = false;
      } else if (__ballot(up)) {
        break;
      }
      const int next = seek(i + 1);
      if (next < nb) load_keys();
      products(sc);
      if (next < nb) load_values();
      i = next;
      if (i >= nb) break;
    }
    if (i >= nb) break;
    fresh = false;
    const int pos0 = (blk0 + wave + 4 * i) * 32;
    scores(sc);
    const bool masked = pos0 + 31 > min(first, end - 1) || (window && pos0 <= last - window);
    if (masked) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) mask_scores(seen_of(pos0, position(qt), window, end, grp), window != 0, sc[qt]);
    }
    softmax_scale(sc, c_log2, w, o);
    if (masked) {
      if (pos0 + 32 > end) clear_past(vf, end - pos0, grp);
      // The values times zero: NaN if one of them is not finite.
      f32x4 zero{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < ND; ++dt) zero = mma8(zero, vf[dt], Frag<T>::zero());
      if (__ballot(zero[0] + zero[1] + zero[2] + zero[3] != 0.f)) {
        int qpos[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) qpos[qt] = position(qt);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) clean_values(vf[dt], pos0, qpos, window, end, grp, o, dt);
      }
    }
    products(sc);
    i = seek(i + 1);
    if (i < nb) {
      load_keys();
      load_values();
    }
  }

  asm volatile("" : "+v"(in16));                   // the rows' places again, not kept through the loop
  float ref[QT], sum[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    ref[qt] = w[qt].ref();
    sum[qt] = w[qt].sum + __shfl_xor(w[qt].sum, 16);
    sum[qt] += __shfl_xor(sum[qt], 32);
  }
  if constexpr (QT == 1) {
    // Every wave joins a quarter of the dims.
    sml[wave * 64 + lane] = make_float2(ref[0], sum[0]);
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) sm[(wave * ND + dt) * 64 + lane] = o[0][dt];
    __syncthreads();
    float2 ml[4];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      ml[x] = sml[x * 64 + lane];
      m = fmaxf(m, ml[x].x);
    }
    const float mu = m == -INFINITY ? 0.f : m;
    f32x4 part[ND / 4] = {};
#pragma unroll
    for (int x = 0; x < 4; ++x) {
      const float a = fast_exp2(ml[x].x - mu);
      l += a * ml[x].y;
#pragma unroll
      for (int d = 0; d < ND / 4; ++d) part[d] += a * sm[(x * ND + wave * (ND / 4) + d) * 64 + lane];
    }
    if (const int t = token(0); t >= 0)
      write_row<T, DH, ND / 4>(c, k, pl, r16, s.r0 + t, pl.kvh * c.G + r16 - t * c.G, grp, wave * (ND / 4), m, l, part,
                               out, ldo, lse, part_o, part_ml);
    return;
  }
  // Waves 2, 3 into 0, 1, then 1 into 0.
#pragma unroll
  for (int half = 2; half; half >>= 1) {
    if (wave >= half && wave < 2 * half) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        sml[((wave - half) * QT + qt) * 64 + lane] = make_float2(ref[qt], sum[qt]);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) sm[(((wave - half) * QT + qt) * ND + dt) * 64 + lane] = o[qt][dt];
      }
    }
    __syncthreads();
    if (wave < half) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        const float2 ml = sml[(wave * QT + qt) * 64 + lane];
        const float m = fmaxf(ref[qt], ml.x), mu = m == -INFINITY ? 0.f : m;
        const float a = fast_exp2(ref[qt] - mu), b = fast_exp2(ml.x - mu);
        ref[qt] = m;
        sum[qt] = a * sum[qt] + b * ml.y;
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) o[qt][dt] = a * o[qt][dt] + b * sm[((wave * QT + qt) * ND + dt) * 64 + lane];
      }
    }
    __syncthreads();
  }
  if (wave) return;
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
    if (const int t = token(qt); t >= 0)
      write_row<T, DH, ND>(c, k, pl, qt * 16 + r16, s.r0 + t, pl.kvh * c.G + qt * 16 + r16 - t * c.G, grp, 0, ref[qt],
                           sum[qt], o[qt], out, ldo, lse, part_o, part_ml);
}

// A class's share of the workspace.
struct Parts {
  float* o;
  float2* ml;
  Join* joins;
  int* count;
};

// Item idx of the first class. The tiles it has are its sequence's (k.tile holds
// all its rows): their own straight code for each number of them, up to QT.
template <typename T, int DH, int QT>
__device__ __forceinline__ void few_group(const PagedView& c, const PagedRows& r, const Class& k, int idx,
                                          const T* __restrict__ q, int64_t ldq, float scale, int window,
                                          T* __restrict__ out, int64_t ldo, float* __restrict__ lse, const Parts& w,
                                          int* err, FewLds<T, DH, QT>& lds) {
  Place pl;
  if (!find_place(c, r, window, k, idx, reinterpret_cast<int*>(lds.o), w.count, err, &pl)) return;
  if (!leave_join(c, k, pl, w.joins)) return;
  const int tiles = (pl.s.n * c.G + 15) / 16;
  if (tiles <= 1)
    few_item<T, DH, 1>(c, k, pl, q, ldq, scale, window, out, ldo, lse, w.o, w.ml, err, lds);
  else if (QT > 1 && (QT == 2 || tiles == 2))
    few_item<T, DH, QT < 2 ? QT : 2>(c, k, pl, q, ldq, scale, window, out, ldo, lse, w.o, w.ml, err, lds);
  else if (QT > 2)
    few_item<T, DH, QT>(c, k, pl, q, ldq, scale, window, out, ldo, lse, w.o, w.ml, err, lds);
}

template <typename T, int DH, int QT>
__global__ __launch_bounds__(256, 2) void paged_few_kernel(PagedView c, PagedRows r, Class k, const T* __restrict__ q,
                                                           int64_t ldq, float scale, int window, T* __restrict__ out,
                                                           int64_t ldo, float* __restrict__ lse, Parts w, int* err) {
  __shared__ FewLds<T, DH, QT> lds;
  few_group<T, DH, QT>(c, r, k, blockIdx.x, q, ldq, scale, window, out, ldo, lse, w, err, lds);
}

// The ranges of a tile's rows joined: 16 lanes per row, four rows per wave (one
// row's loads wait for each other, so rows in flight are what counts).
template <typename T, int DH>
__global__ __launch_bounds__(256) void paged_join_kernel(PagedView c, int tile_rows, const Join* __restrict__ joins,
                                                         const int* __restrict__ count, const float* __restrict__ part_o,
                                                         const float2* __restrict__ part_ml, T* __restrict__ out,
                                                         int64_t ldo, float* __restrict__ lse) {
  constexpr int NV = DH / 64;                      // 4-dim pieces per lane
  const long slot = blockIdx.x;
  const Join j = joins[slot];                      // inside the workspace, written if below the count
  if (slot >= *count || j.ranges == 0) return;
  const int in = blockIdx.y * 16 + static_cast<int>(threadIdx.x >> 4), lane = threadIdx.x & 15;
  const int row = j.tile * tile_rows + in;
  if (row >= j.rows) return;                       // tile_rows is a multiple of 16
  const size_t step = static_cast<size_t>(c.H) * tile_rows;      // from range to range
  const float2* ml = part_ml + slot * tile_rows + in;
  const float* po = part_o + (slot * tile_rows + in) * DH + lane * 4;
  float m = -INFINITY;
  for (int i = lane; i < j.ranges; i += 16) m = fmaxf(m, ml[i * step].x);
#pragma unroll
  for (int o = 1; o < 16; o <<= 1) m = fmaxf(m, __shfl_xor(m, o));
  const float mu = m == -INFINITY ? 0.f : m;
  float l = 0.f;
  f32x4 acc[NV] = {};
#pragma unroll 4
  for (int i = 0; i < j.ranges; ++i) {
    const float2 x = ml[i * step];
    const float wt = fast_exp2(x.x - mu);          // 0 for a range of which the row sees nothing (its partial is zero)
    l += wt * x.y;
#pragma unroll
    for (int v = 0; v < NV; ++v) acc[v] += wt * *reinterpret_cast<const f32x4*>(po + i * step * DH + v * 64);
  }
  const int t = static_cast<int>(static_cast<uint32_t>(row) / static_cast<uint32_t>(c.G));
  const int tok = j.r0 + t, head = j.kvh * c.G + row - t * c.G;
  const float inv = 1.f / l;
#pragma unroll
  for (int v = 0; v < NV; ++v)
    store4_any(out + tok * ldo + head * DH + v * 64 + lane * 4, l == 0.f ? f32x4{0.f, 0.f, 0.f, 0.f} : acc[v] * inv);
  if (lse && lane == 0)
    lse[static_cast<size_t>(tok) * c.H * c.G + head] = l == 0.f ? -INFINITY : 0.69314718f * m + logf(l);
}

// Sequences with many query rows: NW waves of 16 QT rows each against the
// range's blocks, 64 positions at a time through LDS. The page tiles are
// copied there as they lie (global_load_lds, a KiB per wave and copy: no
// registers, no bank conflicts on the way back), the next 64 positions while
// these are computed. What bounds it is the matrix units with the softmax's
// vector work beside them, which the second wave of every SIMD covers: a fragment
// read from LDS serves QT products, so bf16 waves have two tiles (with three
// the registers leave one wave a SIMD: 1050 us where this takes 540, and the
// same rows in eight waves a work-group 712 against 677 at that step); fp32,
// whose tiles take twice the registers, has one and eight waves. Stages of 32
// positions 650 us against 641: more barriers.
__device__ __forceinline__ void copy_to_lds(const void* src, uint32_t lane_offset, uint32_t lds) {
  // Untracked by the compiler's wait counts: it would make every LDS read wait
  // for the copies of the other stage too. Nor does it see that the address may
  // come from v_readfirstlane right before, and a scalar register that a vector
  // instruction wrote takes 5 wait states until a vector memory instruction may
  // read it: s_nop 4 (M0 needs one of them).
  asm volatile("s_nop 4\n\tglobal_load_lds_dwordx4 %0, %1" ::"v"(lane_offset), "s"(src), "{m0}"(lds) : "memory");
}

template <typename T, int DH>
struct ManyLds {
  static constexpr int NB = sizeof(T) == 2 ? 2 : 1;                // blocks per stage
  static constexpr int kTile = 32 * DH;                            // elements of a block's keys or values
  T stage[2][NB][2][kTile];
  static_assert(2 * NB * 2 * kTile * sizeof(T) >= 2 * kMaxPagedB * sizeof(int), "the plan's words");
};

template <typename T, int DH, int QT, int NW>
__device__ __forceinline__ void many_group(const PagedView& c, const PagedRows& r, const Class& k, int idx,
                                           const T* __restrict__ q, int64_t ldq, float scale, int window,
                                           T* __restrict__ out, int64_t ldo, float* __restrict__ lse, const Parts& parts,
                                           int* err, ManyLds<T, DH>& lds) {
  constexpr int ND = DH / 16, WR = 16 * QT;
  constexpr int NB = ManyLds<T, DH>::NB, kTile = ManyLds<T, DH>::kTile;
  constexpr int kCopies = kTile * static_cast<int>(sizeof(T)) / 1024;   // of one KiB
  static_assert(2 * NB * kCopies % NW == 0, "whole copies per wave");
  auto& stage = lds.stage;
  Place pl;
  if (!find_place(c, r, window, k, idx, reinterpret_cast<int*>(stage), parts.count, err, &pl)) return;
  // The last tiles of a prompt see most: they go first.
  const int nrows = pl.s.n * c.G, ntiles = uniform((nrows + k.tile - 1) / k.tile), tile = ntiles - 1 - pl.tile;
  pl.tile = tile;
  if (!leave_join(c, k, pl, parts.joins)) return;
  const int lane = threadIdx.x & 63, wave = uniform(threadIdx.x >> 6);
  const int r16 = lane & 15, grp = lane >> 4;
  const SeqRows& s = pl.s;
  const int cap = c.max_pages << c.page_log2;
  const int row0 = tile * k.tile, wrow0 = row0 + wave * WR;
  const int first = s.p0 + uniform(row0 / c.G), last = s.p0 + uniform((min(row0 + k.tile, nrows) - 1) / c.G);
  const int end = min(max(last + 1, 0), cap);
  const int lo = window ? min(max(first - window + 1, 0), end) : 0;
  const int base = (window ? min(max(s.p0 - window + 1, 0), min(max(s.p0 + s.n, 0), cap)) : 0) / 32;
  const int blk0 = uniform(max(base + pl.range * pl.per, lo / 32));
  const int blk1 = uniform(min(base + (pl.range + 1) * pl.per, (end + 31) / 32));
  // The same of this wave's rows; none: wlast < 0.
  const int wfirst = s.p0 + uniform(wrow0 / c.G);
  const int wlast = wrow0 < nrows ? s.p0 + uniform((min(wrow0 + WR, nrows) - 1) / c.G) : -1;
  const float c_log2 = scale * 1.4426950408889634f;

  // Token of the wave's row qt * 16 + r16 (-1: none), from that of its first.
  const int tok0 = uniform(wrow0 / c.G), part0 = wrow0 - tok0 * c.G;
  const float inv_g = 1.f / c.G;
  auto token = [&](int qt) {
    const int in = qt * 16 + r16;                  // part0 + in < G + 32: the quotient is exact
    return wrow0 + in < nrows ? tok0 + static_cast<int>((part0 + in + 0.5f) * inv_g) : -1;
  };
  Frag<T> qf[QT][DH / 32];
  int qpos[QT];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    const int row = wrow0 + qt * 16 + r16;
    const bool valid = row < nrows;
    const int t = max(token(qt), 0);
    qpos[qt] = valid ? s.p0 + t : -1;
    const T* src = q + (s.r0 + t) * ldq + (pl.kvh * c.G + (valid ? row - t * c.G : 0)) * DH + grp * 8;
#pragma unroll
    for (int dt = 0; dt < DH / 32; ++dt) qf[qt][dt] = valid ? load_frag_any(src + dt * 32) : Frag<T>::zero();
  }
  RowSoftmax w[QT];
  f32x4 o[QT][ND];
#pragma unroll
  for (int qt = 0; qt < QT; ++qt)
#pragma unroll
    for (int dt = 0; dt < ND; ++dt) o[qt][dt] = f32x4{0.f, 0.f, 0.f, 0.f};

  const int32_t* tab = c.table + static_cast<size_t>(pl.b) * c.max_pages;
  const size_t area = static_cast<size_t>(DH) << c.page_log2;
  const int in_page = (1 << c.page_log2) - 1;
  int id = -1, id0 = -64;                          // the pages of blocks id0 .. id0 + 63, one a lane
  auto page_of = [&](int blk) {
    if (blk - id0 >= 64 || id0 < 0) {
      id0 = blk;
      id = -1;
      if (blk + lane < blk1) {
        id = tab[(blk + lane) >> (c.page_log2 - 5)];
        if (id < 0 || id >= c.n_pages) {
          atomicOr(err, kErrBadPage);
          id = -1;
        }
      }
    }
    return __builtin_amdgcn_readlane(id, blk - id0);
  };
  // Copy the blocks from blk on (up to NB) into stage b; bit h of the result:
  // block h is there. A wave's share lies in one block's keys or values.
  constexpr int kShare = 2 * NB * kCopies / NW;
  static_assert(kCopies % kShare == 0, "one plane per wave");
  const int share_h = wave * kShare / (2 * kCopies), share_kv = wave * kShare / kCopies & 1;
  const char* plane = static_cast<const char*>(share_kv ? c.v : c.k) + wave * kShare % kCopies * 1024;
  auto fetch = [&](int blk, int b) {
    uint32_t there = 0;
    int mine = -1;
#pragma unroll
    for (int h = 0; h < NB; ++h) {
      const int page = blk + h < blk1 ? page_of(blk + h) : -1;
      there |= page >= 0 ? 1u << h : 0;
      if (h == share_h) mine = page;
    }
    if (mine >= 0) {
      const size_t off = (static_cast<size_t>(mine) * c.H + pl.kvh) * area + static_cast<size_t>((blk + share_h) * 32 & in_page) * DH;
      const char* src = uniform(plane + off * sizeof(T));
      const uint32_t dst = static_cast<uint32_t>(reinterpret_cast<uintptr_t>(&stage[b])) + wave * kShare * 1024;
#pragma unroll
      for (int j = 0; j < kShare; ++j) copy_to_lds(src + j * 1024, lane * 16, dst + j * 1024);
    }
    return there;
  };
  __syncthreads();                                 // the plan's words have been read
  // A stage's scores: NH blocks from h0 on.
  auto scores = [&](auto& sc, int b, int h0) {
    constexpr int NT = sizeof(sc[0]) / sizeof(f32x4);
#pragma unroll
    for (int pt = 0; pt < NT; ++pt) {
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) sc[qt][pt] = f32x4{0.f, 0.f, 0.f, 0.f};
#pragma unroll
      for (int dt = 0; dt < DH / 32; ++dt) {
        const Frag<T> kf = load_frag(&stage[b][h0 + (pt >> 1)][0][(((pt & 1) * (DH / 32) + dt) * 64 + lane) * 8]);
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) sc[qt][pt] = mma8(sc[qt][pt], kf, qf[qt][dt]);
      }
    }
  };
  // Weights rounded once to the type (bf16: half a step, 2^-8 of each, which
  // averages out over a row like the values' own rounding; a second product
  // of what is left off would cost half as much again).
  auto rounded = [&](const f32x4& x, const f32x4& y) {
    Frag<T> f;
#pragma unroll
    for (int e = 0; e < 4; ++e) {
      f.v[e] = from_f32<T>(x[e]);
      f.v[4 + e] = from_f32<T>(y[e]);
    }
    return f;
  };
  uint32_t there = blk0 < blk1 ? fetch(blk0, 0) : 0, next = 0, on = 0;
  bool ready = false, fresh = true;                // fresh: no reference yet
  int b = 0, blk = blk0;
  while (blk < blk1) {
    // Stages that every row of the wave sees all of, and whose scores need no
    // new reference: one straight run, with nothing but products on the
    // accumulators (other paths through it cost their copies).
    while (true) {
      const int pos0 = blk * 32;
      if (!ready) {
        // This stage's copies have landed, and the other one's reads are over, in every wave.
        asm volatile("s_waitcnt vmcnt(0) lgkmcnt(0)\n\ts_barrier" ::: "memory");
        next = blk + NB < blk1 ? fetch(blk + NB, b ^ 1) : 0;
        on = 0;                                    // blocks this wave's rows see anything of
#pragma unroll
        for (int h = 0; h < NB; ++h)
          on |= pos0 + h * 32 <= wlast && !(window && pos0 + h * 32 + 31 <= wfirst - window) ? there & 1u << h : 0;
        ready = true;
      }
      if (fresh || on != (1u << NB) - 1 || pos0 + NB * 32 - 1 > min(wfirst, end - 1) || (window && pos0 <= wlast - window)) break;
      f32x4 sc[QT][2 * NB];
      scores(sc, b, 0);
      bool up = false;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) up |= scale_scores(sc[qt], c_log2, w[qt]) > w[qt].lim;
      // Key fragments are read four ahead of their products (540 us; left to the
      // compiler's order 552, six ahead 541).
      __builtin_amdgcn_sched_group_barrier(0x100, 4, 0);
#pragma unroll
      for (int g = 0; g < 2 * NB * (DH / 32) - 4; ++g) {
        __builtin_amdgcn_sched_group_barrier(0x008, QT, 0);
        __builtin_amdgcn_sched_group_barrier(0x100, 1, 0);
      }
      __builtin_amdgcn_sched_group_barrier(0x008, 4 * QT, 0);
      if (__ballot(up)) break;
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) softmax_weights(sc[qt], w[qt]);
#pragma unroll
      for (int h = 0; h < NB; ++h) {
        Frag<T> pf[QT];
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) pf[qt] = rounded(sc[qt][2 * h], sc[qt][2 * h + 1]);
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          const Frag<T> vf = load_frag(&stage[b][h][1][(dt * 64 + lane) * 8]);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) o[qt][dt] = mma8(o[qt][dt], vf, pf[qt]);
        }
      }
      ready = false;
      there = next;
      b ^= 1;
      blk += NB;
      if (blk >= blk1) break;
    }
    if (blk >= blk1) break;
    // The others block by block.
    fresh = false;
#pragma unroll 1
    for (int h = 0; h < NB; ++h) {
      if (!(on >> h & 1)) continue;
      const int pos0 = (blk + h) * 32;
      const bool masked = pos0 + 31 > min(wfirst, end - 1) || (window && pos0 <= wlast - window);
      f32x4 sc[QT][2];
      scores(sc, b, h);
      if (masked) {
#pragma unroll
        for (int qt = 0; qt < QT; ++qt) mask_scores(seen_of(pos0, qpos[qt], window, end, grp), window != 0, sc[qt]);
      }
      softmax_scale(sc, c_log2, w, o);
      Frag<T> pf[QT];
#pragma unroll
      for (int qt = 0; qt < QT; ++qt) {
        softmax_weights(sc[qt], w[qt]);
        pf[qt] = rounded(sc[qt][0], sc[qt][1]);
      }
      bool plain = !masked;
      if (masked && pos0 + 32 <= end) {
        // The values times zero: NaN if one of them is not finite.
        f32x4 zero{0.f, 0.f, 0.f, 0.f};
#pragma unroll
        for (int dt = 0; dt < ND; ++dt)
          zero = mma8(zero, load_frag(&stage[b][h][1][(dt * 64 + lane) * 8]), Frag<T>::zero());
        plain = !__ballot(zero[0] + zero[1] + zero[2] + zero[3] != 0.f);
      }
      if (plain) {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          const Frag<T> vf = load_frag(&stage[b][h][1][(dt * 64 + lane) * 8]);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) o[qt][dt] = mma8(o[qt][dt], vf, pf[qt]);
        }
      } else {
#pragma unroll
        for (int dt = 0; dt < ND; ++dt) {
          Frag<T> vf[1] = {load_frag(&stage[b][h][1][(dt * 64 + lane) * 8])};
          if (pos0 + 32 > end) clear_past(vf, end - pos0, grp);
          bool odd = false;
#pragma unroll
          for (int e = 0; e < 8; ++e) odd |= nonfinite(vf[0].v[e]);
          if (__ballot(odd)) clean_values(vf[0], pos0, qpos, window, end, grp, o, dt);
#pragma unroll
          for (int qt = 0; qt < QT; ++qt) o[qt][dt] = mma8(o[qt][dt], vf[0], pf[qt]);
        }
      }
    }
    ready = false;
    there = next;
    b ^= 1;
    blk += NB;
  }
#pragma unroll
  for (int qt = 0; qt < QT; ++qt) {
    float sum = w[qt].sum + __shfl_xor(w[qt].sum, 16);
    sum += __shfl_xor(sum, 32);
    const int row = wrow0 + qt * 16 + r16;
    if (row < nrows) {
      const int t = token(qt);
      write_row<T, DH, ND>(c, k, pl, row - row0, s.r0 + t, pl.kvh * c.G + row - t * c.G, grp, 0, w[qt].ref(), sum, o[qt],
                           out, ldo, lse, parts.o, parts.ml);
    }
  }
}

template <typename T> constexpr int many_qt() { return sizeof(T) == 2 ? 2 : 1; }
template <typename T> constexpr int many_waves() { return kManyTile / (16 * many_qt<T>()); }

template <typename T, int DH>
__global__ __launch_bounds__(64 * many_waves<T>(), 2) void paged_many_kernel(PagedView c, PagedRows r, Class k,
                                                                            const T* __restrict__ q, int64_t ldq,
                                                                            float scale, int window,
                                                                            T* __restrict__ out, int64_t ldo,
                                                                            float* __restrict__ lse, Parts w, int* err) {
  __shared__ __align__(1024) ManyLds<T, DH> lds;
  many_group<T, DH, many_qt<T>(), many_waves<T>()>(c, r, k, blockIdx.x, q, ldq, scale, window, out, ldo, lse, w, err, lds);
}

// Both classes in one launch (bf16: both have four waves): the few rows' items,
// which wait for memory, fill the CUs that the last tiles leave (a mixed batch
// of 27 sequences 338 us in launches of their own, 293 in one).
template <typename T, int DH>
__global__ __launch_bounds__(256, 2) void paged_both_kernel(PagedView c, PagedRows r, Class many, int many_items,
                                                            Class few, const T* __restrict__ q, int64_t ldq, float scale,
                                                            int window, T* __restrict__ out, int64_t ldo,
                                                            float* __restrict__ lse, Parts wm, Parts wf, int* err) {
  constexpr int QT = paged_few_tiles(SPS_DTYPE_BF16);
  constexpr size_t kBytes = sizeof(ManyLds<T, DH>) > sizeof(FewLds<T, DH, QT>) ? sizeof(ManyLds<T, DH>)
                                                                                : sizeof(FewLds<T, DH, QT>);
  __shared__ __align__(1024) char lds[kBytes];
  if (static_cast<int>(blockIdx.x) < many_items)
    many_group<T, DH, many_qt<T>(), many_waves<T>()>(c, r, many, blockIdx.x, q, ldq, scale, window, out, ldo, lse, wm, err,
                                                     reinterpret_cast<ManyLds<T, DH>&>(lds));
  else
    few_group<T, DH, QT>(c, r, few, blockIdx.x - many_items, q, ldq, scale, window, out, ldo, lse, wf, err,
                         reinterpret_cast<FewLds<T, DH, QT>&>(lds));
}

static_assert(sizeof(Join) == kPagedJoinBytes, "the workspace's entries");

template <typename T, int DH>
static hipError_t attn_t(const PagedView& c, const PagedRows& r, const PagedPlan& p, const void* q, int64_t ldq,
                         float scale, int window, void* out, int64_t ldo, float* lse, char* ws, int* err,
                         hipStream_t st) {
  const T* qq = static_cast<const T*>(q);
  T* oo = static_cast<T*>(out);
  // Blocks take about 1 us; an item's start 4 (8: its queries and first stage), a partial of 128 rows 20.
  const Class few{p.few.tile, p.few.target, 0, p.limit, 4, p.qt, static_cast<int>(p.few.items),
                  static_cast<int>(p.few.slots)};
  const Class many{p.many.tile, p.many.target, p.limit, INT32_MAX, 8, 20, static_cast<int>(p.many.items),
                   static_cast<int>(p.many.slots)};
  auto parts = [&](const PagedClass& k) {
    return Parts{reinterpret_cast<float*>(ws + k.o_off), reinterpret_cast<float2*>(ws + k.ml_off),
                 reinterpret_cast<Join*>(ws + k.join_off), reinterpret_cast<int*>(ws + k.count_off)};
  };
  const Parts wf = parts(p.few), wm = parts(p.many);
  const dim3 gf(static_cast<unsigned>(p.few.items)), gm(static_cast<unsigned>(p.many.items));
  hipError_t e = hipSuccess;
  if (sizeof(T) == 2 && p.many.items && p.few.items) {
    if constexpr (sizeof(T) == 2)
      hipLaunchKernelGGL((paged_both_kernel<T, DH>), dim3(gm.x + gf.x), dim3(256), 0, st, c, r, many,
                         static_cast<int>(gm.x), few, qq, ldq, scale, window, oo, ldo, lse, wm, wf, err);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  } else {
    if (p.many.items) {
      hipLaunchKernelGGL((paged_many_kernel<T, DH>), gm, dim3(64 * many_waves<T>()), 0, st, c, r, many, qq, ldq, scale,
                         window, oo, ldo, lse, wm, err);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
    if (p.few.items) {
      // Three tiles are for bf16 alone (paged_few_tiles).
      auto kern = p.qt == 1 ? paged_few_kernel<T, DH, 1> : p.qt == 2 || sizeof(T) == 4 ? paged_few_kernel<T, DH, 2>
                                                                                      : paged_few_kernel<T, DH, sizeof(T) == 2 ? 3 : 2>;
      hipLaunchKernelGGL(kern, gf, dim3(256), 0, st, c, r, few, qq, ldq, scale, window, oo, ldo, lse, wf, err);
      if ((e = hipGetLastError()) != hipSuccess) return e;
    }
  }
  for (const PagedClass* k : {&p.many, &p.few}) {
    if (!k->slots) continue;
    const Parts w = parts(*k);
    hipLaunchKernelGGL((paged_join_kernel<T, DH>), dim3(static_cast<unsigned>(k->slots), k->tile / 16), dim3(256), 0, st, c,
                       k->tile, w.joins, w.count, w.o, w.ml, oo, ldo, lse);
    if ((e = hipGetLastError()) != hipSuccess) return e;
  }
  return e;
}

hipError_t launch_paged_attention(int dtype, const PagedView& c, const PagedRows& r, const PagedPlan& p, const void* q,
                                  int64_t ldq, float scale, int window, void* out, int64_t ldo, float* lse, char* ws,
                                  int* err, hipStream_t st) {
  if (dtype == 1)
    return c.DH == 128 ? attn_t<bf16, 128>(c, r, p, q, ldq, scale, window, out, ldo, lse, ws, err, st)
                       : attn_t<bf16, 64>(c, r, p, q, ldq, scale, window, out, ldo, lse, ws, err, st);
  return c.DH == 128 ? attn_t<float, 128>(c, r, p, q, ldq, scale, window, out, ldo, lse, ws, err, st)
                     : attn_t<float, 64>(c, r, p, q, ldq, scale, window, out, ldo, lse, ws, err, st);
}

}  // namespace sps
