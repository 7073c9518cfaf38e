"""Rotary positions, the paged cache's append and its attention against the
fp64 oracle.

Tolerances. A rounding is off by half a step, u = 2^-8 (bf16) or 2^-24 (fp32) of the
value.
  rope: the angle's cosine and sine come from fp64 angles through fp32
    polynomials of five steps, times the amplitude, then two products and a
    sum: under 16 fp32 roundings of values of at most A (|a| + |b|), and one
    rounding to the type: u |y| + 2^-20 A (|a| + |b|).
  attention: scores are fp32 sums of D products (D 2^-24 of sum |q k|) taken
    through exp2 with a scale and a difference (8 more roundings), so weights
    are off by e = (D + 8) 2^-24 M + 2^-22 with M the largest sum |q k| scale;
    softmax weights may be rounded to the type (u); both the sum of w V and
    the sum of w carry e, and n terms add n 2^-24 each: with W = sum w |V|,
    u |o| + (u + 2 e + 2 n 2^-24) W. lse: e + n 2^-24 + 2^-23 |lse|.
"""
import numpy as np
import pytest
import torch

from oracle import paged as op

pytestmark = pytest.mark.gpu
U = {"bf16": 2.0 ** -8, "f32": 2.0 ** -24}
DT = {"bf16": torch.bfloat16, "f32": torch.float32}


def randn(shape, seed, dtype, std=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * std).to(DT[dtype])


def f64(t):
    return t.double().cpu().numpy()


# ---- rope -----------------------------------------------------------------------
def check_rope(y, x, pos, dtype, rot, layout, amplitude=1.0, backward=False, **kw):
    want = op.rope(f64(x), pos, rot, layout, amplitude, backward, **kw)
    ia, ib = op.pairs(rot, layout)
    mag = np.abs(f64(x))
    lim = U[dtype] * np.abs(want)
    both = 2.0 ** -20 * abs(amplitude) * (mag[..., ia] + mag[..., ib])
    lim[..., ia] += both
    lim[..., ib] += both
    assert (np.abs(f64(y) - want) <= lim).all(), np.abs(f64(y) - want).max()
    assert np.array_equal(f64(y)[..., rot:], f64(x)[..., rot:])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("rows, heads, dim, rot", [
    (1, 1, 2, 2), (1, 64, 128, 128), (3, 5, 128, 64), (17, 24, 64, 64), (33, 3, 64, 20), (2, 7, 80, 80), (5, 2, 256, 256),
    (9, 1, 6, 4), (1030, 4, 128, 96), (257, 33, 64, 32)])
def test_rope(sps, dtype, layout, rows, heads, dim, rot):
    x = randn((rows, heads, dim), rows * 7 + rot, dtype).cuda()
    g = np.random.default_rng(rows)
    pos = g.integers(0, 200000, rows).astype(np.int32)
    p = torch.from_numpy(pos).cuda()
    check_rope(sps.rope(x, p, sps.rope_spec(rot, layout=layout)), x, pos, dtype, rot, layout)
    kw = dict(base=500000.0, factor=8.0, original_len=8192, low_turns=1.0, high_turns=4.0, amplitude=1.25)
    y = sps.rope(x, p, sps.rope_spec(rot, layout=layout, **kw), backward=True)
    check_rope(y, x, pos, dtype, rot, layout, backward=True, **kw)
    y = sps.rope(x, p, sps.rope_spec(rot, layout=layout, factor=4.0))
    check_rope(y, x, pos, dtype, rot, layout, factor=4.0)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("pad", [0, 1, 3, 8])
@pytest.mark.parametrize("rot", [64, 40])
def test_rope_strides_in_place_and_neighbours(sps, dtype, pad, rot):
    """Rows that lie apart at any alignment; nothing between them is written."""
    for layout in ("half", "interleaved"):
        wide = randn((70, 3 * 64 + pad + 5), 5, dtype).cuda()
        x = wide[:, pad:pad + 192].unflatten(1, (3, 64))
        pos = np.arange(70, dtype=np.int32) * 37 - 100        # negative positions turn the other way
        p = torch.from_numpy(pos).cuda()
        before = wide.clone()
        y = sps.rope(x, p, sps.rope_spec(rot, layout=layout))
        assert torch.equal(wide, before)
        out = torch.full((70, 3 * 64 + 9), 7.0, dtype=DT[dtype], device="cuda")
        sps.rope(x, p, sps.rope_spec(rot, layout=layout), out=out[:, 4:196].unflatten(1, (3, 64)))
        assert torch.equal(out[:, 4:196].unflatten(1, (3, 64)), y)
        assert bool((out[:, :4] == 7).all() and (out[:, 196:] == 7).all())
        sps.rope(x, p, sps.rope_spec(rot, layout=layout), out=x)
        assert torch.equal(x, y)
        wide[:, pad:pad + 192] = before[:, pad:pad + 192]
        assert torch.equal(wide, before)
        check_rope(y, x, pos, dtype, rot, layout)


def test_rope_gradient_against_differences(sps):
    """<w, R x> changes by <R^T w, h>: fp32, differences of 2^-3 on a linear map."""
    x, w = randn((4, 2, 64), 1, "f32").cuda(), randn((4, 2, 64), 2, "f32").cuda()
    p = torch.tensor([0, 3, 500, 70000], dtype=torch.int32, device="cuda")
    spec = sps.rope_spec(48, layout="interleaved", amplitude=1.5)
    grad = sps.rope(w, p, spec, backward=True)
    for e in (0, 5, 47, 50, 63):
        h = torch.zeros_like(x)
        h[:, :, e] = 0.125
        d = ((sps.rope(x + h, p, spec).double() - sps.rope(x - h, p, spec).double()) * w.double()).sum(-1) / 0.25
        # 64 products, each side rounded a few times relative to |x| A < 8, over the step 0.25
        assert (d - grad[..., e].double()).abs().max() < 64 * 8 * 8 * 2.0 ** -24 / 0.25


# ---- batches ---------------------------------------------------------------------
class Batch:
    """A paged cache with random contents, scattered pages and new tokens."""

    def __init__(self, sps, dtype, hq, hkv, D, page, prior, new, seed=0, ragged=True, spare=2, extra_rows=0, layers=1,
                 offset=0, before=0):
        self.sps, self.dtype, self.hq, self.hkv, self.D, self.page = sps, dtype, hq, hkv, D, page
        self.prior, self.new, self.B = prior, new, len(prior)
        need = [max(1, -(-(p + offset + n) // page)) for p, n in zip(prior, new)]
        self.n_pages, self.max_pages = sum(need) + spare, max(need) + 1
        g = np.random.default_rng(seed)
        perm = g.permutation(self.n_pages).astype(np.int32)
        self.table = np.full((self.B, self.max_pages), -1, np.int32)
        at = 0
        for b, m in enumerate(need):
            self.table[b, :m] = perm[at:at + m]
            at += m
        self.kv = sps.PagedKV(hq, hkv, D, self.n_pages, page, self.B, self.max_pages, n_layers=layers, dtype=dtype)
        self.kv.buf.copy_(randn(self.kv.buf.shape, seed + 1, dtype))
        self.kv.page_table.copy_(torch.from_numpy(self.table))
        self.kv.lengths.copy_(torch.tensor(prior, dtype=torch.int32))
        self.offset = offset
        self.starts = np.concatenate([[0], np.cumsum(new)]).astype(np.int32) + before
        self.rows = int(self.starts[-1]) + extra_rows
        self.most = max(max(new), 1)
        self.st = torch.from_numpy(self.starts).cuda() if ragged else None
        self.q = randn((self.rows, hq, D), seed + 2, dtype, 1.5).cuda()
        self.out = torch.full((self.rows, hq, D), 99.0, dtype=DT[dtype], device="cuda")
        self.lse = torch.full((self.rows, hq), 99.0, device="cuda")

    def attend(self, window=0, scale=None, lse=True, layer=0, q=None, out=None):
        ws = self.kv.workspace(self.rows, self.most)
        return self.sps.paged_attention(self.kv, layer, self.q if q is None else q, ws, out=self.out if out is None else out,
                                        lse=self.lse if lse else None, starts=self.st, max_tokens=self.most,
                                        pos_offset=self.offset, window=window, scale=scale)

    def planes(self, layer=0):
        return f64(self.kv.buf[layer, 0]), f64(self.kv.buf[layer, 1])

    def check(self, window=0, scale=None, seen=None, layer=0):
        u, D = U[self.dtype], self.D
        scale = np.float64(np.float32(D ** -0.5 if scale is None else scale))
        kp, vp = self.planes(layer)
        out, lse, q = f64(self.out), f64(self.lse), f64(self.q)
        touched = np.zeros(self.rows, bool)
        for b, n in enumerate(self.new):
            if not n:
                continue
            rows = slice(int(self.starts[b]), int(self.starts[b]) + n)
            touched[rows] = True
            L = min(self.prior[b] + self.offset + n, self.max_pages * self.page)
            K = op.gather(kp, self.table[b], max(L, 0), self.page, D, op.key_at)
            V = op.gather(vp, self.table[b], max(L, 0), self.page, D, op.value_at)
            o, z, W, M = op.attention(q[rows], K, V, self.prior[b] + self.offset, scale, window,
                                      None if seen is None else seen[b])
            e = (D + 8) * 2.0 ** -24 * M + 2.0 ** -22
            lim = u * np.abs(o) + (u + 2 * e[..., None] + 2 * max(L, 1) * 2.0 ** -24) * W
            bad = np.abs(out[rows] - o) > lim
            assert not bad.any(), (b, np.argwhere(bad)[:3], np.abs(out[rows] - o).max())
            none = np.isinf(z)
            assert np.array_equal(none, np.isinf(lse[rows]))
            dz = np.abs(np.where(none, 0, lse[rows]) - np.where(none, 0, z))
            assert (dz <= e + max(L, 1) * 2.0 ** -24 + 2.0 ** -23 * np.abs(np.where(none, 0, z))).all(), dz.max()
        assert (out[~touched] == 99).all() and (lse[~touched] == 99).all()     # rows of no sequence


SHAPES = [
    # dtype, query heads, KV heads, dim, page, prior, new
    ("bf16", 4, 4, 128, 32, [0], [1]),
    ("bf16", 32, 8, 128, 64, [2047], [1]),
    ("bf16", 1, 1, 64, 32, [31, 32, 33, 0, 63], [1, 1, 1, 1, 1]),
    ("bf16", 64, 8, 128, 64, [700, 5, 1300], [5, 5, 5]),
    ("bf16", 8, 1, 128, 128, [100, 3000], [2, 2]),
    ("bf16", 20, 4, 64, 256, [511, 512, 1], [3, 3, 3]),
    ("bf16", 24, 4, 128, 32, [90, 0, 400, 17], [1, 40, 0, 5]),
    ("bf16", 4, 2, 64, 32, [0, 0, 10], [130, 1, 65]),
    ("bf16", 3, 3, 128, 64, [0, 77], [300, 33]),
    ("bf16", 16, 2, 128, 1024, [900], [200]),
    ("bf16", 40, 1, 128, 64, [129], [9]),
    ("f32", 4, 4, 64, 32, [100, 40], [5, 5]),
    ("f32", 8, 2, 128, 64, [0, 600], [1, 1]),
    ("f32", 6, 2, 64, 128, [12, 0, 301], [70, 0, 3]),
    ("f32", 2, 1, 128, 32, [0], [150]),
]


@pytest.mark.parametrize("dtype, hq, hkv, D, page, prior, new", SHAPES)
@pytest.mark.parametrize("window", [0, 1, 50])
def test_attention(sps, dtype, hq, hkv, D, page, prior, new, window):
    t = Batch(sps, dtype, hq, hkv, D, page, prior, new, seed=len(prior) + D)
    t.attend(window)
    t.check(window)
    assert sps.device_error() == 0
    if len(set(new)) == 1:                            # rows b n .. b n + n - 1 without starts: the same bits
        got = t.out.clone()
        t.st = None
        t.attend(window, lse=False)
        assert torch.equal(got, t.out)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_attention_peaked_and_flat_scores(sps, dtype):
    t = Batch(sps, dtype, 8, 2, 128, 32, [900, 70], [3, 1], seed=3)
    for scale in (1e-4, 1.0):
        t.attend(scale=scale)
        t.check(scale=scale)


def test_long_context_over_many_ranges(sps):
    """Enough blocks for several ranges per tile, joined in the second launch."""
    for dtype, prior, new in (("bf16", [40000, 300, 9000], [1, 1, 1]), ("bf16", [20000], [7]), ("f32", [9000], [2])):
        t = Batch(sps, dtype, 4, 1, 64, 256, prior, new, seed=9)
        t.attend()
        t.check()
        again = t.out.clone()
        t.attend()
        assert torch.equal(again, t.out)              # a fixed order: the same bits


def test_many_sequences(sps):
    g = np.random.default_rng(11)
    prior, new = g.integers(0, 200, 1024).tolist(), g.integers(0, 4, 1024).tolist()
    t = Batch(sps, "bf16", 2, 1, 64, 32, prior, new, seed=12, extra_rows=3, before=2)
    t.attend()
    t.check()


@pytest.mark.parametrize("dtype, B, window", [("bf16", 65, 0), ("bf16", 130, 100), ("f32", 90, 0), ("bf16", 64, 0)])
def test_many_sequences_of_both_kinds(sps, dtype, B, window):
    """Prompt chunks, drafts, single tokens and waiting requests, some of them
    over long contexts, around the number of sequences whose split is priced."""
    g = np.random.default_rng(B)
    prior, new = g.integers(0, 300, B).tolist(), [(1, 5, 0, 1, 2)[b % 5] for b in range(B)]
    for b, (p, n) in {0: (3000, 1), 3: (10, 70), 40: (900, 33), B - 1: (2500, 9)}.items():
        prior[b], new[b] = p, n
    t = Batch(sps, dtype, 8, 2, 64, 32, prior, new, seed=22, extra_rows=2, before=1)
    t.attend(window)
    t.check(window)
    assert sps.device_error() == 0


def test_two_streams_at_once(sps):
    """Calls that overlap on two streams, each with its workspace, over one cache."""
    t = Batch(sps, "bf16", 16, 2, 128, 64, [9000, 4000, 700], [1, 40, 5], seed=23)
    ws = [t.kv.workspace(t.rows, t.most) for _ in range(2)]
    want = t.attend(lse=False).clone()
    outs, streams = [torch.empty_like(t.out) for _ in range(2)], [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for s in range(2):
            with torch.cuda.stream(streams[s]):
                sps.paged_attention(t.kv, 0, t.q, ws[s], out=outs[s], starts=t.st, max_tokens=t.most)
    torch.cuda.synchronize()
    assert torch.equal(outs[0], want) and torch.equal(outs[1], want)


def test_chunks_over_long_contexts_are_split(sps):
    """Tiles of many rows with several ranges, joined; with a window, and among
    more sequences than the ranges are priced for."""
    for dtype, prior, new, window in (("bf16", [6000], [40], 0), ("bf16", [5000, 10], [33, 1], 3000),
                                      ("f32", [3000], [20], 0), ("bf16", [4000] + [3] * 70, [70] + [1] * 70, 0)):
        t = Batch(sps, dtype, 8, 2, 64, 64, prior, new, seed=19)
        t.attend(window)
        t.check(window)
        again, al = t.out.clone(), t.lse.clone()
        t.attend(window)
        assert torch.equal(again, t.out) and torch.equal(al, t.lse)


@pytest.mark.parametrize("dtype, hq, hkv, D, prior, new, window", [
    ("bf16", 200, 200, 64, [1500, 1571, 1400], [50, 50, 50], 0),
    ("bf16", 40, 40, 128, [1500], [1700], 0),
    ("bf16", 80, 40, 64, [1700], [810], 1300),
    ("bf16", 64, 8, 64, [1500, 40, 900], [1100, 3, 1], 0),
    ("f32", 40, 40, 64, [1500], [1700], 0),
    ("f32", 100, 100, 128, [1900, 0, 2100, 1700], [270, 33, 140, 70], 0)])
def test_tiles_past_whole_rounds_are_split(sps, dtype, hq, hkv, D, prior, new, window):
    """More tiles than the card holds at once, by a part of a round: the first
    stay whole, the last are split and joined. fp64 on the device."""
    t = Batch(sps, dtype, hq, hkv, D, 64, prior, new, seed=21)
    G, L = hq // hkv, [p + n for p, n in zip(prior, new)]
    k, v = randn((sum(L), hkv, D), 1, dtype).cuda(), randn((sum(L), hkv, D), 2, dtype).cuda()
    t.kv.lengths.zero_()
    at = np.concatenate([[0], np.cumsum(L)]).astype(np.int32)
    t.kv.append(0, k, v, starts=torch.from_numpy(at).cuda(), max_tokens=max(L))
    t.kv.lengths.copy_(torch.tensor(prior, dtype=torch.int32))
    t.attend(window)
    first, first_lse = t.out.clone(), t.lse.clone()
    scale = float(np.float32(D ** -0.5))
    for b, n in enumerate(new):
        rows = slice(int(t.starts[b]), int(t.starts[b]) + n)
        pos = prior[b] + torch.arange(n, device="cuda")[:, None]
        p = torch.arange(L[b], device="cuda")[None, :]
        seen = (p <= pos) & ((p > pos - window) if window else (p >= 0))
        for h in range(hkv):
            K, V = k[at[b]:at[b + 1], h].double(), v[at[b]:at[b + 1], h].double()
            for g in range(G):
                q = t.q[rows, h * G + g].double()
                w = (q @ K.T * scale).masked_fill(~seen, -torch.inf)
                z = torch.logsumexp(w, 1)
                w = torch.exp(w - z[:, None])
                o, W = w @ V, w @ V.abs()
                M = (q.abs() @ K.abs().T * scale).amax(1)
                e = (D + 8) * 2.0 ** -24 * M + 2.0 ** -22
                u = U[dtype]
                lim = u * o.abs() + (u + 2 * e[:, None] + 2 * L[b] * 2.0 ** -24) * W
                assert bool(((t.out[rows, h * G + g].double() - o).abs() <= lim).all())
                dz = (t.lse[rows, h * G + g].double() - z).abs()
                assert bool((dz <= e + L[b] * 2.0 ** -24 + 2.0 ** -23 * z.abs()).all())
    t.attend(window)
    assert torch.equal(t.out, first) and torch.equal(t.lse, first_lse)


@pytest.mark.parametrize("seed", range(24))
def test_attention_of_drawn_batches(sps, seed):
    g = np.random.default_rng(1000 + seed)
    H = int(g.choice([1, 2, 3, 8]))
    G = int(g.choice([1, 2, 3, 4, 5, 7, 8, 20]))
    B = int(g.choice([1, 2, 5, 9, 70]))
    D, page = int(g.choice([64, 128])), int(g.choice([32, 64, 128, 512]))
    dtype = "f32" if g.random() < 0.3 else "bf16"
    top = max(2, 600 // B)
    prior = g.integers(0, top, B).tolist()
    new = [int(g.choice([0, 1, 1, 2, 5, int(g.integers(1, 1 + max(1, 200 // B)))])) for _ in range(B)]
    if sum(new) == 0:
        new[0] = 1
    window = int(g.choice([0, 0, 1, 31, 32, 33, 300]))
    t = Batch(sps, dtype, H * G, H, D, page, prior, new, seed=seed, spare=1, extra_rows=int(g.integers(0, 3)))
    # values of very unlike sizes, and keys that make some scores large
    t.kv.buf[0, 1] *= torch.randn(t.kv.buf[0, 1].shape, device="cuda").exp().to(t.kv.dtype)
    t.kv.buf[0, 0, ::3] *= 4
    t.attend(window)
    t.check(window)
    assert sps.device_error() == 0


def test_scores_that_grow_along_the_context(sps):
    """Every few blocks a new largest score, far above the last (the reference
    moves many times), and the same run backwards."""
    for dtype, new in (("bf16", 1), ("bf16", 12), ("bf16", 80), ("f32", 3)):
        t = Batch(sps, dtype, 4, 1, 64, 32, [700], [new], seed=23)
        L = 700 + new
        for grow in (np.linspace(0.0, 12.0, L), np.linspace(12.0, 0.0, L)):
            d = np.arange(64)
            for p in range(L):
                t.kv.buf[0, 0, t.table[0, p // 32], 0, op.key_at(p % 32, d, 64)] = float(grow[p]) / 8
            t.q.fill_(1.0)
            t.attend(scale=1.0)
            t.check(scale=1.0)


def test_rows_outside_the_sequences_are_left(sps):
    t = Batch(sps, "bf16", 8, 2, 128, 64, [10, 400, 0], [2, 0, 70], seed=4, extra_rows=9, before=5)
    t.attend()
    t.check()
    k, v = randn((t.rows, 2, 128), 1, "bf16").cuda(), randn((t.rows, 2, 128), 2, "bf16").cuda()
    qo = torch.full_like(t.q, 99.0)
    t.kv.append(0, k, v, rope=sps.rope_spec(128), q=t.q, q_out=qo, starts=t.st, max_tokens=t.most)
    assert bool((qo[:5] == 99).all() and (qo[-9:] == 99).all())
    assert sps.device_error() == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_nothing_unseen_is_felt(sps, dtype, bad):
    """Pages of nobody, positions behind the last one and, per row, the later
    tokens of its own chunk and what lies before its window hold NaN or Inf."""
    t = Batch(sps, dtype, 8, 2, 64, 64, [70, 3], [5, 40], seed=5)
    t.attend(16)
    want, wl = t.out.clone(), t.lse.clone()
    kp, vp = t.kv.buf[0, 0], t.kv.buf[0, 1]
    d = np.arange(64)
    for b in range(2):
        end = t.prior[b] + t.new[b]
        for p in list(range(end, -(-end // 64) * 64)) + list(range(0, max(0, t.prior[b] - 15))):
            kp[t.table[b, p // 64]][:, op.key_at(p % 64, d, 64)] = bad
            vp[t.table[b, p // 64]][:, op.value_at(p % 64, d, 64)] = bad
    free = sorted(set(range(t.n_pages)) - set(t.table[t.table >= 0].tolist()))
    kp[free], vp[free] = bad, bad
    t.out.fill_(99.0)
    t.attend(16)
    assert torch.equal(t.out, want) and torch.equal(t.lse, wl)
    # The chunk's last token: rows before it are as they were, its own row is not finite.
    for b in range(2):
        p = t.prior[b] + t.new[b] - 1
        vp[t.table[b, p // 64], 0, op.value_at(p % 64, 5, 64)] = bad
    t.attend(16)
    for b in range(2):
        rows = slice(int(t.starts[b]), int(t.starts[b + 1]) - 1)
        assert torch.equal(t.out[rows], want[rows])
        last = t.out[int(t.starts[b + 1]) - 1]
        assert bool((~torch.isfinite(last[:4, 5])).all())
        keep = [i for i in range(64) if i != 5]
        assert torch.equal(last[:, keep], want[int(t.starts[b + 1]) - 1][:, keep])
        if bad == float("inf"):
            assert bool((last[:4, 5] == bad).all())


def test_bad_pages_are_flagged_and_not_read(sps):
    t = Batch(sps, "bf16", 8, 2, 64, 32, [100, 50], [3, 2], seed=6)
    for entry in (-1, t.n_pages, 1 << 30, -(1 << 31)):
        tab = t.table.copy()
        tab[0, 1] = entry
        t.kv.page_table.copy_(torch.from_numpy(tab))
        t.attend()
        assert sps.device_error() == sps.DEV_BAD_PAGE
        seen = [np.ones(200, bool), np.ones(200, bool)]
        seen[0][32:64] = False
        t.check(seen=seen)
    tab[:] = -1                                        # no page at all: rows that see nothing
    t.kv.page_table.copy_(torch.from_numpy(tab))
    t.attend()
    assert sps.device_error() == sps.DEV_BAD_PAGE
    assert bool((t.out == 0).all()) and bool(torch.isneginf(t.lse).all())


def test_positions_before_zero_and_past_the_capacity(sps):
    t = Batch(sps, "bf16", 4, 2, 64, 32, [5, 40], [4, 4], seed=7)
    cap = t.max_pages * 32
    t.table[1] = np.resize(t.table[1, :2], t.max_pages)
    t.kv.page_table.copy_(torch.from_numpy(t.table))
    t.prior = [-2, cap - 2]
    t.kv.lengths.copy_(torch.tensor(t.prior, dtype=torch.int32))
    t.attend()
    t.check()                                          # two rows see nothing, two lie past the capacity
    assert bool((t.out[:2] == 0).all())
    before = t.kv.buf.clone()
    k, v = randn((8, 2, 64), 1, "bf16").cuda(), randn((8, 2, 64), 2, "bf16").cuda()
    t.kv.append(0, k, v)
    assert sps.device_error() == sps.DEV_CAPACITY
    kp, vp = f64(before[0, 0]), f64(before[0, 1])
    op.append(kp, vp, t.table[0], 0, f64(k)[2:4], f64(v)[2:4], 32)
    op.append(kp, vp, t.table[1], cap - 2, f64(k)[4:6], f64(v)[4:6], 32)
    assert np.array_equal(f64(t.kv.buf[0, 0]), kp) and np.array_equal(f64(t.kv.buf[0, 1]), vp)
    for far in (2147483647, -2147483648):              # lengths + offset past 32 bits
        t.kv.lengths.fill_(far)
        t.offset = 1 if far > 0 else -1
        before = t.kv.buf.clone()
        t.kv.append(0, k, v, pos_offset=t.offset)
        assert sps.device_error() == sps.DEV_CAPACITY and torch.equal(before, t.kv.buf)
    t.attend()                                         # all rows before position 0
    assert bool((t.out == 0).all())


def test_starts_that_break_the_rules_are_flagged(sps):
    """Whatever they hold, nothing outside the rows and pages is touched and the flag is set."""
    t = Batch(sps, "bf16", 4, 2, 64, 32, [5, 40, 9], [4, 4, 4], seed=8)
    k, v = randn((12, 2, 64), 1, "bf16").cuda(), randn((12, 2, 64), 2, "bf16").cuda()
    for starts in ([0, 4, 8, 13], [-1, 4, 8, 12], [0, 8, 4, 12], [0, 6, 8, 12], [0, 4, 8, 1 << 30], [8, 0, 12, 0],
                   [-(1 << 31), (1 << 31) - 1, -(1 << 31), (1 << 31) - 1]):
        t.st = torch.tensor(starts, dtype=torch.int32, device="cuda")
        t.attend()
        assert sps.device_error() == sps.DEV_CAPACITY
        t.kv.append(0, k, v, starts=t.st, max_tokens=4)
        assert sps.device_error() == sps.DEV_CAPACITY


def test_starts_that_claim_more_rows_than_there_are(sps):
    """Overlapping claims of many sequences over split contexts: more items and
    partials than the call's rows can have, which the workspace's end and the
    memory behind the outputs do not feel."""
    t = Batch(sps, "bf16", 4, 2, 64, 32, [2000] * 40, [1] * 40, seed=18)
    # 30 tokens from position 2000 on reach a page that the tables do not have.
    for most, flags in ((2, sps.DEV_CAPACITY), (30, sps.DEV_CAPACITY | sps.DEV_BAD_PAGE)):
        rows = most
        starts = [0, rows] * 20 + [0]
        n = t.kv.workspace(rows, most).numel()
        ws = torch.full((n + 4096,), 7, dtype=torch.uint8, device="cuda")
        out = torch.full((rows + 2, 4, 64), 99.0, dtype=torch.bfloat16, device="cuda")
        st = torch.tensor(starts, dtype=torch.int32, device="cuda")
        sps.paged_attention(t.kv, 0, t.q[:rows], ws[:n], out=out[:rows], starts=st, max_tokens=most)
        assert sps.device_error() == flags
        assert bool((ws[n:] == 7).all()) and bool((out[rows:] == 99).all())


def test_claims_of_short_sequences_before_long_ones(sps):
    """Overlapping claims of which the first are not split: partials whose items
    the call does not have are not joined, whatever the workspace holds."""
    for dtype, B in (("bf16", 40), ("f32", 40), ("bf16", 100)):
        t = Batch(sps, dtype, 4, 2, 64, 32, [40] * (B // 2) + [2000] * (B // 2), [1] * B, seed=19)
        n = t.kv.workspace(1, 1).numel()
        ws = torch.full((n + 4096,), 0x7f, dtype=torch.uint8, device="cuda")
        out = torch.full((9, 4, 64), 99.0, dtype=DT[dtype], device="cuda")
        lse = torch.full((9, 4), 99.0, device="cuda")
        st = torch.tensor([0, 1] * (B // 2) + [0], dtype=torch.int32, device="cuda")
        sps.paged_attention(t.kv, 0, t.q[:1], ws[:n], out=out[:1], lse=lse[:1], starts=st, max_tokens=1)
        assert sps.device_error() == sps.DEV_CAPACITY
        assert bool((ws[n:] == 0x7f).all()) and bool((out[1:] == 99).all()) and bool((lse[1:] == 99).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_windows_wider_than_any_context(sps, dtype):
    """The widest window is no window, also for rows before position 0."""
    for prior, new in (([-5, 40], [10, 3]), ([-70, 300], [150, 2])):
        t = Batch(sps, dtype, 4, 2, 64, 32, [max(p, 0) for p in prior], new, seed=20)
        t.prior = prior
        t.kv.lengths.copy_(torch.tensor(prior, dtype=torch.int32))
        t.attend(2147483647)
        t.check()
        wide = t.out.clone()
        t.attend(0)
        assert torch.equal(wide, t.out)


# ---- append ------------------------------------------------------------------------
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D, hq, hkv, page, prior, new", [
    (128, 8, 2, 64, [0], [1]), (64, 4, 4, 32, [31, 32, 0, 5], [1, 1, 1, 1]), (128, 64, 8, 64, [1000, 3, 70], [1, 1, 1]),
    (128, 4, 1, 32, [7, 0, 90], [70, 0, 33]), (64, 6, 3, 128, [100, 250], [64, 300]), (128, 16, 8, 256, [13], [40]),
    (64, 1, 1, 32, [0, 1, 31, 15], [32, 31, 33, 1])])
def test_append(sps, dtype, D, hq, hkv, page, prior, new):
    t = Batch(sps, dtype, hq, hkv, D, page, prior, new, seed=D + len(new), layers=2, extra_rows=2)
    for layout, rot in (("half", D), ("interleaved", D // 2), ("half", 20), (None, 0)):
        # one projection's rows, from an odd element on: q, k, v side by side
        wide = randn((t.rows, (hq + 2 * hkv) * D + 3), rot + 1, dtype).cuda()
        q = wide[:, 1:1 + hq * D].unflatten(1, (hq, D))
        k = wide[:, 1 + hq * D:1 + (hq + hkv) * D].unflatten(1, (hkv, D))
        v = wide[:, 1 + (hq + hkv) * D:1 + (hq + 2 * hkv) * D].unflatten(1, (hkv, D))
        kp, vp = t.planes(1)
        other = t.kv.buf[0].clone()
        spec = None if layout is None else sps.rope_spec(rot, layout=layout, factor=2.0)
        qo = torch.full((t.rows, hq, D), 99.0, dtype=DT[dtype], device="cuda")
        assert t.kv.append(1, k, v, rope=spec, q=q, q_out=qo, starts=t.st, max_tokens=t.most) is qo
        assert sps.device_error() == 0
        pos = np.concatenate([np.arange(p, p + n) for p, n in zip(prior, new)]).astype(np.int32)
        n = len(pos)
        kr = k[:n].contiguous()
        if spec is not None:
            p = torch.from_numpy(pos).cuda()
            # the same rotation as sps_rope, bit for bit, which is checked against the oracle above
            kr = sps.rope(kr, p, spec)
            check_rope(kr, k[:n], pos, dtype, rot, layout, factor=2.0)
            assert torch.equal(qo[:n], sps.rope(q[:n], p, spec))
        else:
            assert torch.equal(qo[:n], q[:n])
        assert bool((qo[n:] == 99).all())
        for b in range(t.B):
            r = slice(int(t.starts[b]), int(t.starts[b + 1]))
            op.append(kp, vp, t.table[b], prior[b], f64(kr)[r], f64(v)[r], page)
        # every other element of the layer, and the other layer, as they were
        assert np.array_equal(f64(t.kv.buf[1, 0]), kp) and np.array_equal(f64(t.kv.buf[1, 1]), vp)
        assert torch.equal(t.kv.buf[0], other)
        before = t.kv.buf.clone()
        t.kv.append(1, k, v, rope=spec, starts=t.st, max_tokens=t.most)        # no queries; the same contents again
        assert torch.equal(before, t.kv.buf)


def test_append_rotates_queries_in_place_and_skips_bad_pages(sps):
    t = Batch(sps, "bf16", 8, 2, 64, 32, [30, 100], [40, 1], seed=6)
    spec = sps.rope_spec(64)
    k, v = randn((41, 2, 64), 1, "bf16").cuda(), randn((41, 2, 64), 2, "bf16").cuda()
    q = t.q.clone()
    want = t.kv.append(0, k, v, rope=spec, q=q, starts=t.st, max_tokens=40).clone()
    t.kv.append(0, k, v, rope=spec, q=q, q_out=q, starts=t.st, max_tokens=40)
    assert torch.equal(q, want) and sps.device_error() == 0
    tab = t.table.copy()
    tab[0, 1] = t.n_pages                              # positions 32 .. 63
    t.kv.page_table.copy_(torch.from_numpy(tab))
    t.kv.buf.zero_()
    t.kv.append(0, k, v, rope=spec, starts=t.st, max_tokens=40)
    assert sps.device_error() == sps.DEV_BAD_PAGE
    kp, vp = np.zeros(t.kv.buf[0, 0].shape), np.zeros(t.kv.buf[0, 1].shape)
    kr = f64(sps.rope(k, torch.tensor(list(range(30, 70)) + [100], dtype=torch.int32, device="cuda"), spec))
    op.append(kp, vp, t.table[0], 30, kr[:2], f64(v)[:2], 32)
    op.append(kp, vp, t.table[0], 64, kr[34:40], f64(v)[34:40], 32)
    op.append(kp, vp, t.table[1], 100, kr[40:], f64(v)[40:], 32)
    assert np.array_equal(f64(t.kv.buf[0, 0]), kp) and np.array_equal(f64(t.kv.buf[0, 1]), vp)


# ---- how they are used ----------------------------------------------------------------
def test_strided_queries_and_outputs(sps):
    t = Batch(sps, "bf16", 8, 2, 64, 32, [100, 7], [3, 20], seed=2)
    want = t.attend().clone()
    wide = torch.zeros((t.rows, 8 * 64 + 7), dtype=torch.bfloat16, device="cuda")
    qv = wide[:, 3:515].unflatten(1, (8, 64))
    qv.copy_(t.q)
    ow = torch.full((t.rows, 8 * 64 + 5), 99.0, dtype=torch.bfloat16, device="cuda")
    t.attend(q=qv, out=ow[:, 1:513].unflatten(1, (8, 64)))
    assert torch.equal(ow[:, 1:513].unflatten(1, (8, 64)), want)
    assert bool((ow[:, :1] == 99).all() and (ow[:, 513:] == 99).all())


def test_speculative_loop_on_pages(sps):
    """Prompts, then rounds that append K + 1 tokens, attend, keep a few of them and
    overwrite the rest in the next round; a sequence that ends frees its pages
    for the next request. Every round against the oracle's own cache."""
    g = np.random.default_rng(21)
    B, hq, hkv, D, page, K = 3, 8, 2, 64, 32, 4
    spec, scale = sps.rope_spec(D, base=50000.0), D ** -0.5
    kv = sps.PagedKV(hq, hkv, D, 16, page, B, 8)
    free, table, hist = list(g.permutation(16)), np.full((B, 8), -1, np.int32), [([], []) for _ in range(B)]
    lengths = [0] * B

    def step(new, seed):
        rows = sum(new)
        for b in range(B):
            for i in range(-(-(lengths[b] + new[b]) // page)):
                if table[b, i] < 0:
                    table[b, i] = free.pop()
        kv.page_table.copy_(torch.from_numpy(table))
        kv.lengths.copy_(torch.tensor(lengths, dtype=torch.int32))
        starts = torch.tensor(np.concatenate([[0], np.cumsum(new)]).astype(np.int32)).cuda()
        q, k, v = (randn((rows, h, D), seed + i, "bf16").cuda() for i, h in enumerate((hq, hkv, hkv)))
        ws = kv.workspace(rows, max(new))
        qr = kv.append(0, k, v, rope=spec, q=q, starts=starts, max_tokens=max(new))
        lse = torch.empty((rows, hq), device="cuda")
        o = sps.paged_attention(kv, 0, qr, ws, lse=lse, starts=starts, max_tokens=max(new))
        assert sps.device_error() == 0
        at = 0
        for b, n in enumerate(new):
            if not n:
                continue
            pos = torch.arange(lengths[b], lengths[b] + n, dtype=torch.int32, device="cuda")
            kr = f64(sps.rope(k[at:at + n], pos, spec))
            hk, hv = hist[b]
            del hk[lengths[b]:], hv[lengths[b]:]
            hk.extend(kr)
            hv.extend(f64(v[at:at + n]))
            out, z, W, M = op.attention(f64(qr[at:at + n]), np.stack(hk, 1), np.stack(hv, 1), lengths[b], scale)
            e = (D + 8) * 2.0 ** -24 * M + 2.0 ** -22
            lim = 2.0 ** -8 * np.abs(out) + (2.0 ** -8 + 2 * e[..., None] + 2 * len(hk) * 2.0 ** -24) * W
            assert (np.abs(f64(o[at:at + n]) - out) <= lim).all()
            at += n

    step([50, 1, 0], 100)
    lengths[0], lengths[1] = 50, 1
    for i in range(12):
        new = [K + 1, K + 1, K + 1 if i > 3 else 0]
        step(new, 200 + 10 * i)
        for b in range(B):
            if new[b]:
                lengths[b] += int(g.integers(1, K + 2))
        if i == 6:                                     # the first request ends, another takes its place
            free.extend(int(x) for x in table[0][table[0] >= 0])
            table[0], lengths[0], hist[0] = -1, 0, ([], [])


def test_results_over_two_caches_join_by_lse(sps):
    """A prefix in one cache and the rest in another, joined with lse, are one cache's result."""
    t = Batch(sps, "f32", 4, 2, 64, 32, [200], [1], seed=13)
    want, wl = t.attend().clone(), t.lse.clone()
    parts = []
    for lo, hi in ((0, 96), (96, 201)):
        tab = t.table.copy()
        tab[0, :] = -1
        m = -(-hi // 32) - lo // 32
        tab[0, :m] = t.table[0, lo // 32:lo // 32 + m]
        t.kv.page_table.copy_(torch.from_numpy(tab))
        t.kv.lengths.fill_(hi - lo - 1)
        o = t.attend().clone()
        parts.append((o, t.lse.clone()))
    (a, x), (b, y) = parts
    z = torch.logaddexp(x, y)
    o = a * (x - z).exp()[..., None] + b * (y - z).exp()[..., None]
    assert (z - wl).abs().max() < 1e-5 and (o - want).abs().max() < 1e-5
    assert sps.device_error() == 0


def test_captured_step_follows_lengths_and_pages(sps):
    """A captured append + attention replays against whatever lengths, table and
    inputs hold then; two graphs share a workspace one after the other."""
    t = Batch(sps, "bf16", 8, 2, 64, 32, [300, 10], [2, 2], seed=14, spare=40)
    t.kv.page_table[:] = torch.randperm(t.n_pages)[:2 * t.max_pages].view(2, -1).to(torch.int32)
    k, v = randn((4, 2, 64), 1, "bf16").cuda(), randn((4, 2, 64), 2, "bf16").cuda()
    spec, ws, q2 = sps.rope_spec(64), t.kv.workspace(4, 2), torch.empty_like(t.q)

    def once():
        t.kv.append(0, k, v, rope=spec, q=t.q, q_out=q2)
        sps.paged_attention(t.kv, 0, q2, ws, out=t.out, lse=t.lse)

    st = torch.cuda.Stream()
    with torch.cuda.stream(st):
        once()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        with torch.cuda.graph(gr):
            once()
        graphs.append(gr)
    start = t.kv.buf.clone()
    for i, (a, b) in enumerate([(300, 10), (0, 0), (31, 330), (5, 64)]):
        t.kv.lengths.copy_(torch.tensor([a, b], dtype=torch.int32))
        t.q.copy_(randn(t.q.shape, 50 + i, "bf16"))
        t.kv.buf.copy_(start)
        once()
        want, wl, wb = t.out.clone(), t.lse.clone(), t.kv.buf.clone()
        for gr in graphs:
            t.kv.buf.copy_(start)
            t.out.fill_(99.0)
            gr.replay()
            torch.cuda.synchronize()
            assert torch.equal(t.out, want) and torch.equal(t.lse, wl) and torch.equal(t.kv.buf, wb)
    assert sps.device_error() == 0


def test_on_another_stream(sps):
    t = Batch(sps, "bf16", 8, 2, 64, 32, [300, 1000], [1, 1], seed=15)
    want = t.attend().clone()
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(st):
        got = t.attend(out=torch.empty_like(t.out))
        got2 = sps.rope(t.q, torch.zeros(2, dtype=torch.int32, device="cuda"), sps.rope_spec(64))
    st.synchronize()
    assert torch.equal(got, want) and torch.equal(got2, t.q)


def test_offsets_past_32_bits(sps):
    """A key plane of more than 2^31 elements: the sequence's pages are its last ones."""
    t = Batch(sps, "bf16", 2, 1, 128, 1024, [1500], [3], seed=16)
    n = (1 << 31) // (1024 * 128) + 8
    big = sps.PagedKV(2, 1, 128, n, 1024, 1, t.max_pages)
    assert big.buf[0, 0].numel() > 1 << 31
    for i in range(2):
        big.buf[0, :, n - 1 - i] = t.kv.buf[0, :, t.table[0, i]]
    big.page_table[0, :2] = torch.tensor([n - 1, n - 2], dtype=torch.int32)
    big.lengths.fill_(1500)
    want = t.attend().clone()
    ws = big.workspace(3, 3)
    assert torch.equal(sps.paged_attention(big, 0, t.q, ws), want)
    k, v = randn((3, 1, 128), 1, "bf16").cuda(), randn((3, 1, 128), 2, "bf16").cuda()
    t.kv.append(0, k, v)
    big.append(0, k, v)
    for i in range(2):
        assert torch.equal(big.buf[0, :, n - 1 - i], t.kv.buf[0, :, t.table[0, i]])
    assert sps.device_error() == 0
    del big
    torch.cuda.empty_cache()


def test_binding_checks(sps):
    t = Batch(sps, "bf16", 8, 2, 64, 32, [30], [2], seed=17)
    ws = t.kv.workspace(2, 2)
    k = randn((2, 2, 64), 1, "bf16").cuda()
    bad = [lambda: sps.paged_attention(t.kv, 0, t.q.float(), ws), lambda: sps.paged_attention(t.kv, 0, t.q[:, :4], ws),
           lambda: sps.paged_attention(t.kv, 0, t.q.transpose(0, 1).contiguous().transpose(0, 1), ws),
           lambda: sps.paged_attention(t.kv, 0, t.q, ws, lse=torch.zeros(2, 4, device="cuda")),
           lambda: sps.paged_attention(t.kv, 0, t.q, ws, starts=torch.zeros(3, dtype=torch.int32, device="cuda")),
           lambda: t.kv.append(0, k, k[:1]), lambda: t.kv.append(0, k, k.cpu()), lambda: t.kv.append(0, k, k, q_out=t.q),
           lambda: sps.rope(t.q, torch.zeros(2, device="cuda"), sps.rope_spec(64)),
           lambda: sps.rope(t.q, torch.zeros(3, dtype=torch.int32, device="cuda"), sps.rope_spec(64))]
    for f in bad:
        with pytest.raises(ValueError):
            f()
    for f in (lambda: sps.paged_attention(t.kv, 0, t.q, ws[:0]), lambda: sps.paged_attention(t.kv, 1, t.q, ws),
              lambda: sps.paged_attention(t.kv, 0, t.q, ws, scale=0.0), lambda: t.kv.append(3, k, k),
              lambda: sps.paged_attention(t.kv, 0, t.q, ws, out=t.q), lambda: sps.rope(t.q, t.st, sps.rope_spec(66))):
        with pytest.raises(sps.SPSError):
            f()
    assert sps.device_error() == 0
