"""Rotary positions and the paged cache on the host: argument checks before
any HIP call, buffer sizes, and the oracle's own pins (CPU only)."""
import ctypes
import os
import random

import numpy as np
import pytest
import torch

from oracle import paged as op

P = ctypes.c_void_p
A = P(4096)                                         # never dereferenced: every call here is refused


@pytest.fixture(scope="module")
def sps():
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    if not os.path.exists(os.path.join(root, "paper_2302_01318_amd", "libsps.so")):
        from paper_2302_01318_amd import build
        build.build()
    from paper_2302_01318_amd import sps as mod
    return mod


def ref(x):
    return ctypes.byref(x)


# ---- refusals ---------------------------------------------------------------
@pytest.mark.parametrize("change, status", [
    ({"rows": -1}, 1), ({"heads": 0}, 1), ({"dim": 7}, 1), ({"dim": 0}, 1), ({"dim": 258}, 2), ({"heads": 1025}, 2),
    ({"rows": (1 << 24) + 1}, 2), ({"dtype": 2}, 4), ({"dtype": 7}, 4), ({"x": None}, 1), ({"out": None}, 1),
    ({"pos": None}, 1), ({"xs": 511}, 1), ({"os": 511}, 1), ({"xs": 1 << 40}, 1), ({"out": A}, 1), ({"x": P(4097)}, 1),
    ({"spec": dict(rot_dim=0)}, 1), ({"spec": dict(rot_dim=3)}, 1), ({"spec": dict(rot_dim=130)}, 1),
    ({"spec": dict(rot_dim=64, base=0.0)}, 1), ({"spec": dict(rot_dim=64, base=float("nan"))}, 1),
    ({"spec": dict(rot_dim=64, base=float("inf"))}, 1), ({"spec": dict(rot_dim=64, factor=0.0)}, 1),
    ({"spec": dict(rot_dim=64, factor=-2.0)}, 1), ({"spec": dict(rot_dim=64, amplitude=float("nan"))}, 1),
    ({"spec": dict(rot_dim=64, original_len=-1)}, 1),
    ({"spec": dict(rot_dim=64, original_len=4096, low_turns=4.0, high_turns=4.0)}, 1),
    ({"spec": dict(rot_dim=64, original_len=4096, low_turns=-1.0)}, 1), ({"spec": None}, 1)])
def test_rope_refuses(sps, change, status):
    a = dict(x=A, xs=600, pos=A, spec=dict(rot_dim=64), rows=3, heads=4, dim=128, dtype=1, out=P(8192), os=512)
    a.update(change)
    spec = None if a["spec"] is None else ref(sps.rope_spec(**a["spec"]))
    assert sps.lib.sps_rope(a["x"], a["xs"], a["pos"], spec, a["rows"], a["heads"], a["dim"], a["dtype"], 0, a["out"],
                            a["os"], None) == status


def test_rope_of_no_rows_is_accepted(sps):
    assert sps.lib.sps_rope(None, 512, None, ref(sps.rope_spec(128)), 0, 4, 128, 1, 0, None, 512, None) == 0


GOOD = dict(n_heads=8, n_kv_heads=2, head_dim=128, dtype=1, n_layers=2, n_pages=10, page_size=64, B=3, max_pages=5)


@pytest.mark.parametrize("change", [
    {"n_heads": 7}, {"n_heads": 0}, {"n_kv_heads": 0}, {"n_kv_heads": 16}, {"n_heads": 2048}, {"head_dim": 96},
    {"dtype": 2}, {"dtype": -1}, {"n_layers": 0}, {"n_layers": 5000}, {"n_pages": 0}, {"n_pages": (1 << 24) + 1},
    {"page_size": 16}, {"page_size": 48}, {"page_size": 2048}, {"B": 0}, {"B": 1025}, {"max_pages": 0},
    {"max_pages": (1 << 16) + 1}, {"n_pages": 1 << 24, "page_size": 1024, "n_kv_heads": 8, "n_layers": 4096}])
def test_paged_config_refused(sps, change):
    c = sps.PagedConfig(**{**GOOD, **change})
    assert sps.lib.sps_paged_bytes(ref(c)) == 0
    h = P()
    assert sps.lib.sps_paged_create(ref(c), A, A, A, ref(h)) == 2 and not h.value
    assert sps.lib.sps_paged_workspace_bytes(ref(c), 4, 4) == 0


def test_paged_sizes(sps):
    c = sps.PagedConfig(**GOOD)
    assert sps.lib.sps_paged_bytes(ref(c)) == 2 * 2 * 10 * 2 * 64 * 128 * 2
    h = P()
    assert sps.lib.sps_paged_create(ref(c), None, A, A, ref(h)) == 1
    assert sps.lib.sps_paged_create(ref(c), P(4096 + 128), A, A, ref(h)) == 1     # 256-byte alignment
    assert sps.lib.sps_paged_create(ref(c), A, A, A, None) == 1
    assert sps.lib.sps_paged_workspace_bytes(ref(c), -1, 1) == 0
    assert sps.lib.sps_paged_workspace_bytes(ref(c), 4, 0) == 0
    assert sps.lib.sps_paged_workspace_bytes(ref(c), (1 << 20) + 1, 1) == 0
    assert sps.lib.sps_paged_workspace_bytes(ref(c), 0, 0) > 0


def test_workspace_for_more_fits_less(sps):
    g = random.Random(1)
    for _ in range(4000):
        H, G = g.choice([1, 2, 8]), g.choice([1, 3, 4, 8, 20])
        c = sps.PagedConfig(H * G, H, g.choice([64, 128]), g.choice([0, 1]), 1, 10, g.choice([32, 64, 256]),
                            g.choice([1, 3, 64, 700]), g.choice([1, 5, 9, 300]))
        r = g.randint(1, 3000)
        m = g.randint(1, r)
        r2 = g.randint(r, 4000)
        m2 = g.randint(m, r2)
        assert sps.lib.sps_paged_workspace_bytes(ref(c), r2, m2) >= sps.lib.sps_paged_workspace_bytes(ref(c), r, m)


@pytest.fixture()
def handle(sps):
    h = P()
    assert sps.lib.sps_paged_create(ref(sps.PagedConfig(**GOOD)), A, A, A, ref(h)) == 0
    yield h
    sps.lib.sps_paged_destroy(h)


@pytest.mark.parametrize("change, status", [
    ({"kv": None}, 1), ({"layer": -1}, 1), ({"layer": 2}, 1), ({"k": None}, 1), ({"v": None}, 1), ({"ks": 255}, 1),
    ({"vs": 255}, 1), ({"rows": -1}, 1), ({"rows": 5}, 1), ({"most": 0}, 1), ({"most": -1}, 1),
    ({"rows": (1 << 20) + 1, "starts": A}, 2), ({"q": A}, 1), ({"qo": A}, 1), ({"q": A, "qo": P(8192), "qs": 1000}, 1),
    ({"q": A, "qo": A, "qs": 1024, "qos": 2048}, 1), ({"k": P(4097)}, 1), ({"spec": dict(rot_dim=256)}, 1),
    ({"spec": dict(rot_dim=64, base=-1.0)}, 1)])
def test_append_refuses(sps, handle, change, status):
    a = dict(kv=handle, layer=1, k=A, ks=256, v=A, vs=256, spec=dict(rot_dim=128), q=None, qs=1024, qo=None, qos=1024,
             starts=None, rows=6, most=2)
    a.update(change)
    assert sps.lib.sps_paged_append(a["kv"], a["layer"], a["k"], a["ks"], a["v"], a["vs"], ref(sps.rope_spec(**a["spec"])),
                                    a["q"], a["qs"], a["qo"], a["qos"], a["starts"], a["rows"], a["most"], 0,
                                    None) == status


@pytest.mark.parametrize("change, status", [
    ({"kv": None}, 1), ({"layer": 2}, 1), ({"q": None}, 1), ({"out": None}, 1), ({"out": A}, 1), ({"qs": 1023}, 1),
    ({"os": 1023}, 1), ({"ws": None}, 1), ({"ws": P(4096 + 64)}, 1), ({"n": 255}, 3), ({"scale": 0.0}, 1),
    ({"scale": -1.0}, 1), ({"scale": float("nan")}, 1), ({"scale": float("inf")}, 1), ({"window": -1}, 1),
    ({"rows": 7}, 1), ({"most": 0, "starts": A}, 1), ({"rows": (1 << 20) + 1, "starts": A}, 2)])
def test_attention_refuses(sps, handle, change, status):
    a = dict(kv=handle, layer=0, q=A, qs=1024, starts=None, rows=6, most=2, scale=0.1, window=0, out=P(1 << 20),
             os=1024, ws=P(1 << 21), n=1 << 30)
    a.update(change)
    assert sps.lib.sps_paged_attention(a["kv"], a["layer"], a["q"], a["qs"], a["starts"], a["rows"], a["most"], 0,
                                       a["scale"], a["window"], a["out"], a["os"], None, a["ws"], a["n"],
                                       None) == status


def test_attention_refuses_a_misaligned_lse(sps, handle):
    assert sps.lib.sps_paged_attention(handle, 0, A, 1024, None, 6, 2, 0, 0.1, 0, P(1 << 20), 1024, P(4098), P(1 << 21),
                                       1 << 30, None) == 1


def test_no_rows_are_accepted(sps, handle):
    assert sps.lib.sps_paged_append(handle, 0, None, 256, None, 256, None, None, 0, None, 0, A, 0, 0, 0, None) == 0
    assert sps.lib.sps_paged_attention(handle, 0, None, 1024, A, 0, 0, 0, 1.0, 0, None, 1024, None, None, 0, None) == 0


def test_binding_refuses_host_tensors(sps):
    with pytest.raises(ValueError):
        sps.rope(torch.zeros(2, 3, 64), torch.zeros(2, dtype=torch.int32), sps.rope_spec(64))
    with pytest.raises(ValueError):
        sps.rope(torch.zeros(2, 64), torch.zeros(2, dtype=torch.int32), sps.rope_spec(64))
    with pytest.raises(ValueError):
        sps.rope(torch.zeros(2, 3, 64, dtype=torch.float64), torch.zeros(2, dtype=torch.int32), sps.rope_spec(64))
    with pytest.raises(ValueError):
        sps.PagedKV(8, 2, 64, 4, 32, 1, 4, device="cpu")
    with pytest.raises(KeyError):
        sps.rope_spec(64, layout="thirds")


# ---- the oracle ---------------------------------------------------------------
def test_oracle_rope_is_a_scaled_rotation_and_backward_its_transpose():
    g = np.random.default_rng(3)
    x, y = g.standard_normal((5, 2, 24)), g.standard_normal((5, 2, 24))
    pos = np.array([0, 1, 7, 1000, 90000])
    for layout in ("half", "interleaved"):
        kw = dict(rot=16, layout=layout, amplitude=1.5, factor=4.0, original_len=64)
        r = op.rope(x, pos, **kw)
        assert np.allclose(np.linalg.norm(r[..., :16], axis=-1), 1.5 * np.linalg.norm(x[..., :16], axis=-1))
        assert np.array_equal(r[..., 16:], x[..., 16:])
        assert np.allclose(r[0, :, :16], 1.5 * x[0, :, :16])
        assert np.isclose((r * y).sum(), (x * op.rope(y, pos, backward=True, **kw)).sum())


def test_oracle_rope_backward_against_differences():
    g = np.random.default_rng(4)
    x, w = g.standard_normal((1, 1, 8)), g.standard_normal((1, 1, 8))
    kw = dict(pos=[37], rot=6, layout="interleaved", amplitude=0.7)
    grad = op.rope(w, backward=True, **kw)
    for i in range(8):
        h = np.zeros_like(x)
        h[0, 0, i] = 1e-4
        d = ((op.rope(x + h, **kw) - op.rope(x - h, **kw)) * w).sum() / 2e-4
        assert abs(d - grad[0, 0, i]) < 1e-9


def test_oracle_scores_depend_on_distance_alone():
    g = np.random.default_rng(5)
    q, k = g.standard_normal((1, 1, 32)), g.standard_normal((1, 1, 32))
    s = [float((op.rope(q, [p + 11], 32) * op.rope(k, [p], 32)).sum()) for p in (0, 5, 4000)]
    assert np.allclose(s, s[0])


def test_frequencies_by_parts():
    f, base = op.frequencies(64, factor=8.0, original_len=4096, low_turns=1.0, high_turns=32.0), op.frequencies(64)
    turns = 4096 * base / (2 * np.pi)
    assert np.allclose(f[turns >= 32], base[turns >= 32]) and np.allclose(f[turns <= 1], base[turns <= 1] / 8)
    assert np.all(f <= base) and np.all(f >= base / 8)


@pytest.mark.parametrize("D", [64, 128])
def test_layout_holds_every_element_once(D):
    p, d = np.meshgrid(np.arange(64), np.arange(D), indexing="ij")
    for at in (op.key_at, op.value_at):
        assert sorted(at(p, d, D).ravel()) == list(range(64 * D))


def test_oracle_append_and_gather_agree():
    g = np.random.default_rng(6)
    kp, vp = np.zeros((6, 2, 32 * 64)), np.zeros((6, 2, 32 * 64))
    k, v = g.standard_normal((70, 2, 64)), g.standard_normal((70, 2, 64))
    table = np.array([4, 0, 3, -1])
    op.append(kp, vp, table, 0, k, v, 32)
    assert np.array_equal(op.gather(kp, table, 70, 32, 64, op.key_at), k.transpose(1, 0, 2))
    assert np.array_equal(op.gather(vp, table, 70, 32, 64, op.value_at), v.transpose(1, 0, 2))


def test_oracle_attention_of_one_position_is_its_value():
    g = np.random.default_rng(7)
    K, V = g.standard_normal((1, 3, 8)), g.standard_normal((1, 3, 8))
    out, lse, _, _ = op.attention(g.standard_normal((3, 2, 8)), K, V, 0, 0.3, window=1)
    assert np.allclose(out, np.repeat(V[0][:, None], 2, 1))
    assert np.isfinite(lse).all()
