"""Host-side checks of the operators around dense experts (no GPU needed): the refusals of each entry point, and the
oracle against the formats' definitions and brute force."""
import ctypes

import numpy as np
import pytest

from oracle import experts as oe

A = 4096   # an aligned stand-in address (never dereferenced: the checks fail first, or nothing is to do)


@pytest.fixture(scope="module")
def bm():
    import __graft_entry__
    __graft_entry__.build_library()
    import paper_2606_00079_gb300 as bm
    return bm


def rows8(bm, rows=4, cols=64, ld=64, codes=A, scales=A):
    return bm._Rowscale(rows, cols, ld, codes, scales)


@pytest.mark.parametrize("which", ["quantize", "dequantize"])
def test_rowscale_refusals(bm, which):
    E = bm.ERR_CODE
    if which == "quantize":
        f = lambda q, x=A, ty=0, ld=64: bm._lib().bitsmoe_rowscale_quantize(x, ty, ld, q, 0)
    else:
        f = lambda q, x=A, ty=0, ld=64: bm._lib().bitsmoe_rowscale_dequantize(q, x, ty, ld, 0)
    assert f(rows8(bm, rows=0)) == 0
    assert f(None) == E["INVALID_ARG"]
    for kw in (dict(rows=-1), dict(cols=0), dict(ld=63), dict(codes=0), dict(scales=0)):
        assert f(rows8(bm, **kw)) == E["INVALID_ARG"], kw
    for ty in (2, -1):
        assert f(rows8(bm), ty=ty) == E["INVALID_ARG"]
    assert f(rows8(bm), ld=63) == E["INVALID_ARG"]
    assert f(rows8(bm), x=0) == E["INVALID_ARG"]
    assert f(rows8(bm), x=A + 2) == E["ALIGNMENT"]
    assert f(rows8(bm), x=A + 1, ty=1) == E["ALIGNMENT"]
    assert f(rows8(bm, scales=A + 2)) == E["ALIGNMENT"]
    assert f(rows8(bm, rows=(1 << 24) + 1)) == E["SHAPE"]
    assert f(rows8(bm, cols=(1 << 20) + 1, ld=1 << 21), ld=1 << 21) == E["SHAPE"]


def test_block_norm_rowscale_refusals(bm):
    E = bm.ERR_CODE

    def f(xs=A, **kw):
        a = bm._BlockNormArgs(T=2, D=8, h=A, y=A, h_out=A, x=A, x_type=2, h_ld=8, y_ld=8, h_out_ld=8, x_ld=8, gate_ld=8)
        for k, v in kw.items():
            setattr(a, k, v)
        return bm._lib().bitsmoe_block_norm_rowscale(ctypes.byref(a), xs, 0)
    assert bm._lib().bitsmoe_block_norm_rowscale(None, A, 0) == E["INVALID_ARG"]
    assert f(T=0) == 0
    assert f(T=0, xs=0, x=0) == 0
    for kw in (dict(x_type=0), dict(x_type=1), dict(x_type=3), dict(x=0), dict(xs=0), dict(x_ld=7), dict(h=0), dict(h_ld=7),
               dict(pre_eps=float("nan")), dict(T=-1), dict(D=0)):
        assert f(**kw) == E["INVALID_ARG"], kw
    assert f(xs=A + 2) == E["ALIGNMENT"]
    assert f(D=32769, h_ld=1 << 16, y_ld=1 << 16, h_out_ld=1 << 16, x_ld=1 << 16) == E["SHAPE"]


def test_route_refusals(bm):
    E = bm.ERR_CODE

    def f(logits=A, ld=16, T=4, E=16, k=2, re=1, experts=A, weights=A, offsets=A, pairs=A, places=A, ws=A, wsb=1 << 30):
        return bm._lib().bitsmoe_route(logits, ld, T, E, k, re, experts, weights, offsets, pairs, places, ws, wsb, 0)
    for kw in (dict(T=-1), dict(E=0), dict(k=0), dict(k=17), dict(E=64, ld=64, k=33), dict(ld=15), dict(logits=0),
               dict(experts=0), dict(weights=0), dict(offsets=0), dict(pairs=0), dict(places=0), dict(T=0, offsets=0)):
        assert f(**kw) == E["INVALID_ARG"], kw
    assert f(E=1025, ld=1025) == E["SHAPE"]
    assert f(T=(1 << 23) + 1) == E["SHAPE"]
    for n in ("logits", "experts", "weights", "offsets", "pairs", "places"):
        assert f(**{n: A + 2}) == E["ALIGNMENT"], n
    assert f(ws=A + 8) == E["ALIGNMENT"]
    need = bm._lib().bitsmoe_route_workspace_bytes(1000, 16, 2)
    assert need > 0
    assert f(T=1000, wsb=need - 1) == E["WORKSPACE_TOO_SMALL"]
    assert f(T=1000, ws=0) == E["WORKSPACE_TOO_SMALL"]
    ws = bm._lib().bitsmoe_route_workspace_bytes
    assert ws(1, 16, 2) == 0
    assert [ws(*a) for a in ((-1, 16, 2), (1000, 0, 1), (1000, 1025, 2), (1000, 16, 17), (1000, 64, 33), (1 << 23, 16, 4))] == [0] * 6


def matrices(bm, ty=1, experts=3, rows=8, cols=16, ld=16, eld=128, sld=8, data=A, scales=A):
    return bm._ExpertMatrices(ty, experts, rows, cols, ld, eld, sld, data, scales)


def test_expert_product_refusals(bm):
    E = bm.ERR_CODE
    m = lambda **kw: matrices(bm, **kw)

    def f(w=None, up=None, **kw):
        w = w if w is not None else m()
        a = bm._ExpertProductArgs(ctypes.addressof(w), ctypes.addressof(up) if up is not None else None, A, A, 16, 5, 7, A, A, 2, 1,
                                  A, 8, 0)
        for k, v in kw.items():
            setattr(a, k, v)
        return bm._lib().bitsmoe_expert_product(ctypes.byref(a), 0)
    assert bm._lib().bitsmoe_expert_product(None, 0) == E["INVALID_ARG"]
    assert f(P=0) == 0
    assert f(w=m(rows=0), y_ld=0) == 0
    a = bm._ExpertProductArgs()
    assert bm._lib().bitsmoe_expert_product(ctypes.byref(a), 0) == E["INVALID_ARG"]
    for w in (m(ty=0), m(ty=3), m(experts=0), m(rows=-1), m(cols=0), m(ld=15), m(data=0), m(eld=-1), m(ty=2, scales=0),
              m(ty=2, sld=-1)):
        assert f(w=w) == E["INVALID_ARG"]
    for w in (m(experts=1025), m(rows=(1 << 20) + 1), m(cols=(1 << 20) + 1, ld=1 << 21)):
        assert f(w=w, x_ld=1 << 22, y_ld=1 << 22) == E["SHAPE"]
    assert f(up=m(ty=2)) == E["INVALID_ARG"]
    assert f(up=m(data=0)) == E["INVALID_ARG"]
    for up in (m(experts=2), m(rows=9), m(cols=15)):
        assert f(up=up) == E["SHAPE"]
    for kw in (dict(P=-1), dict(x_rows=-1), dict(fan=0), dict(y_type=2), dict(x_ld=15), dict(y_ld=7), dict(x=0), dict(offsets=0),
               dict(y=0)):
        assert f(**kw) == E["INVALID_ARG"], kw
    assert f(w=m(ty=2), x_scales=0) == E["INVALID_ARG"]
    assert f(P=(1 << 24) + 1) == E["SHAPE"]
    assert f(x_rows=(1 << 24) + 1) == E["SHAPE"]
    assert f(w=m(rows=1 << 20), P=1 << 24, y_ld=1 << 20) == E["SHAPE"]   # too many tiles
    for kw in (dict(x=A + 1), dict(offsets=A + 2), dict(index=A + 2), dict(y=A + 1), dict(x_scales=A + 1), dict(status=A + 2)):
        assert f(**kw) == E["ALIGNMENT"], kw
    assert f(w=m(data=A + 1)) == E["ALIGNMENT"]
    assert f(w=m(ty=2, scales=A + 1)) == E["ALIGNMENT"]
    assert f(y_type=0, y=A + 2) == E["ALIGNMENT"]


def test_expert_combine_refusals(bm):
    E = bm.ERR_CODE

    def f(y=A, ty=1, y_ld=8, P=6, places=A, weights=A, T=3, k=2, D=8, base=0, base_ld=0, out=A, to=0, out_ld=8):
        return bm._lib().bitsmoe_expert_combine(y, ty, y_ld, P, places, weights, T, k, D, base, base_ld, out, to, out_ld, 0)
    assert f(T=0) == 0
    for kw in (dict(T=-1), dict(P=-1), dict(k=0), dict(k=33), dict(D=0), dict(ty=2), dict(to=2), dict(y_ld=7), dict(out_ld=7),
               dict(base=A, base_ld=7), dict(y=0), dict(places=0), dict(weights=0), dict(out=0), dict(base=A, base_ld=9)):
        assert f(**kw) == E["INVALID_ARG"], kw
    for kw in (dict(T=(1 << 24) + 1), dict(P=(1 << 24) + 1), dict(D=(1 << 20) + 1, y_ld=1 << 21, out_ld=1 << 21)):
        assert f(**kw) == E["SHAPE"], kw
    for kw in (dict(y=A + 1), dict(out=A + 2), dict(places=A + 2), dict(weights=A + 1), dict(base=A + 2, base_ld=8)):
        assert f(**kw) == E["ALIGNMENT"], kw


def test_binding_refusals(bm):
    torch = pytest.importorskip("torch")
    z = lambda *s, dtype=torch.float32: torch.zeros(*s, dtype=dtype)
    f8 = torch.float8_e4m3fn
    for codes, scales in ((z(4, 8), z(4)), (z(4, 8, dtype=f8), z(3)), (z(4, 8, dtype=f8), z(4, dtype=torch.float64)),
                          (z(8, dtype=f8), z(())), (z(4, 8, dtype=f8), z(8)[::2])):
        with pytest.raises(bm.BitsMoEError):
            bm.Rowscale(codes, scales)
    q = bm.Rowscale(z(4, 8, dtype=f8), z(4))
    w = z(2, 4, 8, dtype=torch.bfloat16)
    off = z(3, dtype=torch.int32)
    for call in (lambda: bm.rowscale_quantize(z(4, 8)), lambda: bm.rowscale_dequantize(q), lambda: bm.route(z(4, 8), 2),
                 lambda: bm.expert_product(w, z(4, 8, dtype=torch.bfloat16), off), lambda: bm.expert_product(w, q, off),
                 lambda: bm.expert_combine(z(4, 8), z(2, 2, dtype=torch.int32), z(2, 2))):
        with pytest.raises(bm.BitsMoEError):   # not on a CUDA device, or of two kinds
            call()


def test_rowscale_holds_its_tensors(bm):
    torch = pytest.importorskip("torch")
    q = bm.Rowscale(torch.zeros(4, 8, dtype=torch.float8_e4m3fn), torch.zeros(4))
    for name in ("codes", "scales"):
        with pytest.raises(AttributeError):   # (the library's view of them is kept)
            setattr(q, name, torch.zeros(4))
    e = bm.Rowscale.empty([2, 3, 5], torch.device("cpu"))
    assert e.shape == (2, 3, 5) and e.codes.shape == e.shape and e.codes.stride() == (48, 16, 1) and e.scales.shape == (2, 3)


# ---------------------------------------------------------------------------
# the oracle
# ---------------------------------------------------------------------------
def test_e4m3_values_and_codes():
    v = oe.e4m3_values()
    assert v[0] == 0 and v[1] == 2.0 ** -9 and v[8] == 2.0 ** -6 and v[56] == 1.0 and v[126] == 448.0 and v[0xB8] == -1.0
    fin = np.array([b for b in range(256) if (b & 127) != 127])
    np.testing.assert_array_equal(oe.e4m3_codes(v[fin]), fin)   # (signed zeros too)
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.uniform(-448, 448, 2000), rng.standard_normal(2000) * 2.0 ** rng.integers(-12, 4, 2000)])
    got = v[oe.e4m3_codes(x)]
    best = np.abs(v[fin][None, :] - x[:, None]).min(1)
    np.testing.assert_array_equal(np.abs(got - x), best)
    # ties to the even byte
    assert v[oe.e4m3_codes(np.array([1.0625]))] == 1.0 and v[oe.e4m3_codes(np.array([1.1875]))] == 1.25
    assert oe.e4m3_codes(np.array([2.0 ** -10]))[0] == 0 and oe.e4m3_codes(np.array([3 * 2.0 ** -10]))[0] == 2


def test_rowscale_definition():
    x = np.array([[0, 0, 0], [448, -1, 0], [448.0001, -1, 0], [2.0 ** -90, 0, 0], [3.4e38, 1, 0], [2.0 ** -140, 0, 0]])
    codes, s = oe.rowscale(x)
    np.testing.assert_array_equal(s, np.float32([2.0 ** -100, 1, 2, 2.0 ** -98, 2.0 ** 120, 2.0 ** -100]))
    assert (codes[0] == 0).all() and codes[1, 0] == 126
    codes, s = oe.rowscale(np.array([[np.nan, 1], [np.inf, 1], [1, 2]]))
    assert np.isnan(s[:2]).all() and (codes[:2] == 0).all() and np.isfinite(s[2])


def test_route_oracle_against_brute_force():
    rng = np.random.default_rng(1)
    v = np.round(rng.standard_normal((40, 7)) * 2) / 2      # many ties
    v[3] = -np.inf
    v[4, 2:] = np.nan
    v[5, :5] = -np.inf
    experts, w, off, pairs, places = oe.route(v, 3)
    for t in range(40):
        got = [e for e in experts[t] if e >= 0]
        rest = [e for e in range(7) if e not in got and not np.isnan(v[t, e]) and v[t, e] > -np.inf]
        for a, b in zip(got, got[1:]):
            assert v[t, a] > v[t, b] or (v[t, a] == v[t, b] and a < b)
        if got and rest:
            m = got[-1]
            assert all(v[t, e] < v[t, m] or (v[t, e] == v[t, m] and e > m) for e in rest)
        assert not rest or len(got) == 3
        assert abs(w[t].sum() - (1 if got else 0)) < 1e-12
    assert (experts[3] == -1).all() and (places[3] == -1).all() and (w[3] == 0).all()
    n = off[-1]
    assert (pairs[n:] == -1).all() and sorted(pairs[:n]) == sorted(np.flatnonzero(experts.reshape(-1) >= 0))
    for e in range(7):
        mine = pairs[off[e]:off[e + 1]]
        assert (np.diff(mine) > 0).all() and (experts.reshape(-1)[mine] == e).all()
    for p, at in enumerate(places.reshape(-1)):
        assert at < 0 or pairs[at] == p
    big = np.round(rng.standard_normal((700, 9)) * 2) / 2   # (the other branch of the lists)
    a, b = oe.route(big, 2), oe.route(big[:400], 2)
    assert (a[2] >= b[2]).all() and (a[0][:400] == b[0]).all()
    # softmax over all
    _, w_all, *_ = oe.route(v[:1], 3, renormalize=False)
    np.testing.assert_allclose(w_all[0], np.sort(np.exp(v[0]) / np.exp(v[0]).sum())[::-1][:3])


def test_product_and_combine_oracles():
    rng = np.random.default_rng(2)
    w, up, x = rng.standard_normal((3, 4, 5)), rng.standard_normal((3, 4, 5)), rng.standard_normal((6, 5))
    off = np.array([1, 3, 3, 5])
    idx = np.array([9, 4, 11, 0, 5, 7])
    y, parts = oe.product(w, x, off, idx, 2, up)
    assert np.isnan(y[0]).all() and np.isnan(y[5]).all() and parts[0] is None and parts[5] is None
    for p, e in ((1, 0), (2, 0), (3, 2), (4, 2)):
        g, u = w[e] @ x[idx[p] // 2], up[e] @ x[idx[p] // 2]
        np.testing.assert_allclose(y[p], g / (1 + np.exp(-g)) * u)
    places, wt = np.array([[0, -1], [5, 2], [7, 1]]), rng.standard_normal((3, 2))
    base = rng.standard_normal((3, 5))
    out = oe.combine(x, places, wt, base)
    np.testing.assert_allclose(out[0], base[0] + wt[0, 0] * x[0])
    np.testing.assert_allclose(out[1], base[1] + wt[1, 0] * x[5] + wt[1, 1] * x[2])
    np.testing.assert_allclose(out[2], base[2] + wt[2, 1] * x[1])


def test_what_hands_a_stage_over():
    """Threads that store matrices into a stage beside asynchronous copies of x arrive on its barrier twice: once their copies
    are there, and, as that stands for the copies alone, for their stores."""
    import os
    import re
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    with open(os.path.join(root, "paper_2606_00079_gb300/csrc/expert_product.cu"), encoding="utf-8") as f:
        src = f.read()
    copies = re.findall(r"cp_async_arrive\((\w+)\);\n\s*(.*)", src)
    assert copies and all(re.match(r"if \(!a\.w_vec\) mbar_arrive\(%s\);" % bar, after) for bar, after in copies)
    fills = re.search(r"fills = 32 \* kXWarps \* \(!a\.w_vec && a\.x_vec \? 2 : 1\);", src)
    assert fills and re.search(r"mbar_init_n\(s\.xfull \+ i, fills\)", src) and re.search(r"\(PAIR \? 2 : fills\)", src)


def test_what_hands_a_stage_to_the_other_cta():
    """A pair's second CTA hands the rows in its shared memory over to the first one's products by a release at the cluster's
    scope, and the first one's wait for it acquires at that scope; a relaxed arrival alone stands only for tensor memory."""
    import os
    import re
    folder = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2606_00079_gb300/csrc")
    with open(os.path.join(folder, "expert_product.cu"), encoding="utf-8") as f:
        src = f.read()
    with open(os.path.join(folder, "tc.cuh"), encoding="utf-8") as f:
        tc = f.read()

    def body(name):
        return re.search(r"%s\(.*?\n}\n" % name, tc, re.S).group()
    relaxed = re.findall(r"mbar_arrive_cluster\((\w+)", src)
    assert relaxed and set(relaxed) == {"aempty0"}
    assert "mbar_release_shared_cluster(full0 + " in src and "mbar_wait_shared_cluster(s.full + st" in src
    release, wait = body("void mbar_release_shared_cluster"), body("bool mbar_wait_shared_cluster")
    assert 0 < release.index("fence.release.sync_restrict::shared::cta.cluster;") < release.index("mbar_arrive_cluster(bar)")
    assert 0 < wait.index("mbarrier.try_wait.parity.relaxed.cluster") < wait.index("fence.acquire.sync_restrict::shared::cluster.cluster;")
