"""GPU checks of the routing, the products grouped by expert and their weighted sum against float64.

Tolerances, by arithmetic (u = 2^-24).  A sum of K exact products in fp32, in any order and with the tensor core's
truncating additions (an addition loses less than 2^-23 of the largest operand, and every partial sum is at most the sum M of
the products' magnitudes): (K + 8) 2^-23 M; its scales add 2 u each of the sum.  SiLU(g) u: |SiLU'| <= 1.1, expf and
the division at most 8 u (and |g| u through the exponent's argument).  A bf16 result adds half a step, 2^-8 relative.
Softmax weights: the exponent's argument is off by u |l - l_max|, expf by 2 units in the last place, the sum of n by n u,
the division by u."""
import ctypes

import numpy as np
import pytest

from oracle import experts as oe

pytestmark = pytest.mark.gpu
u = 2.0 ** -24


@pytest.fixture(scope="module")
def env():
    torch = pytest.importorskip("torch")
    if not torch.cuda.is_available():
        pytest.skip("no CUDA device")
    import __graft_entry__
    __graft_entry__.build()
    import paper_2606_00079_gb300 as bm
    torch.cuda.set_device(0)
    return torch, bm


# ---------------------------------------------------------------------------
# routing
# ---------------------------------------------------------------------------
def logits_of(rng, T, E):
    v = rng.standard_normal((T, E)) * 2
    v = np.where(rng.random((T, 1)) < 0.5, np.round(v * 2) / 2, v).astype(np.float32)   # many ties in half of the rows
    kinds = rng.integers(0, 12, T)
    v[kinds == 0] = -np.inf
    v[kinds == 1] = np.nan
    v[kinds == 2, E // 2:] = -np.inf
    v[kinds == 3, :E // 3] = np.nan
    v[kinds == 4] *= 0.0    # signed zeros
    v[kinds == 5] = 1e30 * v[kinds == 5]
    return v


@pytest.mark.parametrize("T,E,k", [(1, 1, 1), (1, 128, 8), (3, 7, 7), (31, 33, 4), (32, 64, 8), (64, 128, 8), (65, 128, 8),
                                   (70, 1024, 32), (200, 300, 5), (1000, 2, 2), (4999, 61, 6), (6000, 1000, 3), (20000, 16, 4)])
@pytest.mark.parametrize("renorm", [True, False])
def test_route(env, T, E, k, renorm):
    torch, bm = env
    v = logits_of(np.random.default_rng([T, E, k]), T, E)
    wide = torch.full((T, E + 3), 99.0, device="cuda")
    wide[:, 1:1 + E] = torch.from_numpy(v).cuda()
    r = bm.route(wide[:, 1:1 + E], k, renormalize=renorm)
    experts, weights, offsets, pairs, places = oe.route(v, k, renorm)
    for name, want in (("experts", experts), ("offsets", offsets), ("pairs", pairs), ("places", places)):
        np.testing.assert_array_equal(getattr(r, name).cpu().numpy(), want, err_msg=name)
    got = r.weights.double().cpu().numpy()
    none = experts < 0
    assert (got[none] == 0).all()
    with np.errstate(invalid="ignore", divide="ignore"):
        span = np.where(weights > 0, np.abs(np.log(weights / np.maximum(weights.max(1, keepdims=True), 1e-300))), 0)
        # (over all: the largest argument that counts is below 104, where expf underflows)
        tol = (2 * np.maximum(span, 0 if renorm else 104) + (k if renorm else E) + 16) * u * weights + 1e-40
    assert (np.abs(got - weights) <= tol).all()
    again = bm.route(torch.from_numpy(v).cuda(), k, renormalize=renorm)
    for a, b in zip(r, again):
        assert torch.equal(a, b)


def test_route_no_tokens_infinity_and_refusals(env):
    torch, bm = env
    r = bm.route(torch.empty(0, 16, device="cuda"), 4)
    assert r.offsets.tolist() == [0] * 17 and r.pairs.numel() == 0 and r.experts.shape == (0, 4)
    r = bm.route(torch.tensor([[0.0, float("inf"), 1.0]], device="cuda"), 2)
    assert r.experts.tolist() == [[1, 2]] and torch.isnan(r.weights).all()
    for bad in (0, 17, 33):
        with pytest.raises(bm.BitsMoEError):
            bm.route(torch.zeros(4, 16, device="cuda"), bad)
    with pytest.raises(bm.BitsMoEError):
        bm.route(torch.zeros(4, 16, device="cuda", dtype=torch.bfloat16), 2)


def test_route_in_two_graphs_and_on_a_stream(env):
    torch, bm = env
    rng = np.random.default_rng(5)
    data = [torch.from_numpy(logits_of(rng, 500, 64)).cuda() for _ in range(3)]
    buf = [torch.zeros(500, 64, device="cuda") for _ in range(2)]
    graphs, outs = [], []
    for b in buf:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(bm.route(b, 6))
        graphs.append(g)
    for i in range(2):
        buf[0].copy_(data[i])
        buf[1].copy_(data[i + 1])
        graphs[1].replay()
        graphs[0].replay()
        torch.cuda.synchronize()
        for o, d in zip(outs, (data[i], data[i + 1])):
            for a, b in zip(o, bm.route(d, 6)):
                assert torch.equal(a, b)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    r = bm.route(data[0], 6, stream=st)
    st.synchronize()
    for a, b in zip(r, bm.route(data[0], 6)):
        assert torch.equal(a, b)


# ---------------------------------------------------------------------------
# products
# ---------------------------------------------------------------------------
def pitched(torch, x, ty, shift=0):
    """bf16 rows, or codes with odd scales, on 16-byte boundaries (shift 0) or off them; and their float64 values."""
    n = 8 if ty == "bf16" else 16
    if ty == "bf16":
        t, scale = x.to(torch.bfloat16), None
        vals = t.double()
    else:
        scale = x.abs().amax(-1) / 300 + 1e-3
        t = (x / scale[..., None]).to(torch.float8_e4m3fn)
        vals = t.double() * scale.double()[..., None]
    C = x.shape[-1]
    pitch = (C + n - 1) // n * n if not shift else C + 1 + (C % 2)
    flat = torch.zeros(*x.shape[:-1], pitch + (2 if shift else 0), dtype=torch.float32).to(t.dtype).cuda()[..., shift:shift + C]
    (flat.view(torch.uint8) if ty == "e4m3" else flat).copy_((t.view(torch.uint8) if ty == "e4m3" else t).cuda())
    return flat, scale.cuda() if scale is not None else None, vals.numpy()


def wrap(bm, t, s):
    return t if s is None else bm.Rowscale(t, s)


def run_product(env, counts, R, C, ty="bf16", glu=False, fan=0, out="bf16", shift=0, lead=0, tail=0, seed=0, tokens=None):
    """counts: rows of each expert; fan: 0 (rows in order) or the index's divisor."""
    torch, bm = env
    E = len(counts)
    off = lead + np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    P = int(off[-1]) + tail
    g = torch.Generator().manual_seed(1000 * seed + 7 * R + C + P)
    w, ws, wv = pitched(torch, torch.randn(E, R, C, generator=g) * (0.5 + torch.rand(E, R, 1, generator=g)) / C ** 0.5, ty, shift)
    up, us, uv = pitched(torch, torch.randn(E, R, C, generator=g) / C ** 0.5, ty, shift) if glu else (None, None, None)
    rows = P if not fan else tokens or max(1, P // fan)
    x, xs, xv = pitched(torch, torch.randn(rows, C, generator=g) * 3, ty, shift)
    idx = torch.randint(0, rows * fan, (P,), generator=g, dtype=torch.int32) if fan else None
    dt = torch.float32 if out == "f32" else torch.bfloat16
    ybuf = torch.full((P, R + 3), 77.0, dtype=dt, device="cuda")
    y = ybuf[:, 1:1 + R]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), torch.from_numpy(off).cuda(), index=idx.cuda() if fan else None,
                            fan=max(fan, 1), up=wrap(bm, up, us) if glu else None, y=y, status=status)
    assert got is y
    ybuf = ybuf.double().cpu().numpy()
    assert int(status.item()) == 0
    assert (ybuf[:, 0] == 77).all() and (ybuf[:, 1 + R:] == 77).all()
    # float64, expert by expert
    q = idx.numpy() // fan if fan else np.arange(P)
    for e in range(E):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        xr = xv[q[a:b]]
        gs, gm = xr @ wv[e].T, np.abs(xr) @ np.abs(wv[e]).T
        eg = (C + 8) * 2.0 ** -23 * gm + 8 * u * np.abs(gs)
        if glu:
            us_, um = xr @ uv[e].T, np.abs(xr) @ np.abs(uv[e]).T
            eu = (C + 8) * 2.0 ** -23 * um + 8 * u * np.abs(us_)
            silu = gs / (1 + np.exp(-gs))
            want = silu * us_
            tol = 1.1 * eg * (np.abs(us_) + eu) + np.abs(silu) * eu + (16 + np.abs(gs)) * u * np.abs(want)
        else:
            want, tol = gs, eg
        tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if out == "bf16" else 2 * u * np.abs(want)) + 1e-37
        d = np.abs(ybuf[a:b, 1:1 + R] - want)
        assert (d <= tol).all(), (e, np.argwhere(~(d <= tol))[:4].tolist(), float(np.nanmax(d / tol)))
    assert (ybuf[:off[0]] == 77).all() and (ybuf[off[-1]:] == 77).all()


def ragged(rng, E, most, empty=0.3):
    c = rng.integers(0, most + 1, E)
    c[rng.random(E) < empty] = 0
    return c


PRODUCTS = [
    # counts of each expert, rows, cols
    ([1], 1, 1), ([1], 64, 64), ([3], 17, 40), ([0, 5, 0, 1], 100, 72), ([0, 0, 0], 64, 64), ([16, 17, 15, 1], 128, 128),
    ([33, 0, 2], 200, 264), ([1, 1, 1, 1, 1, 1, 1, 1], 96, 512), ([255, 256, 257], 130, 136), ([513, 1, 70], 64, 200),
    ([40, 3], 1001, 2041), ([700], 65, 33),
]


@pytest.mark.parametrize("case", range(len(PRODUCTS)))
@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("fan", [0, 1, 3])
def test_expert_product(env, case, ty, glu, fan):
    counts, R, C = PRODUCTS[case]
    run_product(env, counts, R, C, ty, glu, fan, out="f32" if case % 2 else "bf16", lead=case % 3, tail=2 * (case % 2), seed=case)


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("fan", [0, 2])
def test_expert_product_off_the_boundaries(env, ty, glu, fan):
    run_product(env, [5, 0, 70, 1], 67, 129, ty, glu, fan, out="f32", shift=1, lead=1, tail=1)


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("counts,R,C", [([1], 64, 64), ([5, 0, 70, 1], 67, 129), ([300, 2], 300, 517), ([3, 9], 40, 4095), ([2], 33, 1),
                                          ([700, 900], 700, 2041)])
@pytest.mark.parametrize("shift", [1, 3, 8, 15])
def test_expert_product_rows_of_x_off_the_boundaries(env, ty, counts, R, C, shift):
    """Matrices on 16-byte boundaries, rows of x anywhere: the bits of the same rows on boundaries."""
    torch, bm = env
    g = torch.Generator().manual_seed(C)
    E, P = len(counts), sum(counts)
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)
    raw = torch.full((P, C + 17), 127, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) if ty == "e4m3" else torch.full(
        (P, C + 17), float("nan"), dtype=torch.bfloat16, device="cuda")   # (NaN between the rows)
    off_x = raw[:, shift:shift + C]
    (off_x.view(torch.uint8) if ty == "e4m3" else off_x).copy_(x.view(torch.uint8) if ty == "e4m3" else x)
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    idx = torch.randint(0, 2 * P, (P,), generator=g, dtype=torch.int32).cuda()
    for kw in (dict(), dict(index=idx, fan=2, up=wrap(bm, up, us))):
        for dt in (torch.float32, torch.bfloat16):
            a = bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), off, dtype=dt, **kw)
            b = bm.expert_product(wrap(bm, w, ws), wrap(bm, off_x, xs), off, dtype=dt, **kw)
            assert torch.equal(a, b)


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("counts,R,C", [([1], 64, 64), ([5, 0, 70, 1], 67, 129), ([300, 2], 300, 517), ([3, 9], 40, 4095), ([2], 33, 1)])
@pytest.mark.parametrize("shift", [1, 6])
def test_expert_product_matrices_off_the_boundaries(env, ty, counts, R, C, shift):
    """Matrices anywhere (with or without U, x on boundaries or off them): the bits of the same matrices on boundaries."""
    torch, bm = env
    g = torch.Generator().manual_seed(C)
    E, P = len(counts), sum(counts)
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)

    def moved(t):
        raw = torch.full((*t.shape[:-1], C + 9), 127, dtype=torch.uint8, device="cuda").view(t.dtype) if ty == "e4m3" else torch.full(
            (*t.shape[:-1], C + 9), float("nan"), dtype=t.dtype, device="cuda")
        v = raw[..., shift:shift + C]
        (v.view(torch.uint8) if ty == "e4m3" else v).copy_(t.view(torch.uint8) if ty == "e4m3" else t)
        return v
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    for u_ in (None, up):
        for dt in (torch.float32, torch.bfloat16):
            a = bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), off, up=None if u_ is None else wrap(bm, u_, us), dtype=dt)
            for xx in (x, moved(x)):
                b = bm.expert_product(wrap(bm, moved(w), ws), wrap(bm, xx, xs), off, up=None if u_ is None else wrap(bm, moved(u_), us), dtype=dt)
                assert torch.equal(a, b)


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("E,P,R,C", [(3, 100, 300, 1030), (40, 400, 200, 2050)])
def test_expert_product_matrices_off_the_boundaries_beside_copies(env, ty, E, P, R, C):
    """Matrices that threads store into a stage beside their own asynchronous copies of x, more steps than stages: the bits of
    matrices on boundaries, every time."""
    torch, bm = env
    g = torch.Generator().manual_seed(P)
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    w1, up1 = (torch.zeros(E, R, C + 1, dtype=torch.uint8 if ty == "e4m3" else torch.bfloat16, device="cuda").view(w.dtype)[..., 1:] for _ in range(2))
    for a, b in ((w1, w), (up1, up)):
        (a.view(torch.uint8) if ty == "e4m3" else a).copy_(b.view(torch.uint8) if ty == "e4m3" else b)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)
    x = wrap(bm, x, xs)
    off = torch.linspace(0, P, E + 1).int().cuda()
    for u_, u1_ in ((None, None), (wrap(bm, up, us), wrap(bm, up1, us))):
        for dt in (torch.float32, torch.bfloat16):
            ref = bm.expert_product(wrap(bm, w, ws), x, off, up=u_, dtype=dt)
            for _ in range(10):
                assert torch.equal(bm.expert_product(wrap(bm, w1, ws), x, off, up=u1_, dtype=dt), ref)


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("matrices", [0, 1])
@pytest.mark.parametrize("rows", [0, 1])
def test_expert_product_of_pairs_on_and_off_the_boundaries(env, ty, matrices, rows):
    """Pairs of CTAs (100 rows each of 15 experts: 30 tiles of pairs, with U 45; below the size from which rows of x are copied),
    more steps than stages: every way that matrices and rows of x reach a stage, the same bits every time, and within the
    bounds of the values."""
    torch, bm = env
    g = torch.Generator().manual_seed(2 * matrices + rows)
    E, P, R, C = 15, 1500, 600, 1500
    w, ws, wv = pitched(torch, torch.randn(E, R, C, generator=g) / C ** 0.5, ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g) / C ** 0.5, ty)
    x, xs, xv = pitched(torch, torch.randn(P, C, generator=g), ty)
    assert P * R * C <= 2 ** 31   # (rows of x: read as they lie)

    def off_by_one(t):
        flat = torch.zeros(*t.shape[:-1], C + 3, dtype=torch.uint8 if ty == "e4m3" else torch.bfloat16, device="cuda").view(t.dtype)[..., 1:1 + C]
        (flat.view(torch.uint8) if ty == "e4m3" else flat).copy_(t.view(torch.uint8) if ty == "e4m3" else t)
        return flat
    counts = torch.full((E,), P // E)
    counts[3], counts[4] = 0, 2 * (P // E)
    off = torch.cat([torch.zeros(1, dtype=torch.long), counts.cumsum(0)]).int().cuda()
    idx = torch.randperm(P, generator=g).int()
    kw = dict(index=idx.cuda(), dtype=torch.bfloat16)
    w1, up1, x1 = (off_by_one(t) if m else t for t, m in ((w, matrices), (up, matrices), (x, rows)))
    for glu in (False, True):
        ref = bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), off, up=wrap(bm, up, us) if glu else None, **kw)
        for _ in range(8):
            y = bm.expert_product(wrap(bm, w1, ws), wrap(bm, x1, xs), off, up=wrap(bm, up1, us) if glu else None, **kw)
            assert torch.equal(y, ref)
        if not glu:
            o = off.tolist()
            for e in range(E):
                xr = xv[idx.numpy()[o[e]:o[e + 1]]]
                want, mag = xr @ wv[e].T, np.abs(xr) @ np.abs(wv[e]).T
                tol = (C + 8) * 2.0 ** -23 * mag + 8 * u * np.abs(want)
                assert (np.abs(ref[o[e]:o[e + 1]].double().cpu().numpy() - want) <= tol + 2.0 ** -8 * (np.abs(want) + tol)).all()


@pytest.mark.parametrize("times", [1, 4, 5, 60])
def test_expert_product_of_few_of_many_rows_off_the_boundaries(env, times):
    """Large products of rows of x off boundaries: x is copied only where it has up to four rows for each of y, whatever it holds
    beside them; the same bits either way."""
    torch, bm = env
    g = torch.Generator().manual_seed(times)
    E, P, R, C = 2, 600, 2048, 2047
    n = times * P
    w, _, _ = pitched(torch, torch.randn(E, R, C, generator=g), "bf16")
    x = torch.randn(n, C, dtype=torch.bfloat16, device="cuda")   # (an odd pitch)
    off = torch.tensor([0, 250, P], dtype=torch.int32).cuda()
    idx = torch.randint(0, n, (P,), generator=g, dtype=torch.int32).cuda()
    y = torch.zeros(P, R, device="cuda")
    assert P * R * C > 2 ** 31
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    before = torch.cuda.memory_allocated()
    bm.expert_product(w, x, off, index=idx, y=y)
    used = torch.cuda.max_memory_allocated() - before
    assert (n * 2048 * 2 <= used < n * 2048 * 2 + 2 ** 21) if times <= 4 else used == 0
    rows = torch.zeros(P, 2048, dtype=torch.bfloat16, device="cuda")[:, :C]
    rows.copy_(x[idx.long()])
    assert torch.equal(bm.expert_product(w, rows, off), y)


@pytest.mark.parametrize("E,most,R,C,ty,glu", [(128, 6, 96, 256, "bf16", True), (300, 3, 40, 128, "e4m3", False), (1024, 2, 16, 64, "bf16", False),
                                               (60, 40, 320, 512, "e4m3", True), (7, 400, 384, 256, "bf16", True), (5, 600, 520, 384, "e4m3", False)])
def test_expert_product_many_experts_and_tiles(env, E, most, R, C, ty, glu):
    rng = np.random.default_rng([E, most])
    run_product(env, ragged(rng, E, most), R, C, ty, glu, fan=4, out="f32", lead=3, tail=5)
    run_product(env, ragged(rng, E, most), R, C, ty, glu, fan=0, out="bf16")


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_expert_product_large(env, ty, glu, shift, out):
    """Many rows an expert, several turns of every CTA, more than one chain of sums of an fp32 result."""
    rng = np.random.default_rng(12)
    counts = rng.integers(200, 700, 12)
    counts[4] = 0
    run_product(env, counts, 1300, 1230, ty, glu, fan=2, out=out, shift=shift, lead=2, tail=3)


def test_expert_product_deep(env):
    run_product(env, [9, 40], 64, 14336, "bf16", False, 0, "f32")
    run_product(env, [9, 40], 64, 14336, "e4m3", True, 2, "bf16")


def test_expert_product_strided_and_shared_matrices(env):
    """Gate and up as halves of one tensor, an expert's pitch that is not rows * pitch, one matrix for all experts."""
    torch, bm = env
    g = torch.Generator().manual_seed(3)
    both = torch.randn(4, 96, 128, generator=g).to(torch.bfloat16).cuda()
    x = torch.randn(20, 128, generator=g).to(torch.bfloat16).cuda()
    off = torch.tensor([0, 4, 4, 15, 20], dtype=torch.int32).cuda()
    a = bm.expert_product(both[:, :48], x, off, up=both[:, 48:])
    b = bm.expert_product(both[:, :48].contiguous(), x, off, up=both[:, 48:].contiguous())
    assert torch.equal(a, b)
    a = bm.expert_product(both[::2, :48], x, off[:3])
    b = bm.expert_product(both[::2, :48].contiguous(), x, off[:3])
    assert torch.equal(a[:4], b[:4])
    turned = both.transpose(0, 1).contiguous().transpose(0, 1)   # experts between the rows
    assert turned.stride() == (128, 512, 1)
    assert torch.equal(bm.expert_product(turned, x, off), bm.expert_product(both, x, off))
    one = both[:1].expand(4, 96, 128)
    a = bm.expert_product(one, x, off)
    b = bm.expert_product(both[:1], x, torch.tensor([0, 20], dtype=torch.int32).cuda())
    # (the sums' order may depend on a tile's size)
    tol = (128 + 8) * 2.0 ** -22 * (x.double().abs() @ both[0].double().abs().T)
    assert ((a.double() - b.double()).abs() <= tol).all()


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("shift", [0, 1])
def test_expert_product_rows_that_are_not_there(env, ty, shift):
    """Indices that are no row of x give NaN rows and nothing else; offsets outside 0 .. P are held there."""
    torch, bm = env
    g = torch.Generator().manual_seed(4)
    w, ws, _ = pitched(torch, torch.randn(3, 80, 96, generator=g), ty, shift)
    x, xs, _ = pitched(torch, torch.randn(10, 96, generator=g), ty, shift)
    w, x = wrap(bm, w, ws), wrap(bm, x, xs)
    idx = torch.randint(0, 20, (40,), generator=g, dtype=torch.int32)
    bad = idx.clone()
    for p, v in ((0, -1), (5, 20), (17, 2 ** 31 - 1), (18, -2 ** 31), (39, 21)):
        bad[p] = v
    off = torch.tensor([0, 18, 18, 40], dtype=torch.int32).cuda()
    good = bm.expert_product(w, x, off, index=idx.cuda(), fan=2)
    y = bm.expert_product(w, x, off, index=bad.cuda(), fan=2)
    lost = torch.tensor([0, 5, 17, 18, 39])
    keep = torch.ones(40, dtype=torch.bool)
    keep[lost] = False
    assert torch.isnan(y[lost.cuda()]).all() and torch.equal(y[keep.cuda()], good[keep.cuda()])
    y = torch.zeros(40, 80, device="cuda")
    bm.expert_product(w, x, torch.tensor([-5, 18, 18, 4000], dtype=torch.int32).cuda(), index=idx.cuda(), fan=2, y=y)
    assert torch.equal(y, good)
    y.zero_()
    bm.expert_product(w, x, torch.tensor([30, 18, 50, 18], dtype=torch.int32).cuda(), index=idx.cuda(), fan=2, y=y)
    assert (y[:18] == 0).all()
    # rows in order: past x's last row
    y = bm.expert_product(w, x, torch.tensor([0, 4, 4, 10], dtype=torch.int32).cuda())
    assert torch.isfinite(y).all()


@pytest.mark.parametrize("E,P,R,C", [(6, 20, 130, 1100), (200, 400, 130, 200), (40, 3000, 600, 200)])   # split columns, single CTAs, pairs
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_expert_product_offsets_that_do_not_ascend(env, E, P, R, C, out):
    """Every second expert has all rows, so that there are many more tiles than rows of y allow: nothing but y's rows is
    touched, and the next call is as ever."""
    torch, bm = env
    dt = torch.float32 if out == "f32" else torch.bfloat16
    w, x = torch.randn(E, R, C, device="cuda").bfloat16(), torch.randn(P, C, device="cuda").bfloat16()
    good = torch.linspace(0, P, E + 1).int().cuda()
    ref = bm.expert_product(w, x, good, up=w, dtype=dt)
    bad = torch.tensor([(-1, P + 1)[e % 2] for e in range(E + 1)], dtype=torch.int32).cuda()
    buf = torch.full((P + 2, R + 3), 77.0, dtype=dt, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.expert_product(w, x, bad, up=w, y=buf[1:1 + P, 1:1 + R], status=status)
    rest = buf.clone()
    rest[1:1 + P, 1:1 + R] = 77.0
    assert bool((rest == 77).all()) and int(status.item()) == 0
    assert torch.equal(bm.expert_product(w, x, good, up=w, dtype=dt), ref)


def far_apart(torch, big, x, gap):
    """x's rows (or matrices), gap elements of `big` apart."""
    view = big.view(x.dtype).as_strided(x.shape, ((gap, x.shape[2] + 16, 1) if x.dim() == 3 else (gap, 1)))
    (view.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else view).copy_(x.view(torch.uint8) if x.dtype is torch.float8_e4m3fn else x)
    return view


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("P,R", [(6, 300), (300, 96), (1600, 520)])   # split columns, single CTAs, (with U) pairs
@pytest.mark.parametrize("shift", [0, 1])   # of the gaps: on 16-byte boundaries and off them
def test_expert_product_past_32_bits(env, ty, P, R, shift):
    """Rows of x and y, and matrices, of which the last begin past 2^32 elements: the bits of the same close together."""
    torch, bm = env
    g = torch.Generator().manual_seed(P + R)
    E, C = 12, 272
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)
    off = torch.linspace(0, P, E + 1).int().cuda()
    one = 2 if ty == "bf16" else 1
    big = [torch.empty((2 ** 32 + 2 ** 26) * b, dtype=torch.uint8, device="cuda") for b in (one, one, 2)]
    gap_w, gap_p = (2 ** 32 // (E - 1) + 1) // 16 * 16 + 16 + shift, (2 ** 32 // (P - 1) + 1) // 16 * 16 + 16 + shift
    wide_w, wide_x = far_apart(torch, big[0], w, gap_w), far_apart(torch, big[1], x, gap_p)
    y = far_apart(torch, big[2], torch.zeros(P, R, dtype=torch.bfloat16, device="cuda"), gap_p)
    assert min((E - 1) * gap_w, (P - 1) * gap_p) >= 2 ** 32
    for up, wide_up in ((None, None), (wrap(bm, w, ws), wrap(bm, wide_w, ws))):
        ref = bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), off, up=up, dtype=torch.bfloat16)
        y.zero_()
        bm.expert_product(wrap(bm, wide_w, ws), wrap(bm, wide_x, xs), off, up=wide_up, y=y)
        assert torch.equal(y, ref)


@pytest.mark.parametrize("shift", [0, 1])
def test_rows_and_sums_past_32_bits(env, shift):
    """The coder, its inverse, the norm to 8 bits and the weighted sum on rows of which the last begin past 2^32 elements."""
    torch, bm = env
    g = torch.Generator().manual_seed(7)
    T, k, D = 9, 3, 264
    gap = 2 ** 32 // (T - 1) + 16 + shift
    big = [torch.empty(2 ** 32 + 2 ** 26, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    codes = torch.empty(2 ** 32 + 2 ** 26, dtype=torch.uint8, device="cuda")
    x = torch.randn(T, D, generator=g).bfloat16().cuda()
    wide, back = far_apart(torch, big[0], x, gap), far_apart(torch, big[1], torch.zeros_like(x), gap)
    q = bm.Rowscale(far_apart(torch, codes, torch.zeros(T, D, dtype=torch.float8_e4m3fn, device="cuda"), gap), torch.zeros(T, device="cuda"))
    ref = bm.rowscale_quantize(x)
    bm.rowscale_quantize(wide, q)
    assert torch.equal(q.codes.view(torch.uint8), ref.codes.view(torch.uint8)) and torch.equal(q.scales, ref.scales)
    bm.rowscale_dequantize(q, out=back)
    assert torch.equal(back, bm.rowscale_dequantize(ref, torch.bfloat16))
    ref = bm.block_norm(x, x_dtype=torch.float8_e4m3fn)[1]
    bm.block_norm(wide, x=q)
    assert torch.equal(q.codes.view(torch.uint8), ref.codes.view(torch.uint8)) and torch.equal(q.scales, ref.scales)
    places = torch.randint(-1, T, (T, k), generator=g, dtype=torch.int32).cuda()
    weights = torch.rand(T, k, generator=g).cuda()
    bm.expert_combine(wide, places, weights, out=back)
    assert torch.equal(back, bm.expert_combine(x, places, weights, dtype=torch.bfloat16))


def test_expert_product_nothing_to_do(env):
    torch, bm = env
    w = torch.randn(2, 8, 16, device="cuda").to(torch.bfloat16)
    x = torch.randn(4, 16, device="cuda").to(torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    y = torch.full((4, 8), 5.0, device="cuda")
    assert (bm.expert_product(w, x, off, y=y) == 5).all()
    assert bm.expert_product(w, x[:0], off).shape == (0, 8)
    assert bm.expert_product(w[:, :0], x, off).shape == (4, 0)
    # no rows of x at all, all of them asked for
    y = bm.expert_product(w, x[:0], torch.tensor([0, 2, 3], dtype=torch.int32).cuda(), index=torch.zeros(3, dtype=torch.int32).cuda())
    assert torch.isnan(y).all()


def test_expert_product_not_finite_stays_in_its_row(env):
    torch, bm = env
    w = torch.randn(2, 64, 128, device="cuda").to(torch.bfloat16)
    x = torch.randn(40, 128, device="cuda").to(torch.bfloat16)
    off = torch.tensor([0, 17, 40], dtype=torch.int32).cuda()
    good = bm.expert_product(w, x, off)
    x[16, 3], x[17, 9] = float("nan"), float("inf")
    y = bm.expert_product(w, x, off)
    keep = torch.ones(40, dtype=torch.bool, device="cuda")
    keep[16:18] = False
    assert torch.equal(y[keep], good[keep]) and torch.isnan(y[16]).all() and not torch.isfinite(y[17]).any()
    w[0, 5, 7] = float("nan")
    y = bm.expert_product(w, x, off)
    rows = torch.ones(64, dtype=torch.bool, device="cuda")
    rows[5] = False
    assert torch.equal(y[:16, rows], good[:16, rows]) and torch.isnan(y[:16, 5]).all()


def test_expert_product_in_a_graph_and_on_a_stream(env):
    torch, bm = env
    rng = np.random.default_rng(9)
    E, k, T = 16, 3, 50
    w = torch.randn(E, 96, 128, device="cuda").to(torch.bfloat16)
    up = torch.randn(E, 96, 128, device="cuda").to(torch.bfloat16)
    x = torch.randn(T, 128, device="cuda").to(torch.bfloat16)
    data = [torch.from_numpy(logits_of(rng, T, E)).cuda() for _ in range(3)]
    logits = data[0].clone()
    y = torch.zeros(T * k, 96, device="cuda")

    def step():
        r = bm.route(logits, k)
        return bm.expert_product(w, x, r.offsets, index=r.pairs, fan=k, up=up, y=y)
    step()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        step()
    for d in data[1:]:
        logits.copy_(d)
        y.zero_()
        g.replay()
        got = y.clone()
        y.zero_()
        assert torch.equal(got, step())
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    r = bm.route(logits, k)
    st.wait_stream(torch.cuda.current_stream())
    a = bm.expert_product(w, x, r.offsets, index=r.pairs, fan=k, up=up, stream=st)
    st.synchronize()
    n = int(r.offsets[-1])
    assert torch.equal(a[:n], y[:n])


# experts, rows of a matrix, columns, rows of y, first rows of y and of the matrices that are lost with block 0's first tile:
# pairs (many rows an expert; fp32: single CTAs), large (fp32: tiles of 128 rows), single CTAs (few), columns split over a
# cluster (few tiles: all of the tile is lost)
LOST = {"pairs": (12, 700, 4096, 1200, 64, 128), "large": (12, 2600, 4096, 4800, 64, 128), "single": (80, 520, 4096, 400, 5, 128), "split": (3, 520, 8192, 15, 5, 128)}


@pytest.mark.parametrize("kind", sorted(LOST))
@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("fan", [0, 2])
def test_expert_product_lost_waits(env, kind, ty, glu, fan):
    """An arrival of block 0 is left out, so that its waits run out: the call reports it, what it lost is NaN, every other
    result stands, and the next call is as ever."""
    torch, bm = env
    g = torch.Generator().manual_seed(8)
    E, R, C, P, rows, cols = LOST[kind]
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty) if glu else (None, None, None)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)
    w, x = wrap(bm, w, ws), wrap(bm, x, xs)
    up = wrap(bm, up, us) if glu else None
    off = torch.arange(0, P + 1, P // E, dtype=torch.int32).cuda()
    idx = torch.randint(0, 2 * P, (P,), generator=g, dtype=torch.int32).cuda() if fan else None
    kw = dict(index=idx, fan=max(fan, 1), up=up)
    for dt in (torch.float32, torch.bfloat16):
        ref = bm.expert_product(w, x, off, dtype=dt, **kw)
        for with_status in (True, False):
            buf = torch.full((P, R + 8), 7.0, dtype=dt, device="cuda")
            y, status = buf[:, :R], torch.zeros(1, dtype=torch.int32, device="cuda")
            bm.bitsmoe_debug_wait_limit(1, 2_000_000)
            try:
                bm.expert_product(w, x, off, y=y, status=status if with_status else None, **kw)
                torch.cuda.synchronize()
            finally:
                bm.bitsmoe_debug_wait_limit(0, 0)
            assert int(status.item()) == (bm.ERR_CODE["TIMEOUT"] if with_status else 0)
            lost = torch.isnan(y)
            assert bool(lost[:rows, :cols].all()) and not bool(lost.all())
            assert torch.equal(y[~lost], ref[~lost])
            assert (buf[:, R:] == 7).all()
            status.zero_()
            assert torch.equal(bm.expert_product(w, x, off, y=y, status=status, **kw), ref)
            assert int(status.item()) == 0


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("strips", [2, 8])   # 192 tiles of pairs, and 768
def test_expert_product_lost_plan(env, ty, glu, strips):
    """Pairs of CTAs with several waves of tiles; block 0's warps are not told which tiles come after the first.  The call
    reports it, every result is NaN or as ever (none keeps what y held), and the next call is as ever."""
    torch, bm = env
    g = torch.Generator().manual_seed(strips)
    E, C, P, wide = 48, 256, 24000, 256 if glu else 512   # two tiles of 256 and 244 rows of y an expert, by 256 or 512 of the matrices
    R = wide * (strips - 1) + 60
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty) if glu else (None, None, None)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)
    w, x = wrap(bm, w, ws), wrap(bm, x, xs)
    kw = dict(up=wrap(bm, up, us) if glu else None, dtype=torch.bfloat16)
    off = torch.arange(0, P + 1, P // E, dtype=torch.int32).cuda()
    ref = bm.expert_product(w, x, off, **kw)
    assert bool(torch.isfinite(ref).all())
    for with_status in (True, False):
        buf = torch.full((P, R + 8), 77.0, dtype=torch.bfloat16, device="cuda")
        y, status = buf[:, :R], torch.zeros(1, dtype=torch.int32, device="cuda")
        bm.bitsmoe_debug_wait_limit(2, 2_000_000)
        try:
            bm.expert_product(w, x, off, y=y, status=status if with_status else None, **kw)
            torch.cuda.synchronize()
        finally:
            bm.bitsmoe_debug_wait_limit(0, 0)
        assert int(status.item()) == (bm.ERR_CODE["TIMEOUT"] if with_status else 0)
        lost = torch.isnan(y)
        assert bool(lost.any()) and torch.equal(y[~lost], ref[~lost])
        # a pair has one tile of a wave: of the first it is there, of the others lost
        pairs = torch.cuda.get_device_properties(0).multi_processor_count // 2
        assert 244 * 60 <= int(lost.sum()) <= (2 * E * strips - 1) // pairs * 256 * wide
        assert (buf[:, R:] == 77).all()
        status.zero_()
        assert torch.equal(bm.expert_product(w, x, off, y=y, status=status, **kw), ref)
        assert int(status.item()) == 0


@pytest.mark.parametrize("kind", sorted(LOST) + ["waves"])
@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("glu", [False, True])
def test_expert_product_short_waits(env, kind, ty, glu):
    """Waits bounded to less than what they take, so that they run out in some warps and not in others, at any place: results
    are NaN (and the call says so) or as ever, and the next call is as ever."""
    torch, bm = env
    g = torch.Generator().manual_seed(9)
    E, R, C, P = LOST[kind][:4] if kind != "waves" else (48, 2100, 256, 24000)
    w, ws, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(E, R, C, generator=g), ty) if glu else (None, None, None)
    x, xs, _ = pitched(torch, torch.randn(P, C, generator=g), ty)
    w, x = wrap(bm, w, ws), wrap(bm, x, xs)
    kw = dict(up=wrap(bm, up, us) if glu else None)
    off = torch.arange(0, P + 1, P // E, dtype=torch.int32).cuda()
    for dt in (torch.float32, torch.bfloat16):
        ref = bm.expert_product(w, x, off, dtype=dt, **kw)
        for clocks in (1, 100, 500, 1000, 2000, 3000, 5000, 8000, 15000, 40000):
            y, status = torch.full((P, R), 77.0, dtype=dt, device="cuda"), torch.zeros(1, dtype=torch.int32, device="cuda")
            bm.bitsmoe_debug_wait_limit(0, clocks)
            try:
                bm.expert_product(w, x, off, y=y, status=status, **kw)
                torch.cuda.synchronize()
            finally:
                bm.bitsmoe_debug_wait_limit(0, 0)
            lost = torch.isnan(y)
            assert torch.equal(y[~lost], ref[~lost]), clocks
            assert int(status.item()) == bm.ERR_CODE["TIMEOUT"] or (int(status.item()) == 0 and not bool(lost.any())), clocks
            status.zero_()
            assert torch.equal(bm.expert_product(w, x, off, y=y, status=status, **kw), ref) and int(status.item()) == 0


@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
@pytest.mark.parametrize("R", [64, 250, 256, 300, 1000])
@pytest.mark.parametrize("shift", [0, 1, 8])
def test_expert_product_16_bit_results(env, ty, R, shift):
    """bf16 rows of y on 16-byte boundaries (turned on their way out) and off them: the same bits; nothing beside them is
    touched."""
    torch, bm = env
    g = torch.Generator().manual_seed(R)
    C = 320
    w, ws, _ = pitched(torch, torch.randn(4, R, C, generator=g), ty)
    up, us, _ = pitched(torch, torch.randn(4, R, C, generator=g), ty)
    x, xs, _ = pitched(torch, torch.randn(700, C, generator=g), ty)
    off = torch.tensor([1, 3, 300, 300, 698], dtype=torch.int32).cuda()
    for u_ in (None, wrap(bm, up, us)):
        other = torch.full((700, (R + 7) // 8 * 8 + (8 if shift == 1 else 1)), 7.0, dtype=torch.bfloat16, device="cuda")[:, :R]
        bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), off, up=u_, y=other)
        buf = torch.full((700, (R + 24) // 8 * 8 + (1 if shift == 1 else 0)), 7.0, dtype=torch.bfloat16, device="cuda")
        y = buf[:, shift:shift + R]
        bm.expert_product(wrap(bm, w, ws), wrap(bm, x, xs), off, up=u_, y=y)
        assert torch.equal(y, other)
        rest = buf.clone()
        rest[:, shift:shift + R] = 7.0
        assert (rest == 7).all() and (y[0] == 7).all() and (y[698:] == 7).all()


def test_expert_product_waves_of_unequal_tiles(env):
    """Many waves of tiles of all sizes: every row's result, whoever had it."""
    torch, bm = env
    rng = np.random.default_rng(11)
    counts = rng.integers(0, 900, 40)
    counts[rng.random(40) < 0.2] = 0
    E, R, C = 40, 1300, 64
    off = torch.from_numpy(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)).cuda()
    P = int(off[-1])
    w = torch.randn(E, R, C, device="cuda").to(torch.bfloat16)
    x = torch.randn(P, C, device="cuda").to(torch.bfloat16)
    for up in (None, torch.randn(E, R, C, device="cuda").to(torch.bfloat16)):
        y = bm.expert_product(w, x, off, up=up)
        half = bm.expert_product(w, x, off, up=up, dtype=torch.bfloat16).float()   # (by pairs of CTAs)
        o = off.tolist()
        for e in range(E):
            if o[e] == o[e + 1]:
                continue
            xr = x[o[e]:o[e + 1]].float()
            a = xr @ w[e].float().T
            m = xr.abs() @ w[e].float().abs().T
            if up is not None:
                b = xr @ up[e].float().T
                want = a / (1 + torch.exp(-a)) * b
                tol = (C + 16) * 2.0 ** -22 * (1.1 * m * b.abs() + a.abs() * (xr.abs() @ up[e].float().abs().T)) + 1e-5 * want.abs()
            else:
                want, tol = a, (C + 16) * 2.0 ** -22 * m
            assert ((y[o[e]:o[e + 1]] - want).abs() <= tol).all(), e
            assert ((half[o[e]:o[e + 1]] - want).abs() <= tol + 2.0 ** -8 * (want.abs() + tol)).all(), e


def test_expert_products_beside_the_forward_on_another_stream(env):
    """Kernels of one stream wait inside pairs and clusters and hold whole SMs; forwards of the tensor-core projections and
    microscaled products run on another: every result as alone."""
    import synth
    torch, bm = env
    spec = synth.scaled_spec(synth.WORKLOADS["tiny"], D=256, E=8, I=256, n=128, group=128, top_k=2)
    L = bm.bitsmoe_pack(synth.make_layer(spec, seed=5, bits_dist={0: .1, 1: .2, 2: .4, 3: .2, 4: .1}), device=0)
    xf, logits = synth.make_inputs(spec, 40, seed=5)
    xd, ld = torch.from_numpy(xf.view(np.int16)).cuda(), torch.from_numpy(logits).cuda()
    ws = bm.Workspace(L, 40, spec.top_k)
    y_ref = bm.moe_forward(L, xd, ld, spec.top_k, ws).clone()
    mw = bm.microscale_quantize(torch.randn(300, 4096, device="cuda"))
    mx = torch.randn(40, 4096, device="cuda").to(torch.bfloat16)
    m_ref = bm.microscale_product(mw, mx)
    cases = []
    for E, R, C, P in ((3, 520, 2048, 15), (40, 520, 512, 200), (6, 700, 512, 1500)):
        w = torch.randn(E, R, C, device="cuda").to(torch.bfloat16)
        x = torch.randn(P, C, device="cuda").to(torch.bfloat16)
        off = torch.arange(0, P + 1, P // E, dtype=torch.int32).cuda()
        cases.append((w, x, off, bm.expert_product(w, x, off, up=w)))
    torch.cuda.synchronize()
    st = torch.cuda.Stream()
    got, other = [], []
    for _ in range(30):
        with torch.cuda.stream(st):
            for w, x, off, ref in cases:
                got.append((bm.expert_product(w, x, off, up=w), ref))
        other.append((bm.moe_forward(L, xd, ld, spec.top_k, ws).clone(), y_ref))
        other.append((bm.microscale_product(mw, mx), m_ref))
    torch.cuda.synchronize()
    for a, b in got:
        assert torch.equal(a, b)
    for a, b in other:
        torch.testing.assert_close(a, b, rtol=1e-4, atol=1e-5)


# ---------------------------------------------------------------------------
# the weighted sum
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("T,k,D,P", [(1, 1, 1, 1), (1, 8, 2048, 8), (5, 3, 100, 20), (37, 8, 2050, 296), (70, 32, 64, 2000), (9, 2, 8200, 18),
                                     (600, 8, 256, 4800), (3, 4, 1, 0)])
@pytest.mark.parametrize("ty,out", [("bf16", "f32"), ("f32", "bf16"), ("bf16", "bf16"), ("f32", "f32")])
@pytest.mark.parametrize("base", [None, "own", "place"])
@pytest.mark.parametrize("shift", [0, 1])
def test_expert_combine(env, T, k, D, P, ty, out, base, shift):
    torch, bm = env
    g = torch.Generator().manual_seed(T + k + D + P)
    dts = {"f32": torch.float32, "bf16": torch.bfloat16}

    def rows(n, dt):
        buf = torch.randn(n, D + 9 if shift else (D + 7) // 8 * 8, generator=g).to(dts[dt]).cuda()
        return buf[:, shift:shift + D]
    y = rows(P, ty)
    places = torch.randint(-2, P + 3, (T, k), generator=g, dtype=torch.int32)
    places[0, 0] = -1
    weights = torch.rand(T, k, generator=g)
    obuf = torch.full((T, D + 9 if shift else (D + 7) // 8 * 8 + 8), 77.0, dtype=dts[out], device="cuda")
    o = obuf[:, shift:shift + D]
    b = None
    if base:
        b = rows(T, out)
        if base == "place":
            o.copy_(b)
            b = o
    bv = b.double().cpu().numpy() if base else None
    got = bm.expert_combine(y, places.cuda(), weights.cuda(), base=b, out=o)
    assert got is o
    yv, wv = y.double().cpu().numpy(), weights.double().numpy()
    want = oe.combine(yv, places.numpy(), wv, bv)
    mag = oe.combine(np.abs(yv), places.numpy(), wv, np.abs(bv) if base else None)
    tol = (k + 2) * u * mag
    tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if out == "bf16" else u * np.abs(want))
    assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()
    rest = obuf.clone()
    rest[:, shift:shift + D] = 77.0
    assert (rest == 77).all()


def test_expert_combine_of_experts_that_do_not_count(env):
    """A place outside the rows adds nothing, whatever its weight and whatever lies in the rows."""
    torch, bm = env
    y = torch.full((4, 64), float("nan"), device="cuda")
    y[2] = 3.0
    places = torch.tensor([[-1, 2, 4], [-1, -1, -1]], dtype=torch.int32).cuda()
    w = torch.tensor([[float("inf"), 2.0, float("nan")], [1.0, 1.0, 1.0]]).cuda()
    out = bm.expert_combine(y, places, w)
    assert (out[0] == 6).all() and (out[1] == 0).all()
    assert bm.expert_combine(y, places[:0], w[:0]).shape == (0, 64)
    with pytest.raises(bm.BitsMoEError):
        bm.expert_combine(y, places, w[:, :2])
    with pytest.raises(bm.BitsMoEError):
        bm.expert_combine(y, places, w, base=torch.zeros(2, 64, device="cuda", dtype=torch.bfloat16), dtype=torch.float32)


# ---------------------------------------------------------------------------
# together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("T", [1, 6, 90, 400])
def test_a_block_of_coded_experts(env, T):
    """Norm in 8 bits, routing, gate and up, SwiGLU's rows in 8 bits, down, weighted sum onto the shared branch, the next
    norm: as a decoder block runs them, against float64 on the values that each step was given."""
    torch, bm = env
    E, k, D, I = 12, 3, 192, 160
    g = torch.Generator().manual_seed(T)
    mats = {n: bm.rowscale_quantize((torch.randn(E, *s, generator=g) / s[1] ** 0.5).cuda())
            for n, s in (("gate", (I, D)), ("up", (I, D)), ("down", (D, I)))}
    router = (torch.randn(E, D, generator=g) / D ** 0.5).cuda()
    h = torch.randn(T, D, generator=g).cuda()
    gain = (1 + 0.1 * torch.randn(D, generator=g)).cuda()
    shared = torch.randn(T, D, generator=g).cuda()
    _, x = bm.block_norm(h, pre_gain=gain, x_dtype=torch.float8_e4m3fn)
    xv = bm.rowscale_dequantize(x)
    logits = xv @ router.T
    if T > 2:
        logits[-1] = float("-inf")
    r = bm.route(logits, k)
    hid = bm.expert_product(mats["gate"], x, r.offsets, index=r.pairs, fan=k, up=mats["up"], dtype=torch.bfloat16)
    n = int(r.offsets[-1])
    hid[n:] = 0
    hq = bm.rowscale_quantize(hid)
    yd = bm.expert_product(mats["down"], hq, r.offsets, dtype=torch.float32)
    out = bm.expert_combine(yd, r.places, r.weights, base=shared)
    h2, x2 = bm.block_norm(h, out, x_dtype=torch.float8_e4m3fn)
    vals = {n_: bm.rowscale_dequantize(m).double().cpu().numpy() for n_, m in mats.items()}
    off, pairs = r.offsets.cpu().numpy(), r.pairs.cpu().numpy()
    want, parts = oe.product(vals["gate"], xv.double().cpu().numpy(), off, pairs, k, vals["up"])
    got = hid.double().cpu().numpy()
    for p in range(n):
        gs, gm, us, um = parts[p]
        eg, eu = (D + 16) * 2.0 ** -23 * gm, (D + 16) * 2.0 ** -23 * um
        silu = gs / (1 + np.exp(-gs))
        tol = 1.1 * eg * (np.abs(us) + eu) + np.abs(silu) * eu + (16 + np.abs(gs)) * u * np.abs(want[p])
        assert (np.abs(got[p] - want[p]) <= tol + 2.0 ** -8 * (np.abs(want[p]) + tol)).all()
    hv = bm.rowscale_dequantize(hq).double().cpu().numpy()
    down, parts = oe.product(vals["down"], hv, off)
    got = yd.double().cpu().numpy()
    for p in range(n):
        assert (np.abs(got[p] - down[p]) <= (I + 16) * 2.0 ** -23 * parts[p][1] + 4 * u * np.abs(down[p])).all()
    wt, pl = r.weights.double().cpu().numpy(), r.places.cpu().numpy()
    sv = shared.double().cpu().numpy()
    want = oe.combine(got, pl, wt, sv)
    mag = oe.combine(np.abs(np.nan_to_num(got)), pl, wt, np.abs(sv))
    assert (np.abs(out.double().cpu().numpy() - want) <= (k + 3) * u * mag).all()
    if T > 2:
        assert torch.equal(out[-1], shared[-1])
    want_h = h.double().cpu().numpy() + out.double().cpu().numpy()
    assert (np.abs(h2.double().cpu().numpy() - want_h) <= 2 * u * (np.abs(want_h) + np.abs(h.double().cpu().numpy()))).all()
    assert torch.isfinite(bm.rowscale_dequantize(x2)).all()


def test_refusals_of_the_binding(env):
    torch, bm = env
    w = torch.randn(2, 8, 16, device="cuda").to(torch.bfloat16)
    x = torch.randn(4, 16, device="cuda").to(torch.bfloat16)
    off = torch.zeros(3, dtype=torch.int32, device="cuda")
    ok = dict(w=w, x=x, offsets=off)
    for kw in (dict(w=w.float()), dict(w=w[0]), dict(x=x[:, :8]), dict(x=x.float()), dict(offsets=off[:2]), dict(offsets=off.long()),
               dict(offsets=off.cpu()), dict(index=off.float()), dict(fan=0), dict(up=w[:, :4]), dict(up=w[:1]), dict(y=torch.zeros(4, 7, device="cuda")),
               dict(y=torch.zeros(4, 8, device="cuda", dtype=torch.float16)), dict(status=torch.zeros(2, dtype=torch.int32, device="cuda")),
               dict(w=w.transpose(1, 2)), dict(x=x.cpu())):
        with pytest.raises(bm.BitsMoEError):
            bm.expert_product(**{**ok, **kw})


FIRST = """
import sys, torch
sys.path.insert(0, sys.argv[1])
import paper_2606_00079_gb300 as bm
torch.cuda.set_device(0)
T, E, k, D, I = int(sys.argv[2]), 8, 2, 256, 192
w, up = (torch.randn(E, I, D, device="cuda").to(torch.bfloat16) for _ in range(2))
logits, h = torch.randn(T, E, device="cuda"), torch.randn(T, D, device="cuda")
dn = torch.randn(E, D, I, device="cuda")
def step():
    _, x = bm.block_norm(h, x_dtype=torch.float8_e4m3fn)
    xd = bm.rowscale_dequantize(x, torch.bfloat16)
    r = bm.route(logits, k)
    a = bm.expert_product(w, xd, r.offsets, index=r.pairs, fan=k, up=up)
    y = bm.expert_product(bm.rowscale_quantize(dn), bm.rowscale_quantize(a), r.offsets)
    return bm.expert_combine(y, r.places, r.weights, base=h)
g = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(g):
    out = step()
g.replay()
torch.cuda.synchronize()
assert torch.equal(out, step()) and bool(torch.isfinite(out).all())
print("same")
"""


@pytest.mark.parametrize("T", [3, 400])
def test_first_calls_inside_a_capture(env, T):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", FIRST, root, str(T)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]


@pytest.mark.parametrize("T,E,R", [(1, 1, 200), (40, 2, 130), (900, 3, 300), (3000, 40, 161)])   # split columns, single CTAs, pairs
@pytest.mark.parametrize("out", ["f32", "bf16"])
def test_swiglu_of_large_gates(env, T, E, R, out):
    """Sums of one product, so exact: y is SiLU's own error.  expf and a quotient of 2 units in the last place each are 4 u
    each, the sum below the quotient u, two products u each; bf16 adds half a step."""
    torch, bm = env
    C = 1024   # (columns to split; all but one of x are 0)
    g = torch.linspace(-80, 80, E * R, device="cuda").view(E, R).bfloat16()
    w, up = (torch.randn(E, R, C, device="cuda").bfloat16() for _ in range(2))
    w[:, :, 5], up[:, :, 5] = g, 1.5
    x = torch.zeros(T, C, dtype=torch.bfloat16, device="cuda")
    x[:, 5] = 1
    off = torch.linspace(0, T, E + 1, device="cuda").int()
    y = bm.expert_product(w, x, off, up=up, dtype=torch.float32 if out == "f32" else torch.bfloat16).double()
    o, gd = off.tolist(), g.double()
    want = torch.cat([(gd[e] / (1 + torch.exp(-gd[e])) * 1.5).expand(o[e + 1] - o[e], R) for e in range(E)])
    rel = 12 * u if out == "f32" else 2.0 ** -8 + 13 * u
    assert ((y - want).abs() <= rel * want.abs()).all()


# columns split; single CTAs; pairs, and of fp32 results tiles of 64 and of 128 rows of y
@pytest.mark.parametrize("E,P,R", [(1, 3, 300), (40, 300, 200), (12, 3000, 700), (3, 4000, 2700)])
@pytest.mark.parametrize("out", ["f32", "bf16"])
@pytest.mark.parametrize("glu", [False, True])
@pytest.mark.parametrize("shift", [0, 1])   # of y
def test_scales_whose_product_leaves_the_range(env, E, P, R, out, glu, shift):
    """Rows' scales from 2^-100 to 2^120, as the coder gives them, and zeros.  The codes are small whole numbers, so the sums are
    exact: a result is its sum times both scales, two roundings of fp32 (and SiLU's 12, and half a step of bf16), wherever the
    sum, the scaled sums and the result are normal numbers or zeros, whatever the scales' product alone is."""
    torch, bm = env
    g = torch.Generator().manual_seed(P + R)
    C = 288

    def coded(*shape):
        codes = torch.randint(-2, 3, (*shape, C), generator=g).float()
        codes.view(-1, C)[::7] = 0   # (sums that are zero)
        e = torch.tensor([-100.0, -75, -60, -8, 0, 3, 60, 70, 120])[torch.randint(0, 9, shape, generator=g)]
        s = (2.0 ** e.double() * (1 + torch.rand(shape, generator=g).double()) / 2).float()
        s[torch.rand(shape, generator=g) < 0.02] = 0
        return bm.Rowscale(codes.to(torch.float8_e4m3fn).cuda(), s.cuda()), codes.double(), s.double()
    w, wv, ws = coded(E, R)
    up, uv, us = coded(E, R) if glu else (None, None, None)
    x, xv, xs = coded(P)
    off = torch.linspace(0, P, E + 1).int()
    dt = torch.float32 if out == "f32" else torch.bfloat16
    y = torch.zeros(P, R + 8 - R % 8 + shift, dtype=dt, device="cuda")[:, shift:shift + R]
    bm.expert_product(w, x, off.cuda(), up=up, y=y)
    got, o, low, high = y.double().cpu(), off.tolist(), 2.0 ** -126, 2.0 ** 127
    normal = lambda v: (v == 0) | ((v.abs() >= low) & (v.abs() <= high))
    checked = 0
    for e in range(E):
        a, b = o[e], o[e + 1]
        want = (xv[a:b] @ wv[e].T) * xs[a:b, None] * ws[e]
        ok, rel = normal(want), 3 * u
        if glu:
            other = (xv[a:b] @ uv[e].T) * xs[a:b, None] * us[e]
            ok = ok & normal(other) & (want.abs() < 80)   # (SiLU of others underflows, or is the gate itself)
            silu = want / (1 + torch.exp(-want))
            ok = ok & normal(silu)
            want = silu * other
            ok, rel = ok & normal(want), (3 * 81 + 3 + 12) * u   # (|SiLU'(g) g| is at most (1 + |g|) |SiLU(g)|)
        tol = rel * want.abs() + (2.0 ** -8 * want.abs() * (1 + rel) if out == "bf16" else 0)
        d = (got[a:b] - want).abs()
        assert bool((d <= tol)[ok].all()), (e, int((~(d <= tol) & ok).sum()), int(ok.sum()))
        checked += int((ok & (want != 0)).sum())
    assert checked > P


@pytest.mark.parametrize("E,P", [(1, 3), (5, 300), (4, 2000)])   # columns split, and whole
@pytest.mark.parametrize("ty", ["bf16", "e4m3"])
def test_fp32_results_of_many_columns(env, E, P, ty):
    """Sums of products of one sign, where cutting off adds up.  Registers add what accumulators of at most 8 additions (bf16; 32)
    hold: of 8 (32) additions that lose less than 2^-23 of the sum so far each, their n sums u each, and the clusters' 8; the
    scales' products, and the decoded values' roundings in fp32, 5."""
    torch, bm = env
    g = torch.Generator().manual_seed(E)
    C, R = 8192, 300
    w, ws, _ = pitched(torch, torch.rand(E, R, C, generator=g) + 0.1, ty)
    x, xs, _ = pitched(torch, torch.rand(P, C, generator=g) + 0.1, ty)
    off = torch.linspace(0, P, E + 1).int().cuda()
    w, x = wrap(bm, w, ws), wrap(bm, x, xs)
    y = bm.expert_product(w, x, off, dtype=torch.float32).double()
    wd = w.double() if ty == "bf16" else bm.rowscale_dequantize(w).double()
    xd = x.double() if ty == "bf16" else bm.rowscale_dequantize(x).double()
    o = off.tolist()
    want = torch.cat([xd[o[e]:o[e + 1]] @ wd[e].T for e in range(E)])
    chains, adds = (64, 8) if ty == "bf16" else (8, 32)
    assert ((y - want).abs() <= (2 * adds + chains + 8 + 5) * u * want).all()
