"""GPU parity of block_norm against the fp64 oracle, and the run of it with the routed experts and a
microscaled shared expert, as a decoder block uses them.

Tolerance, by arithmetic (u = 2^-24, half a step of fp32): a mean of D squares is off by at most D + 2
roundings of itself, its inverse root by half of that and 4 more; a branch value by that and 8 roundings of
factors and the sigmoid: eb = ((D + 2) / 2 + 12) u |branch|; h' = a h + branch by eb + 2 u (|a h| + |branch|).
x = h' r g: |g r| eh + ((D + 2) / 2 + 8) u |x| and the effect of eh on r, at most |x| ||eh|| / ||h'||.
A bf16 output adds half a step, 2^-8.
"""
import numpy as np
import pytest

from oracle import microscale as om

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


def typed(torch, a, ty):
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.float32 if ty == "f32" else torch.bfloat16)


def check(got, want, tol, ty, name):
    tol = tol + (2.0 ** -8 * (np.abs(want) + tol) if ty == "bf16" else 0) + 1e-37
    d = np.abs(got.double().cpu().numpy() - want)
    assert (d <= tol).all(), (name, np.argwhere(~(d <= tol))[:4].tolist(), float(np.nanmax(d / tol)))


def run_case(env, T, D, h="f32", y="f32", gains="bf16", x="bf16", post=True, gate="none", sigmoid=False, channel=False,
             offset=0.0, a=1.0, b=1.0, eps=1e-6, seed=0, pre=True, amp=1.0):
    torch, bm = env
    rng = np.random.default_rng([T, D, seed])
    dev = {}
    dev["h"] = typed(torch, amp * 3 * rng.standard_normal((T, D)), h)
    dev["y"] = typed(torch, amp * rng.standard_normal((T, D)) * np.exp(rng.uniform(-3, 3, (T, 1))), y)
    if T > 2:
        dev["y"][1] = 0.0
        dev["h"][2] = 0.0
        dev["y"][2] = 0.0
    for n in ("post", "pre", "channel"):
        dev[n] = typed(torch, (0 if offset else 1) + 0.3 * rng.standard_normal(D), gains)
    dev["gate"] = {"none": None, "token": typed(torch, rng.standard_normal(T) * 2, y),
                   "element": typed(torch, rng.standard_normal((T, D)), y)}[gate]
    kw = dict(post_norm=post, post_gain=dev["post"].cuda() if post else None, post_eps=eps,
              gate=dev["gate"].cuda() if gate != "none" else None, gate_sigmoid=sigmoid,
              channel_scale=dev["channel"].cuda() if channel else None, branch_scale=b, residual_scale=a,
              pre_gain=dev["pre"].cuda() if pre else None, pre_eps=eps, gain_offset=offset,
              x_dtype=torch.float32 if x == "f32" else torch.bfloat16)
    hn, xn = bm.block_norm(dev["h"].cuda(), dev["y"].cuda(), **kw)
    f = {k: v.double().numpy() for k, v in dev.items() if v is not None}
    g = f.get("gate")
    if g is not None:
        g = 1 / (1 + np.exp(-g)) if sigmoid else g
        g = g[:, None] if gate == "token" else g
    a, b, eps = (float(np.float32(v)) for v in (a, b, eps))
    wh, br, wx = om.block_norm(f["h"], f["y"], offset + f["post"] if post else None, g, f["channel"] if channel else None,
                               b, a, offset + f["pre"] if pre else None, eps, eps)
    eb = ((D + 2) / 2 + 12) * u * np.abs(br)
    eh = eb + 2 * u * (np.abs(a * f["h"]) + np.abs(br))
    check(hn, wh, eh, h, "h")
    r = 1 / np.sqrt((wh * wh).mean(axis=1, keepdims=True) + eps)
    nh = np.linalg.norm(wh, axis=1, keepdims=True)
    rel = np.where(nh > 0, np.linalg.norm(eh, axis=1, keepdims=True) / np.where(nh > 0, nh, 1), 0)
    gp = np.abs(offset + f["pre"]) if pre else 1.0
    check(xn, wx, gp * r * eh + (((D + 2) / 2 + 8) * u + rel) * np.abs(wx), x, "x")


WIDTHS = [1, 2, 7, 8, 31, 64, 100, 256, 257, 1000, 1024, 2048, 2050, 4096, 4104, 5120, 8192, 8200, 12288, 16384, 20001, 32768]


@pytest.mark.parametrize("D", WIDTHS)
def test_widths(env, D):
    run_case(env, 5, D)
    run_case(env, 1, D, h="bf16", y="bf16", post=False, gate="element", channel=True, seed=1)


@pytest.mark.parametrize("T", [1, 2, 3, 17, 151, 153, 1000, 5000])
def test_rows(env, T):
    run_case(env, T, 256, gate="token", sigmoid=True)
    run_case(env, T, 520, h="bf16", channel=True, a=0.5, b=-2.0)


@pytest.mark.parametrize("T,D", [(700, 5001), (400, 8191), (5000, 515), (2500, 1030), (1300, 4095), (20000, 259)])
def test_many_rows_off_boundaries(env, T, D):
    """Several rows a block, whose ends share 16 bytes with their neighbours'; in place, and the same rows alone."""
    torch, bm = env
    run_case(env, T, D, channel=True)
    run_case(env, T, D, h="bf16", y="f32", gate="element", sigmoid=True, seed=1)
    run_case(env, T, D, h="bf16", y="bf16", gains="bf16", x="f32", post=False, gate="token", seed=2)
    g = torch.Generator().manual_seed(D)
    h, y = torch.randn(T, D, generator=g).cuda(), torch.randn(T, D, generator=g).bfloat16().cuda()
    ho, x = bm.block_norm(h, y, post_norm=True)
    for i in (0, 1, T - 1):
        ah, ax = bm.block_norm(h[i:i + 1], y[i:i + 1], post_norm=True)
        assert torch.equal(ho[i:i + 1], ah) and torch.equal(x[i:i + 1], ax)
    _, x2 = bm.block_norm(h, y, post_norm=True, h_out=h)
    assert torch.equal(h, ho) and torch.equal(x2, x)


@pytest.mark.parametrize("h", ["f32", "bf16"])
@pytest.mark.parametrize("y", ["f32", "bf16"])
@pytest.mark.parametrize("gains", ["f32", "bf16"])
@pytest.mark.parametrize("x", ["f32", "bf16"])
def test_types(env, h, y, gains, x):
    for D in (512, 515):
        run_case(env, 4, D, h, y, gains, x, gate="element", sigmoid=True, channel=True, offset=1.0)


@pytest.mark.parametrize("post", [False, True])
@pytest.mark.parametrize("gate,sigmoid", [("none", False), ("token", False), ("token", True), ("element", False), ("element", True)])
@pytest.mark.parametrize("channel", [False, True])
@pytest.mark.parametrize("D", [384, 386])
def test_options(env, post, gate, sigmoid, channel, D):
    run_case(env, 6, D, post=post, gate=gate, sigmoid=sigmoid, channel=channel, a=0.7, b=1.3, pre=channel)


def test_magnitudes(env):
    """Rows whose squares pass fp32's range would be infinite in any order; rows near it are not.  Tiny rows
    live on the epsilon."""
    run_case(env, 4, 256, amp=1e15, eps=1e-6)
    run_case(env, 4, 256, amp=1e-12, eps=1e-6)
    run_case(env, 4, 256, amp=1e-12, eps=1e-20)


def test_parts(env):
    """Pre-norm alone, post-norm and residual alone, in place, and y None with a residual scale."""
    torch, bm = env
    g = torch.Generator().manual_seed(0)
    for D in (768, 771):
        h = torch.randn(9, D, generator=g).cuda()
        y = torch.randn(9, D, generator=g).cuda()
        w = torch.rand(D, generator=g).cuda()
        none, x = bm.block_norm(h, pre_gain=w)
        assert none is None
        _, br, want = om.block_norm(h.double().cpu().numpy(), pre=w.double().cpu().numpy())
        check(x, want, (D / 2 + 12) * u * np.abs(want), "bf16", "x")
        both, x = bm.block_norm(h, y, post_norm=True, pre_gain=w)
        alone, nox = bm.block_norm(h, y, post_norm=True, pre_norm=False)
        assert nox is None and torch.equal(alone, both)
        keep = h.clone()
        out, x2 = bm.block_norm(h, y, post_norm=True, pre_gain=w, h_out=h)
        assert out is h and torch.equal(h, both) and torch.equal(x2, x)
        o = torch.empty_like(keep)
        bm.block_norm(keep, residual_scale=0.25, h_out=o, pre_norm=False)
        assert torch.equal(o, 0.25 * keep)


def test_strides_and_alignment(env):
    """Every operand on a pitch of its own, on and off 16-byte boundaries; nothing outside the rows is written."""
    torch, bm = env
    g = torch.Generator().manual_seed(2)
    T, D = 7, 512
    mk = lambda dt: torch.randn(T, D, generator=g).to(dt).cuda()  # noqa: E731
    h, y, e = mk(torch.float32), mk(torch.bfloat16), mk(torch.bfloat16)
    gains = torch.rand(3, D, generator=g).cuda()
    ref_h, ref_x = bm.block_norm(h, y, post_norm=True, post_gain=gains[0], gate=e, channel_scale=gains[1], pre_gain=gains[2])

    def placed(src, ld, off):
        buf = torch.full((T * ld + off + 3,), 7.0, dtype=src.dtype, device="cuda")
        v = buf[off:off + T * ld].view(T, ld)[:, :D]
        v.copy_(src)
        return buf, v

    for ld, off in ((512, 0), (528, 8), (513, 0), (520, 1), (600, 3)):
        _, hv = placed(h, ld, off)
        _, yv = placed(y, ld + 8, off)
        _, ev = placed(e, ld + 16, off)
        ob, ov = placed(torch.zeros_like(h), ld + 24, off)
        xb, xv = placed(torch.zeros_like(ref_x), ld + 32, off)
        vec = [torch.cat([torch.zeros(off, device="cuda"), v])[off:] for v in gains]
        bm.block_norm(hv, yv, post_norm=True, post_gain=vec[0], gate=ev, channel_scale=vec[1], pre_gain=vec[2], h_out=ov, x=xv)
        # another order of the sums where the rows are read otherwise: one more rounding of each partial sum
        torch.testing.assert_close(ov, ref_h, rtol=1e-5, atol=1e-6)
        torch.testing.assert_close(xv.float(), ref_x.float(), rtol=2.0 ** -7, atol=1e-6)
        for buf, p in ((ob, ld + 24), (xb, ld + 32)):
            rest = torch.ones_like(buf, dtype=torch.bool)
            rest[off:off + T * p].view(T, p)[:, :D] = False
            assert (buf[rest] == 7).all()
    # a gate per token with a stride
    gt = torch.randn(T, 3, generator=g).cuda()
    a = bm.block_norm(h, y, gate=gt[:, 1], gate_sigmoid=True)
    b = bm.block_norm(h, y, gate=gt[:, 1].contiguous(), gate_sigmoid=True)
    assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_no_rows(env):
    torch, bm = env
    h, y = torch.zeros(0, 96, device="cuda"), torch.zeros(0, 96, device="cuda")
    w = torch.ones(96, device="cuda")
    ho, x = bm.block_norm(h, y, post_norm=True, post_gain=w, pre_gain=w, gate=torch.zeros(0, device="cuda"))
    assert ho.shape == x.shape == (0, 96)


def test_non_finite_rows_stay_apart(env):
    torch, bm = env
    g = torch.Generator().manual_seed(3)
    for D in (256, 259):
        h, y = torch.randn(8, D, generator=g).cuda(), torch.randn(8, D, generator=g).cuda()
        ref = bm.block_norm(h, y, post_norm=True)
        y[3, 5] = float("nan")
        y[5, 0] = float("inf")
        got = bm.block_norm(h, y, post_norm=True)
        keep = [0, 1, 2, 4, 6, 7]
        assert torch.equal(got[0][keep], ref[0][keep]) and torch.equal(got[1][keep], ref[1][keep])
        assert torch.isnan(got[0][3]).all() and torch.isnan(got[1][3]).all()


def test_rows_past_32_bits(env):
    """More than 2^31 elements: the last rows equal the same rows alone."""
    torch, bm = env
    T, D = 140000, 16384
    h = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    y = torch.zeros(T, D, dtype=torch.bfloat16, device="cuda")
    h[-2:], y[-2:] = torch.randn(2, D, device="cuda").bfloat16(), torch.randn(2, D, device="cuda").bfloat16()
    ho, x = bm.block_norm(h, y, post_norm=True, h_out=h.clone())
    ah, ax = bm.block_norm(h[-2:], y[-2:], post_norm=True)
    assert torch.equal(ho[-2:], ah) and torch.equal(x[-2:], ax)
    assert int(torch.count_nonzero(x[:-2])) == 0


def test_streams_and_graph(env):
    torch, bm = env
    g = torch.Generator().manual_seed(4)
    h, y = torch.randn(33, 1024, generator=g).cuda(), torch.randn(33, 1024, generator=g).cuda()
    ref = bm.block_norm(h, y, post_norm=True)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bm.block_norm(h, y, post_norm=True, stream=s)
    s.synchronize()
    assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    hs, ho, x = h.clone(), torch.empty_like(h), torch.empty(33, 1024, dtype=torch.bfloat16, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bm.block_norm(hs, y, post_norm=True, h_out=ho, x=x)
    for k in (1.0, 2.0):
        hs.copy_(k * h)
        graph.replay()
        torch.cuda.synchronize()
        want = bm.block_norm(k * h, y, post_norm=True)
        assert torch.equal(ho, want[0]) and torch.equal(x, want[1])


@pytest.mark.parametrize("T", [1, 13])
@pytest.mark.parametrize("act", ["bf16", "coded"])
def test_a_block_with_routed_experts_and_a_shared_expert(env, T, act):
    """pre-norm -> routed experts + sigmoid-gated microscaled shared expert -> post-norm, residual, next
    pre-norm, against the same in fp64 from the values that each step read.  The routed part has the
    forward's tolerance (2e-3 of the largest value)."""
    import oracle
    import synth
    torch, bm = env
    spec = synth.scaled_spec(synth.WORKLOADS["tiny"], D=256, E=8, I=256, n=128, group=64, top_k=2)
    layer = synth.make_layer(spec, seed=8)
    L = bm.bitsmoe_pack(layer, device=0)
    rng = np.random.default_rng(8)
    D, I = spec.D, 320
    W = [torch.from_numpy((rng.standard_normal(s) / np.sqrt(s[1])).astype(np.float32)).cuda() for s in ((I, D), (I, D), (D, I))]
    gate_w, up_w, down_w = (bm.microscale_quantize(w, "e4m3", 2.0 ** -8) for w in W)
    h = torch.from_numpy((3 * rng.standard_normal((T, D))).astype(np.float32)).cuda()
    gain = [torch.from_numpy((1 + 0.1 * rng.standard_normal(D)).astype(np.float32)).cuda() for _ in range(3)]
    logits = torch.from_numpy(rng.standard_normal((T, spec.E)).astype(np.float32)).cuda()
    sg = torch.from_numpy(rng.standard_normal(T).astype(np.float32)).cuda()
    _, x = bm.block_norm(h, pre_gain=gain[0])
    routed = bm.moe_forward(L, x, logits, spec.top_k)
    xin = bm.microscale_quantize(x, "e4m3", 2.0 ** -6) if act == "coded" else x
    mid = bm.microscale_product(gate_w, xin, up=up_w, dtype=torch.bfloat16)
    min_ = bm.microscale_quantize(mid, "e4m3", 2.0 ** -6) if act == "coded" else mid
    shared = bm.microscale_product(down_w, min_)
    h1, _ = bm.block_norm(h, shared, gate=sg, gate_sigmoid=True, pre_norm=False)
    h2, xn = bm.block_norm(h1, routed, post_norm=True, post_gain=gain[1], pre_gain=gain[2])
    torch.cuda.synchronize()
    f = lambda t: t.double().cpu().numpy()  # noqa: E731
    xv = f(bm.microscale_dequantize(xin)) if act == "coded" else f(x)
    mv = f(bm.microscale_dequantize(min_)) if act == "coded" else f(mid)
    wg, wu, wd = (f(bm.microscale_dequantize(m)) for m in (gate_w, up_w, down_w))
    g_, ag, u_, au = om.product(wg, xv, wu)
    want_mid = om.silu(g_) * u_
    eg, eu = (D + 4) * 2 * u * ag, (D + 4) * 2 * u * au
    e = 1.1 * eg * np.abs(u_) + np.abs(om.silu(g_)) * eu + 1.1 * eg * eu + 32 * u * np.abs(want_mid)
    check(mid, want_mid, e, "bf16", "mid")
    want_sh, mag = om.product(wd, mv)
    check(shared, want_sh, (I + 4) * 2 * u * mag, "f32", "shared")
    ref = oracle.moe_forward_factored(layer, x.view(torch.int16).cpu().numpy().view(np.uint16), f(logits).astype(np.float32), spec.top_k)
    assert np.max(np.abs(f(routed) - ref)) <= 2e-3 * np.max(np.abs(ref))
    w1, _, _ = om.block_norm(f(h), f(shared), gate=1 / (1 + np.exp(-f(sg)))[:, None])
    check(h1, w1, 16 * u * (np.abs(f(h)) + np.abs(f(shared))), "f32", "h1")
    w2, br, wx = om.block_norm(f(h1), f(routed), f(gain[1]), pre=f(gain[2]))
    eh = (D / 2 + 13) * u * np.abs(br) + 2 * u * (np.abs(f(h1)) + np.abs(br))
    check(h2, w2, eh, "f32", "h2")
    r = 1 / np.sqrt((w2 * w2).mean(axis=1, keepdims=True) + 1e-6)
    rel = np.linalg.norm(eh, axis=1, keepdims=True) / np.linalg.norm(w2, axis=1, keepdims=True)
    check(xn, wx, np.abs(f(gain[2])) * r * eh + ((D / 2 + 9) * u + rel) * np.abs(wx), "bf16", "x")


@pytest.mark.parametrize("T,D", [(2600, 512), (700, 2048), (500, 4096), (300, 4104), (300, 8192), (200, 12288), (200, 16384)])
def test_many_rows_on_boundaries(env, T, D):
    """More rows than run at once: they come through the ring of the 8-wide kernel.  The formula, with the gate per
    element and per token, in place, and the same rows alone (one block a row, in registers) to the bit."""
    torch, bm = env
    run_case(env, T, D, gate="element", sigmoid=True, channel=True)
    run_case(env, T, D, h="bf16", y="f32", gate="element", seed=1)
    run_case(env, T, D, h="bf16", y="bf16", x="f32", post=False, gate="token", sigmoid=True, seed=2)
    g = torch.Generator().manual_seed(D)
    h, y = torch.randn(T, D, generator=g).cuda(), torch.randn(T, D, generator=g).bfloat16().cuda()
    e, w = torch.randn(T, D, generator=g).bfloat16().cuda(), torch.rand(D, generator=g).cuda()
    f = lambda a, b, c, **kw: bm.block_norm(a, b, post_norm=True, post_gain=w, gate=c, gate_sigmoid=True, pre_gain=w, **kw)  # noqa: E731
    ho, x = f(h, y, e)
    for i in (0, 1, T // 2, T - 1):
        ah, ax = f(h[i:i + 1], y[i:i + 1], e[i:i + 1])
        assert torch.equal(ho[i:i + 1], ah) and torch.equal(x[i:i + 1], ax)
    _, x2 = f(h, y, e, h_out=h)
    assert torch.equal(h, ho) and torch.equal(x2, x)


@pytest.mark.parametrize("D", [96, 512, 4096])
def test_an_aligned_row_of_an_odd_pitch_alone(env, D):
    """One row has no pitch and is read eight elements at a time; in its batch it is not.  The sums take different orders,
    both near the formula."""
    torch, bm = env
    g = torch.Generator().manual_seed(D)
    buf = torch.randn(9 * (D + 1), generator=g).cuda()
    h = buf.view(9, D + 1)[:, :D]
    w = torch.rand(D, generator=g).cuda()
    _, _, want = om.block_norm(h.double().cpu().numpy(), pre=w.double().cpu().numpy())
    _, many = bm.block_norm(h, pre_gain=w, x_dtype=torch.float32)
    _, one = bm.block_norm(h[8:], pre_gain=w, x_dtype=torch.float32)   # (it starts on a 16-byte boundary)
    check(many, want, (D / 2 + 12) * u * np.abs(want), "f32", "many")
    check(one, want[8:], (D / 2 + 12) * u * np.abs(want[8:]), "f32", "one")
