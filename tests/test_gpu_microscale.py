"""GPU parity of the microscaled 4-bit quantiser, its inverse and the product (through the C ABI) against
the oracle (oracle/microscale.py, fp64).

The quantiser is bit-exact.  Product tolerance, by arithmetic: the products of two codes or of a code with a
bf16 value are exact in fp32, a sum of K of them in any order is off by at most (K - 1) roundings, each at
most a step (2^-23, truncation counted) of the sum of magnitudes, and the tensor scale, its application and
a split of the sum add 4 more: (K + 4) 2^-23 sum |w x|.  A bf16 result adds half a step, 2^-8 |y|.  For
silu(g) u: |silu'| <= 1.1, so 1.1 eg |u| + |silu(g)| eu + 1.1 eg eu, and 16 roundings (exp, sum, quotient and
product) of 2^-23 |y|.
"""
import numpy as np
import pytest

from oracle import microscale as om

pytestmark = pytest.mark.gpu
U = 2.0 ** -23


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


def bf16(a):
    import torch
    return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(torch.bfloat16)


def check_quantized(q, x, fmt, scale):
    codes, byte = om.quantize(x, fmt, scale)
    rows = x.shape[0]
    np.testing.assert_array_equal(q.scales.cpu().numpy(), om.tile_scales(byte))
    np.testing.assert_array_equal(q.codes.cpu().numpy().reshape(rows, -1), om.pack_codes(codes))
    return om.values(codes, byte, fmt, scale)


SHAPES = [(1, 1), (1, 31), (3, 33), (2, 16), (5, 1001), (33, 130), (129, 64), (257, 512), (130, 2048), (300, 2050)]


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("dt", ["f32", "bf16"])
@pytest.mark.parametrize("shape", SHAPES)
def test_quantizer_is_bit_exact(env, fmt, dt, shape):
    torch, bm = env
    rng = np.random.default_rng([*shape, len(fmt), len(dt)])
    x = rng.standard_normal(shape) * np.exp(rng.uniform(-12, 4, (shape[0], 1)))
    x[:, 0::7] *= 20
    x[shape[0] // 2] = 0.0
    t = torch.from_numpy(x.astype(np.float32))
    if dt == "bf16":
        t = t.to(torch.bfloat16)
    scale = 1.0 if fmt == "e8m0" else 2.0 ** -6
    q = bm.microscale_quantize(t.cuda(), fmt, scale)
    v = check_quantized(q, t.float().numpy(), fmt, scale)
    for out in (torch.float32, torch.bfloat16):
        got = bm.microscale_dequantize(q, out).cpu()
        assert torch.equal(got, torch.from_numpy(v).to(out))


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_quantizer_at_the_borders(env, fmt):
    """Ties between codes and between scales with their fp32 neighbours, powers of two and their neighbours,
    subnormals, the largest values, both zeros."""
    torch, bm = env
    blk = om.BLOCK[fmt]
    rng = np.random.default_rng(11)
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.0], np.float32)
    around = np.concatenate([mids, np.nextafter(mids, np.float32(0)), np.nextafter(mids, np.float32(9))])
    rows = []
    if fmt == "e8m0":
        tops = np.float32(2.0) ** np.array([-140, -127, -126, -125, -60, -3, 0, 1, 60, 125, 126], np.float32)
        tops = np.concatenate([tops, np.nextafter(tops, np.float32(0)), tops * np.float32(1.5),
                               [np.float32(3.4e38), np.float32(2e-45)]])
        for top in tops:
            x = (2.0 ** np.floor(np.log2(np.float64(top))) / 4) * rng.choice(around, 2 * blk).astype(np.float64)
            x = np.where(np.abs(x) > top, top, x).astype(np.float32)
            x[0], x[blk], x[3], x[5] = top, -top, 0.0, -0.0
            rows.append(x * rng.choice([-1, 1], 2 * blk).astype(np.float32))
    else:
        s = om.E4M3[:127].astype(np.float64)
        tops = np.concatenate([6 * s, 3 * (s[1:] + s[:-1])]).astype(np.float32)   # scales and their midpoints
        tops = np.concatenate([tops, np.nextafter(tops, np.float32(0)), np.nextafter(tops, np.float32(1e9)),
                               np.float32([1e4, 1e-6, 1e-30, 3e38])])
        for top in tops:
            sc = om.E4M3[om.nearest_even(np.minimum(np.float64(top) / 6, 448.0), om.E4M3[:127])]
            m = rng.choice(mids[:7], 2 * blk) * sc                                # exact in fp32: 7 bits
            x = m.astype(np.float32)
            j = rng.integers(0, 3, 2 * blk)
            x = np.where(j == 1, np.nextafter(x, np.float32(0)), np.where(j == 2, np.nextafter(x, np.float32(1e9)), x))
            x = np.minimum(x, top)
            x[0], x[blk] = top, top
            x = (x * rng.choice([-1, 1], 2 * blk)).astype(np.float32)
            rows.append(x)
    x = np.stack(rows)
    for scale in (1.0, 2.0 ** -40, 2.0 ** 3):
        with np.errstate(over="ignore"):
            xs = (x * np.float32(scale)).astype(np.float32)
        q = bm.microscale_quantize(torch.from_numpy(xs).cuda(), fmt, scale)
        if scale == 1.0:
            check_quantized(q, xs, fmt, scale)
            xb = bf16(xs)
            check_quantized(bm.microscale_quantize(xb.cuda(), fmt, 1.0), xb.float().numpy(), fmt, 1.0)
        else:
            # v = x / scale in fp32: what the definition quantises (x may have lost bits, the quotient may too)
            with np.errstate(over="ignore", under="ignore"):
                check_quantized(q, (xs / np.float32(scale)).astype(np.float32), fmt, 1.0)


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_quantizer_blocks_without_a_scale(env, fmt):
    """A NaN or an infinity makes its own block NaN and no other; the product passes it on to that row only."""
    torch, bm = env
    rng = np.random.default_rng(5)
    x = rng.standard_normal((6, 70)).astype(np.float32)
    x[1, 40] = np.nan
    x[2, 3] = np.inf
    x[3, 69] = -np.inf
    q = bm.microscale_quantize(torch.from_numpy(x).cuda(), fmt, 1.0)
    v = check_quantized(q, x, fmt, 1.0)
    got = bm.microscale_dequantize(q).cpu().numpy()
    np.testing.assert_array_equal(got, v.astype(np.float32))
    assert np.isnan(got[1]).sum() in (16, 32) and np.isnan(got).any(axis=1).tolist() == [False, True, True, True, False, False]
    act = bf16(rng.standard_normal((3, 70)))
    y = bm.microscale_product(q, act.cuda()).cpu().numpy()
    assert np.isnan(y).any(axis=0).tolist() == [False, True, True, True, False, False]
    aq = bm.microscale_quantize(act.cuda(), fmt, 1.0)
    y = bm.microscale_product(q, aq).cpu().numpy()
    assert np.isnan(y).any(axis=0).tolist() == [False, True, True, True, False, False]
    assert np.isnan(y).all(axis=0).tolist() == [False, True, True, True, False, False]


@pytest.mark.parametrize("ty", ["f32", "bf16"])
def test_quantizer_strides_and_alignment(env, ty):
    """Rows apart and on odd addresses; what lies between the rows is neither read into a block nor written."""
    torch, bm = env
    dt = torch.float32 if ty == "f32" else torch.bfloat16
    g = torch.Generator().manual_seed(1)
    for ld, off, cols in ((72, 0, 64), (67, 1, 64), (133, 3, 130), (1040, 8, 1024)):
        base = torch.randn(9 * ld + off, generator=g).to(dt)
        x = base[off:off + 9 * ld].view(9, ld)[:, :cols]
        dev = base.cuda()[off:off + 9 * ld].view(9, ld)[:, :cols]
        q = bm.microscale_quantize(dev, "e4m3", 1.0)
        check_quantized(q, x.float().numpy(), "e4m3", 1.0)
        out = torch.full((9 * ld + off,), 7.0, dtype=dt, device="cuda")
        view = out[off:off + 9 * ld].view(9, ld)[:, :cols]
        bm.microscale_dequantize(q, out=view)
        assert torch.equal(view, bm.microscale_dequantize(q, dt))
        rest = torch.ones_like(out, dtype=torch.bool)
        rest[off:off + 9 * ld].view(9, ld)[:, :cols] = False
        assert (out[rest] == 7).all()


def test_quantizer_offsets_past_32_bits(env):
    """More than 2^32 elements and 2^31 code bytes: the last rows equal the same rows quantised alone."""
    torch, bm = env
    rows, cols = 70000, 65536
    x = torch.zeros(rows, cols, dtype=torch.bfloat16, device="cuda")
    x[-3:] = torch.randn(3, cols, device="cuda").to(torch.bfloat16)
    q = bm.microscale_quantize(x, "e8m0")
    alone = bm.microscale_quantize(x[-3:], "e8m0")
    assert torch.equal(q.codes.view(rows, -1)[-3:], alone.codes.view(3, -1))
    assert torch.equal(q.block_scales()[-3:], alone.block_scales())
    assert int(q.codes.view(rows, -1)[:-3].max()) == 0
    act = torch.randn(1, cols, device="cuda").to(torch.bfloat16)
    y = bm.microscale_product(q, act)
    # the two calls may split their sums differently: each is within (K + 4) 2^-23 sum |w x| of the exact sum
    mag = act.double().abs() @ bm.microscale_dequantize(alone).double().abs().t()
    assert ((y[:, -3:] - bm.microscale_product(alone, act)).abs() <= 2 * (cols + 4) * U * mag).all()
    assert int(torch.count_nonzero(y[:, :-3])) == 0


def make(rng, rows, cols, fmt, scale=None):
    """A random matrix of any codes and varied block scales: (Microscale arrays, fp64 values)."""
    codes = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
    nb = -(-cols // om.BLOCK[fmt])
    byte = rng.integers(110, 130, (rows, nb)) if fmt == "e8m0" else rng.integers(1, 100, (rows, nb))
    scale = scale or float(np.float32(0.37))
    return codes, byte.astype(np.uint8), scale, om.values(codes, byte, fmt, float(np.float32(scale)))


def upload(env, m, fmt):
    torch, bm = env
    codes, byte, scale, _ = m
    p = np.pad(codes, ((0, 0), (0, codes.shape[1] % 2)))
    return bm.Microscale.from_rows(torch.from_numpy(p[:, 0::2] | (p[:, 1::2] << 4)).cuda(),
                                   torch.from_numpy(byte).cuda(), codes.shape[1], fmt, scale)


def check_product(env, T, rows, cols, fmt, coded, glu, out, seed=0):
    torch, bm = env
    rng = np.random.default_rng([seed, T, rows, cols])
    w = make(rng, rows, cols, fmt)
    u = make(rng, rows, cols, fmt, 0.01) if glu else None
    if coded:
        a = make(rng, T, cols, fmt, 0.5)
        x, xv = upload(env, a, fmt), a[3]
    else:
        t = bf16(rng.standard_normal((T, cols)) * np.exp(rng.uniform(-3, 3, (T, 1))))
        x, xv = t.cuda(), t.double().numpy()
    dt = torch.float32 if out == "f32" else torch.bfloat16
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = bm.microscale_product(upload(env, w, fmt), x, up=upload(env, u, fmt) if glu else None, dtype=dt, status=status)
    got = y.double().cpu().numpy()
    assert int(status.item()) == 0
    r = om.product(w[3], xv, u[3] if glu else None)
    e = (cols + 4) * U * r[1]
    want = r[0]
    if glu:
        eu = (cols + 4) * U * r[3]
        want = om.silu(r[0]) * r[2]
        e = 1.1 * e * np.abs(r[2]) + np.abs(om.silu(r[0])) * eu + 1.1 * e * eu + 16 * U * np.abs(want)
    tol = e + (2.0 ** -8 * (np.abs(want) + e) if out == "bf16" else 0) + 1e-37
    bad = ~(np.abs(got - want) <= tol)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), int(bad.sum()), float((np.abs(got - want) / tol).max()))


PRODUCTS = [   # T, rows, cols
    (1, 1, 1), (1, 128, 64), (2, 3, 31), (1, 130, 33), (3, 127, 129), (5, 256, 256), (8, 129, 500), (16, 200, 1001),
    (17, 384, 2048), (31, 150, 300), (33, 65, 255), (64, 300, 320), (100, 257, 640), (128, 128, 512), (129, 140, 257), (255, 128, 96),
    (256, 256, 1024), (257, 130, 130), (300, 512, 768), (520, 1000, 200),
]


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("x", ["bf16", "coded"])
@pytest.mark.parametrize("shape", PRODUCTS)
def test_product(env, fmt, x, shape):
    check_product(env, *shape, fmt, x == "coded", False, "f32")


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("x", ["bf16", "coded"])
@pytest.mark.parametrize("shape", PRODUCTS[::2])
def test_product_swiglu(env, fmt, x, shape):
    check_product(env, *shape, fmt, x == "coded", True, "bf16")
    check_product(env, *shape, fmt, x == "coded", True, "f32", seed=1)


@pytest.mark.parametrize("x", ["bf16", "coded"])
@pytest.mark.parametrize("T,rows,cols", [(1, 4096, 14336), (7, 2048, 8192), (24, 6000, 2048), (16, 21000, 1536), (40, 1536, 4096), (700, 640, 4096)])
def test_product_large(env, x, T, rows, cols):
    check_product(env, T, rows, cols, "e4m3", x == "coded", False, "f32")
    check_product(env, T, rows, cols, "e8m0", x == "coded", False, "bf16")


@pytest.mark.parametrize("x", ["bf16", "coded"])
@pytest.mark.parametrize("T,rows,cols", [(600, 4900, 1300), (513, 5003, 777), (290, 9900, 600), (300, 12900, 700), (90, 20400, 330),
                                         (20, 20400, 1090), (5, 20400, 2300)])
def test_product_many_tiles(env, x, T, rows, cols):
    """More tiles than SMs or half as many (no split of the columns), odd numbers of row and token tiles, several
    stages."""
    check_product(env, T, rows, cols, "e4m3", x == "coded", False, "f32")
    check_product(env, T, rows, cols, "e8m0", x == "coded", False, "bf16")
    check_product(env, T, rows, cols, "e8m0", x == "coded", True, "f32")
    check_product(env, T, rows, cols, "e4m3", x == "coded", True, "bf16")


@pytest.mark.parametrize("coded", [False, True])
@pytest.mark.parametrize("T", [1, 9, 140])
def test_product_strides(env, coded, T):
    """x rows apart and off 16-byte boundaries, y rows apart and off them: the same values as dense ones, and
    what lies between and behind y's rows stays."""
    torch, bm = env
    rng = np.random.default_rng(T)
    rows, cols = 150, 264
    w = upload(env, make(rng, rows, cols, "e4m3"), "e4m3")
    x = bf16(rng.standard_normal((T, cols))).cuda()
    xq = bm.microscale_quantize(x, "e4m3", 1.0)
    ref = bm.microscale_product(w, xq if coded else x)
    for ld, off in ((264, 0), (272, 8), (265, 0), (300, 1), (267, 3)):
        buf = torch.full((T * ld + 8,), float("nan"), dtype=torch.bfloat16, device="cuda")
        xv = buf[off:off + T * ld].view(T, ld)[:, :cols]
        xv.copy_(x)
        for dt in (torch.float32, torch.bfloat16):
            out = torch.full(((T + 1) * 161 + 5,), 7.0, dtype=dt, device="cuda")
            yv = out[off:off + T * 161].view(T, 161)[:, :rows]
            bm.microscale_product(w, xq if coded else xv, y=yv)
            assert torch.equal(yv, ref.to(dt)), (ld, off, dt)
            rest = torch.ones_like(out, dtype=torch.bool)
            rest[off:off + T * 161].view(T, 161)[:, :rows] = False
            assert (out[rest] == 7).all()


@pytest.mark.parametrize("cols", [1, 7, 8, 9, 64, 255, 777, 2041])
def test_rows_brought_onto_16_byte_boundaries(env, cols):
    """Every offset and odd pitches: the columns as they were, zeros up to the next eight, nothing behind."""
    torch, bm = env
    g = torch.Generator().manual_seed(cols)
    for T, ld, off in ((1, cols, 0), (1, cols, 5), (9, cols, 1), (9, cols + 1, 2), (40, cols + 3, 3), (40, cols + 8, 4), (17, cols + 5, 7)):
        buf = torch.full((T * ld + off,), float("nan"), dtype=torch.bfloat16, device="cuda")
        x = buf[off:off + T * ld].view(T, ld)[:, :cols]
        x.copy_(torch.randn(T, cols, generator=g).bfloat16())
        pad = (cols + 7) // 8 * 8
        out = torch.full((T + 1, pad + 8), 3.0, dtype=torch.bfloat16, device="cuda")
        rc = bm._lib().bitsmoe_microscale_align(x.data_ptr(), ld, T, cols, out.data_ptr(), pad + 8, bm._raw_stream(0))
        assert rc == 0
        assert torch.equal(out[:T, :cols], x) and int(torch.count_nonzero(out[:T, cols:pad])) == 0
        assert (out[:T, pad:] == 3).all() and (out[T] == 3).all()


@pytest.mark.parametrize("T,rows,cols", [(20, 300, 777), (70, 140, 2041), (300, 260, 515)])
def test_product_reads_rows_off_boundaries_itself(env, T, rows, cols):
    """The C entry takes such rows as they are; the binding brings many of them onto boundaries: the same values."""
    torch, bm = env
    rng = np.random.default_rng(T)
    w, u = (upload(env, make(rng, rows, cols, "e4m3"), "e4m3") for _ in range(2))
    x = bf16(rng.standard_normal((T, cols))).cuda()
    for up in (None, u):
        y = torch.empty(T, rows, device="cuda")
        rc = bm._lib().bitsmoe_microscale_product(w._c, up._c if up else None, x.data_ptr(), cols, None, T, y.data_ptr(), 0, rows, None,
                                                  bm._raw_stream(0))
        assert rc == 0
        assert torch.equal(y, bm.microscale_product(w, x, up=up))


def test_large_product_of_rows_off_boundaries_in_a_graph_and_on_a_stream(env):
    torch, bm = env
    T, rows, cols = 300, 1500, 1301
    rng = np.random.default_rng(8)
    w = upload(env, make(rng, rows, cols, "e8m0"), "e8m0")
    xs = [bf16(rng.standard_normal((T, cols))).cuda() for _ in range(3)]
    pad = [torch.nn.functional.pad(x, (0, 3)).contiguous()[:, :cols] for x in xs]   # the same rows on boundaries
    want = [bm.microscale_product(w, x) for x in pad]
    for x, v in zip(xs, want):
        assert torch.equal(bm.microscale_product(w, x), v)
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = bm.microscale_product(w, xs[1], stream=s)
    s.synchronize()
    assert torch.equal(got, want[1])
    x, y = xs[0].clone(), torch.empty(T, rows, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bm.microscale_product(w, x, y=y)
    for k in (2, 1):
        x.copy_(xs[k])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, want[k])


def test_product_with_values_that_are_not_finite(env):
    """A NaN or infinite activation reaches its own row of y only."""
    torch, bm = env
    rng = np.random.default_rng(2)
    w = upload(env, make(rng, 70, 100, "e8m0"), "e8m0")
    x = bf16(rng.standard_normal((20, 100)))
    clean = bm.microscale_product(w, x.cuda())
    x[3, 50] = float("nan")
    x[7, 0] = float("inf")
    y = bm.microscale_product(w, x.cuda())
    keep = [t for t in range(20) if t not in (3, 7)]
    assert torch.equal(y[keep], clean[keep])
    assert not torch.isfinite(y[3]).any() and not torch.isfinite(y[7]).all()
    q = bm.microscale_product(w, bm.microscale_quantize(x.cuda(), "e8m0"))
    assert torch.isnan(q[3]).all() and torch.isnan(q[7]).all() and torch.isfinite(q[keep]).all()


def test_product_scale_extremes(env):
    """E8M0 scales far from 1 whose products stay in fp32's range."""
    torch, bm = env
    rng = np.random.default_rng(9)
    for lo, hi, xs in ((0, 4, 2.0 ** 100), (240, 245, 2.0 ** -60)):
        codes = rng.integers(0, 16, (130, 96)).astype(np.uint8)
        byte = rng.integers(lo, hi, (130, 3)).astype(np.uint8)
        v = om.values(codes, byte, "e8m0", 1.0)
        t = bf16(rng.standard_normal((5, 96)) * xs)
        y = bm.microscale_product(upload(env, (codes, byte, 1.0, None), "e8m0"), t.cuda()).double().cpu().numpy()
        want, mag = om.product(v, t.double().numpy())
        assert (np.abs(y - want) <= 100 * U * mag).all()


@pytest.mark.parametrize("T", [3, 12, 30])
def test_product_scale_extremes_with_a_range_of_activations(env, T):
    """Activations that are not all exact in fp16 as they are: small ones on small scales (sums of 2^-110 and
    less), and small ones on a block of large scales beside large ones on a block of small scales."""
    torch, bm = env
    rng = np.random.default_rng(T)
    codes = rng.integers(0, 16, (130, 96)).astype(np.uint8)
    for scales, xs in (((1, 8, 12), (0.5, 0.125, 2.0 ** -30)), ((80, 83, 86), (2.0 ** -80, 2.0 ** -83, 2.0 ** -85)),
                       ((247, 127, 100), (0.125, 2.0 ** 27, 1.0)), ((250, 127, 120), (2.0 ** -16, 2.0 ** 14, 2.0 ** 13))):
        byte = np.tile(np.array(scales, np.uint8), (130, 1))
        v = om.values(codes, byte, "e8m0", 1.0)
        t = bf16(rng.uniform(0.5, 1, (T, 96)) * rng.choice([-1, 1], (T, 96)) * np.repeat(xs, 32))
        y = bm.microscale_product(upload(env, (codes, byte, 1.0, None), "e8m0"), t.cuda()).double().cpu().numpy()
        want, mag = om.product(v, t.double().numpy())
        assert (np.abs(y - want) <= 100 * U * mag).all(), (scales, xs)


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("T", [1, 7, 16, 40])
def test_product_activation_range(env, fmt, T):
    """Activations over many binades within a row and between rows, with the large ones on zero codes: the small
    ones still count in full.  Rows of zeros, rows all tiny and all large."""
    torch, bm = env
    rng = np.random.default_rng(T)
    rows, cols = 140, 600
    for lo, hi in ((-40, 0), (-100, -60), (30, 60), (-60, 60), (-2, 2)):
        codes, byte, scale, _ = make(rng, rows, cols, fmt)
        big = np.arange(cols) % 5 == 0
        codes[:, big] = 0
        v = om.values(codes, byte, fmt, float(np.float32(scale)))
        x = rng.standard_normal((T, cols)) * 2.0 ** rng.uniform(lo, hi, (T, cols))
        x[:, big] *= 2.0 ** 12
        x[T // 2, :300] = 0.0
        t = bf16(x)
        y = bm.microscale_product(upload(env, (codes, byte, scale, None), fmt), t.cuda()).double().cpu().numpy()
        want, mag = om.product(v, t.double().numpy())
        assert (np.abs(y - want) <= (cols + 4) * U * mag).all(), (lo, hi)


def test_sizes_past_32_bits_are_refused(env):
    """2^32 + 5 rows or columns are not cut to 5 on their way to the library."""
    torch, bm = env
    n = 2 ** 32 + 5
    x = torch.empty(n, dtype=torch.bfloat16, device="cuda")
    w = bm.microscale_quantize(torch.ones(4, 1, device="cuda"))
    for call in (lambda: bm.microscale_quantize(x.view(n, 1)), lambda: bm.microscale_quantize(x.view(1, n)),
                 lambda: bm.microscale_product(w, x.view(n, 1)), lambda: bm.block_norm(x.view(n, 1)),
                 lambda: bm.block_norm(x.view(1, n)), lambda: bm.Microscale.empty(n, 1), lambda: bm.Microscale.empty(1, n)):
        with pytest.raises(bm.BitsMoEError):
            call()


def test_empty_calls_write_nothing(env):
    torch, bm = env
    rng = np.random.default_rng(0)
    w = upload(env, make(rng, 5, 64, "e8m0"), "e8m0")
    assert bm.microscale_product(w, torch.zeros(0, 64, dtype=torch.bfloat16, device="cuda")).shape == (0, 5)
    assert bm.microscale_product(w, bm.Microscale.empty(0, 64)).shape == (0, 5)
    assert bm.microscale_quantize(torch.zeros(0, 64, device="cuda")).rows == 0
    assert bm.microscale_dequantize(bm.Microscale.empty(0, 64)).shape == (0, 64)
    none = bm.Microscale.empty(0, 64)
    assert bm.microscale_product(none, torch.zeros(3, 64, dtype=torch.bfloat16, device="cuda")).shape == (3, 0)


@pytest.mark.parametrize("coded", [False, True])
def test_product_on_streams_in_graphs_and_again(env, coded):
    """The same bits on the current stream, on another one, on two at once, captured and replayed with new
    inputs in the same buffers."""
    torch, bm = env
    rng = np.random.default_rng(4)
    w = upload(env, make(rng, 700, 1024, "e4m3"), "e4m3")
    u = upload(env, make(rng, 700, 1024, "e4m3", 0.01), "e4m3")
    xs = [bf16(rng.standard_normal((24, 1024))).cuda() for _ in range(2)]
    xq = [bm.microscale_quantize(x, "e4m3", 1.0) for x in xs] if coded else xs
    ref = [bm.microscale_product(w, x, up=u) for x in xq]
    assert torch.equal(bm.microscale_product(w, xq[0], up=u), ref[0])
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(5):
        got = [bm.microscale_product(w, xq[i], up=u, stream=s[i]) for i in range(2)]
        torch.cuda.synchronize()
        assert torch.equal(got[0], ref[0]) and torch.equal(got[1], ref[1])
    x = xs[0].clone()
    y = torch.empty_like(ref[0])
    q = bm.Microscale.empty(24, 1024, "e4m3", 1.0)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        if coded:
            bm.microscale_quantize(x, "e4m3", 1.0, out=q)
        bm.microscale_product(w, q if coded else x, up=u, y=y)
    for i in (0, 1, 0):
        x.copy_(xs[i])
        y.zero_()
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, ref[i])


@pytest.mark.parametrize("case", ["few", "few_split", "coded", "coded_split", "coded_pair", "coded_pair_swiglu", "wide", "wide_split", "wide_swiglu"])
def test_product_reports_a_wait_that_ran_out(env, case):
    """A block that never reports a slot of its ring free (testing hook): the bounded waits run out, the status word
    says so, and the next call is right.  Every case has more stages than its ring."""
    torch, bm = env
    rng = np.random.default_rng(6)
    T = {"few": 3, "few_split": 2, "coded_pair": 256, "coded_pair_swiglu": 256}.get(case, 40)
    rows, cols = {"few": (152 * 128, 8192), "few_split": (130, 65536), "coded": (152 * 128, 8192), "coded_pair": (152 * 128, 4096),
                  "coded_pair_swiglu": (80 * 128, 4096), "coded_split": (130, 65536),
                  "wide": (152 * 128, 2048), "wide_split": (130, 16384), "wide_swiglu": (152 * 128, 1024)}[case]
    w = bm.microscale_quantize(torch.randn(rows, cols, device="cuda"), "e4m3", 1.0)
    x = bf16(rng.standard_normal((T, cols))).cuda()
    if case.startswith("coded"):
        x = bm.microscale_quantize(x, "e4m3", 1.0)
    up = w if case.endswith("swiglu") else None
    ref = bm.microscale_product(w, x, up=up)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    bm.bitsmoe_debug_wait_limit(1, 2_000_000)
    try:
        bm.microscale_product(w, x, up=up, status=status)
        torch.cuda.synchronize()
    finally:
        bm.bitsmoe_debug_wait_limit(0, 0)
    assert int(status.item()) == bm.ERR_CODE["TIMEOUT"]
    status.zero_()
    assert torch.equal(bm.microscale_product(w, x, up=up, status=status), ref)
    assert int(status.item()) == 0


def test_products_beside_the_forward_on_another_stream(env):
    """Both allocate tensor memory and wait inside clusters: split and paired products on one stream, forwards of the
    tensor-core projections on another, many at a time; every result as alone."""
    import synth
    torch, bm = env
    rng = np.random.default_rng(12)
    spec = synth.scaled_spec(synth.WORKLOADS["tiny"], D=256, E=8, I=256, n=128, group=128, top_k=2)
    L = bm.bitsmoe_pack(synth.make_layer(spec, seed=5, bits_dist={0: .1, 1: .2, 2: .4, 3: .2, 4: .1}), device=0)
    x, logits = synth.make_inputs(spec, 40, seed=5)
    xd, ld = torch.from_numpy(x.view(np.int16)).cuda(), torch.from_numpy(logits).cuda()
    ws = bm.Workspace(L, 40, spec.top_k)
    y_ref = bm.moe_forward(L, xd, ld, spec.top_k, ws)
    cases = []
    for T, rows, cols in ((40, 300, 4096), (256, 1500, 1024), (3, 400, 2048)):
        w = upload(env, make(rng, rows, cols, "e4m3"), "e4m3")
        a = bf16(rng.standard_normal((T, cols))).cuda()
        for v in (a, bm.microscale_quantize(a, "e4m3", 1.0)):
            cases.append((w, v, bm.microscale_product(w, v)))
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    for _ in range(20):
        y = torch.empty_like(y_ref)
        with torch.cuda.stream(s[0]):
            for _ in range(3):
                bm.moe_forward(L, xd, ld, spec.top_k, ws, y=y)
        got = [bm.microscale_product(w, v, stream=s[1]) for w, v, _ in cases]
        torch.cuda.synchronize()
        assert all(torch.equal(g, r) for g, (_, _, r) in zip(got, cases))
        assert bm.bitsmoe_last_device_status(ws.ptr) == 0
        torch.testing.assert_close(y, y_ref, rtol=1e-5, atol=1e-6)


_FIRST_IN_CAPTURE = r"""
import sys
import torch
sys.path.insert(0, sys.argv[1])
import paper_2606_00079_gb300 as bm
torch.manual_seed(0)
w, x = torch.randn(300, 512, device="cuda"), torch.randn(40, 512, device="cuda").bfloat16()
q, xq = bm.Microscale.empty(300, 512, "e4m3", 1.0), bm.Microscale.empty(40, 512, "e4m3", 1.0)
o = [torch.zeros(n, 300, device="cuda") for n in (40, 40, 3, 3)]
d, hx = torch.zeros(300, 512, device="cuda"), torch.zeros(40, 512, dtype=torch.bfloat16, device="cuda")
torch.cuda.synchronize()
def calls():
    bm.microscale_quantize(w, "e4m3", 1.0, out=q)
    bm.microscale_quantize(x, "e4m3", 1.0, out=xq)
    bm.microscale_dequantize(q, out=d)
    bm.microscale_product(q, x, y=o[0])
    bm.microscale_product(q, xq, y=o[1])
    bm.microscale_product(q, x[:3], y=o[2])
    bm.microscale_product(q, x[:3], up=q, y=o[3])
    bm.block_norm(x, x=hx)
g = torch.cuda.CUDAGraph()
with torch.cuda.graph(g):
    calls()
g.replay()
torch.cuda.synchronize()
first = [t.clone() for t in (*o, d, hx)]
calls()
torch.cuda.synchronize()
assert all(torch.equal(a, b) for a, b in zip(first, (*o, d, hx))) and float(o[0].abs().max()) > 0
print("CAPTURED")
"""


def test_first_calls_of_a_process_inside_a_capture(env):
    import os
    import subprocess
    import sys
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", _FIRST_IN_CAPTURE, root], capture_output=True, text=True, timeout=300)
    assert "CAPTURED" in r.stdout, (r.stdout, r.stderr[-2000:])


WAITS = {"few": (3, 152 * 128, 8192), "few_split": (2, 130, 65536), "few_tiles": (3, 300 * 128, 4096), "few_swiglu": (3, 152 * 128, 4096),
         "few_split_tiles": (3, 200 * 128, 2304), "few_split_tiles_swiglu": (3, 200 * 128, 1280),
         "coded": (40, 152 * 128, 8192), "coded_tiles": (256, 152 * 128, 4096), "coded_swiglu": (256, 80 * 128, 4096),
         "coded_split": (40, 130, 65536), "wide": (40, 152 * 128, 2048), "wide_split": (40, 130, 16384), "wide_swiglu": (40, 152 * 128, 1024)}


@pytest.mark.parametrize("case", list(WAITS))
def test_a_wait_that_ran_out_leaves_nan(env, case):
    """The ordinary call, without a status word: what a block that gave up has lost is NaN (its first tile, where that has
    more stages than its ring), every other value is right, nothing between the rows is touched, and the next call is
    right."""
    torch, bm = env
    T, rows, cols = WAITS[case]
    g = torch.Generator().manual_seed(6)
    w = bm.microscale_quantize(torch.randn(rows, cols, device="cuda"), "e4m3", 1.0)
    x = torch.randn(T, cols, generator=g).bfloat16().cuda()
    if case.startswith("coded"):
        x = bm.microscale_quantize(x, "e4m3", 1.0)
    up = w if case.endswith("swiglu") else None
    ref = bm.microscale_product(w, x, up=up)
    for dt in (torch.float32, torch.bfloat16):
        buf = torch.full((T, rows + 5), 7.0, dtype=dt, device="cuda")
        y = buf[:, :rows]
        bm.bitsmoe_debug_wait_limit(1, 2_000_000)
        try:
            bm.microscale_product(w, x, up=up, y=y)
            torch.cuda.synchronize()
        finally:
            bm.bitsmoe_debug_wait_limit(0, 0)
        lost = torch.isnan(y)
        assert bool(lost.any())
        if "split_tiles" not in case:
            assert bool(lost[:min(T, 128), :min(rows, 128)].all())
        assert torch.equal(y[~lost], ref.to(dt)[~lost])
        assert (buf[:, rows:] == 7).all()
        if not case.endswith("split"):
            assert not bool(lost.all())
        bm.microscale_product(w, x, up=up, y=y)
        assert torch.equal(y, ref.to(dt))


def test_a_refused_quantisation_leaves_out_as_it_was(env):
    """A tensor scale that the library does not take: `out` keeps its codes and its own scale."""
    torch, bm = env
    x = torch.randn(9, 70, device="cuda")
    q = bm.microscale_quantize(x, "e4m3", 0.5)
    before = bm.microscale_dequantize(q)
    s = torch.cuda.Stream()
    for scale in (3.0, 2.0 ** 101, 0.0, float("nan")):
        for kw in ({}, {"stream": s}):
            with pytest.raises(bm.BitsMoEError):
                bm.microscale_quantize(x, "e4m3", scale, out=q, **kw)
            assert q.scale == 0.5
    torch.cuda.synchronize()
    assert torch.equal(bm.microscale_dequantize(q), before)
    bm.microscale_quantize(x, "e4m3", 2.0, out=q)
    assert q.scale == 2.0 and torch.equal(bm.microscale_dequantize(q), bm.microscale_dequantize(bm.microscale_quantize(x, "e4m3", 2.0)))


def test_quantizer_where_the_quotient_is_subnormal(env):
    """x / scale below fp32's normal range: its lost bits would move values next to a midpoint between codes onto it
    (E8M0's smallest block scale is 2^-127, the midpoints 2^-129 and up)."""
    torch, bm = env
    rng = np.random.default_rng(21)
    mids = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, 7.5], np.float64)
    for k in (1, 3, 10, 24, 60, 100):
        x = rng.choice(mids, (40, 64)) * 2.0 ** -127 * 2.0 ** k
        x[20:] *= 2.0 ** rng.integers(0, 4, (20, 1))
        with np.errstate(under="ignore"):
            x = x.astype(np.float32)
            j = rng.integers(0, 3, x.shape)
            x = np.where(j == 1, np.nextafter(x, np.float32(0)), np.where(j == 2, np.nextafter(x, np.float32(1)), x))
        x *= rng.choice([-1, 1], x.shape).astype(np.float32)
        for fmt in ("e8m0", "e4m3"):
            check_quantized(bm.microscale_quantize(torch.from_numpy(x).cuda(), fmt, 2.0 ** k), x, fmt, 2.0 ** k)
            xb = bf16(x)
            check_quantized(bm.microscale_quantize(xb.cuda(), fmt, 2.0 ** k), xb.float().numpy(), fmt, 2.0 ** k)


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_quantizer_tensor_scales_far_from_one(env, fmt):
    """Every block scale and quotient that the extremes of the tensor scale reach, normal and subnormal, and quotients
    past fp32's range (a block without a scale)."""
    torch, bm = env
    rng = np.random.default_rng(22)
    for k in (-100, -37, 37, 100):
        e = rng.uniform(-149, 127.9, (64, 1)) if k > 0 else rng.uniform(-149, 127.9 + k / 2, (64, 1))
        with np.errstate(under="ignore", over="ignore"):
            x = (rng.standard_normal((64, 96)) * 2.0 ** e).astype(np.float32)
        x = np.where(np.isfinite(x), x, np.float32(1.0))
        check_quantized(bm.microscale_quantize(torch.from_numpy(x).cuda(), fmt, 2.0 ** k), x, fmt, 2.0 ** k)
        xb = bf16(x)
        xb = torch.where(torch.isfinite(xb), xb, torch.ones_like(xb))
        check_quantized(bm.microscale_quantize(xb.cuda(), fmt, 2.0 ** k), xb.float().numpy(), fmt, 2.0 ** k)


def test_product_takes_subclasses_of_microscale(env):
    torch, bm = env

    class Mine(bm.Microscale):
        pass

    rng = np.random.default_rng(3)
    w = upload(env, make(rng, 40, 96, "e4m3"), "e4m3")
    a = bm.microscale_quantize(torch.randn(5, 96, device="cuda"), "e4m3")
    mine = Mine(a.codes, a.scales, 5, 96, "e4m3", a.scale)
    assert torch.equal(bm.microscale_product(w, mine), bm.microscale_product(w, a))


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
@pytest.mark.parametrize("T,rows,cols", [(3, 130, 777), (14, 300, 1301), (20, 300, 777), (70, 140, 2041), (300, 260, 515), (300, 1500, 1301)])
def test_rows_off_boundaries_against_rows_on_them(env, fmt, T, rows, cols):
    """What the kernels read element by element, what the binding copies first (the last case) and what comes by TMA:
    the same values, with and without the second matrix."""
    torch, bm = env
    rng = np.random.default_rng([T, cols])
    w, u = (upload(env, make(rng, rows, cols, fmt), fmt) for _ in range(2))
    x = bf16(rng.standard_normal((T, cols))).cuda()
    on = torch.nn.functional.pad(x, (0, -cols % 8)).contiguous()[:, :cols]
    assert on.stride(0) % 8 == 0 and on.data_ptr() % 16 == 0 and x.stride(0) % 8
    for up in (None, u):
        want = bm.microscale_product(w, on, up=up)
        y = torch.empty(T, rows, device="cuda")
        rc = bm._lib().bitsmoe_microscale_product(w._c, up._c if up else None, x.data_ptr(), cols, None, T, y.data_ptr(), 0, rows, None,
                                                  bm._raw_stream(0))
        assert rc == 0
        assert torch.equal(y, want)
        assert torch.equal(bm.microscale_product(w, x, up=up), want)


@pytest.mark.parametrize("x", ["bf16", "coded"])
@pytest.mark.parametrize("T,rows,cols", [(13, 14336, 4096), (16, 130, 40000), (1, 5, 1 << 20), (3, 7, (1 << 20) - 37)])
def test_product_where_few_tokens_take_the_other_kernels(env, x, T, rows, cols):
    """More slots a CTA than the kernel of few tokens gains with, and activations that its shared memory does not hold."""
    check_product(env, T, rows, cols, "e4m3", x == "coded", False, "f32")
    check_product(env, T, rows, cols, "e8m0", x == "coded", True, "bf16")


def test_largest_numbers_of_rows_and_tokens(env):
    """2^24 rows or tokens: the last ones equal the same ones alone."""
    torch, bm = env
    n = 1 << 24
    g = torch.Generator().manual_seed(1)
    big = torch.zeros(n, 32, dtype=torch.bfloat16, device="cuda")
    big[-200:] = torch.randn(200, 32, generator=g).bfloat16().cuda()
    small = torch.randn(3, 32, generator=g).bfloat16().cuda()
    q, last, few = bm.microscale_quantize(big), bm.microscale_quantize(big[-200:]), bm.microscale_quantize(small)
    for a in (small, few):
        y = bm.microscale_product(q, a)
        assert torch.equal(y[:, -200:], bm.microscale_product(last, a)) and int(torch.count_nonzero(y[:, :-200])) == 0
        del y
    for a, b in ((big, big[-200:]), (q, last)):
        y = bm.microscale_product(few, a)
        assert torch.equal(y[-200:], bm.microscale_product(few, b)) and int(torch.count_nonzero(y[:-200])) == 0
    y = bm.microscale_dequantize(q, torch.bfloat16)
    assert torch.equal(y[-200:], bm.microscale_dequantize(last, torch.bfloat16)) and int(torch.count_nonzero(y[:-200])) == 0
    _, x = bm.block_norm(big)
    assert torch.equal(x[-200:], bm.block_norm(big[-200:])[1]) and int(torch.count_nonzero(x[:-200])) == 0
