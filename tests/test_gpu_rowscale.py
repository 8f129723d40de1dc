"""GPU checks of rows in 8 bits: the coder and its inverse to the bit against the oracle, and the norm between blocks
with an 8-bit output.

The norm's codes are compared to the bit with the coder's of the same kernel's fp32 output, and its values with float64:
a value within half a step of E4M3, 2^-4 of it (2^-10 of the scale below the normal codes), plus the error of the fp32 norm
before it (the bound in tests/test_gpu_block_norm.py, at most (1.5 D + 40) 2^-24 of the row's norm per element for the
gains used here), plus half of a step where that error moves the scale: twice the steps in all."""
import numpy as np
import pytest

from oracle import experts as oe, microscale as om

pytestmark = pytest.mark.gpu


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


def special_rows(rng, rows, cols, amp=1.0):
    """Rows of all sizes: normal, tiny, huge, zeros, largest values on and next to a border, not finite."""
    x = (amp * rng.standard_normal((rows, cols))).astype(np.float32)
    kinds = rng.integers(0, 10, rows)
    for r in range(rows):
        c = int(rng.integers(0, cols))
        if kinds[r] == 0:
            x[r] = 0
        elif kinds[r] == 1:
            x[r] *= np.float32(2.0 ** -120)
        elif kinds[r] == 2:
            x[r] *= np.float32(2.0 ** 122)
        elif kinds[r] == 3:
            x[r] = np.clip(x[r], -1, 1)
            x[r, c] = np.float32(-448 * 2.0 ** -7)
        elif kinds[r] == 4:
            x[r] = np.clip(x[r], -1, 1)
            x[r, c] = np.nextafter(np.float32(448 * 2.0 ** -7), np.float32(9))
        elif kinds[r] == 5:
            x[r] *= np.float32(2.0) ** rng.integers(-20, 1, cols).astype(np.float32)
        elif kinds[r] == 6:   # midpoints between codes
            x[r] = (oe.e4m3_values()[rng.integers(0, 126, cols)] + oe.e4m3_values()[rng.integers(0, 126, cols)]) / 2
    if rows > 4:
        x[1, cols // 2] = np.nan
        x[3, cols - 1] = -np.inf
    return x


SHAPES = [(1, 1), (3, 7), (5, 64), (33, 256), (33, 257), (17, 1000), (9, 1024), (9, 1025), (7, 2050), (4, 4096), (3, 4104),
          (2, 16384), (2, 16392), (3, 20001)]


@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("ty", ["f32", "bf16"])
@pytest.mark.parametrize("shift", [0, 1])   # elements off a 16-byte boundary, on a pitch that is not a multiple of 16 bytes
def test_rowscale_to_the_bit(env, rows, cols, ty, shift):
    torch, bm = env
    rng = np.random.default_rng([rows, cols, shift])
    with np.errstate(over="ignore", under="ignore"):
        x = torch.from_numpy(special_rows(rng, rows, cols)).to(torch.float32 if ty == "f32" else torch.bfloat16)
    buf = torch.zeros(rows, cols + 2 + shift, dtype=x.dtype, device="cuda") if shift else torch.zeros(rows, (cols + 7) // 8 * 8, dtype=x.dtype, device="cuda")
    dev = buf[:, shift:shift + cols]
    dev.copy_(x)
    q = bm.rowscale_quantize(dev)
    codes, scales = oe.rowscale(x.double().numpy())
    np.testing.assert_array_equal(q.scales.cpu().numpy(), scales)
    np.testing.assert_array_equal(q.codes.view(torch.uint8).cpu().numpy(), codes)
    # into codes off the boundaries, nothing between the rows touched
    raw = torch.full((rows, cols + 3), 77, dtype=torch.uint8, device="cuda")
    out = bm.Rowscale(raw[:, 1:1 + cols].view(torch.float8_e4m3fn), torch.empty(rows, device="cuda"))
    assert bm.rowscale_quantize(dev, out=out) is out
    raw = raw.cpu().numpy()
    np.testing.assert_array_equal(raw[:, 1:1 + cols], codes)
    assert (raw[:, 0] == 77).all() and (raw[:, 1 + cols:] == 77).all()
    # back: code * scale rounded once
    want = oe.e4m3_values()[codes] * scales[:, None].astype(np.float64)
    for src in (q, out):
        for dt in (torch.float32, torch.bfloat16):
            back = bm.rowscale_dequantize(src, dt)
            np.testing.assert_array_equal(back.double().cpu().numpy(), want)
            wide = torch.full((rows, cols + 5), 7.0, dtype=dt, device="cuda")
            bm.rowscale_dequantize(src, out=wide[:, 1:1 + cols])
            wide = wide.double().cpu().numpy()
            np.testing.assert_array_equal(wide[:, 1:1 + cols], want)
            assert (wide[:, 0] == 7).all() and (wide[:, 1 + cols:] == 7).all()


def test_rowscale_any_scale_and_every_code(env):
    torch, bm = env
    codes = torch.arange(256, dtype=torch.uint8).repeat(3, 1).cuda()
    s = torch.tensor([0.3, -1.7e-30, 5e37]).cuda()
    v = oe.e4m3_values().astype(np.float32)
    with np.errstate(over="ignore"):
        want = v[None, :] * s.cpu().numpy()[:, None]
        got = bm.rowscale_dequantize(bm.Rowscale(codes.view(torch.float8_e4m3fn), s)).cpu().numpy()
    np.testing.assert_array_equal(got, want)


def test_rowscale_matrices_of_experts(env):
    torch, bm = env
    x = torch.randn(5, 33, 70, device="cuda")
    q = bm.rowscale_quantize(x)
    assert q.shape == (5, 33, 70) and q.scales.shape == (5, 33)
    flat = bm.rowscale_quantize(x.view(165, 70))
    assert torch.equal(q.codes.reshape(165, 70).view(torch.uint8), flat.codes.contiguous().view(torch.uint8))
    assert torch.equal(bm.rowscale_dequantize(q).view(165, 70), bm.rowscale_dequantize(flat))
    with pytest.raises(bm.BitsMoEError):
        bm.rowscale_quantize(x[:, :30])   # matrices with rows between them
    for empty in (x[:0], x[:, :0]):
        assert bm.rowscale_dequantize(bm.rowscale_quantize(empty)).shape == empty.shape


def test_rowscale_stream_and_graph(env):
    torch, bm = env
    x = torch.randn(300, 512, device="cuda", dtype=torch.bfloat16)
    st = torch.cuda.Stream()
    st.wait_stream(torch.cuda.current_stream())
    q = bm.rowscale_quantize(x, stream=st)
    v = bm.rowscale_dequantize(q, stream=st)
    st.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        gv = bm.rowscale_dequantize(bm.rowscale_quantize(x))
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(gv, v)
    x.mul_(3.0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(gv, bm.rowscale_dequantize(bm.rowscale_quantize(x)))


WIDTHS = [1, 2, 7, 8, 100, 256, 257, 1000, 2048, 2050, 4096, 4104, 8192, 8200, 12288, 16384, 20001]


@pytest.mark.parametrize("D", WIDTHS)
@pytest.mark.parametrize("T", [1, 5, 700])
def test_norm_in_eight_bits(env, D, T):
    torch, bm = env
    if T * D > 4_000_000:
        pytest.skip("covered by fewer rows")
    rng = np.random.default_rng([T, D])
    h = torch.from_numpy((3 * rng.standard_normal((T, D))).astype(np.float32))
    y = torch.from_numpy(rng.standard_normal((T, D)).astype(np.float32)).to(torch.bfloat16)
    if T > 2:
        h[1], y[1] = 0.0, 0.0
    pre = torch.from_numpy((1 + 0.2 * rng.standard_normal(D)).astype(np.float32))
    gate = torch.from_numpy(rng.standard_normal(T).astype(np.float32))
    kw = dict(post_norm=True, gate=gate.cuda(), gate_sigmoid=True, branch_scale=0.5, residual_scale=0.875, pre_gain=pre.cuda())
    hn, q = bm.block_norm(h.cuda(), y.cuda(), x_dtype=torch.float8_e4m3fn, **kw)
    hd, xd = bm.block_norm(h.cuda(), y.cuda(), x_dtype=torch.float32, **kw)
    assert torch.equal(hn, hd)
    want = bm.rowscale_quantize(xd)
    assert torch.equal(q.scales, want.scales)
    assert torch.equal(q.codes.contiguous().view(torch.uint8), want.codes.contiguous().view(torch.uint8))
    # against float64
    g = 1 / (1 + np.exp(-gate.double().numpy()))[:, None]
    _, _, wx = om.block_norm(h.double().numpy(), y.double().numpy(), np.ones(D), g, None, 0.5, 0.875, pre.double().numpy(), 1e-6, 1e-6)
    got = bm.rowscale_dequantize(q).double().cpu().numpy()
    s = q.scales.double().cpu().numpy()[:, None]
    err = (1.5 * D + 40) * 2.0 ** -24 * np.linalg.norm(wx, axis=1, keepdims=True)
    assert (np.abs(got - wx) <= 2 * np.maximum(2.0 ** -4 * np.abs(wx), 2.0 ** -10 * s) + err).all()


@pytest.mark.parametrize("T,D", [(3, 64), (3, 2048), (3, 2050), (900, 512), (900, 515), (2, 20001)])
def test_norm_in_eight_bits_rows_that_are_not_finite(env, T, D):
    torch, bm = env
    h = torch.randn(T, D, device="cuda")
    h[0, D // 2] = float("nan")
    h[2 % T, D - 1] = float("inf")
    raw = torch.full((T, D + 3), 77, dtype=torch.uint8, device="cuda")
    x = bm.Rowscale(raw[:, 1:1 + D].view(torch.float8_e4m3fn), torch.empty(T, device="cuda"))
    _, q = bm.block_norm(h, x=x)
    assert q is x
    bad = torch.zeros(T, dtype=torch.bool)
    bad[0] = bad[2 % T] = True
    assert torch.equal(torch.isnan(q.scales).cpu(), bad)
    assert (raw[:, 1:1 + D][bad.cuda()] == 0).all() and (raw[:, 0] == 77).all() and (raw[:, 1 + D:] == 77).all()
    _, dense = bm.block_norm(h, x_dtype=torch.float32)
    want = bm.rowscale_quantize(dense)   # (rows read element by element take another order of sums: within a step)
    a, b = bm.rowscale_dequantize(q)[~bad.cuda()], bm.rowscale_dequantize(want)[~bad.cuda()]
    assert ((a - b).abs() <= 2.0 ** -3 * b.abs() + 2.0 ** -9 * want.scales[~bad.cuda()][:, None]).all()


def test_norm_in_eight_bits_in_a_graph_and_in_place(env):
    torch, bm = env
    h = torch.randn(64, 2048, device="cuda")
    y = torch.randn(64, 2048, device="cuda", dtype=torch.bfloat16)
    h0 = h.clone()
    want_h, want = bm.block_norm(h0, y, x_dtype=torch.float8_e4m3fn)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _, q = bm.block_norm(h, y, h_out=h, x_dtype=torch.float8_e4m3fn)
    h.copy_(h0)
    g.replay()
    torch.cuda.synchronize()
    assert torch.equal(h, want_h) and torch.equal(q.scales, want.scales)
    assert torch.equal(q.codes.view(torch.uint8), want.codes.view(torch.uint8))
    with pytest.raises(bm.BitsMoEError):
        bm.block_norm(h, y, pre_norm=False, x_dtype=torch.float8_e4m3fn)
    with pytest.raises(bm.BitsMoEError):
        bm.block_norm(h, y, x=bm.Rowscale.empty((64, 2047)))
