"""Host-side checks of the microscaled 4-bit operators and block_norm (no GPU needed): the refusals of
each entry point, the sizes, and the oracle against the formats' definitions."""
import ctypes

import numpy as np
import pytest

from oracle import microscale as om

A = 4096   # an aligned stand-in address (never dereferenced: the checks fail first, or nothing is to do)


@pytest.fixture(scope="module")
def bm():
    import __graft_entry__
    __graft_entry__.build_library()
    import paper_2606_00079_gb300 as bm
    return bm


def micro(bm, fmt=0, rows=4, cols=64, scale=1.0, codes=A, scales=A):
    return bm._Microscale(fmt, rows, cols, scale, codes, scales)


def test_sizes(bm):
    assert bm.microscale_bytes("e8m0", 1, 1) == (16, 512)
    assert bm.microscale_bytes("e8m0", 129, 129) == (129 * 80, 2 * 2 * 512)
    assert bm.microscale_bytes("e4m3", 128, 64) == (128 * 32, 512)
    assert bm.microscale_bytes("e4m3", 128, 65) == (128 * 48, 2 * 512)
    assert bm.microscale_bytes("e4m3", 0, 65) == (0, 0)
    for bad in ((0, -1, 4), (0, 4, 0), (2, 4, 4), (-1, 4, 4)):
        a, b = ctypes.c_size_t(), ctypes.c_size_t()
        assert bm._lib().bitsmoe_microscale_bytes(*bad, ctypes.byref(a), ctypes.byref(b)) == bm.ERR_CODE["INVALID_ARG"]
    with pytest.raises(bm.BitsMoEError):
        bm.microscale_bytes("e8m0", (1 << 24) + 1, 4)
    with pytest.raises(bm.BitsMoEError):
        bm.microscale_bytes("fp4", 4, 4)


@pytest.mark.parametrize("which", ["quantize", "dequantize"])
def test_quantizer_refusals(bm, which):
    E = bm.ERR_CODE
    if which == "quantize":
        f = lambda m, x=A, ty=0, ld=64: bm._lib().bitsmoe_microscale_quantize(x, ty, ld, m, 0)
    else:
        f = lambda m, x=A, ty=0, ld=64: bm._lib().bitsmoe_microscale_dequantize(m, x, ty, ld, 0)
    assert f(micro(bm, rows=0)) == 0
    assert f(None) == E["INVALID_ARG"]
    for kw in (dict(fmt=2), dict(rows=-1), dict(cols=0), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("inf")),
               dict(scale=float("nan")), dict(codes=0), dict(scales=0)):
        assert f(micro(bm, **kw)) == E["INVALID_ARG"], kw
    assert f(micro(bm), ty=2) == E["INVALID_ARG"]
    assert f(micro(bm), ld=63) == E["INVALID_ARG"]
    assert f(micro(bm), x=0) == E["INVALID_ARG"]
    assert f(micro(bm), x=A + 2) == E["ALIGNMENT"]
    assert f(micro(bm), x=A + 1, ty=1) == E["ALIGNMENT"]
    assert f(micro(bm, codes=A + 8)) == E["ALIGNMENT"]
    assert f(micro(bm, scales=A + 8)) == E["ALIGNMENT"]
    assert f(micro(bm, rows=(1 << 24) + 1)) == E["SHAPE"]
    assert f(micro(bm, cols=(1 << 20) + 1), ld=1 << 21) == E["SHAPE"]
    if which == "quantize":
        for s in (3.0, 0.7, 2.0 ** -101, 2.0 ** 101):
            assert f(micro(bm, scale=s)) == E["INVALID_ARG"], s


def test_product_refusals(bm):
    E = bm.ERR_CODE

    def f(w=None, up=None, x=A, x_ld=64, xq=None, T=3, y=A, ty=0, y_ld=4, status=0):
        return bm._lib().bitsmoe_microscale_product(w if w is not None else micro(bm), up, x, x_ld, xq, T, y, ty, y_ld,
                                                    status, 0)
    assert f(T=0) == 0
    assert f(w=micro(bm, rows=0), y_ld=0) == 0
    assert f(T=-1) == E["INVALID_ARG"]
    assert f(T=(1 << 24) + 1) == E["SHAPE"]
    assert f(w=micro(bm, scale=0.0)) == E["INVALID_ARG"]
    assert f(x=0) == E["INVALID_ARG"]
    assert f(y=0) == E["INVALID_ARG"]
    assert f(ty=7) == E["INVALID_ARG"]
    assert f(x_ld=63) == E["INVALID_ARG"]
    assert f(y_ld=3) == E["INVALID_ARG"]
    assert f(x=A + 1) == E["ALIGNMENT"]
    assert f(y=A + 2) == E["ALIGNMENT"]
    assert f(status=A + 2) == E["ALIGNMENT"]
    assert f(up=micro(bm, fmt=1)) == E["INVALID_ARG"]
    assert f(up=micro(bm, rows=5)) == E["SHAPE"]
    assert f(up=micro(bm, cols=32)) == E["SHAPE"]
    assert f(up=micro(bm, codes=0)) == E["INVALID_ARG"]
    assert f(xq=micro(bm, rows=3)) == E["INVALID_ARG"]                  # x and xq
    assert f(x=0, xq=micro(bm, rows=4)) == E["SHAPE"]
    assert f(x=0, xq=micro(bm, rows=3, cols=65)) == E["SHAPE"]
    assert f(x=0, xq=micro(bm, rows=3, fmt=1)) == E["INVALID_ARG"]
    assert f(x=0, xq=micro(bm, rows=3, scale=float("nan"))) == E["INVALID_ARG"]


def test_block_norm_refusals(bm):
    E = bm.ERR_CODE

    def f(**kw):
        a = bm._BlockNormArgs(T=2, D=8, h=A, y=A, h_out=A, x=A, h_ld=8, y_ld=8, h_out_ld=8, x_ld=8, gate_ld=8)
        for k, v in kw.items():
            setattr(a, k, v)
        return bm._lib().bitsmoe_block_norm(ctypes.byref(a), 0)
    assert bm._lib().bitsmoe_block_norm(None, 0) == E["INVALID_ARG"]
    assert f(T=0) == 0
    for kw in (dict(T=-1), dict(D=0), dict(h=0), dict(h_type=2), dict(y_type=-1), dict(x_type=3), dict(gain_type=9),
               dict(gate_type=2), dict(gate_kind=3), dict(gate_kind=1), dict(post_eps=-1.0), dict(pre_eps=float("nan")),
               dict(residual_scale=float("inf")), dict(branch_scale=float("nan")), dict(gain_offset=float("nan")),
               dict(h_ld=7), dict(y_ld=7), dict(h_out_ld=7), dict(x_ld=7), dict(gate_kind=2, gate=A, gate_ld=7),
               dict(gate_kind=1, gate=A, gate_ld=0), dict(y=0, post_norm=1), dict(y=0, gate_kind=1, gate=A),
               dict(y=0, channel_scale=A), dict(post_gain=A), dict(x=0, pre_gain=A), dict(h_out=0, x=0)):
        assert f(**kw) == E["INVALID_ARG"], kw
    assert f(D=bm.BLOCK_NORM_MAX_D + 1, h_ld=1 << 20, y_ld=1 << 20, h_out_ld=1 << 20, x_ld=1 << 20) == E["SHAPE"]
    assert f(T=(1 << 24) + 1) == E["SHAPE"]
    for kw in (dict(h=A + 2), dict(y=A + 2), dict(x=A + 2), dict(h_out=A + 2), dict(pre_gain=A + 2),
               dict(h_type=1, h=A + 1), dict(gate_kind=1, gate=A + 2), dict(channel_scale=A + 2),
               dict(post_norm=1, post_gain=A + 2)):
        assert f(**kw) == E["ALIGNMENT"], kw


def test_align_refusals(bm):
    E, A, f = bm.ERR_CODE, 1 << 20, bm._lib().bitsmoe_microscale_align
    for args in ((A, 8, -1, 8, A, 8, None), (A, 8, 1, 0, A, 8, None), (A, 7, 1, 8, A, 8, None), (A, 9, 1, 9, A, 8, None),
                 (A, 9, 1, 9, A, 12, None), (None, 8, 1, 8, A, 8, None), (A, 8, 1, 8, None, 8, None)):
        assert f(*args) == E["INVALID_ARG"], args
    assert f(A, 8, (1 << 24) + 1, 8, A, 8, None) == E["SHAPE"]
    assert f(A, 1 << 21, 1, (1 << 20) + 1, A, 1 << 21, None) == E["SHAPE"]
    assert f(A + 1, 8, 1, 8, A, 8, None) == E["ALIGNMENT"] and f(A, 8, 1, 8, A + 8, 8, None) == E["ALIGNMENT"]
    assert f(None, 8, 0, 8, None, 8, None) == bm.OK


def test_torch_wrappers_refuse_before_the_library(bm):
    torch = pytest.importorskip("torch")
    codes = torch.zeros(4, 32, dtype=torch.uint8)
    q = bm.Microscale.from_rows(codes, torch.zeros(4, 2, dtype=torch.uint8), 64, "e8m0")
    with pytest.raises(bm.BitsMoEError):   # host memory
        bm.microscale_product(q, torch.zeros(1, 64, dtype=torch.bfloat16))
    with pytest.raises(bm.BitsMoEError):
        bm.microscale_quantize(torch.zeros(2, 64))
    with pytest.raises(bm.BitsMoEError):
        bm.block_norm(torch.zeros(2, 64))
    with pytest.raises(bm.BitsMoEError):
        bm.Microscale(codes.view(-1)[:-1], q.scales, 4, 64)
    with pytest.raises(bm.BitsMoEError):
        bm.Microscale.from_rows(codes, torch.zeros(4, 3, dtype=torch.uint8), 64, "e8m0")


@pytest.mark.parametrize("fmt", ["e8m0", "e4m3"])
def test_from_rows_stores_the_documented_layout(bm, fmt):
    torch = pytest.importorskip("torch")
    rng = np.random.default_rng(3)
    for rows, cols in ((1, 1), (3, 33), (130, 200), (257, 513)):
        c = rng.integers(0, 16, (rows, cols)).astype(np.uint8)
        s = rng.integers(0, 127, (rows, -(-cols // om.BLOCK[fmt]))).astype(np.uint8)
        p = np.pad(c, ((0, 0), (0, cols % 2)))
        packed = p[:, 0::2] | (p[:, 1::2] << 4)
        if cols % 2:
            packed[:, -1] |= 0xF0              # what lies past the last column is not stored
        q = bm.Microscale.from_rows(torch.from_numpy(packed), torch.from_numpy(s), cols, fmt)
        np.testing.assert_array_equal(q.codes.numpy().reshape(rows, -1), om.pack_codes(c))
        np.testing.assert_array_equal(q.scales.numpy(), om.tile_scales(s))
        np.testing.assert_array_equal(q.block_scales().numpy(), s)


def test_oracle_against_the_definitions():
    """Known values: the E4M3 extremes, a block whose largest element is on each side of a power of two,
    ties to even, saturation."""
    assert om.E4M3[126] == 448 and om.E4M3[1] == 2.0 ** -9 and om.E4M3[8] == 2.0 ** -6 and om.E4M3[56] == 1.0
    x = np.zeros((1, 32), np.float32)
    x[0, :9] = [4.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, -5.0, 7.9]
    c, s = om.quantize(x, "e8m0", 1.0)
    assert s[0, 0] == 127
    assert list(c[0, :9]) == [6, 0, 2, 2, 4, 4, 6, 14, 7]     # 5 lies between 4 and 6: the even index is 4's
    x[0, 8] = 8.0
    c, s = om.quantize(x, "e8m0", 1.0)
    assert s[0, 0] == 128 and c[0, 8] == 6
    c, s = om.quantize(np.full((1, 16), 6.0 * 448 * 4, np.float32), "e4m3", 1.0)
    assert s[0, 0] == 126 and (c == 7).all()
    np.testing.assert_array_equal(om.values(c, s, "e4m3", 0.5), np.full((1, 16), 1344.0))


def test_sources_name_no_multicast():
    """The library also runs as replicas on several GPUs, where no load or arrival is spread over a cluster."""
    import os
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    for folder in ("paper_2606_00079_gb300/csrc", "include"):
        for name in sorted(os.listdir(os.path.join(root, folder))):
            with open(os.path.join(root, folder, name), encoding="utf-8") as f:
                assert "multicast" not in f.read(), name


def test_product_refuses_tensor_scales_whose_product_leaves_the_range(bm):
    """Both scales alone are in the quantiser's range; the sums times their product would be 0 inf or lost."""
    E = bm.ERR_CODE

    def f(sw, su, sx, T=3):
        w, u = micro(bm, scale=sw), micro(bm, scale=su)
        return bm._lib().bitsmoe_microscale_product(w, u, 0, 0, micro(bm, rows=T, scale=sx), T, A, 0, 4, 0, 0)
    for bad in ((2.0 ** 100, 1.0, 2.0 ** 100), (1.0, 2.0 ** 64, 2.0 ** 64), (2.0 ** -100, 1.0, 2.0 ** -100), (1.0, 2.0 ** -27, 2.0 ** -100)):
        assert f(*bad) == E["INVALID_ARG"], bad
    for good in ((2.0 ** 100, 2.0 ** -100, 2.0 ** 27), (2.0 ** -26, 1.0, 2.0 ** -100), (3e38, 1e-37, 1.0)):
        assert f(*good, T=0) == 0, good


def test_wrappers_do_without_torch_internals(bm, monkeypatch):
    """Where torch lacks the fast forms of the current device and stream, its public ones are used."""
    torch = pytest.importorskip("torch")
    for name in ("_torch", "_DENSE", "_raw_stream", "_current"):
        monkeypatch.setattr(bm, name, getattr(bm, name))
    for name in ("_cuda_getDevice", "_cuda_getCurrentRawStream"):
        monkeypatch.delattr(torch._C, name, raising=False)
    bm._load_torch()
    assert bm._current is torch.cuda.current_device
    monkeypatch.setattr(torch.cuda, "current_stream", lambda i: type("S", (), {"cuda_stream": 40 + i}))
    assert bm._raw_stream(2) == 42
