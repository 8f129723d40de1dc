"""The dense 4-bit operators and the norms between blocks, as single passes that a serving program makes:
their plain forms in torch and the library's calls, with their inputs, their work and their 64-bit values.

A case is a dict of plain values; its "kind" says which operator it goes through:

  quantize  rows -> microscaled 4-bit codes and block scales, and back to the values they stand for
  product   y = x W^T with W in 4 bits, x in bf16 or in 4 bits; "glu": silu(x Wg^T) * (x Wu^T)
  norm      post-norm of a block's output, its gate and scales, the residual sum, and the next pre-norm

A 4-bit matrix is (codes, scales): codes uint8 [rows][16 ceil(cols / 32)], two E2M1 codes a byte, the lower
column in the lower half; scales one byte for each block of 32 (format "e8m0") or 16 ("e4m3") columns, in
tiles of 128 rows x 4 blocks: byte ((r / 128) ceil(blocks / 4) + b / 4) 512 + (r % 32) 16 + (r % 128 / 32) 4
+ b % 4 for block b of row r.
"""
import math

import numpy as np
import torch
import torch.nn.functional as F

own = False

BLOCK = {"e8m0": 32, "e4m3": 16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
EPS = 1e-6


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def _quantize(name, rows, cols, fmt, dtype):
    return dict(name=name, kind="quantize", rows=rows, cols=cols, fmt=fmt, dtype=dtype)


def _product(name, T, rows, cols, fmt, x, out, glu=False):
    return dict(name=name, kind="product", T=T, rows=rows, cols=cols, fmt=fmt, x=x, out=out, glu=glu)


def _norm(name, T, D, h, y, post, gate, channel):
    return dict(name=name, kind="norm", T=T, D=D, h=h, y=y, post=post, gate=gate, channel=channel)


def listed():
    return [
        # activations of a decode batch, before a product that reads them in 4 bits
        _quantize("quantize_T32", 32, 2048, "e4m3", "bf16"),
        # a dense matrix of a large layer, quantised once from its float weights
        _quantize("quantize_matrix", 14336, 4096, "e8m0", "f32"),
        # one token through a large down projection
        _product("product_T1", 1, 4096, 14336, "e8m0", "bf16", "f32"),
        # a batch and sizes that are multiples of nothing
        _product("product_odd_T37", 37, 1001, 2041, "e4m3", "bf16", "f32"),
        # prefill of a prompt with 16-bit activations
        _product("product_T4096", 4096, 14336, 4096, "e4m3", "bf16", "bf16"),
        # small decode batch with 4-bit activations
        _product("coded_T8", 8, 14336, 4096, "e4m3", "fp4", "f32"),
        # prefill of long prompts with 4-bit activations, the largest call
        _product("coded_T8192", 8192, 14336, 4096, "e4m3", "fp4", "bf16"),
        # gate and up of a shared expert with their activation, decode batch
        _product("swiglu_T16", 16, 14336, 4096, "e8m0", "bf16", "bf16", True),
        # the same of a small expert at a prompt's length, 4-bit activations
        _product("swiglu_coded_T1024", 1024, 768, 2048, "e8m0", "fp4", "bf16", True),
        # between two blocks for one token: post-norm, a gate for the token, residual, pre-norm
        _norm("norm_T1", 1, 2048, "f32", "f32", True, "token", False),
        # an odd width and batch, 16-bit residual, a gate for each element, no post-norm
        _norm("norm_odd_T77", 77, 2050, "bf16", "bf16", False, "element", True),
        # the same point of a long prefill: post-norm and a scale for each channel
        _norm("norm_T16384", 16384, 4096, "f32", "f32", True, "none", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["quantize", "quantize", "product", "product", "product", "coded", "coded", "coded", "norm", "norm"])
    fmt = rng.choice(["e8m0", "e4m3"])
    if kind == "norm":
        D = _log(rng, 64, 8192)
        return dict(kind=kind, T=_log(rng, 1, min(16384, 16384 * 4096 // D)), D=D, h=rng.choice(["f32", "bf16"]),
                    y=rng.choice(["f32", "bf16"]), post=rng.random() < 0.6,
                    gate=rng.choice(["none", "token", "element"]), channel=rng.random() < 0.5)
    rows = _log(rng, 64, 14336)
    cols = _log(rng, 64, 14336)
    if rng.random() < 0.5:   # sizes as models have them; the others are odd
        rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
    if kind == "quantize":
        return dict(kind=kind, rows=min(rows, 14336 * 4096 // cols), cols=cols, fmt=fmt, dtype=rng.choice(["f32", "bf16"]))
    rows = min(rows, 14336 * 4096 // cols)
    glu = rng.random() < 0.35
    if glu:
        rows = max(32, rows // 2)
    most = (8192 if kind == "coded" else 4096) * 14336 * 4096 // (rows * cols * (2 if glu else 1))
    return dict(kind="product", T=_log(rng, 1, min(8192, most)), rows=rows, cols=cols, fmt=fmt,
                x="fp4" if kind == "coded" else "bf16", out=rng.choice(["f32", "bf16"]), glu=glu)


# --------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------
def _tile(s):
    """Block scales [rows][blocks] (uint8) in the stored order, zeros where a tile has no block."""
    r, b = s.shape
    s = F.pad(s, (0, -b % 4, 0, -r % 128))
    return s.view(s.shape[0] // 128, 4, 32, s.shape[1] // 4, 4).permute(0, 3, 2, 1, 4).reshape(-1)


def _untile(s, rows, blocks):
    t = s.view((rows + 127) // 128, (blocks + 3) // 4, 32, 4, 4).permute(0, 3, 2, 1, 4)
    return t.reshape((rows + 127) // 128 * 128, (blocks + 3) // 4 * 4)[:rows, :blocks]


def _scale_values(dev, fmt):
    """The 256 values of a scale byte in fp32 (the last of e8m0, and 127 of e4m3, are NaN)."""
    if fmt == "e4m3":
        return torch.arange(256, device=dev).to(torch.uint8).view(torch.float8_e4m3fn).float()
    v = torch.exp2(torch.arange(256, device=dev, dtype=torch.float64) - 127.0)
    v[255] = math.nan
    return v.float()


def _encode(x, fmt, s):
    """Codes (0..15, one a byte) and scale bytes of the rows of x (fp32); s is a power of two."""
    blk = BLOCK[fmt]
    v = F.pad(x.float() / s, (0, -x.shape[1] % blk)).view(x.shape[0], -1, blk)
    a = v.abs()
    top = a.amax(2)
    if fmt == "e8m0":
        e = (torch.frexp(top).exponent - 3).clamp(-127, 125)
        e = torch.where(top > 0, e, torch.full_like(e, -127))
        scale = torch.exp2(e.double()).float()
        byte = (e + 127).to(torch.uint8)
    else:
        q = (top / 6.0).clamp(max=448.0).to(torch.float8_e4m3fn)
        scale, byte = q.float(), q.view(torch.uint8)
    m = scale.unsqueeze(2)
    c = ((a > 0.25 * m).to(torch.uint8) + (a >= 0.75 * m) + (a > 1.25 * m) + (a >= 1.75 * m) + (a > 2.5 * m)
         + (a >= 3.5 * m) + (a > 5.0 * m)) * (m > 0)
    return (c + 8 * torch.signbit(v).to(torch.uint8)).view(x.shape[0], -1), byte


def _store(codes, byte, cols):
    c = F.pad(codes[:, :cols], (0, -cols % 32))
    return (c[:, 0::2] | (c[:, 1::2] << 4)).contiguous(), _tile(byte)


def _decode(codes, scales, rows, cols, fmt, s):
    """fp32 values [rows][cols] of a stored matrix."""
    blk = BLOCK[fmt]
    nb = (cols + blk - 1) // blk
    grid = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    q = torch.stack((codes & 15, codes >> 4), 2).view(rows, -1)[:, :nb * blk]
    m = _scale_values(codes.device, fmt)[_untile(scales, rows, nb).long()]
    v = grid[q.int()].view(rows, nb, blk) * m.unsqueeze(2)
    return v.view(rows, -1)[:, :cols] * s


def _run_plain(c, s):
    if c["kind"] == "quantize":
        codes, byte = _encode(s["x"], c["fmt"], s["s"])
        return _decode(*_store(codes, byte, c["cols"]), c["rows"], c["cols"], c["fmt"], s["s"])
    if c["kind"] == "product":
        x = s["x"].float() if c["x"] == "bf16" else _decode(*s["x"], c["T"], c["cols"], c["fmt"], s["xs"])
        y = x @ _decode(*s["w"], c["rows"], c["cols"], c["fmt"], s["ws"]).t()
        if c["glu"]:
            u = x @ _decode(*s["up"], c["rows"], c["cols"], c["fmt"], s["us"]).t()
            y = y / (1.0 + torch.exp(-y)) * u
        return y.to(TYPE[c["out"]])
    h, y = s["h"].float(), s["y"].float()
    if c["post"]:
        y = y * torch.rsqrt((y * y).mean(1, keepdim=True) + EPS) * s["post"].float()
    if c["gate"] == "token":
        y = y / (1.0 + torch.exp(-s["gate"].float().unsqueeze(1)))
    elif c["gate"] == "element":
        y = y * s["gate"].float()
    if c["channel"]:
        y = y * s["channel"].float()
    h = 0.875 * h + 0.5 * y
    x = h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["pre"].float()
    return {"h": h.to(TYPE[c["h"]]), "x": x.to(torch.bfloat16)}


# --------------------------------------------------------------------------
# the library's calls
# --------------------------------------------------------------------------
def _run_own(c, s):
    import paper_2606_00079_gb300 as bm
    if c["kind"] == "quantize":
        return bm.microscale_dequantize(bm.microscale_quantize(s["x"], c["fmt"], s["s"]))
    if c["kind"] == "product":
        w = bm.Microscale(*s["w"], c["rows"], c["cols"], c["fmt"], s["ws"])
        up = bm.Microscale(*s["up"], c["rows"], c["cols"], c["fmt"], s["us"]) if c["glu"] else None
        x = s["x"] if c["x"] == "bf16" else bm.Microscale(*s["x"], c["T"], c["cols"], c["fmt"], s["xs"])
        return bm.microscale_product(w, x, up=up, dtype=TYPE[c["out"]])
    h, x = bm.block_norm(s["h"], s["y"], post_norm=c["post"], post_gain=s["post"] if c["post"] else None, post_eps=EPS,
                         gate=s["gate"], gate_sigmoid=c["gate"] == "token", channel_scale=s["channel"],
                         branch_scale=0.5, residual_scale=0.875, pre_gain=s["pre"], pre_eps=EPS)
    return {"h": h, "x": x}


def run(state):
    c = state["case"]
    return _run_own(c, state) if own else _run_plain(c, state)


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------
def _gen(*key):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(np.random.SeedSequence([abs(int(k)) for k in key]).generate_state(1)[0]))
    return g


def _acts(g, T, D):
    """Activations: normal, a few channels much larger, the last row of a batch all zeros (a padded token)."""
    x = torch.randn(T, D, generator=g, device="cuda")
    big = torch.rand(D, generator=g, device="cuda") < 0.01
    x = torch.where(big, 12.0 * x, x)
    if T > 2:
        x[-1] = 0.0
    return x


def _weights(g, R, K):
    """Weights of a dense projection: normal over sqrt(K), rows of unequal norms."""
    return torch.randn(R, K, generator=g, device="cuda") * (0.5 + torch.rand(R, 1, generator=g, device="cuda")) / math.sqrt(K)


def _tensor_scale(x, fmt):
    """The power of two that brings the largest block scale of e4m3 just under its largest value."""
    if fmt == "e8m0":
        return 1.0
    return 2.0 ** math.ceil(math.log2(max(float(x.abs().max()), 1e-30) / (6.0 * 448.0)))


def _coded(x, fmt):
    s = _tensor_scale(x, fmt)
    codes, byte = _encode(x, fmt, s)
    return _store(codes, byte, x.shape[1]), s


def prepare(case, seed):
    c = case
    g = _gen(seed, sum(ord(ch) * (i + 1) for i, ch in enumerate(c["kind"])), c.get("T", 0), c.get("rows", 0), c.get("cols", 0))
    s = {"case": c}
    if c["kind"] == "quantize":
        x = _weights(g, c["rows"], c["cols"]) if c["dtype"] == "f32" else _acts(g, c["rows"], c["cols"])
        s["x"] = x.to(TYPE[c["dtype"]])
        s["s"] = _tensor_scale(s["x"], c["fmt"])
    elif c["kind"] == "product":
        s["w"], s["ws"] = _coded(_weights(g, c["rows"], c["cols"]), c["fmt"])
        if c["glu"]:
            s["up"], s["us"] = _coded(_weights(g, c["rows"], c["cols"]), c["fmt"])
        x = _acts(g, c["T"], c["cols"]).to(torch.bfloat16)
        if c["x"] == "bf16":
            s["x"] = x
        else:
            s["x"], s["xs"] = _coded(x, c["fmt"])
    else:
        T, D = c["T"], c["D"]
        s["h"] = (3.0 * _acts(g, T, D)).to(TYPE[c["h"]])
        s["y"] = _acts(g, T, D).to(TYPE[c["y"]])
        gain = 1.0 + 0.2 * torch.randn(3, D, generator=g, device="cuda")
        s["post"], s["pre"] = gain[0].to(torch.bfloat16), gain[1].to(torch.bfloat16)
        s["channel"] = gain[2].to(torch.bfloat16) if c["channel"] else None
        s["gate"] = None
        if c["gate"] == "token":
            s["gate"] = torch.randn(T, generator=g, device="cuda")
        elif c["gate"] == "element":
            s["gate"] = torch.rand(T, D, generator=g, device="cuda").to(TYPE[c["y"]])
    return s


# --------------------------------------------------------------------------
# work and values
# --------------------------------------------------------------------------
def _size(dtype):
    return 2 if dtype == "bf16" else 4


def work(case):
    c = case
    if c["kind"] == "norm":
        n = c["T"] * c["D"]
        vec = 1 + int(c["post"]) + int(c["channel"])
        gate = {"none": 0, "token": 4 * c["T"], "element": n * _size(c["y"])}[c["gate"]]
        return {"bytes": n * (2 * _size(c["h"]) + _size(c["y"]) + 2) + 2 * vec * c["D"] + gate, "flops": 12 * n}

    def coded(rows):
        return rows * ((c["cols"] + 1) // 2 + (c["cols"] + BLOCK[c["fmt"]] - 1) // BLOCK[c["fmt"]])

    if c["kind"] == "quantize":
        n = c["rows"] * c["cols"]
        return {"bytes": n * _size(c["dtype"]) + coded(c["rows"]) + 4 * n, "flops": 8 * n}
    mats = 2 if c["glu"] else 1
    x = 2 * c["T"] * c["cols"] if c["x"] == "bf16" else coded(c["T"])
    return {"bytes": mats * coded(c["rows"]) + x + c["T"] * c["rows"] * _size(c["out"]),
            "flops": 2 * mats * c["T"] * c["rows"] * c["cols"]}


def _exact_values(stored, rows, cols, fmt, s):
    """A stored matrix in 64 bits: the codes' fields taken apart, the scale bytes fetched by the layout's formula."""
    codes, scales = stored
    r = torch.arange(rows, device=codes.device).unsqueeze(1)
    k = torch.arange(cols, device=codes.device).unsqueeze(0)
    n = (codes[:, :(cols + 1) // 2].unsqueeze(2) >> torch.tensor([0, 4], device=codes.device, dtype=torch.uint8)) & 15
    n = n.reshape(rows, -1)[:, :cols].to(torch.int32)
    e, m = (n >> 1) & 3, n & 1
    v = torch.where(e > 0, (2 + m).double() * torch.exp2(e.double() - 2.0), m.double() * 0.5)
    v = torch.where(n >= 8, -v, v)
    del n, e, m
    blk = BLOCK[fmt]
    b = torch.arange((cols + blk - 1) // blk, device=codes.device).unsqueeze(0)
    tiles = (b.shape[1] + 3) // 4
    byte = scales[((r // 128) * tiles + b // 4) * 512 + (r % 32) * 16 + (r % 128 // 32) * 4 + b % 4].to(torch.int32)
    if fmt == "e8m0":
        sc = torch.exp2(byte.double() - 127.0)
    else:
        f, p = byte & 7, byte >> 3
        sc = torch.where(p > 0, (8 + f).double() * torch.exp2(p.double() - 10.0), f.double() * 2.0 ** -9)
    return v * sc.gather(1, (k // blk).expand(rows, cols)) * s


def _half_even(v, step):
    return torch.round(v / step) * step


def _exact_quantize(x, fmt, s):
    x = x.double() / s
    blk = BLOCK[fmt]
    rows, cols = x.shape
    nb = (cols + blk - 1) // blk
    v = torch.zeros(rows, nb * blk, dtype=torch.float64, device=x.device)
    v[:, :cols] = x
    v = v.view(rows, nb, blk)
    top = v.abs().amax(2, keepdim=True)
    if fmt == "e8m0":
        sc = torch.exp2(torch.clamp(torch.floor(torch.log2(top.clamp(min=2.0 ** -140))) - 2.0, min=-127.0))
    else:
        a = top / 6.0
        step = torch.exp2(torch.floor(torch.log2(a.clamp(min=2.0 ** -6))) - 3.0)
        sc = _half_even(a, step).clamp(max=448.0)
    w = torch.where(sc > 0, v / sc.clamp(min=2.0 ** -140), torch.zeros_like(v))
    m = w.abs()
    step = torch.where(m < 2.0, 0.5, torch.where(m < 4.0, 1.0, 2.0))
    q = _half_even(m, step).clamp(max=6.0)
    return (torch.copysign(q, v) * sc).view(rows, -1)[:, :cols] * s


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "quantize":
        return _exact_quantize(s["x"], c["fmt"], s["s"])
    if c["kind"] == "product":
        x = s["x"].double() if c["x"] == "bf16" else _exact_values(s["x"], c["T"], c["cols"], c["fmt"], s["xs"])
        y = torch.matmul(x, _exact_values(s["w"], c["rows"], c["cols"], c["fmt"], s["ws"]).t())
        if c["glu"]:
            y = y * torch.sigmoid(y) * torch.matmul(x, _exact_values(s["up"], c["rows"], c["cols"], c["fmt"], s["us"]).t())
        return y
    h, y = s["h"].double(), s["y"].double()
    if c["post"]:
        y = y / torch.sqrt(y.pow(2).sum(1, keepdim=True) / c["D"] + EPS) * s["post"].double()
    if c["gate"] != "none":
        y = y * (torch.sigmoid(s["gate"].double())[:, None] if c["gate"] == "token" else s["gate"].double())
    if c["channel"]:
        y = y * s["channel"].double()
    h = 0.875 * h + 0.5 * y
    return {"h": h, "x": h / torch.sqrt(h.pow(2).sum(1, keepdim=True) / c["D"] + EPS) * s["pre"].double()}
