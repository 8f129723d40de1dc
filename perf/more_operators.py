"""The operators around experts that are dense matrices, as single passes that a serving program makes: their plain
forms in torch and the library's calls, with their inputs, their work and their 64-bit values.

A case is a dict of plain values; its "kind" says which operator it goes through:

  rows8    rows -> 8-bit codes (E4M3) with a power-of-two scale a row, and back to the values they stand for
  norm8    post-norm of a block's output, its gate and scales, the residual sum, the next pre-norm, in 8 bits
  route    router logits -> each token's experts and weights, and the pairs (token, expert) in the experts' order
  experts  y[p] = W_e x of the rows that each expert has, ragged; "glu": silu(Wg_e x) * (Wu_e x); 16 or 8 bits
  combine  the weighted sum of each token's rows

Rows in 8 bits are (codes, scales): torch.float8_e4m3fn on a pitch of a multiple of 16, a fp32 scale a row;
value = code * scale.  Pairs: pair t * k + j is token t's j-th expert; the pairs in the order of their experts (and
by number within one) are the rows that the experts take, `offsets` where each expert's begin.  A token that routes
nowhere (padding: its logits are all -inf) has expert -1, weight 0 and place -1.
"""
import math

import numpy as np
import torch
import torch.nn.functional as F

own = False

TYPE = {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}
EPS = 1e-6


# --------------------------------------------------------------------------
# cases
# --------------------------------------------------------------------------
def _rows8(name, rows, cols, dtype):
    return dict(name=name, kind="rows8", rows=rows, cols=cols, dtype=dtype)


def _norm8(name, T, D, h, y, post, gate, channel):
    return dict(name=name, kind="norm8", T=T, D=D, h=h, y=y, post=post, gate=gate, channel=channel)


def _route(name, T, E, k, renorm):
    return dict(name=name, kind="route", T=T, E=E, k=k, renorm=renorm)


def _experts(name, T, E, k, rows, cols, dtype, out, glu, gather):
    return dict(name=name, kind="experts", T=T, E=E, k=k, rows=rows, cols=cols, dtype=dtype, out=out, glu=glu, gather=gather)


def _combine(name, T, k, D, y, out, base):
    return dict(name=name, kind="combine", T=T, k=k, D=D, y=y, out=out, base=base)


def listed():
    return [
        # activations of a decode batch, before a product that reads them in 8 bits
        _rows8("rows8_T32", 32, 2048, "bf16"),
        # a dense matrix of a large layer, coded once from its float weights
        _rows8("rows8_matrix", 14336, 4096, "f32"),
        # between two blocks of a small batch of an odd width, 16-bit residual, gates for each element
        _norm8("norm8_odd_T77", 77, 2050, "bf16", "bf16", False, "element", True),
        # the same point of a long prefill: post-norm and a scale for each channel
        _norm8("norm8_T16384", 16384, 4096, "f32", "f32", True, "none", True),
        # one token among 128 experts
        _route("route_T1", 1, 128, 8, True),
        # a long prefill's routing
        _route("route_T16384", 16384, 128, 8, True),
        # one token through gate and up of its eight experts
        _experts("swiglu_T1", 1, 128, 8, 768, 2048, "bf16", "bf16", True, True),
        # a decode batch through the down matrices in 8 bits
        _experts("down8_T32", 32, 128, 8, 2048, 768, "e4m3", "bf16", False, False),
        # a long prefill through gate and up of small experts, 512 rows each on average
        _experts("swiglu_T8192", 8192, 128, 8, 768, 2048, "bf16", "bf16", True, True),
        # a prefill through a matrix of large experts in 8 bits
        _experts("gate8_T4096", 4096, 8, 2, 14336, 4096, "e4m3", "bf16", False, True),
        # the end of a decode batch's block, an odd width
        _combine("combine_odd_T37", 37, 8, 2050, "bf16", "f32", False),
        # the end of a long prefill's block, added to the shared expert's output
        _combine("combine_T8192", 8192, 8, 2048, "bf16", "bf16", True),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rows8", "norm8", "route", "experts", "experts", "experts", "combine"])
    if kind == "rows8":
        cols = _log(rng, 64, 14336)
        return dict(kind=kind, rows=_log(rng, 1, min(65536, 14336 * 4096 // cols)), cols=cols, dtype=rng.choice(["f32", "bf16"]))
    if kind == "norm8":
        D = _log(rng, 64, 8192)
        return dict(kind=kind, T=_log(rng, 1, min(16384, 16384 * 4096 // D)), D=D, h=rng.choice(["f32", "bf16"]),
                    y=rng.choice(["f32", "bf16"]), post=rng.random() < 0.6,
                    gate=rng.choice(["none", "token", "element"]), channel=rng.random() < 0.5)
    if kind == "route":
        E = _log(rng, 2, 1024)
        return dict(kind=kind, T=_log(rng, 1, min(65536, 16384 * 512 // E)), E=E, k=_log(rng, 1, min(16, E)), renorm=rng.random() < 0.7)
    if kind == "combine":
        D, k = _log(rng, 64, 8192), _log(rng, 1, 16)
        return dict(kind=kind, T=_log(rng, 1, min(16384, 8192 * 8 * 2048 // (D * k))), k=k, D=D, y=rng.choice(["f32", "bf16"]),
                    out=rng.choice(["f32", "bf16"]), base=rng.random() < 0.5)
    E = _log(rng, 1, 256)
    glu = rng.random() < 0.5
    mats = 2 if glu else 1
    most = 8 * 14336 * 4096 // (E * mats)   # elements of a matrix
    cols = _log(rng, 64, min(14336, most // 64))
    rows = _log(rng, 64, min(14336, most // cols))
    if rng.random() < 0.5:   # sizes as models have them; the others are odd
        rows, cols = max(64, rows // 64 * 64), max(64, cols // 64 * 64)
    k = _log(rng, 1, min(8, E))
    return dict(kind=kind, T=_log(rng, 1, max(1, min(8192, 8192 * 14336 * 4096 // (k * rows * cols * mats)))), E=E, k=k, rows=rows,
                cols=cols, dtype=rng.choice(["bf16", "e4m3"]), out=rng.choice(["bf16", "bf16", "f32"]), glu=glu,
                gather=rng.random() < 0.6)


# --------------------------------------------------------------------------
# plain forms
# --------------------------------------------------------------------------
def _encode(x):
    """E4M3 codes and scales of the rows of x (fp32)."""
    m, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(m > 0, e - 9 + (m > 0.875).int(), torch.full_like(e, -100)).clamp(min=-100)
    s = torch.exp2(e.double())
    return (x.double() / s).float().to(torch.float8_e4m3fn), s.float().squeeze(-1)


def _norm_plain(c, s):
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
    codes, scale = _encode(h * torch.rsqrt((h * h).mean(1, keepdim=True) + EPS) * s["pre"].float())
    return {"h": h.to(TYPE[c["h"]]), "x": (codes.float() * scale.unsqueeze(1)).to(torch.bfloat16)}


def _lists(experts, E):
    """Offsets, the pairs in the experts' order (-1 behind them) and each pair's place (-1: none)."""
    T, k = experts.shape
    key = torch.where(experts < 0, E, experts).view(-1).long()
    order = torch.sort(key, stable=True).indices
    count = torch.zeros(E + 1, dtype=torch.int64, device=key.device).scatter_add_(0, key, torch.ones_like(key))
    offsets = F.pad(count[:E].cumsum(0), (1, 0))
    at = torch.arange(T * k, device=key.device)
    here = at < offsets[E]
    place = torch.empty_like(at)
    place[order] = torch.where(here, at, -1)
    return offsets.int(), torch.where(here, order, -1).int(), place.view(T, k).int()


def _route_plain(logits, k, renorm):
    v = torch.where(torch.isnan(logits), -math.inf, logits).float()
    top, at = torch.sort(v, dim=1, descending=True, stable=True)
    top, at = top[:, :k], at[:, :k]
    none = torch.isneginf(top)
    first = top[:, :1].clamp(min=-3e38)
    w = torch.exp(top - first)
    w = torch.where(none, 0.0, w / (w if renorm else torch.exp(v - first)).sum(1, keepdim=True))
    experts = torch.where(none, -1, at).int()
    offsets, pairs, places = _lists(experts, logits.shape[1])
    return {"experts": experts, "weights": w, "offsets": offsets, "pairs": pairs, "places": places}


def _experts_plain(c, s):
    E, M, P = c["E"], s["most"], s["y"].shape[0]
    off = s["offsets"].long()
    p = torch.arange(P, device=off.device)
    e = torch.searchsorted(off[1:].contiguous(), p, right=True)
    here = e < E
    slot = torch.where(here, e * M + p - off[e.clamp(max=E - 1)], E * M)
    x = s["x"].float() * s["xs"].unsqueeze(1) if c["dtype"] == "e4m3" else s["x"].float()
    if c["gather"]:
        x = x[torch.where(here, s["pairs"].long(), 0) // c["k"]]
    pad = torch.zeros(E * M + 1, c["cols"], device=off.device)
    pad[slot] = x
    pad = pad[:E * M].view(E, M, -1)

    def product(w, ws):
        v = w.float() * ws.unsqueeze(2) if c["dtype"] == "e4m3" else w.float()
        return torch.bmm(pad, v.transpose(1, 2)).view(E * M, -1)

    y = product(s["w"], s["ws"])
    if c["glu"]:
        y = y / (1.0 + torch.exp(-y)) * product(s["up"], s["us"])
    return torch.where(here.unsqueeze(1), y[slot.clamp(max=E * M - 1)], 0.0).to(TYPE[c["out"]])


def _combine_plain(c, s):
    here = s["places"] >= 0
    y = s["y"].float()[torch.where(here, s["places"], 0).long()]
    y = (torch.where(here.unsqueeze(2), y, 0.0) * s["weights"].unsqueeze(2)).sum(1)
    return (s["base"].float() + y if c["base"] else y).to(TYPE[c["out"]])


def _run_plain(c, s):
    if c["kind"] == "rows8":
        codes, scale = _encode(s["x"].float())
        return {"values": codes.float() * scale.unsqueeze(1), "scales": scale}
    if c["kind"] == "norm8":
        return _norm_plain(c, s)
    if c["kind"] == "route":
        return _route_plain(s["logits"], c["k"], c["renorm"])
    return _experts_plain(c, s) if c["kind"] == "experts" else _combine_plain(c, s)


# --------------------------------------------------------------------------
# the library's calls
# --------------------------------------------------------------------------
def _run_own(c, s):
    import paper_2606_00079_gb300 as bm
    if c["kind"] == "rows8":
        q = bm.rowscale_quantize(s["x"])
        return {"values": bm.rowscale_dequantize(q), "scales": q.scales}
    if c["kind"] == "norm8":
        h, x = bm.block_norm(s["h"], s["y"], post_norm=c["post"], post_gain=s["post"] if c["post"] else None, post_eps=EPS,
                             gate=s["gate"], gate_sigmoid=c["gate"] == "token", channel_scale=s["channel"],
                             branch_scale=0.5, residual_scale=0.875, pre_gain=s["pre"], pre_eps=EPS, x_dtype=torch.float8_e4m3fn)
        return {"h": h, "x": bm.rowscale_dequantize(x, torch.bfloat16)}
    if c["kind"] == "route":
        r = bm.route(s["logits"], c["k"], renormalize=c["renorm"])
        return {"experts": r.experts, "weights": r.weights, "offsets": r.offsets, "pairs": r.pairs, "places": r.places}
    if c["kind"] == "combine":
        return bm.expert_combine(s["y"], s["places"], s["weights"], base=s["base"], dtype=TYPE[c["out"]])
    w, up, x = s["w"], s["up"], s["x"]
    if c["dtype"] == "e4m3":
        w, x = bm.Rowscale(w, s["ws"]), bm.Rowscale(x, s["xs"])
        up = bm.Rowscale(up, s["us"]) if c["glu"] else None
    return bm.expert_product(w, x, s["offsets"], index=s["pairs"] if c["gather"] else None, fan=c["k"] if c["gather"] else 1, up=up, y=s["y"])


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


def _pitch(x, n):
    """x with its rows on a pitch of a multiple of n elements."""
    out = torch.zeros(*x.shape[:-1], (x.shape[-1] + n - 1) // n * n, dtype=x.dtype, device=x.device)[..., :x.shape[-1]]
    return out.copy_(x)


def _stored(x, dtype):
    """Rows as they are kept: bf16, or codes; with the codes' scales."""
    if dtype == "bf16":
        return _pitch(x.to(torch.bfloat16), 8), None
    codes, scale = _encode(x)
    return _pitch(codes, 16), scale


def _logits(g, T, E):
    """Router logits: some experts likelier than others, an expert out of use here and there (-inf), equal values (they
    come from 16 bits), and a padded token, which routes nowhere, at the end of a batch."""
    v = torch.randn(T, E, generator=g, device="cuda") + 0.5 * torch.randn(E, generator=g, device="cuda")
    v = v.to(torch.bfloat16).float()
    if E > 8:
        v = torch.where(torch.rand(E, generator=g, device="cuda") < 0.02, -math.inf, v)
    if T > 2:
        v[-1] = -math.inf
    return v


def prepare(case, seed):
    c = case
    g = _gen(seed, sum(ord(ch) * (i + 1) for i, ch in enumerate(c["kind"])), c.get("T", 0), c.get("rows", 0), c.get("cols", 0))
    s = {"case": c}
    if c["kind"] == "rows8":
        x = _weights(g, c["rows"], c["cols"]) if c["dtype"] == "f32" else _acts(g, c["rows"], c["cols"])
        s["x"] = x.to(TYPE[c["dtype"]])
    elif c["kind"] == "norm8":
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
    elif c["kind"] == "route":
        s["logits"] = _logits(g, c["T"], c["E"])
    elif c["kind"] == "combine":
        T, k, D = c["T"], c["k"], c["D"]
        r = _route_plain(_logits(g, T, 4 * k), k, True)
        s["places"], s["weights"] = r["places"], r["weights"]
        s["y"] = torch.randn(T * k, D, generator=g, device="cuda").to(TYPE[c["y"]])
        s["base"] = torch.randn(T, D, generator=g, device="cuda").to(TYPE[c["out"]]) if c["base"] else None
    else:
        T, E, k = c["T"], c["E"], c["k"]
        r = _route_plain(_logits(g, T, E), k, True)
        s["offsets"], s["pairs"] = r["offsets"], r["pairs"]
        s["most"] = max(1, int(torch.diff(r["offsets"]).max()))
        for name, scales in (("w", "ws"), ("up", "us")):
            s[name] = s[scales] = None
            if name == "w" or c["glu"]:
                s[name], s[scales] = _stored(_weights(g, E * c["rows"], c["cols"]).view(E, c["rows"], -1), c["dtype"])
        s["x"], s["xs"] = _stored(_acts(g, T if c["gather"] else T * k, c["cols"]), c["dtype"])
        s["y"] = torch.zeros(T * k, c["rows"], dtype=TYPE[c["out"]], device="cuda")   # rows behind the last expert's stay
    return s


# --------------------------------------------------------------------------
# work and values
# --------------------------------------------------------------------------
def _size(dtype):
    return {"e4m3": 1, "bf16": 2, "f32": 4}[dtype]


def work(case):
    c = case
    if c["kind"] == "rows8":
        n = c["rows"] * c["cols"]
        return {"bytes": n * (_size(c["dtype"]) + 1 + 4) + 4 * c["rows"], "flops": 4 * n}
    if c["kind"] == "norm8":
        n = c["T"] * c["D"]
        vec = 1 + int(c["post"]) + int(c["channel"])
        gate = {"none": 0, "token": 4 * c["T"], "element": n * _size(c["y"])}[c["gate"]]
        return {"bytes": n * (2 * _size(c["h"]) + _size(c["y"]) + 1 + 2) + 4 * c["T"] + 2 * vec * c["D"] + gate, "flops": 16 * n}
    if c["kind"] == "route":
        return {"bytes": 4 * c["T"] * c["E"] + 16 * c["T"] * c["k"] + 4 * c["E"] + 4, "flops": 4 * c["T"] * c["E"]}
    if c["kind"] == "combine":
        n = c["T"] * c["D"]
        return {"bytes": n * (c["k"] * _size(c["y"]) + (1 + int(c["base"])) * _size(c["out"])) + 8 * c["T"] * c["k"], "flops": 2 * n * c["k"]}
    mats = 2 if c["glu"] else 1
    P = c["T"] * c["k"]
    active = c["E"] * (1.0 - (1.0 - c["k"] / c["E"]) ** c["T"])   # of evenly liked experts
    matrix = c["rows"] * c["cols"] * _size(c["dtype"]) + (4 * c["rows"] if c["dtype"] == "e4m3" else 0)
    x = (c["T"] if c["gather"] else P) * c["cols"] * _size(c["dtype"])
    return {"bytes": mats * active * matrix + x + P * c["rows"] * _size(c["out"]), "flops": 2.0 * mats * P * c["rows"] * c["cols"]}


def _exact_coded(x):
    """The values of rows in 8 bits, in 64: steps of an eighth of a binade, of 2^-9 below 2^-6, in units of the scale."""
    a = x.abs().amax(-1, keepdim=True)
    s = torch.exp2(torch.ceil(torch.log2(a.clamp(min=2.0 ** -92) / 448.0)).clamp(min=-100.0))
    s = torch.where(a <= 224.0 * s, 0.5 * s, s).clamp(min=2.0 ** -100)   # (log2 may round up past a whole number,
    s = torch.where(a > 448.0 * s, 2.0 * s, s)                           # or down)
    v = x / s
    step = torch.exp2(torch.floor(torch.log2(v.abs().clamp(min=2.0 ** -6))) - 3.0)
    return torch.round(v / step) * step * s, s.squeeze(-1)


def exact(case, seed):
    c = case
    s = prepare(case, seed)
    if c["kind"] == "rows8":
        values, scales = _exact_coded(s["x"].double())
        return {"values": values, "scales": scales}
    if c["kind"] == "norm8":
        h, y = s["h"].double(), s["y"].double()
        if c["post"]:
            y = y / torch.sqrt(y.pow(2).sum(1, keepdim=True) / c["D"] + EPS) * s["post"].double()
        if c["gate"] != "none":
            y = y * (torch.sigmoid(s["gate"].double())[:, None] if c["gate"] == "token" else s["gate"].double())
        if c["channel"]:
            y = y * s["channel"].double()
        h = 0.875 * h + 0.5 * y
        return {"h": h, "x": _exact_coded(h / torch.sqrt(h.pow(2).sum(1, keepdim=True) / c["D"] + EPS) * s["pre"].double())[0]}
    if c["kind"] == "route":
        v = s["logits"].double()
        low = -1e300
        top = torch.topk(v, c["k"], 1).values   # (which of equal ones does not matter to the weights)
        z = torch.logsumexp((top if c["renorm"] else v).clamp(min=low), 1, keepdim=True)
        w = torch.where(torch.isneginf(top), 0.0, torch.exp(top.clamp(min=low) - z))
        return {"experts": None, "weights": w, "offsets": None, "pairs": None, "places": None}
    if c["kind"] == "combine":
        out = s["base"].double() if c["base"] else torch.zeros(c["T"], c["D"], dtype=torch.float64, device="cuda")
        for j in range(c["k"]):
            p = s["places"][:, j].long()
            w = torch.where(p >= 0, s["weights"][:, j].double(), 0.0)
            out = out + w[:, None] * s["y"].double()[p.clamp(min=0)]
        return out
    off = s["offsets"].tolist()
    out = torch.zeros(c["T"] * c["k"], c["rows"], dtype=torch.float64, device="cuda")

    def values(x, scale):
        return x.double() if scale is None else x.double() * scale.double()[..., None]

    x = values(s["x"], s["xs"])
    for e in range(c["E"]):
        a, b = off[e], off[e + 1]
        if a == b:
            continue
        rows = x[s["pairs"][a:b].long() // c["k"]] if c["gather"] else x[a:b]
        y = rows @ values(s["w"][e], None if s["ws"] is None else s["ws"][e]).t()
        if c["glu"]:
            y = y * torch.sigmoid(y) * (rows @ values(s["up"][e], None if s["us"] is None else s["us"][e]).t())
        out[a:b] = y
    return out
