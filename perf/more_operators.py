"""Performance cases of the operators around a block's attention: the layer norm of its hidden rows, modulated as
diffusion transformers do, and the projections to and from Q, K and V as products of microscaled operands.

Operators (field ``op``):

* ``norm``         layer norm of rows, with an affine map, a modulation (scale and shift of each batch entry), both or
                   neither;
* ``norm_grad``    the same with its gradients: of the rows, the weight, the bias, the scale and the shift;
* ``linear``       rows quantised in blocks of 32 elements that share a power-of-two scale (``mxfp4``: e2m1 codes,
                   ``mxfp8``: e4m3 codes) times weights kept so, plus a bias;
* ``norm_linear``  a norm whose rows, rounded to their type, go to such a product as codes;
* ``linear_grad``  the product with the gradients of its rows (through weights that stay as they are: the rounding of the
                   rows passes a gradient on as it is) and of its bias.

Row counts are those of the package's workloads (4096-token images, 4352 with text, 16384-token video, edited regions,
single rows such as a block's modulation vector); widths are heads x head dim of 64 or 128, and generic ones. ``run`` is
the operators' plain form, or with ``own`` the package's calls.
"""

import math

import torch

own = False

DEV = "cuda:0"
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 32  # elements that share a scale
# largest exponent of a code, significand up to which the largest code is within half a step, largest code,
# bits of the significand after its first, smallest normal exponent, smallest exponent of a scale
FORMATS = {"mxfp4": (2, 1.75, 6.0, 1, 0, -127), "mxfp8": (8, 1.8125, 448.0, 3, -6, -124)}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
EPS = 1e-6


def listed():
    return [
        # The target rows of an image block ahead of its attention: no affine map, the block's modulation.
        dict(name="norm_image", op="norm", dtype="bf16", pdtype="bf16", batch=1, rows=4096, width=4096, affine=False,
             modulated=True, ahead=0),
        # One row, a time embedding: the smallest call.
        dict(name="norm_row", op="norm", dtype="bf16", pdtype="bf16", batch=1, rows=1, width=1536, affine=True,
             modulated=False, ahead=0),
        # Training on video rows, every parameter with its gradient.
        dict(name="norm_grad_video", op="norm_grad", dtype="bf16", pdtype="f32", batch=1, rows=16384, width=2048,
             affine=True, modulated=True, ahead=0),
        # An fp32 verification run of two entries, odd rows and an odd width, behind the reference rows.
        dict(name="norm_grad_odd", op="norm_grad", dtype="f32", pdtype="f32", batch=2, rows=1009, width=1001,
             affine=True, modulated=True, ahead=77),
        # Q, K and V of an image's rows, both sides in 4 bits: 16 heads of 128.
        dict(name="linear_qkv", op="linear", dtype="bf16", xfmt="mxfp4", wfmt="mxfp4", batch=1, rows=4096, width=2048,
             out=6144, bias=True, ahead=0),
        # The wide layer behind the attention of video rows: 8-bit rows, 4-bit weights.
        dict(name="linear_video", op="linear", dtype="bf16", xfmt="mxfp8", wfmt="mxfp4", batch=1, rows=16384,
             width=2048, out=8192, bias=True, ahead=0),
        # One row against all the modulation vectors of a block: bound by the weights' bytes.
        dict(name="linear_row", op="linear", dtype="bf16", xfmt="mxfp8", wfmt="mxfp4", batch=1, rows=1, width=4096,
             out=24576, bias=True, ahead=0),
        # The rows of an edited region, 8 bits on both sides: 24 heads of 64.
        dict(name="linear_region", op="linear", dtype="bf16", xfmt="mxfp8", wfmt="mxfp8", batch=1, rows=61, width=1536,
             out=4608, bias=True, ahead=0),
        # An image block's norm and its Q, K, V in one chain, text rows included: 32 heads of 128.
        dict(name="norm_linear_text", op="norm_linear", dtype="bf16", pdtype="bf16", xfmt="mxfp4", wfmt="mxfp4",
             batch=1, rows=4352, width=4096, out=12288, affine=False, modulated=True, bias=True, ahead=0),
        # The same chain at a region of odd size, one GPU's share of the heads, rows behind the reference's.
        dict(name="norm_linear_region", op="norm_linear", dtype="bf16", pdtype="bf16", xfmt="mxfp8", wfmt="mxfp4",
             batch=2, rows=131, width=1536, out=1152, affine=True, modulated=True, bias=False, ahead=77),
        # Training through frozen 4-bit weights.
        dict(name="linear_grad_image", op="linear_grad", dtype="bf16", xfmt="mxfp8", wfmt="mxfp4", batch=1, rows=4096,
             width=2048, out=6144, bias=True, ahead=0),
        # An fp32 verification run of odd sizes: 6 heads of 64.
        dict(name="linear_grad_f32", op="linear_grad", dtype="f32", xfmt="mxfp8", wfmt="mxfp8", batch=1, rows=323,
             width=384, out=1153, bias=True, ahead=0),
    ]


MOST_FLOPS = {"linear": 2.0 * 16384 * 2048 * 8192, "norm_linear": 2.0 * 4352 * 4096 * 12288,
              "linear_grad": 4.0 * 4096 * 2048 * 6144}
MOST_ELEMENTS = {"norm": 4096 * 4096, "norm_grad": 16384 * 2048}


def draw(rng):
    def size(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    while True:
        op = rng.choice(("norm", "norm_grad", "linear", "linear", "norm_linear", "linear_grad"))
        dtype = "bf16" if op == "norm_linear" else rng.choice(("bf16", "bf16", "bf16", "f32"))
        c = dict(op=op, dtype=dtype, batch=rng.choice((1, 1, 1, 2, 3)), rows=size(1, 16384),
                 ahead=rng.choice((0, 0, 0, 77, 256)))
        if op in ("norm", "norm_grad"):
            c.update(pdtype=rng.choice((dtype, "f32")), width=size(8, 8192), affine=rng.random() < 0.5,
                     modulated=rng.random() < 0.6)
            if rng.random() < 0.6:  # most widths are whole heads
                c["width"] = max(64, c["width"] // 64 * 64)
            if c["batch"] * (c["rows"] + c["ahead"]) * c["width"] <= MOST_ELEMENTS[op]:
                return c
            continue
        c.update(xfmt=rng.choice(("mxfp4", "mxfp8")), wfmt=rng.choice(("mxfp4", "mxfp4", "mxfp8")),
                 width=32 * size(1, 256), out=size(1, 24576), bias=rng.random() < 0.7)
        if rng.random() < 0.6:
            c["out"] = max(64, c["out"] // 64 * 64)
        if op == "norm_linear":
            c.update(pdtype=rng.choice(("bf16", "f32")), affine=rng.random() < 0.5, modulated=rng.random() < 0.6)
        cost = work(c)["flops"] * (4 if dtype == "f32" and op == "linear_grad" else 1)
        if cost <= MOST_FLOPS[op] and c["batch"] * (c["rows"] + c["ahead"]) * max(c["width"], c["out"]) <= 16384 * 8192:
            return c


# ---- inputs


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _hidden(gen, c):
    """Hidden rows [batch, rows, width]: channels of unlike size around unlike means, a few loud ones. With ``ahead``
    rows of a buffer that holds as many others in front of them."""
    W = c["width"]
    size = torch.exp(0.5 * torch.randn((W,), generator=gen, device=DEV))
    size = size * (1.0 + 15.0 * (torch.rand((W,), generator=gen, device=DEV) < 0.005))
    x = torch.randn((c["batch"], c["ahead"] + c["rows"], W), generator=gen, device=DEV)
    x = x * size + 0.3 * torch.randn((W,), generator=gen, device=DEV)
    return x.to(DTYPES[c["dtype"]])[:, c["ahead"]:]


def _norm_inputs(gen, c):
    dt, W = DTYPES[c["pdtype"]], c["width"]

    def vector(mean, std, *shape):
        return (mean + std * torch.randn((*shape, W), generator=gen, device=DEV)).to(dt)

    s = {"weight": None, "bias": None, "scale": None, "shift": None}
    if c["affine"]:
        s.update(weight=vector(1.0, 0.2), bias=vector(0.0, 0.2))
    if c["modulated"]:
        s.update(scale=vector(0.0, 0.3, c["batch"]), shift=vector(0.0, 0.3, c["batch"]))
    return s


def prepare(case, seed):
    c = case
    gen = _gen(seed)
    s = {"c": c, "x": _hidden(gen, c)}
    if c["op"] in ("norm", "norm_grad", "norm_linear"):
        s.update(_norm_inputs(gen, c))
    if c["op"] in ("linear", "norm_linear", "linear_grad"):
        w = torch.randn((c["out"], c["width"]), generator=gen, device=DEV) / math.sqrt(c["width"])
        w = w * torch.exp(0.3 * torch.randn((c["out"], 1), generator=gen, device=DEV))
        s["w_codes"], s["w_scales"] = _pack(*_quantise(w, c["wfmt"]), c["wfmt"])
        s["b"] = (0.2 * torch.randn((c["out"],), generator=gen, device=DEV)).to(DTYPES[c["dtype"]]) if c["bias"] else None
    if c["op"] == "norm_grad":
        s["g"] = torch.randn(s["x"].shape, generator=gen, device=DEV).to(DTYPES[c["dtype"]])
        s["leaves"] = [s[n].requires_grad_(True) for n in ("x", "weight", "bias", "scale", "shift") if s[n] is not None]
    if c["op"] == "linear_grad":
        s["g"] = torch.randn((c["batch"], c["rows"], c["out"]), generator=gen, device=DEV).to(DTYPES[c["dtype"]])
        s["leaves"] = [s[n].requires_grad_(True) for n in ("x", "b") if s[n] is not None]
    return s


# ---- the operators' plain forms


def _normalised(x, wide):
    """((x - mean) / sqrt(variance + eps), 1 / sqrt(variance + eps)) of rows in ``wide`` bits."""
    x = x.to(wide)
    off = x - x.mean(-1, keepdim=True)
    r = (off.square().mean(-1, keepdim=True) + EPS).rsqrt()
    return off * r, r


def _mapped(h, s):
    """The affine map and the modulation of normalised rows."""
    f = h.dtype
    n = h if s["weight"] is None else h * s["weight"].to(f) + s["bias"].to(f)
    return n if s["scale"] is None else n * (1.0 + s["scale"].to(f)[:, None]) + s["shift"].to(f)[:, None]


def _norm_plain(s):
    return _mapped(_normalised(s["x"], torch.float32)[0], s).to(s["x"].dtype)


def _norm_grad_plain(s):
    f = torch.float32
    h, r = _normalised(s["x"], f)
    out = {"y": _mapped(h, s).to(s["x"].dtype)}
    g = s["g"].to(f)
    e = g
    if s["scale"] is not None:
        n = h if s["weight"] is None else h * s["weight"].to(f) + s["bias"].to(f)
        out["scale"] = (g * n).sum(1).to(s["scale"].dtype)
        out["shift"] = g.sum(1).to(s["shift"].dtype)
        e = g * (1.0 + s["scale"].to(f)[:, None])
    if s["weight"] is not None:
        out["weight"] = (e * h).sum((0, 1)).to(s["weight"].dtype)
        out["bias"] = e.sum((0, 1)).to(s["bias"].dtype)
        e = e * s["weight"].to(f)
    dx = r * (e - e.mean(-1, keepdim=True) - h * (e * h).mean(-1, keepdim=True))
    out["x"] = dx.to(s["x"].dtype)
    return out


def _power(e):
    """2^e as fp32 for whole e of -126 to 127, from its bits."""
    return ((e + 127) << 23).view(torch.float32)


def _quantise(x, fmt):
    """(signed values in steps of a block's scale, scale bytes) of x [..., width]."""
    emax, most, top, bits, low, lowest = FORMATS[fmt]
    y = x.to(torch.float32).unflatten(-1, (-1, BLOCK))
    word = y.abs().amax(-1).view(torch.int32)
    cut = int((most - 1.0) * (1 << 23))
    e = (word >> 23) - 127 - emax + ((word & 0x7FFFFF) > cut).to(torch.int32)
    e = e.clamp(lowest, 127 - emax)
    y = y * _power(-e)[..., None]
    step = _power(((y.abs().view(torch.int32) >> 23) - 127).clamp(min=low) - bits)
    q = (torch.round(y / step) * step).clamp(-top, top)
    return q.flatten(-2), (e + 127).to(torch.uint8)


def _values(q, scales):
    """What codes of value q and their scale bytes stand for."""
    e = scales.to(torch.int32) - 127
    lo = e.clamp(min=-126)
    y = q.unflatten(-1, (-1, BLOCK)) * _power(lo)[..., None] * _power(e - lo)[..., None]  # 2^-127 in two steps
    return y.flatten(-2)


def _pack(q, scales, fmt):
    """Bytes of the codes: e4m3, or two e2m1 codes a byte, the first in the low half."""
    if fmt == "mxfp8":
        return q.to(torch.float8_e4m3fn).view(torch.uint8), scales
    at = torch.bucketize(q.abs(), torch.tensor(E2M1, device=q.device)).to(torch.uint8)
    at = at | (torch.signbit(q).to(torch.uint8) << 3)
    return at[..., 0::2] | (at[..., 1::2] << 4), scales


def _unpack(codes, scales, fmt):
    if fmt == "mxfp8":
        return _values(codes.view(torch.float8_e4m3fn).to(torch.float32), scales)
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=codes.device)
    return _values(table[torch.stack((codes & 15, codes >> 4), -1).flatten(-2).int()], scales)


def _product_plain(x, s, w):
    c = s["c"]
    rows = _values(*_quantise(x, c["xfmt"])).flatten(0, 1)
    y = torch.mm(rows, w.t())
    if s["b"] is not None:
        y = y + s["b"].to(torch.float32)
    return y.view(*x.shape[:2], c["out"]).to(DTYPES[c["dtype"]])


def _linear_plain(s):
    return _product_plain(s["x"], s, _unpack(s["w_codes"], s["w_scales"], s["c"]["wfmt"]))


def _norm_linear_plain(s):
    # in 64 bits up to the rounding that decides the codes
    n = _mapped(_normalised(s["x"], torch.float64)[0], s).to(s["x"].dtype)
    return _product_plain(n, s, _unpack(s["w_codes"], s["w_scales"], s["c"]["wfmt"]))


def _linear_grad_plain(s):
    w = _unpack(s["w_codes"], s["w_scales"], s["c"]["wfmt"])
    out = {"y": _product_plain(s["x"], s, w)}
    g = s["g"].to(torch.float32).flatten(0, 1)
    out["x"] = torch.mm(g, w).view(s["x"].shape).to(s["x"].dtype)
    if s["b"] is not None:
        out["b"] = g.sum(0).to(s["b"].dtype)
    return out


# ---- the package's calls


def _own_weights(s):
    from paper_2609_32415_amd import ops

    return ops.MxTensor(s["w_codes"][None, None], s["w_scales"][None, None], s["c"]["wfmt"])


def _norm_own(s):
    from paper_2609_32415_amd import ops

    return ops.layer_norm(s["x"], s["weight"], s["bias"], scale=s["scale"], shift=s["shift"], eps=EPS)


def _norm_grad_own(s):
    with torch.enable_grad():
        y = _norm_own(s)
        grads = torch.autograd.grad(y, s["leaves"], s["g"])
    names = [n for n in ("x", "weight", "bias", "scale", "shift") if s[n] is not None]
    return {"y": y.detach(), **dict(zip(names, grads))}


def _linear_own(s):
    from paper_2609_32415_amd import ops

    return ops.mx_linear(s["x"], _own_weights(s), s["b"], fmt=s["c"]["xfmt"])


def _norm_linear_own(s):
    from paper_2609_32415_amd import ops

    n = ops.layer_norm_mx(s["x"], s["c"]["xfmt"], s["weight"], s["bias"], scale=s["scale"], shift=s["shift"], eps=EPS)
    return ops.mx_linear(n, _own_weights(s), s["b"])


def _linear_grad_own(s):
    with torch.enable_grad():
        y = _linear_own(s)
        grads = torch.autograd.grad(y, s["leaves"], s["g"])
    return {"y": y.detach(), **dict(zip([n for n in ("x", "b") if s[n] is not None], grads))}


PLAIN = {"norm": _norm_plain, "norm_grad": _norm_grad_plain, "linear": _linear_plain,
         "norm_linear": _norm_linear_plain, "linear_grad": _linear_grad_plain}
OWN = {"norm": _norm_own, "norm_grad": _norm_grad_own, "linear": _linear_own, "norm_linear": _norm_linear_own,
       "linear_grad": _linear_grad_own}


def run(state):
    op = state["c"]["op"]
    if own:
        return OWN[op](state)
    with torch.no_grad():
        return PLAIN[op](state)


# ---- the least that a pass reads, writes and computes


def work(case):
    c = case
    esz = 2 if c["dtype"] == "bf16" else 4
    rows, W = c["batch"] * c["rows"], c["width"]
    small = 0.0
    if c["op"] in ("norm", "norm_grad", "norm_linear"):
        psz = 2 if c["pdtype"] == "bf16" else 4
        small = psz * W * ((2 if c["affine"] else 0) + (2 * c["batch"] if c["modulated"] else 0))
    if c["op"] == "norm":
        return {"bytes": 2.0 * rows * W * esz + small, "flops": 9.0 * rows * W}
    if c["op"] == "norm_grad":
        return {"bytes": 4.0 * rows * W * esz + 2 * small, "flops": 25.0 * rows * W}
    per = (0.5 if c["wfmt"] == "mxfp4" else 1.0) + 1.0 / BLOCK
    bias = c["out"] * esz if c["bias"] else 0
    b = rows * W * esz + c["out"] * W * per + rows * c["out"] * esz + bias
    flops = 2.0 * rows * W * c["out"]
    if c["op"] == "linear_grad":
        return {"bytes": float(b + rows * c["out"] * esz + rows * W * esz + bias), "flops": 2 * flops}
    return {"bytes": float(b + small), "flops": flops}


# ---- from the definitions, in 64 bits


def _norm_terms(s):
    """(normalised rows, what multiplies and what is added to them, 1 / deviation), each entry by itself."""
    d = torch.float64
    h, r = [], []
    for rows in s["x"].detach().to(d):
        var, mean = torch.var_mean(rows, -1, correction=0, keepdim=True)
        r.append(1.0 / torch.sqrt(var + EPS))
        h.append((rows - mean) / torch.sqrt(var + EPS))
    one, zero = torch.ones((), dtype=d, device=DEV), torch.zeros((), dtype=d, device=DEV)
    w, b = (one, zero) if s["weight"] is None else (s["weight"].detach().to(d), s["bias"].detach().to(d))
    S = [one] * len(h) if s["scale"] is None else list(1.0 + s["scale"].detach().to(d))
    t = [zero] * len(h) if s["shift"] is None else list(s["shift"].detach().to(d))
    return h, r, w, b, S, t


def _norm_exact(s):
    h, _, w, b, S, t = _norm_terms(s)
    return torch.stack([a * (w * m) + (b * m + u) for a, m, u in zip(h, S, t)])


def _norm_grad_exact(s):
    d = torch.float64
    h, r, w, b, S, _ = _norm_terms(s)
    W = s["c"]["width"]
    out = {"y": _norm_exact(s), "x": [], "scale": [], "shift": [], "weight": 0.0, "bias": 0.0}
    for a, q, m, g in zip(h, r, S, s["g"].to(d)):
        along = torch.einsum("rc,rc->c", g, a)  # sums over the rows
        total = torch.einsum("rc->c", g)
        out["scale"].append(w * along + b * total)
        out["shift"].append(total)
        out["weight"] = out["weight"] + m * along
        out["bias"] = out["bias"] + m * total
        e = g * (m * w)
        # the derivative of the norm: e less its parts along the ones and along the row itself
        coef = torch.einsum("rc,rc->r", e, a)[:, None] / W
        out["x"].append((e - e.sum(-1, keepdim=True) / W - a * coef) * q)
    for n in ("x", "scale", "shift"):
        out[n] = torch.stack(out[n])
    return {n: v for n, v in out.items() if n in ("y", "x") or s[n] is not None}


def _code_values(fmt):
    """The non-negative values of a format's codes, in order."""
    if fmt == "mxfp4":
        return list(E2M1)
    return [(m if e == 0 else 8 + m) * 2.0 ** (max(e, 1) - 10) for e in range(16) for m in range(8)][:127]


def _rounded_exact(x, fmt):
    """Every element against the format's table of values: the nearest one, on a tie the even code."""
    emax, most = FORMATS[fmt][:2]
    vals = _code_values(fmt)
    table = torch.tensor(vals, dtype=torch.float64, device=DEV)
    mids = (table[1:] + table[:-1]) / 2
    lowest = FORMATS[fmt][5]

    def power(e):  # from the bits of a double: pow() need not be exact
        return ((e.to(torch.int64) + 1023) << 52).view(torch.float64)

    y = x.to(torch.float64).unflatten(-1, (-1, BLOCK))
    amax = y.abs().amax(-1)
    e = torch.ceil(torch.log2(amax / (most * 2.0 ** emax))).clamp(lowest, 127 - emax)  # log2 rounds: set right below
    e = torch.where(amax > most * 2.0 ** emax * power(e), e + 1, e)
    e = torch.where(amax <= most * 2.0 ** emax * power(e - 1), e - 1, e).clamp(lowest, 127 - emax)
    m = (y.abs() / power(e)[..., None]).contiguous()
    down, up = torch.bucketize(m, mids), torch.bucketize(m, mids, right=True)
    at = torch.where(down % 2 == 0, down, up).clamp(max=len(vals) - 1)  # on a tie the two differ: the even one
    return (torch.sign(y) * table[at] * power(e)[..., None]).flatten(-2)


def _weights_exact(s):
    fmt, d = s["c"]["wfmt"], torch.float64
    table = torch.tensor(_code_values(fmt), dtype=d, device=DEV)
    b = s["w_codes"].to(torch.int64)
    if fmt == "mxfp4":
        b = torch.stack((b % 16, b // 16), -1).flatten(-2)
    n = 8 if fmt == "mxfp4" else 128
    y = torch.where(b >= n, -table[b % n], table[b % n])
    return y * ((s["w_scales"].to(torch.int64) - 127 + 1023) << 52).view(d).repeat_interleave(BLOCK, -1)


def _linear_exact(s, x, w):
    out = []
    for rows in x:
        y = _rounded_exact(rows, s["c"]["xfmt"]) @ w.T
        out.append(y if s["b"] is None else y + s["b"].detach().to(torch.float64))
    return torch.stack(out)


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        return _norm_exact(s)
    if op == "norm_grad":
        return _norm_grad_exact(s)
    w = _weights_exact(s)
    if op == "linear":
        return _linear_exact(s, s["x"], w)
    if op == "norm_linear":
        return _linear_exact(s, _norm_exact(s).to(s["x"].dtype), w)
    g = s["g"].to(torch.float64)
    out = {"y": _linear_exact(s, s["x"].detach(), w), "x": torch.stack([rows @ w for rows in g])}
    if s["b"] is not None:
        out["b"] = g.flatten(0, 1).sum(0)
    return out
