"""Norms and 4-bit products: what is measured, and their plain forms.

Four kinds of pass:

  norm           Y = (x - mean) * rstd * gamma + beta of every row (rms: mean taken as 0), with mean and rstd kept
  norm_backward  dX, dgamma, dbeta of the same from dY; dX with the gradient that goes past the norm added
  quantize       X -> 4-bit blocks with a scale each, and the values they stand for read back
  fp4_linear     X quantised, then Y = act(z) + R or act(z_gate) * z_up + R with z = alpha * (X W) + b over the
                 4-bit values of X and of W (which is in hand quantised)

``run`` computes them with elementary torch operations in 32 bits, or, where ``own`` is true, through the
library's entry points.  ``exact`` computes the definition in 64 bits.  The layout of 4-bit tensors is part of the
interface: a tensor of `rows` rows (in `parts` equal parts) and k columns is

    q[rows][16 * ceil(k / 32)] bytes, column 2 i in the low half of byte i, 2 i + 1 in the high one, zeros past k
    scales[parts][ceil(rows / parts / 128)][ceil(k / (4 * block))][32][4][4] bytes: the scale of row r of a part and
      block j at [r / 128][j / 4][r % 32][r % 128 / 32][j % 4], zeros where there is none

with blocks of 32 and scales 2^(byte - 127) (mx) or blocks of 16 and scales in e4m3 (nv).
"""
import math

import torch

own = False

ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
FORMATS = {"mx": 0, "nv": 1}
BLOCK = {"mx": 32, "nv": 16}
E2M1 = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # The norm in front of a layer in a decoding step: one token.
        dict(name="norm 1 row", op="norm", m=1, n=2048, x="bf16", rms=False, affine=True),
        # A short prompt, a residual stream in f32, rows of odd length.
        dict(name="norm odd rows f32", op="norm", m=333, n=2047, x="f32", rms=False, affine=True),
        # A training batch.
        dict(name="norm 16384 x 4096", op="norm", m=16384, n=4096, x="bf16", rms=False, affine=True),
        # Training backward: a ragged batch on a middle-sized layer ...
        dict(name="norm_backward ragged", op="norm_backward", m=1000, n=2056, x="bf16", rms=True, affine=True,
             residual=False),
        # ... and a full one, the gradient of the residual stream added.
        dict(name="norm_backward 16384 x 4096", op="norm_backward", m=16384, n=4096, x="bf16", rms=False, affine=True,
             residual=True),
        # Activations of a decoding batch, rows of odd length, a scale for the whole tensor.
        dict(name="quantize 16 rows", op="quantize", format="nv", x="bf16", rowmajor=False, rows=16, parts=1, k=2047,
             scaled=True),
        # A layer's weights stored [in][out], once per load: the 2048 x 16384 of the headline product.
        dict(name="quantize weights", op="quantize", format="mx", x="bf16", rowmajor=True, rows=16384, parts=2, k=2048,
             scaled=False),
        # Activations of a prompt.
        dict(name="quantize 8192 x 4096", op="quantize", format="nv", x="bf16", rowmajor=False, rows=8192, parts=1,
             k=4096, scaled=True),
        # One token of a decoding step through a gated layer: 16.8 MB of weights in 4 bits.
        dict(name="fp4_linear 1 row gated", op="fp4_linear", format="mx", m=1, k=2048, n=8192, act="silu", gated=True,
             bias=False, residual=False, scaled=False, y="bf16"),
        # A decoding batch of 16 on the same weights, with bias, activation and residual.
        dict(name="fp4_linear 16 rows", op="fp4_linear", format="nv", m=16, k=2048, n=16384, act="gelu", gated=False,
             bias=True, residual=True, scaled=True, y="bf16"),
        # A short prompt through a layer whose sizes are no multiple of anything.
        dict(name="fp4_linear odd sizes", op="fp4_linear", format="nv", m=333, k=2047, n=2049, act="gelu_tanh",
             gated=False, bias=True, residual=True, scaled=True, y="bf16"),
        # A prompt through a square layer.
        dict(name="fp4_linear 4096 cube", op="fp4_linear", format="nv", m=4096, k=4096, n=4096, act="gelu", gated=False,
             bias=True, residual=True, scaled=True, y="bf16"),
    ]


def _log(rng, low, high, step=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(low, min(high, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["norm", "norm_backward", "quantize", "fp4_linear", "fp4_linear"])
    step = rng.choice([1, 8, 32])
    flag = lambda: rng.random() < 0.5  # noqa: E731
    if op in ("norm", "norm_backward"):
        n = _log(rng, 64, 16384, step)
        case = dict(op=op, m=_log(rng, 1, min(16384, (1 << 26) // n)), n=n, x=rng.choice(["bf16", "bf16", "f32"]), rms=flag(),
                    affine=rng.random() < 0.8)
        if case["x"] == "f32":
            case["m"] = (case["m"] + 1) // 2
        if op == "norm_backward":
            case.update(residual=flag())
        return case
    case = dict(op=op, format=rng.choice(list(FORMATS)))
    if op == "quantize":
        k, parts = _log(rng, 64, 4096, step), rng.choice([1, 1, 2])
        return dict(case, x=rng.choice(["bf16", "bf16", "f32"]), rowmajor=flag(), rows=parts * _log(rng, 1, 4096), parts=parts,
                    k=k, scaled=flag())
    gated = flag()
    return dict(case, m=_log(rng, 1, 4096), k=_log(rng, 256, 4096, step), n=_log(rng, 256, 2048 if gated else 4096, step),
                act=rng.choice(["silu", "gelu", "relu"] if gated else list(ACTS)), gated=gated, bias=flag(), residual=flag(),
                scaled=flag(), y=rng.choice(["bf16", "bf16", "f32"]))


# --- sizes ---------------------------------------------------------------------------------

def _pitch(k):
    return (k + 31) // 32 * 16


def _atoms(rows, k, block):
    """Blocks of 128 rows x 4 scales of a part: (down, across)"""
    return (rows + 127) // 128, (k + 4 * block - 1) // (4 * block)


def _packed_bytes(rows, k, block):
    return rows * ((k + 1) // 2 + (k + block - 1) // block)


def work(case):
    c = case
    if c["op"] in ("norm", "norm_backward"):
        m, n, size = c["m"], c["n"], 4 if c["x"] == "f32" else 2
        weights = 2 * n if c["affine"] else 0
        if c["op"] == "norm":
            return {"bytes": (size + 2) * m * n + (1 if c["rms"] else 2) * (weights + 4 * m), "flops": 8 * m * n}
        tensors = m * n * (2 + size * (3 if c["residual"] else 2))
        return {"bytes": tensors + weights + (1 if c["rms"] else 2) * 4 * (m + n), "flops": 14 * m * n}
    block = BLOCK[c["format"]]
    if c["op"] == "quantize":
        rows, k = c["rows"], c["k"]
        return {"bytes": (4 if c["x"] == "f32" else 2) * rows * k + _packed_bytes(rows, k, block) + 2 * rows * k,
                "flops": 4 * rows * k}
    m, k, n = c["m"], c["k"], c["n"]
    wide = 2 * n if c["gated"] else n
    return {"bytes": 2 * m * k + _packed_bytes(wide, k, block) + (2 * wide if c["bias"] else 0) +
            (2 * m * n if c["residual"] else 0) + (4 if c["y"] == "f32" else 2) * m * n, "flops": 2 * m * k * wide}


# --- inputs --------------------------------------------------------------------------------

def _type(name):
    return torch.float32 if name == "f32" else torch.bfloat16


def _activations(g, m, n, kind):
    """Rows of different sizes and means, some columns much larger than the others."""
    x = torch.randn(m, n, generator=g, device="cuda")
    column = torch.exp(0.5 * torch.randn(n, generator=g, device="cuda"))
    row = torch.exp(0.3 * torch.randn(m, 1, generator=g, device="cuda"))
    return ((x * column + 0.2) * row).to(_type(kind))


def _quantized(x, parts, name, mult):
    """Plain quantisation of x [rows][k] f32: (q, scales) in the interface's layout."""
    rows, k = x.shape
    block = BLOCK[name]
    values, scale, codes = _codes(x, name, mult)
    pitch = _pitch(k)
    nibbles = torch.zeros(rows, 2 * pitch, dtype=torch.uint8, device=x.device)
    nibbles[:, :k] = codes[:, :k]
    q = nibbles[:, 0::2] + 16 * nibbles[:, 1::2]
    each = rows // parts
    down, across = _atoms(each, k, block)
    byte = torch.zeros(parts, down * 128, across * 4, dtype=torch.uint8, device=x.device)
    if name == "mx":
        coded = (torch.frexp(scale).exponent + 126).to(torch.uint8)
    else:
        coded = scale.to(torch.float8_e4m3fn).view(torch.uint8)
    byte[:, :each, :scale.shape[1]] = coded.view(parts, each, -1)
    scales = byte.view(parts, down, 4, 32, across, 4).permute(0, 1, 4, 3, 2, 5).contiguous()
    return q.contiguous(), scales


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, s = case, {"case": dict(case)}
    dev, bf, f32 = "cuda", torch.bfloat16, torch.float32
    randn = lambda *shape: torch.randn(*shape, generator=g, device=dev)  # noqa: E731
    if c["op"] in ("norm", "norm_backward"):
        m, n = c["m"], c["n"]
        s["x"] = _activations(g, m, n, c["x"])
        s["gamma"] = (1 + 0.2 * randn(n)).to(bf) if c["affine"] else None
        s["beta"] = (0.2 * randn(n)).to(bf) if c["affine"] and not c["rms"] else None
        if c["op"] == "norm":
            s["y"] = torch.empty(m, n, device=dev, dtype=bf)
            s["mean"] = None if c["rms"] else torch.empty(m, device=dev)
            s["rstd"] = torch.empty(m, device=dev)
            return s
        x = s["x"].double()
        mean = torch.zeros(m, 1, device=dev, dtype=torch.float64) if c["rms"] else x.mean(1, keepdim=True)
        s["mean"] = None if c["rms"] else mean[:, 0].float()
        s["rstd"] = torch.rsqrt(((x - mean) ** 2).mean(1) + EPS).float()
        s["dy"] = randn(m, n).to(bf)
        s["r"] = randn(m, n).to(_type(c["x"])) if c["residual"] else None
        s["dx"] = torch.empty_like(s["x"])
        s["dgamma"] = torch.empty(n, device=dev) if c["affine"] else None
        s["dbeta"] = torch.empty(n, device=dev) if c["affine"] and not c["rms"] else None
        return s
    block = BLOCK[c["format"]]
    u8 = torch.uint8
    rows, k = (c["rows"], c["k"]) if c["op"] == "quantize" else (c["m"], c["k"])
    parts = c.get("parts", 1)
    x = _activations(g, rows, k, c.get("x", "bf16"))
    s["x"] = x.t().contiguous() if c.get("rowmajor") else x
    down, across = _atoms(rows // parts, k, block)
    s["q"] = torch.empty(rows, _pitch(k), device=dev, dtype=u8)
    s["scales"] = torch.empty(parts, down, across, 32, 4, 4, device=dev, dtype=u8)
    # A factor for the whole tensor that puts its largest scale near the top of the scales' range.
    s["mult"] = (448 * 6 / x.float().abs().max()).reshape(1) if c["scaled"] else None
    if c["op"] == "quantize":
        s["values"] = torch.empty(rows, k, device=dev, dtype=bf)
        return s
    n = c["n"]
    wide = 2 * n if c["gated"] else n
    w = (randn(wide, k) / math.sqrt(k)).to(bf).float()
    w_mult = (448 * 6 / w.abs().max()).reshape(1) if c["scaled"] else None
    s["wq"], s["wscales"] = _quantized(w, 2 if c["gated"] else 1, c["format"], w_mult)
    s["alpha"] = 1 / (s["mult"] * w_mult) if c["scaled"] else None
    s["b"] = (0.5 * randn(wide)).to(bf) if c["bias"] else None
    s["r"] = randn(c["m"], n).to(bf) if c["residual"] else None
    s["y"] = torch.empty(c["m"], n, device=dev, dtype=f32 if c["y"] == "f32" else bf)
    return s


EPS = 1e-5


# --- the framework's calls -----------------------------------------------------------------

def _own(s):
    from paper_2505_01637_b200 import binding as mb

    c = s["case"]
    kind = 1 if c.get("x") == "f32" else 0
    if c["op"] == "norm":
        mb.morello_layer_norm(c["rms"], kind, c["m"], c["n"], EPS, s["x"], s["gamma"], s["beta"], s["y"], s["mean"], s["rstd"])
        return {"y": s["y"], "mean": s["mean"], "rstd": s["rstd"]}
    if c["op"] == "norm_backward":
        mb.morello_layer_norm_backward(c["rms"], kind, 0, c["m"], c["n"], s["x"], s["gamma"], s["mean"], s["rstd"], s["dy"],
                                       s["r"], s["dx"], s["dgamma"], s["dbeta"])
        return {"dx": s["dx"], "dgamma": s["dgamma"], "dbeta": s["dbeta"]}
    form = FORMATS[c["format"]]
    if c["op"] == "quantize":
        layout = 0 if c["rowmajor"] else 1
        mb.morello_fp4_quantize(form, kind, layout, c["rows"], c["parts"], c["k"], s["x"], s["mult"], s["q"], s["scales"])
        mb.morello_fp4_dequantize(form, 0, c["rows"], c["parts"], c["k"], s["q"], s["scales"], None, s["values"])
        return {"values": s["values"]}
    mb.morello_fp4_quantize(form, 0, 1, c["m"], 1, c["k"], s["x"], s["mult"], s["q"], s["scales"])
    mb.morello_fp4_linear(form, ACTS[c["act"]], c["gated"], c["y"] == "f32", c["m"], c["k"], c["n"], s["q"], s["scales"],
                          s["wq"], s["wscales"], s["alpha"], s["b"], s["r"], s["y"])
    return {"y": s["y"]}


# --- the plain forms -----------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if act == "gelu":
        return 0.5 * z * (1 + torch.erf(z * math.sqrt(0.5)))
    if act == "gelu_tanh":
        return 0.5 * z * (1 + torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z)))
    if act == "silu":
        return z / (1 + torch.exp(-z))
    return z


def _power(e):
    """2^e for -127 <= e <= 127, f32 without a rounding."""
    return torch.tensor([2.0 ** i for i in range(-127, 128)], device=e.device)[e.long() + 127]


def _codes(x, name, mult):
    """(values [rows][k padded to blocks] over their scale, scale [rows][blocks], codes) of x [rows][k], f32.

    The quotients are rounded to f32 before they are rounded to 4 bits (and amax / 6 before e4m3): with 24 bits in
    the numerator and at most 4 in the denominator that never moves one onto a midpoint."""
    rows, k = x.shape
    block = BLOCK[name]
    x = x.float()
    if mult is not None:
        x = x * mult
    blocks = (k + block - 1) // block
    padded = torch.zeros(rows, blocks * block, device=x.device)
    padded[:, :k] = x
    grouped = padded.view(rows, blocks, block)
    amax = grouped.abs().amax(dim=2)
    if name == "mx":
        # amax = f * 2^e with f in [1/2, 1): its exponent is e - 1, the largest of a 4-bit value is 2
        scale = _power((torch.frexp(amax).exponent - 3).clamp(-127, 127))
        scale = torch.where(amax > 0, scale, torch.full_like(scale, 2.0 ** -127))
        v = grouped / scale[..., None]
    else:
        y = amax / 6
        step = _power((torch.frexp(y).exponent - 1).clamp(-6, 127) - 3)
        scale = (torch.round(y / step) * step).clamp(max=448)
        v = torch.where(scale[..., None] > 0, grouped / scale[..., None], torch.zeros_like(grouped))
    a = v.abs().clamp(max=6)
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0))
    a = torch.round(a / step) * step                                  # round half to even, in codes as in values
    code = torch.where(a < 2, 2 * a, torch.where(a < 4, a + 2, a / 2 + 4)).to(torch.uint8)
    code = code + 8 * torch.signbit(v).to(torch.uint8)
    return torch.copysign(a, v).view(rows, -1), scale, code.view(rows, -1)


def _decoded(q, scales, name, k):
    """f32 values of a 4-bit tensor [rows][k] in the interface's layout."""
    rows, parts, block = q.shape[0], scales.shape[0], BLOCK[name]
    codes = torch.stack([q & 15, q >> 4], dim=2).view(rows, -1)[:, :k]
    table = torch.tensor(E2M1 + tuple(-v for v in E2M1), device=q.device)
    down, across = scales.shape[1:3]
    byte = scales.permute(0, 1, 4, 3, 2, 5).reshape(parts, down * 128, across * 4)[:, :rows // parts].reshape(rows, -1)
    if name == "mx":
        scale = _power(byte.long() - 127)
    else:
        scale = byte.contiguous().view(torch.float8_e4m3fn).float()
    return table[codes.long()] * scale.repeat_interleave(block, dim=1)[:, :k]


def _values(x, name, mult):
    """What x stands for once quantised, f32 (over mult)."""
    v, scale, _ = _codes(x, name, mult)
    return (v * scale.repeat_interleave(BLOCK[name], dim=1))[:, :x.shape[1]]


def _plain(s):
    c, bf = s["case"], torch.bfloat16
    if c["op"] == "norm":
        x = s["x"].float()
        mean = torch.zeros(c["m"], 1, device=x.device) if c["rms"] else x.mean(dim=1, keepdim=True)
        d = x - mean
        rstd = 1 / torch.sqrt((d * d).mean(dim=1, keepdim=True) + EPS)
        y = d * rstd
        if s["gamma"] is not None:
            y = y * s["gamma"].float()
        if s["beta"] is not None:
            y = y + s["beta"].float()
        return {"y": y.to(bf), "mean": None if c["rms"] else mean[:, 0], "rstd": rstd[:, 0]}
    if c["op"] == "norm_backward":
        x, dy, rstd = s["x"].float(), s["dy"].float(), s["rstd"][:, None]
        h = (x if c["rms"] else x - s["mean"][:, None]) * rstd
        g = dy if s["gamma"] is None else dy * s["gamma"].float()
        inner = g - h * (g * h).mean(dim=1, keepdim=True)
        if not c["rms"]:
            inner = inner - g.mean(dim=1, keepdim=True)
        dx = rstd * inner
        if s["r"] is not None:
            dx = dx + s["r"].float()
        return {"dx": dx.to(s["dx"].dtype), "dgamma": (dy * h).sum(dim=0) if s["dgamma"] is not None else None,
                "dbeta": dy.sum(dim=0) if s["dbeta"] is not None else None}
    if c["op"] == "quantize":
        x = s["x"].t() if c["rowmajor"] else s["x"]
        return {"values": _values(x, c["format"], s["mult"]).to(bf)}
    z = torch.matmul(_values(s["x"], c["format"], s["mult"]), _decoded(s["wq"], s["wscales"], c["format"], c["k"]).t())
    if s["alpha"] is not None:
        z = z * s["alpha"]
    if s["b"] is not None:
        z = z + s["b"].float()
    y = _act(z[:, :c["n"]], c["act"]) * z[:, c["n"]:] if c["gated"] else _act(z, c["act"])
    if s["r"] is not None:
        y = y + s["r"].float()
    return {"y": y.to(s["y"].dtype)}


def run(state):
    return _own(state) if own else _plain(state)


# --- the definitions in 64 bits ------------------------------------------------------------

def _nearest(v, grid):
    """The member of a sorted grid nearest to v, ties to the even place, beyond its end the last."""
    middle = (grid[:-1] + grid[1:]) / 2
    place = torch.bucketize(v, middle)
    tie = (place < len(middle)) & (v == middle[place.clamp(max=len(middle) - 1)]) & (place % 2 == 1)
    return grid[place + tie.long()]


def _values64(x, name, mult):
    if mult is not None:
        x = x.float() * mult          # the product is rounded to f32 by definition
    x = x.double()
    rows, k = x.shape
    out = torch.empty_like(x)
    four = torch.tensor(E2M1, dtype=torch.float64, device=x.device)
    powers = torch.tensor([2.0 ** e for e in range(-127, 128)], dtype=torch.float64, device=x.device)
    eight = torch.arange(127, dtype=torch.uint8, device=x.device).view(torch.float8_e4m3fn).double()
    for first in range(0, k, BLOCK[name]):
        part = x[:, first:first + BLOCK[name]]
        amax = part.abs().amax(dim=1, keepdim=True)
        if name == "mx":
            scale = powers[(torch.bucketize(amax, powers, right=True) - 3).clamp(min=0)]   # floor(log2) - 2
        else:
            scale = _nearest(amax / 6, eight)
        over = torch.where(scale > 0, part.abs() / scale, torch.zeros_like(part))
        out[:, first:first + BLOCK[name]] = torch.sign(part) * _nearest(over, four) * scale
    return out


def _stored64(q, scales, name, k):
    """A 4-bit tensor's values, read place by place."""
    rows, parts, block = q.shape[0], scales.shape[0], BLOCK[name]
    r = torch.arange(rows, device=q.device)[:, None]
    j = torch.arange(k, device=q.device)[None, :]
    code = (q.long()[r, j // 2] >> (4 * (j % 2))) & 15
    part, row = r // (rows // parts), r % (rows // parts)
    b = j // block
    byte = scales[part, row // 128, b // 4, row % 32, row % 128 // 32, b % 4]
    scale = torch.ldexp(torch.ones_like(byte, dtype=torch.float64), byte.long() - 127) if name == "mx" else byte.view(torch.float8_e4m3fn).double()
    four = torch.tensor(E2M1, dtype=torch.float64, device=q.device)
    return torch.where(code >= 8, -four[code % 8], four[code % 8]) * scale


def _act64(z, act):
    one = {"none": lambda: z, "relu": lambda: z.clamp(min=0),
           "gelu": lambda: z * torch.special.ndtr(z),
           "gelu_tanh": lambda: z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)),
           "silu": lambda: z * torch.sigmoid(z)}
    return one[act]()


def _norm64(x, gamma, beta, rms):
    mean = x.new_zeros(x.shape[0], 1) if rms else x.sum(dim=1, keepdim=True) / x.shape[1]
    rstd = torch.rsqrt(((x - mean) ** 2).sum(dim=1, keepdim=True) / x.shape[1] + EPS)
    y = (x - mean) * rstd
    y = y if gamma is None else y * gamma
    return y if beta is None else y + beta, mean, rstd


def exact(case, seed):
    c, s = case, prepare(case, seed)
    dbl = lambda v: None if v is None else v.double()  # noqa: E731
    if c["op"] == "norm":
        y, mean, rstd = _norm64(s["x"].double(), dbl(s["gamma"]), dbl(s["beta"]), c["rms"])
        return {"y": y, "mean": None if c["rms"] else mean[:, 0], "rstd": rstd[:, 0]}
    if c["op"] == "norm_backward":
        with torch.enable_grad():
            x = s["x"].double().requires_grad_(True)
            gamma = (s["gamma"].double() if c["affine"] else torch.ones(c["n"], dtype=torch.float64, device="cuda")).requires_grad_(True)
            y, _, _ = _norm64(x, gamma, None, c["rms"])
            dx, dgamma = torch.autograd.grad(y, (x, gamma), s["dy"].double())
        return {"dx": dx if s["r"] is None else dx + s["r"].double(), "dgamma": dgamma if s["dgamma"] is not None else None,
                "dbeta": s["dy"].double().sum(dim=0) if s["dbeta"] is not None else None}
    if c["op"] == "quantize":
        return {"values": _values64(s["x"].t() if c["rowmajor"] else s["x"], c["format"], s["mult"])}
    x, w = _values64(s["x"], c["format"], s["mult"]), _stored64(s["wq"], s["wscales"], c["format"], c["k"])
    z = x @ w.t()
    if s["alpha"] is not None:
        z = z * s["alpha"].double()
    if s["b"] is not None:
        z = z + s["b"].double()
    y = _act64(z, c["act"]) if not c["gated"] else _act64(z[:, :c["n"]], c["act"]) * z[:, c["n"]:]
    return {"y": y if s["r"] is None else y + s["r"].double()}
