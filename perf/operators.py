"""The feed-forward operators: what is measured, and their plain forms.

Five kinds of pass:

  linear            Y = act(X W + b) + R, or Y = act(X Wg + bg) * (X Wu + bu) + R with W = [Wg | Wu]
  linear_backward   dX, dW, db of the same from dY and the kept Z = X W + b
  route             logits -> experts and weights of every token, and the plan that sorts the tokens' rows by
                    expert; with "train" also the gradient of the logits
  experts           gated product of every row with its expert's first weights, product with its second
                    weights, weighted sum of a token's rows
  experts_backward  dX, dW, db of the first (gated, gathering) product

``run`` computes them with elementary torch operations in 32 bits, or, where ``own`` is true, through the
library's entry points.  ``exact`` computes the definition in 64 bits.  The row layout of the experts' products is
part of the interface: the rows of an expert begin at a multiple of 128; plan = row_src[R], block_expert[R / 128],
offsets[E + 1], counts[E], slot[T * K] (then scratch), R = 128 * floor((T K + 127 min(E, T K)) / 128).
"""
import math

import torch

own = False

ACTS = {"none": 0, "relu": 1, "gelu": 2, "gelu_tanh": 3, "silu": 4}
SCORES = {"softmax": 0, "sigmoid": 1}
BLOCK = 128          # rows of a block of the experts' row layout
PLAN_CHUNK = 2048    # entries per chunk of the plan's scratch


def listed():
    return [
        # One token of a decoding step through a gated feed-forward layer: the 2048 x 16384 weights of the
        # headline vector-matrix product, read once.
        dict(name="linear 1 row gated", op="linear", m=1, k=2048, n=8192, act="silu", gated=True, colmajor=False,
             bias=False, residual=False, keep_z=False, y="bf16"),
        # A decoding batch of 16 on the same weights, stored [out][in], with bias, activation and residual.
        dict(name="linear 16 rows", op="linear", m=16, k=2048, n=16384, act="gelu", gated=False, colmajor=True,
             bias=True, residual=True, keep_z=False, y="bf16"),
        # A short prompt through a layer whose sizes are no multiple of anything.
        dict(name="linear odd sizes", op="linear", m=333, k=2047, n=2049, act="gelu_tanh", gated=False, colmajor=False,
             bias=True, residual=True, keep_z=False, y="bf16"),
        # The training forward of a square layer: Z is kept for the backward pass.
        dict(name="linear 4096 cube", op="linear", m=4096, k=4096, n=4096, act="gelu", gated=False, colmajor=False,
             bias=True, residual=True, keep_z=True, y="bf16"),
        # Training backward: a ragged batch on a middle-sized layer.
        dict(name="linear_backward ragged", op="linear_backward", m=1000, k=1024, n=2056, act="gelu", gated=False,
             colmajor=True, bias=True),
        # Training backward of a gated layer, the largest weights.
        dict(name="linear_backward gated", op="linear_backward", m=4096, k=2048, n=8192, act="silu", gated=True,
             colmajor=False, bias=False),
        # Routing in a decoding step: scores with a balance bias, limited to groups of experts.
        dict(name="route 16 tokens", op="route", tokens=16, experts=64, topk=8, score="sigmoid", groups=8, topk_groups=4,
             renorm=True, bias=True, logits="f32", train=False),
        # Routing of a training batch, with the logits' gradient.
        dict(name="route 16384 tokens", op="route", tokens=16384, experts=256, topk=8, score="softmax", groups=1,
             topk_groups=1, renorm=True, bias=False, logits="f32", train=True),
        # Four decoding sequences: each live expert sees a row or two, the weights are what is read.
        dict(name="experts 4 tokens", op="experts", tokens=4, experts=64, topk=4, d=2048, f=1024, colmajor=False),
        # A prompt through the same kind of layer.
        dict(name="experts 4096 tokens", op="experts", tokens=4096, experts=32, topk=4, d=2048, f=1024, colmajor=False),
        # Training backward of the experts' first product: a ragged batch on few experts ...
        dict(name="experts_backward ragged", op="experts_backward", tokens=777, experts=16, topk=2, d=1024, f=1000,
             colmajor=True, bias=True),
        # ... and a full one.
        dict(name="experts_backward 4096", op="experts_backward", tokens=4096, experts=32, topk=4, d=2048, f=1024,
             colmajor=False, bias=False),
    ]


def _log(rng, low, high, step=1):
    v = math.exp(rng.uniform(math.log(low), math.log(high)))
    return max(low, min(high, int(round(v / step)) * step))


def draw(rng):
    op = rng.choice(["linear", "linear", "linear_backward", "route", "experts", "experts_backward"])
    step = rng.choice([1, 8, 8, 64])
    flag = lambda: rng.random() < 0.5  # noqa: E731
    if op in ("linear", "linear_backward"):
        back = op == "linear_backward"
        gated = flag()
        case = dict(op=op, m=_log(rng, 64 if back else 1, 4096), k=_log(rng, 256, 4096, step),
                    n=_log(rng, 256, 4096, step), act=rng.choice(["silu", "gelu", "relu"] if gated else list(ACTS)),
                    gated=gated, colmajor=flag(), bias=flag())
        if not back:
            case.update(residual=flag(), keep_z=flag(), y=rng.choice(["bf16", "bf16", "f32"]))
        return case
    if op == "route":
        experts = rng.choice([8, 16, 64, 128, 256])
        groups = rng.choice([1, 1, 4])
        return dict(op=op, tokens=_log(rng, 1, 16384), experts=experts, topk=rng.choice([1, 2, 4]), score=rng.choice(list(SCORES)),
                    groups=groups, topk_groups=2 if groups > 1 else 1, renorm=flag(), bias=flag(),
                    logits=rng.choice(["f32", "bf16"]), train=flag())
    experts = rng.choice([8, 16, 32])
    case = dict(op=op, tokens=_log(rng, 64 if op == "experts_backward" else 1, 4096), experts=experts, topk=rng.choice([1, 2, 4]),
                d=_log(rng, 256, 2048, step), f=_log(rng, 256, 1024, step), colmajor=flag())
    if op == "experts_backward":
        case.update(bias=flag())
    return case


# --- sizes ---------------------------------------------------------------------------------

def _rows(tokens, topk, experts):
    pairs = tokens * topk
    return (pairs + (BLOCK - 1) * min(experts, pairs)) // BLOCK * BLOCK


def work(case):
    c = case
    if c["op"] in ("linear", "linear_backward"):
        m, k, n = c["m"], c["k"], c["n"]
        wide = 2 * n if c["gated"] else n
        if c["op"] == "linear":
            out = m * n * (4 if c["y"] == "f32" else 2) + (2 * m * wide if c["keep_z"] else 0)
            return {"bytes": 2 * (m * k + k * wide) + (2 * wide if c["bias"] else 0) + (2 * m * n if c["residual"] else 0) + out,
                    "flops": 2 * m * k * wide}
        z = 2 * m * wide if c["gated"] or c["act"] != "none" else 0
        return {"bytes": 2 * (m * k + k * wide) + z + 2 * m * n + 2 * (m * k + k * wide) + (4 * wide if c["bias"] else 0),
                "flops": 4 * m * k * wide}
    t, e, kk = c["tokens"], c["experts"], c["topk"]
    if c["op"] == "route":
        size = 4 if c["logits"] == "f32" else 2
        rows = _rows(t, kk, e)
        byte = size * t * e + (4 * e if c["bias"] else 0) + 8 * t * kk + 4 * (rows + rows // BLOCK + 2 * e + 1 + t * kk)
        if c["train"]:
            byte += 4 * t * kk + size * t * e
        return {"bytes": byte, "flops": 4 * t * e}
    d, f = c["d"], c["f"]
    live = min(e, t * kk)    # experts whose weights a pass can need
    if c["op"] == "experts":
        return {"bytes": 2 * live * 3 * d * f + 4 * t * d + 8 * t * kk, "flops": 6 * t * kk * d * f}
    return {"bytes": 2 * live * 2 * d * f + 2 * e * 2 * d * f + 4 * t * d + 2 * t * kk * 3 * f, "flops": 8 * t * kk * d * f}


# --- inputs --------------------------------------------------------------------------------

def _randn(g, *shape, scale=1.0):
    return (torch.randn(*shape, generator=g, device="cuda") * scale).to(torch.bfloat16)


def _weights(g, experts, k, wide, colmajor):
    lead = () if experts is None else (experts,)
    shape = lead + ((wide, k) if colmajor else (k, wide))
    return _randn(g, *shape, scale=1.0 / math.sqrt(k))


def _pick(g, tokens, experts, topk):
    """Experts of every token, some of them far more popular than others, and weights that sum to 1."""
    lean = torch.randn(experts, generator=g, device="cuda")
    score = torch.randn(tokens, experts, generator=g, device="cuda") + lean
    top, idx = torch.sort(score, dim=1, descending=True, stable=True)
    top, idx = top[:, :topk], idx[:, :topk]
    return idx.to(torch.int32).contiguous(), torch.softmax(top, dim=1).contiguous()


def _plan(idx, experts):
    """The plan of the rows of idx [T][K], as a dict of int32 tensors."""
    pairs, rows = idx.numel(), _rows(idx.shape[0], idx.shape[1], experts)
    dev = idx.device
    flat = idx.reshape(-1).long()
    counts = torch.zeros(experts, dtype=torch.long, device=dev).scatter_add_(0, flat, torch.ones_like(flat))
    ends = torch.cumsum((counts + BLOCK - 1) // BLOCK * BLOCK, 0)
    starts = ends - (counts + BLOCK - 1) // BLOCK * BLOCK
    order = torch.sort(flat, stable=True).indices
    sorted_experts = flat[order]
    at = starts[sorted_experts] + torch.arange(pairs, device=dev) - (torch.cumsum(counts, 0) - counts)[sorted_experts]
    slot = torch.empty(pairs, dtype=torch.long, device=dev)
    slot[order] = at
    row_src = torch.full((rows,), -1, dtype=torch.long, device=dev)
    row_src[at] = order
    first = torch.arange(rows // BLOCK, device=dev) * BLOCK
    block_expert = torch.searchsorted(ends, first, right=True)
    block_expert = torch.where(first < ends[-1], block_expert, torch.full_like(block_expert, -1))
    offsets = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), ends])
    return {k: v.to(torch.int32) for k, v in dict(row_src=row_src, block_expert=block_expert, offsets=offsets, counts=counts,
                                                  slot=slot.view_as(idx)).items()}


def _packed(plan, scratch):
    """The same as the one buffer the entry points take."""
    parts = [plan[k].reshape(-1) for k in ("row_src", "block_expert", "offsets", "counts", "slot")]
    return torch.cat(parts + [torch.zeros(scratch, dtype=torch.int32, device=parts[0].device)])


def _scratch(tokens, topk, experts):
    return (tokens * topk + PLAN_CHUNK - 1) // PLAN_CHUNK * experts


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    c, s = case, {"case": dict(case)}
    dev, bf, f32 = "cuda", torch.bfloat16, torch.float32
    if c["op"] in ("linear", "linear_backward"):
        m, k, n = c["m"], c["k"], c["n"]
        wide = 2 * n if c["gated"] else n
        s["x"] = _randn(g, m, k)
        s["w"] = _weights(g, None, k, wide, c["colmajor"])
        if c["op"] == "linear":
            s["b"] = _randn(g, wide, scale=0.5) if c["bias"] else None
            s["r"] = _randn(g, m, n) if c["residual"] else None
            s["y"] = torch.empty(m, n, device=dev, dtype=f32 if c["y"] == "f32" else bf)
            s["z"] = torch.empty(m, wide, device=dev, dtype=bf) if c["keep_z"] else None
        else:
            s["z"] = _randn(g, m, wide)
            s["dy"] = _randn(g, m, n)
            s["dx"] = torch.empty_like(s["x"])
            s["dw"] = torch.empty_like(s["w"])
            s["db"] = torch.empty(wide, device=dev, dtype=f32) if c["bias"] else None
        return s
    t, e, kk = c["tokens"], c["experts"], c["topk"]
    if c["op"] == "route":
        kind = f32 if c["logits"] == "f32" else bf
        lean = torch.randn(e, generator=g, device=dev) * 0.5
        s["logits"] = (torch.randn(t, e, generator=g, device=dev) * 1.5 + lean).to(kind)
        s["bias"] = torch.randn(e, generator=g, device=dev) * 0.1 if c["bias"] else None
        s["idx"] = torch.empty(t, kk, device=dev, dtype=torch.int32)
        s["weights"] = torch.empty(t, kk, device=dev, dtype=f32)
        rows = _rows(t, kk, e)
        ends = [rows, rows // BLOCK, e + 1, e, t * kk, _scratch(t, kk, e)]
        s["plan"] = torch.zeros(sum(ends), device=dev, dtype=torch.int32)
        s["parts"] = torch.split(s["plan"], ends)
        if c["train"]:
            s["dweights"] = torch.randn(t, kk, generator=g, device=dev)
            s["dlogits"] = torch.empty_like(s["logits"])
        return s
    d, f = c["d"], c["f"]
    rows = _rows(t, kk, e)
    idx, s["weights"] = _pick(g, t, e, kk)
    s["parts"] = _plan(idx, e)
    s["plan"] = _packed(s["parts"], _scratch(t, kk, e))
    s["x"] = _randn(g, t, d)
    s["w1"] = _weights(g, e, d, 2 * f, c["colmajor"])
    if c["op"] == "experts":
        s["idx"] = idx
        s["w2"] = _weights(g, e, f, d, c["colmajor"])
        s["r"] = _randn(g, t, d)
        s["h"] = torch.empty(rows, f, device=dev, dtype=bf)
        s["y"] = torch.empty(rows, d, device=dev, dtype=f32)
        s["out"] = torch.empty(t, d, device=dev, dtype=bf)
    else:
        live = (s["parts"]["row_src"] >= 0)[:, None]
        s["z"] = _randn(g, rows, 2 * f) * live
        s["dy"] = _randn(g, rows, f) * live
        s["dx"] = torch.empty_like(s["x"])
        s["dw"] = torch.empty_like(s["w1"])
        s["db"] = torch.empty(e, 2 * f, device=dev, dtype=f32) if c["bias"] else None
    return s


# --- the framework's calls -----------------------------------------------------------------

def _own(s):
    from paper_2505_01637_b200 import binding as mb

    c = s["case"]
    layout = 1 if c.get("colmajor") else 0
    if c["op"] == "linear":
        mb.morello_linear(ACTS[c["act"]], c["gated"], c["y"] == "f32", layout, c["m"], c["k"], c["n"],
                          s["x"], s["w"], s["b"], s["r"], s["y"], s["z"])
        return {"y": s["y"], "z": s["z"]}
    if c["op"] == "linear_backward":
        mb.morello_linear_backward(ACTS[c["act"]], c["gated"], 0, 0, layout, c["m"], c["k"], c["n"],
                                   s["x"], s["w"], s["z"], s["dy"], s["dx"], s["dw"], s["db"])
        return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}
    t, e, kk = c["tokens"], c["experts"], c["topk"]
    if c["op"] == "route":
        kind = c["logits"] == "f32"
        mb.morello_route(SCORES[c["score"]], c["renorm"], 1.0, kind, t, e, kk, c["groups"], c["topk_groups"],
                         s["logits"], s["bias"], s["idx"], s["weights"])
        mb.morello_expert_plan(t, kk, e, s["idx"], s["plan"])
        row_src, block_expert, offsets, counts, slot, _ = s["parts"]
        out = {"idx": s["idx"], "weights": s["weights"], "row_src": row_src, "block_expert": block_expert,
               "offsets": offsets, "counts": counts, "slot": slot}
        if c["train"]:
            mb.morello_route_backward(SCORES[c["score"]], c["renorm"], 1.0, kind, t, e, kk, s["logits"], s["idx"],
                                      s["dweights"], s["dlogits"])
            out["dlogits"] = s["dlogits"]
        return out
    d, f = c["d"], c["f"]
    if c["op"] == "experts":
        mb.morello_expert_linear(ACTS["silu"], 1, 0, layout, 1, t, kk, e, d, f, s["plan"], s["x"], s["w1"], None, s["h"])
        mb.morello_expert_linear(ACTS["none"], 0, 1, layout, 0, t, kk, e, f, d, s["plan"], s["h"], s["w2"], None, s["y"])
        mb.morello_expert_combine(1, t, kk, e, d, s["plan"], s["weights"], s["y"], s["r"], s["out"])
        return {"out": s["out"]}
    mb.morello_expert_linear_backward(ACTS["silu"], 1, 0, 0, layout, 1, t, kk, e, d, f, s["plan"], s["x"], s["w1"],
                                      s["z"], s["dy"], s["dx"], s["dw"], s["db"])
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


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


def _slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return 0.5 * (1 + torch.erf(z * math.sqrt(0.5))) + z * torch.exp(-0.5 * z * z) * (1 / math.sqrt(2 * math.pi))
    if act == "gelu_tanh":
        u = torch.tanh(math.sqrt(2 / math.pi) * (z + 0.044715 * z * z * z))
        return 0.5 * (1 + u) + 0.5 * z * (1 - u * u) * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * z * z)
    if act == "silu":
        p = 1 / (1 + torch.exp(-z))
        return p * (1 + z * (1 - p))
    return torch.ones_like(z)


def _dz(z, dy, act, gated):
    if not gated:
        return dy * _slope(z, act)
    n = dy.shape[-1]
    gate, up = z[..., :n], z[..., n:]
    return torch.cat([dy * up * _slope(gate, act), dy * _act(gate, act)], dim=-1)


def _route_keys(c, x, bias):
    """(score of every expert, key it is chosen by)"""
    score = 1 / (1 + torch.exp(-x)) if c["score"] == "sigmoid" else x
    return score, score if bias is None else score + bias


def _chosen(c, key):
    if c["groups"] > 1:
        t, per = key.shape[0], c["experts"] // c["groups"]
        grouped = key.view(t, c["groups"], per)
        best = torch.sort(grouped, dim=2, descending=True, stable=True).values
        rank = best[..., 0] + best[..., 1] if c["score"] == "sigmoid" else best[..., 0]
        keep = torch.sort(rank, dim=1, descending=True, stable=True).indices[:, :c["topk_groups"]]
        dead = torch.ones(t, c["groups"], dtype=torch.bool, device=key.device).scatter_(1, keep, False)
        key = grouped.masked_fill(dead[..., None], -math.inf).view(t, -1)
    return torch.sort(key, dim=1, descending=True, stable=True).indices[:, :c["topk"]]


def _route_weights(c, x, idx):
    """Weights of the chosen experts, in x's type."""
    if c["score"] == "sigmoid":
        w = 1 / (1 + torch.exp(-torch.gather(x, 1, idx)))
    else:
        e = torch.exp(x - x.max(dim=1, keepdim=True).values)
        w = torch.gather(e, 1, idx) / e.sum(dim=1, keepdim=True)
    return w / w.sum(dim=1, keepdim=True) if c["renorm"] else w


def _route_slope(c, x, idx, g):
    """Gradient of the logits from the gradient g of the weights."""
    w = _route_weights(c, x, idx)
    full = torch.zeros_like(x)
    if c["score"] == "sigmoid":
        s = 1 / (1 + torch.exp(-torch.gather(x, 1, idx)))
        inner = w * (g - (g * w).sum(dim=1, keepdim=True)) * (1 - s) if c["renorm"] else g * s * (1 - s)
        return full.scatter(1, idx, inner)
    dot = (g * w).sum(dim=1, keepdim=True)
    if c["renorm"]:
        return full.scatter(1, idx, w * (g - dot))
    e = torch.exp(x - x.max(dim=1, keepdim=True).values)
    return full.scatter(1, idx, g * w) - dot * e / e.sum(dim=1, keepdim=True)


def _plain_experts(s, x, w, colmajor):
    """Rows x [R][k] times their experts' weights, block by block."""
    block = s["parts"]["block_expert"].long().clamp(min=0)
    w = w[block].float()
    rows = x.view(len(block), BLOCK, -1)
    return torch.matmul(rows, w.transpose(1, 2) if colmajor else w).view(x.shape[0], -1)


def _gathered(s, x):
    src = s["parts"]["row_src"].long()
    live = (src >= 0)[:, None]
    return torch.where(live, x.float()[src.clamp(min=0) // s["case"]["topk"]], torch.zeros((), device=x.device)), live


def _plain(s):
    c, bf = s["case"], torch.bfloat16
    if c["op"] == "linear":
        w = s["w"].float()
        z = torch.matmul(s["x"].float(), w.t() if c["colmajor"] else w)
        if s["b"] is not None:
            z = z + s["b"].float()
        y = _act(z[:, :c["n"]], c["act"]) * z[:, c["n"]:] if c["gated"] else _act(z, c["act"])
        if s["r"] is not None:
            y = y + s["r"].float()
        return {"y": y.to(s["y"].dtype), "z": z.to(bf) if c["keep_z"] else None}
    if c["op"] == "linear_backward":
        x, w = s["x"].float(), s["w"].float()
        dz = _dz(s["z"].float(), s["dy"].float(), c["act"], c["gated"])
        dx = torch.matmul(dz, w if c["colmajor"] else w.t())
        dw = torch.matmul(dz.t(), x) if c["colmajor"] else torch.matmul(x.t(), dz)
        return {"dx": dx.to(bf), "dw": dw.to(bf), "db": dz.sum(dim=0) if c["bias"] else None}
    if c["op"] == "route":
        x = s["logits"].float()
        _, key = _route_keys(c, x, s["bias"])
        idx = _chosen(c, key)
        plan = _plan(idx.to(torch.int32), c["experts"])
        out = {"idx": idx.to(torch.int32), "weights": _route_weights(c, x, idx), **plan, "slot": plan["slot"].reshape(-1)}
        if c["train"]:
            out["dlogits"] = _route_slope(c, x, idx, s["dweights"]).to(s["logits"].dtype)
        return out
    rows, live = _gathered(s, s["x"])
    if c["op"] == "experts":
        z = _plain_experts(s, rows, s["w1"], c["colmajor"])
        h = _act(z[:, :c["f"]], "silu") * z[:, c["f"]:]
        y = _plain_experts(s, h, s["w2"], c["colmajor"])
        slot = s["parts"]["slot"].long()
        out = (y[slot] * s["weights"][..., None]).sum(dim=1) + s["r"].float()
        return {"out": out.to(bf)}
    dz = _dz(s["z"].float(), s["dy"].float(), "silu", True) * live
    block = s["parts"]["block_expert"].long()
    # dX of a row, block by block, then the sum over a token's rows
    dx = _plain_experts(s, dz, s["w1"], not c["colmajor"])
    slot = s["parts"]["slot"].long()
    dx = dx[slot].sum(dim=1)
    a, b = rows.view(len(block), BLOCK, -1), dz.view(len(block), BLOCK, -1)
    each = torch.matmul(b.transpose(1, 2), a) if c["colmajor"] else torch.matmul(a.transpose(1, 2), b)
    dw = torch.zeros(s["w1"].shape, device=each.device).index_add_(0, block.clamp(min=0), each)
    db = torch.zeros(c["experts"], 2 * c["f"], device=each.device).index_add_(0, block.clamp(min=0), b.sum(dim=1))
    return {"dx": dx.to(bf), "dw": dw.to(bf), "db": db if c["bias"] else None}


def run(state):
    return _own(state) if own else _plain(state)


# --- the definitions in 64 bits ------------------------------------------------------------

def _act64(z, act):
    one = {"none": lambda: z, "relu": lambda: z.clamp(min=0),
           "gelu": lambda: z * torch.special.ndtr(z),
           "gelu_tanh": lambda: z * torch.sigmoid(2 * math.sqrt(2 / math.pi) * (z + 0.044715 * z ** 3)),
           "silu": lambda: z * torch.sigmoid(z)}
    return one[act]()


def _forward64(x, w, b, r, act, gated):
    z = x @ w
    if b is not None:
        z = z + b
    if gated:
        gate, up = z.chunk(2, dim=-1)
        y = _act64(gate, act) * up
    else:
        y = _act64(z, act)
    return z, y if r is None else y + r


def _dz64(z, dy, act, gated):
    """dY carried back to Z by differentiating the definition."""
    with torch.enable_grad():
        z = z.clone().requires_grad_(True)
        if gated:
            gate, up = z.chunk(2, dim=-1)
            y = _act64(gate, act) * up
        else:
            y = _act64(z, act)
        return torch.autograd.grad(y, z, dy)[0]


def _route64(c, s):
    x = s["logits"].double()
    x32 = s["logits"].float()
    _, key = _route_keys(c, x32, s["bias"])    # the choice is made on 32-bit keys: that is its definition
    idx = _chosen(c, key)
    out = {"idx": None, "row_src": None, "block_expert": None, "offsets": None, "counts": None, "slot": None}
    with torch.enable_grad():
        x = x.clone().requires_grad_(True)
        p = torch.sigmoid(x) if c["score"] == "sigmoid" else torch.softmax(x, dim=1)
        w = torch.gather(p, 1, idx)
        if c["renorm"]:
            w = w / w.sum(dim=1, keepdim=True)
        out["weights"] = w.detach()
        if c["train"]:
            out["dlogits"] = torch.autograd.grad(w, x, s["dweights"].double())[0]
    return out


def exact(case, seed):
    c, s = case, prepare(case, seed)
    dbl = lambda v: None if v is None else v.double()  # noqa: E731
    if c["op"] == "linear":
        w = s["w"].double()
        z, y = _forward64(s["x"].double(), w.t() if c["colmajor"] else w, dbl(s["b"]), dbl(s["r"]), c["act"], c["gated"])
        return {"y": y, "z": z if c["keep_z"] else None}
    if c["op"] == "linear_backward":
        w = s["w"].double()
        dz = _dz64(s["z"].double(), s["dy"].double(), c["act"], c["gated"])
        dw = s["x"].double().t() @ dz
        return {"dx": dz @ (w if c["colmajor"] else w.t()), "dw": dw.t() if c["colmajor"] else dw,
                "db": dz.sum(dim=0) if c["bias"] else None}
    if c["op"] == "route":
        return _route64(c, s)
    # Experts: token by token is the definition; the rows of one expert are taken together.
    parts = {k: v.cpu() for k, v in s["parts"].items()}
    x = s["x"].double()
    result = torch.zeros_like(x)
    if c["op"] == "experts":
        result += s["r"].double()
        weight = s["weights"].double()
    else:
        dw = torch.zeros(s["w1"].shape, dtype=torch.float64, device="cuda")
        db = torch.zeros(c["experts"], 2 * c["f"], dtype=torch.float64, device="cuda")
    for e in range(c["experts"]):
        first, count = int(parts["offsets"][e]), int(parts["counts"][e])
        if count == 0:
            continue
        src = parts["row_src"][first:first + count].long().cuda()
        token, place = src // c["topk"], src % c["topk"]
        w1 = s["w1"][e].double()
        w1 = w1.t() if c["colmajor"] else w1
        if c["op"] == "experts":
            w2 = s["w2"][e].double()
            _, h = _forward64(x[token], w1, None, None, "silu", True)
            result.index_add_(0, token, (h @ (w2.t() if c["colmajor"] else w2)) * weight[token, place][:, None])
        else:
            z, dy = (s[k][first:first + count].double() for k in ("z", "dy"))
            dz = _dz64(z, dy, "silu", True)
            result.index_add_(0, token, dz @ w1.t())
            one = x[token].t() @ dz
            dw[e] = one.t() if c["colmajor"] else one
            db[e] = dz.sum(dim=0)
    if c["op"] == "experts":
        return {"out": result}
    return {"dx": result, "dw": dw, "db": db if c["bias"] else None}
