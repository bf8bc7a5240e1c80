"""What is timed of layers in 8 bits: layer norm with 8-bit rows, and its gradient
from sums that were kept in 8 bits; rows and weights put into 8 bits; the product of
8-bit rows with 8-bit weights, a scale for each 128 elements of a row and each 128 x
128 elements of the weights; and the weights' gradient from the rows kept in 8 bits.

A case is a dict of plain sizes and options, `op` naming the operator.
`prepare` makes a case's seeded inputs on the GPU, with the output buffers (and
the workspace) a training or serving program keeps; `run` is one call of the
operator.  Where `own` is false, `run` computes the same from elementary torch
operations in 32 bits.
"""
import math

import torch

own = False

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E4M3 = torch.float8_e4m3fn
TORCH = {"fp32": F32, "fp16": F16, "bf16": BF16}
SIZE = {"fp32": 4, "fp16": 2, "bf16": 2}
QMAX = 448.0            # the largest e4m3 number
TINY = 2.0 ** -126      # the smallest scale
BLOCK = 128             # rows and columns of the weights that share a scale


def _norm(name, n, dim, x, res, group=BLOCK, y=False, kept=False):
    return _named(name, dict(op="norm", n=n, dim=dim, x=x, res=res, group=group, y=y, kept=kept))


def _norm_grad(name, n, dim, x, res, kept, group=BLOCK):
    return _named(name, dict(op="norm_grad", n=n, dim=dim, x=x, res=res, kept=kept, group=group))


def _rows(name, n, dim, x, group=BLOCK):
    return _named(name, dict(op="rows", n=n, dim=dim, x=x, group=group))


def _blocks(name, n, dim, x, both=True):
    return _named(name, dict(op="blocks", n=n, dim=dim, x=x, both=both))


def _product(name, n, k, m, out, group=BLOCK):
    return _named(name, dict(op="product", n=n, k=k, m=m, out=out, group=group))


def _product_grad(name, n, k, m, dz, out, group=BLOCK, add=False):
    return _named(name, dict(op="product_grad", n=n, k=k, m=m, dz=dz, out=out, group=group, add=add))


def _named(name, c):
    return dict(c, name=name) if name else c


def listed():
    return [
        # Four tokens of a decoding step: residual, normed row in 16 and 8 bits; latency.
        _norm("layernorm_tokens", 4, 8192, "bf16", True, y=True),
        # A training step: residual, its 16-bit sum, the 8-bit row for the next
        # product and the sum in 8 bits for the way back.
        _norm("layernorm_prompt", 32_768, 4096, "bf16", True, kept=True),
        # The way back from sums kept in 8 bits, an odd number of tokens.
        _norm_grad("layernorm_grad_kept", 16_383, 4096, "bf16", True, True),
        # Learned rows of the width of Reddit-shaped features, all in fp32.
        _norm_grad("layernorm_grad_nodes", 233_000, 602, "fp32", False, False),
        # The gradient of a wide layer's output, before it meets the weights in 8 bits.
        _rows("rows_gradient", 8191, 16_384, "bf16"),
        # A layer's master weights after a step, for the product and its way back.
        _blocks("blocks_weights", 16_384, 4096, "fp32"),
        # One token of a decoding step: latency, and the weights' bytes.
        _product("product_token", 1, 4096, 16_384, "bf16"),
        # The tokens of a decoding step of 96 sequences.
        _product("product_batch", 96, 8192, 8192, "bf16"),
        # A batch of seeds of a 47-class graph, learned rows of 100 with one scale each: the
        # student's head; latency.
        _product("product_classes", 1024, 100, 47, "fp32", group=0),
        # A prompt or training step of a wide layer, an odd number of tokens.
        _product("product_prompt", 8191, 4096, 16_384, "bf16"),
        # The gradient of a wide layer's weights.
        _product_grad("product_grad_tokens", 16_384, 4096, 8192, "bf16", "bf16"),
        # Reddit-shaped features and 41 classes, the whole graph's rows at once: few
        # sums, each over many rows.
        _product_grad("product_grad_nodes", 233_000, 602, 41, "fp32", "fp32", group=0),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    while True:
        c = _drawn(rng)
        w = work(c)
        if w["bytes"] <= 1.8e9 and w["flops"] <= 1.0e12:
            return c


def _drawn(rng):
    op = rng.choice(["norm", "norm_grad", "rows", "blocks", "product", "product_grad"])
    t16 = rng.choice(["fp16", "bf16"])
    t = rng.choice(["fp32", t16])
    if op == "norm":
        return _norm("", _log(rng, 1, 300_000), _log(rng, 16, 8192), t, rng.random() < 0.6,
                     rng.choice([0, 32, 64, 128, 128]), rng.random() < 0.4, rng.random() < 0.5)
    if op == "norm_grad":
        return _norm_grad("", _log(rng, 1, 300_000), _log(rng, 16, 8192), t, rng.random() < 0.6,
                          rng.random() < 0.6, rng.choice([0, 32, 64, 128, 128]))
    if op == "rows":
        return _rows("", _log(rng, 1, 300_000), _log(rng, 16, 128_000), t,
                     rng.choice([0, 32, 128, 128]))
    if op == "blocks":
        return _blocks("", _log(rng, 16, 65_536), _log(rng, 16, 16_384), t, rng.random() < 0.7)
    n, k, m = _log(rng, 1, 65_536), _log(rng, 16, 16_384), _log(rng, 16, 65_536)
    if rng.random() < 0.5:      # the widths of a layer that was made for the machine
        k, m = -(-k // BLOCK) * BLOCK, -(-m // 64) * 64
    group = rng.choice([0, BLOCK, BLOCK])
    if op == "product":
        return _product("", n, k, m, t, group)
    return _product_grad("", n, k, m, t, rng.choice([t, "fp32"]), group, rng.random() < 0.3)


# ---------------------------------------------------------------------------
# Work.
# ---------------------------------------------------------------------------
def _groups(dim, group):
    return -(-dim // group) if group else 1


def _row8(dim, group):
    """Bytes of an 8-bit row and its scales."""
    return dim + 4 * _groups(dim, group)


def _block8(rows, cols):
    """Bytes of 8-bit weights and their scales."""
    return rows * cols + 4 * _groups(rows, BLOCK) * _groups(cols, BLOCK)


def work(c):
    n, op = c["n"], c["op"]
    if op in ("norm", "norm_grad"):
        d, x, q = c["dim"], c["dim"] * SIZE[c["x"]], _row8(c["dim"], c["group"])
        if op == "norm":
            b = x * (1 + 2 * c["res"] + c["y"]) + q * (1 + c["kept"]) + 8
            return {"bytes": n * b + 2 * x, "flops": 9 * n * d}
        b = x * (2 + c["res"]) + (q if c["kept"] else x) + 8
        return {"bytes": n * b + x + 8 * d, "flops": 13 * n * d}
    if op == "rows":
        d = c["dim"]
        return {"bytes": n * (d * SIZE[c["x"]] + _row8(d, c["group"])), "flops": 3 * n * d}
    if op == "blocks":
        d = c["dim"]
        return {"bytes": n * d * SIZE[c["x"]] + _block8(n, d) * (1 + c["both"]), "flops": 3 * n * d}
    k, m = c["k"], c["m"]
    rows = n * _row8(k, c["group"])
    if op == "product":
        b = rows + _block8(m, k) + n * m * SIZE[c["out"]]
    else:
        b = rows + n * m * SIZE[c["dz"]] + m * k * SIZE[c["out"]] * (1 + c["add"])
    return {"bytes": b, "flops": 2 * n * m * k}


# ---------------------------------------------------------------------------
# Seeded inputs.
# ---------------------------------------------------------------------------
def _randn(g, n, d, dtype=F32, std=1.0):
    return (torch.randn(n, d, generator=g, device="cuda") * std).to(dtype)


def _strong(g, n, d):
    """Rows with a few strong columns, as residual streams have."""
    x = _randn(g, n, d)
    x[:, :: max(1, d // 7)] *= 12
    return x


def _empty(*shape, dtype=F32):
    return torch.empty(shape, dtype=dtype, device="cuda")


def _as_rows8(x, group):
    """Codes and scales of x in 8 bits."""
    d = x.shape[1]
    scales = (_tops(x, group) / QMAX).clamp(min=TINY)
    return (x / _spread(scales, d, group)).clamp(-QMAX, QMAX).to(E4M3), scales


def _as_blocks8(w):
    n, d = w.shape
    scales = (_tops(_tops(w, BLOCK).t(), BLOCK).t().contiguous() / QMAX).clamp(min=TINY)
    return (w / _spread_blocks(scales, n, d)).clamp(-QMAX, QMAX).to(E4M3), scales


def _tops(x, group):
    """Largest magnitude of each group of a row's elements."""
    n, d = x.shape
    group = group or d
    k = -(-d // group)
    return torch.nn.functional.pad(x.abs(), (0, k * group - d)).view(n, k, group).amax(2)


def _spread(scales, dim, group):
    """A scale for each of a row's elements."""
    return scales.repeat_interleave(group, 1)[:, :dim] if group else scales


def _spread_blocks(scales, n, d):
    return scales.repeat_interleave(BLOCK, 0)[:n].repeat_interleave(BLOCK, 1)[:, :d]


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    c, s = case, {"c": case}
    n, op, group = c["n"], c["op"], c.get("group", 0)
    if op in ("norm", "norm_grad"):
        d, dt = c["dim"], TORCH[c["x"]]
        s["eps"] = 1e-5
        s["w"] = (1 + 0.2 * torch.randn(d, generator=g, device="cuda")).to(dt)
        s["b"] = (0.1 * torch.randn(d, generator=g, device="cuda")).to(dt)
        x = _strong(g, n, d) + 0.5       # means that are not zero
        s["mean"], s["rstd"] = _empty(n), _empty(n)
        if op == "norm":
            s["x"] = x.to(dt)
            s["res"] = _randn(g, n, d, dt, 2.0) if c["res"] else None
            s["sum"] = _empty(n, d, dtype=dt) if c["res"] else None
            s["y"] = _empty(n, d, dtype=dt) if c["y"] else None
            s["q"], s["q_scales"] = _empty(n, d, dtype=E4M3), _empty(n, _groups(d, group))
            if c["kept"]:
                s["kept"], s["kept_scales"] = _empty(n, d, dtype=E4M3), _empty(n, _groups(d, group))
        else:
            x = x.to(dt)
            x64 = x.double()
            var, mean = torch.var_mean(x64, 1, correction=0)
            s["mean"], s["rstd"] = mean.float(), torch.rsqrt(var + s["eps"]).float()
            if c["kept"]:
                s["s"], s["s_scales"] = _as_rows8(x.float(), group)
            else:
                s["s"] = x
            s["dy"] = _randn(g, n, d, dt, 0.01)
            s["dsum"] = _randn(g, n, d, dt, 0.01) if c["res"] else None
            s["dx"], s["dw"], s["db"] = _empty(n, d, dtype=dt), _empty(d), _empty(d)
    elif op == "rows":
        # gradients: rows of very different size
        d = c["dim"]
        x = _randn(g, n, d) * torch.exp(_randn(g, n, 1) * 2 - 6)
        s["x"] = x.to(TORCH[c["x"]])
        s["q"], s["q_scales"] = _empty(n, d, dtype=E4M3), _empty(n, _groups(d, group))
    elif op == "blocks":
        d = c["dim"]
        s["x"] = _randn(g, n, d, TORCH[c["x"]], d ** -0.5)
        s["q"], s["q_scales"] = _empty(n, d, dtype=E4M3), _empty(_groups(n, BLOCK), _groups(d, BLOCK))
        if c["both"]:
            s["qt"] = _empty(d, n, dtype=E4M3)
            s["qt_scales"] = _empty(_groups(d, BLOCK), _groups(n, BLOCK))
    else:
        k, m = c["k"], c["m"]
        s["a"], s["a_scales"] = _as_rows8(_strong(g, n, k), group)
        if op == "product":
            s["w"], s["w_scales"] = _as_blocks8(_randn(g, m, k, std=k ** -0.5))
            s["out"] = _empty(n, m, dtype=TORCH[c["out"]])
        else:
            s["dz"] = (_randn(g, n, m) * torch.exp(_randn(g, n, 1) - 4)).to(TORCH[c["dz"]])
            s["dw"] = _empty(m, k, dtype=TORCH[c["out"]])
            if c["add"]:        # what an earlier part of the batch gave
                s["before"] = _randn(g, m, k, TORCH[c["out"]], 0.02)
    if own:
        _keep(s)
    return s


def _keep(s):
    """The descriptions of the tensors and the workspace that a program keeps
    beside its buffers."""
    from paper_2606_02916_amd import gg
    c = s["c"]
    group, op = c.get("group", 0), c["op"]
    s["r"] = r = {}
    for k in ("x", "res", "sum", "y", "q", "kept", "s", "dy", "dsum", "dx", "a", "out", "dz", "dw",
              "qt", "w"):
        t = s.get(k)
        if t is None or t.dim() != 2:
            continue
        if t.dtype != E4M3:
            r[k] = gg.make_rows(t)
        elif op == "blocks" or k == "w":
            r[k] = gg.make_blocks(t, s[k + "_scales"])
        else:
            r[k] = gg.make_rows(t, scales=s[k + "_scales"], group=group)
    size = {"norm_grad": lambda: gg.gg_ws_layernorm(c["n"], c["dim"]),
            "product_grad": lambda: gg.gg_ws_product(c["n"], c["k"], c["m"]),
            }.get(op, lambda: 0)()
    s["ws"] = torch.empty(max(size, 1), dtype=torch.uint8, device="cuda")


# ---------------------------------------------------------------------------
# One pass.
# ---------------------------------------------------------------------------
def run(s):
    return (_run_own if own else _run_plain)[s["c"]["op"]](s)


def _norm_outputs(s, o):
    c, out = s["c"], {k: o[k] for k in ("mean", "rstd", "q", "q_scales")}
    for k, wanted in (("sum", c["res"]), ("y", c["y"]), ("kept", c["kept"]),
                      ("kept_scales", c["kept"])):
        if wanted:
            out[k] = o[k]
    return out


def _own_norm(s):
    from paper_2606_02916_amd import gg
    c, r = s["c"], s["r"]
    gg.gg_layernorm_forward(r["x"], r.get("res"), c["n"], c["dim"], s["w"], s["b"], s["eps"],
                            r.get("sum"), r.get("y"), r["q"], r.get("kept"), s["mean"], s["rstd"])
    return _norm_outputs(s, s)


def _own_norm_grad(s):
    from paper_2606_02916_amd import gg
    c, r = s["c"], s["r"]
    gg.gg_layernorm_backward(r["dy"], r.get("dsum"), r["s"], s["mean"], s["rstd"], c["n"], c["dim"],
                             s["w"], r["dx"], s["dw"], s["db"], s["ws"])
    return {"dx": s["dx"], "dw": s["dw"], "db": s["db"]}


def _own_rows(s):
    from paper_2606_02916_amd import gg
    c, r = s["c"], s["r"]
    gg.gg_quantise_rows(r["x"], c["n"], c["dim"], r["q"])
    return {"q": s["q"], "q_scales": s["q_scales"]}


def _own_blocks(s):
    from paper_2606_02916_amd import gg
    c, r = s["c"], s["r"]
    gg.gg_quantise_blocks(r["x"], c["n"], c["dim"], r["q"], r.get("qt"))
    out = {"q": s["q"], "q_scales": s["q_scales"]}
    if c["both"]:
        out["qt"], out["qt_scales"] = s["qt"], s["qt_scales"]
    return out


def _own_product(s):
    from paper_2606_02916_amd import gg
    c, r = s["c"], s["r"]
    gg.gg_product_forward(r["a"], c["n"], c["k"], r["w"], c["m"], r["out"])
    return {"out": s["out"]}


def _own_product_grad(s):
    from paper_2606_02916_amd import gg
    c, r = s["c"], s["r"]
    if c["add"]:
        s["dw"].copy_(s["before"])
    gg.gg_product_backward(r["a"], c["n"], c["k"], r["dz"], c["m"], r["dw"],
                           gg.GG_PRODUCT_ADD if c["add"] else 0, s["ws"])
    return {"dw": s["dw"]}


def _plain_norm(s):
    c = s["c"]
    x, o = s["x"].float(), {}
    if c["res"]:
        x = x + s["res"].float()
        o["sum"] = x.to(s["x"].dtype)
    if c["kept"]:
        o["kept"], o["kept_scales"] = _as_rows8(x, c["group"])
    o["mean"] = x.mean(1)
    x = x - o["mean"][:, None]
    o["rstd"] = torch.rsqrt(x.square().mean(1) + s["eps"])
    y = x * o["rstd"][:, None] * s["w"].float() + s["b"].float()
    if c["y"]:
        o["y"] = y.to(s["x"].dtype)
    o["q"], o["q_scales"] = _as_rows8(y, c["group"])
    return _norm_outputs(s, o)


def _plain_norm_grad(s):
    c, r = s["c"], s["rstd"][:, None]
    x = s["s"].float()
    if c["kept"]:
        x = x * _spread(s["s_scales"], c["dim"], c["group"])
    dy = s["dy"].float()
    xhat = (x - s["mean"][:, None]) * r
    g = dy * s["w"].float()
    dx = r * (g - g.mean(1, keepdim=True) - xhat * (g * xhat).mean(1, keepdim=True))
    if s["dsum"] is not None:
        dx = dx + s["dsum"].float()
    return {"dx": dx.to(s["dy"].dtype), "dw": (dy * xhat).sum(0), "db": dy.sum(0)}


def _plain_rows(s):
    q, scales = _as_rows8(s["x"].float(), s["c"]["group"])
    return {"q": q, "q_scales": scales}


def _plain_blocks(s):
    q, scales = _as_blocks8(s["x"].float())
    out = {"q": q, "q_scales": scales}
    if s["c"]["both"]:
        # 8-bit tensors are moved as bytes
        out["qt"] = q.view(torch.uint8).t().contiguous().view(E4M3)
        out["qt_scales"] = scales.t().contiguous()
    return out


def _numbers(s):
    """The 8-bit rows a as fp32 numbers."""
    return s["a"].float() * _spread(s["a_scales"], s["c"]["k"], s["c"]["group"])


def _plain_product(s):
    c = s["c"]
    w = s["w"].float() * _spread_blocks(s["w_scales"], c["m"], c["k"])
    return {"out": (_numbers(s) @ w.t()).to(s["out"].dtype)}


def _plain_product_grad(s):
    dw = s["dz"].float().t() @ _numbers(s)
    if s["c"]["add"]:
        dw = dw + s["before"].float()
    return {"dw": dw.to(s["dw"].dtype)}


_run_own = {"norm": _own_norm, "norm_grad": _own_norm_grad, "rows": _own_rows, "blocks": _own_blocks,
            "product": _own_product, "product_grad": _own_product_grad}
_run_plain = {"norm": _plain_norm, "norm_grad": _plain_norm_grad, "rows": _plain_rows,
              "blocks": _plain_blocks, "product": _plain_product,
              "product_grad": _plain_product_grad}


# ---------------------------------------------------------------------------
# The definitions in 64 bits, rows at a time.
# ---------------------------------------------------------------------------
def exact(case, seed):
    global own
    was, own = own, False
    try:
        s = prepare(case, seed)
    finally:
        own = was
    op, n = case["op"], case["n"]
    if op == "blocks":
        return _exact_blocks(s)
    piece = {"norm": _exact_norm, "norm_grad": _exact_norm_grad, "rows": _exact_rows,
             "product": _exact_product, "product_grad": _exact_product_grad}[op]
    step = max(1, (1 << 27) // max(case.get(k, 1) for k in ("dim", "k", "m")))
    got, sums = {}, {}
    for i in range(0, n, step):
        rows, added = piece(s, slice(i, min(n, i + step)))
        for k, x in rows.items():
            got.setdefault(k, []).append(x)
        for k, x in added.items():
            sums[k] = sums[k] + x if k in sums else x
    return {**{k: torch.cat(x) for k, x in got.items()}, **sums}


def _exact_codes(y, group):
    """Scales, and codes that are not rounded."""
    parts = y.split(group or y.shape[1], 1)
    scales = (torch.stack([p.abs().max(1).values for p in parts], 1) / QMAX).clamp_min(TINY)
    return torch.cat([p / scales[:, j, None] for j, p in enumerate(parts)], 1), scales


def _exact_numbers(codes, scales, group):
    """code * scale; codes as bytes through a table of their values."""
    table = torch.arange(256, dtype=torch.uint8, device="cuda").view(E4M3).double()
    col = torch.arange(codes.shape[1], device="cuda") // (group or codes.shape[1])
    return table[codes.view(torch.uint8).long()] * scales.double()[:, col]


def _exact_norm(s, b):
    c, got = s["c"], {}
    x = s["x"][b].double()
    if c["res"]:
        x += s["res"][b].double()
        got["sum"] = x.clone()
    if c["kept"]:
        got["kept"], got["kept_scales"] = _exact_codes(x, c["group"])
    got["mean"] = x.sum(1) / c["dim"]
    x -= got["mean"][:, None]
    got["rstd"] = 1 / torch.sqrt((x * x).sum(1) / c["dim"] + s["eps"])
    y = torch.addcmul(s["b"].double(), x, s["w"].double() * got["rstd"][:, None])
    if c["y"]:
        got["y"] = y
    got["q"], got["q_scales"] = _exact_codes(y, c["group"])
    return got, {}


def _exact_norm_grad(s, b):
    c, d = s["c"], s["c"]["dim"]
    if c["kept"]:
        x = _exact_numbers(s["s"][b], s["s_scales"][b], c["group"])
    else:
        x = s["s"][b].double()
    r = s["rstd"][b].double()[:, None]
    x = x - s["mean"][b].double()[:, None]
    dy = s["dy"][b].double()
    g = dy * s["w"].double()
    dx = r * g - r * g.sum(1, keepdim=True) / d - x * (r ** 3 * (g * x).sum(1, keepdim=True) / d)
    if s["dsum"] is not None:
        dx += s["dsum"][b].double()
    return {"dx": dx}, {"dw": (dy * x * r).sum(0), "db": dy.sum(0)}


def _exact_rows(s, b):
    q, scales = _exact_codes(s["x"][b].double(), s["c"]["group"])
    return {"q": q, "q_scales": scales}, {}


def _exact_blocks(s):
    x = s["x"].double()
    scales = torch.stack([torch.stack([p.abs().max() for p in band.split(BLOCK, 1)])
                          for band in x.split(BLOCK, 0)]) / QMAX
    scales.clamp_min_(TINY)
    row = torch.arange(x.shape[0], device="cuda") // BLOCK
    col = torch.arange(x.shape[1], device="cuda") // BLOCK
    x /= scales[row][:, col]
    out = {"q": x, "q_scales": scales}
    if s["c"]["both"]:
        out["qt"], out["qt_scales"] = x.t().contiguous(), scales.t().contiguous()
    return out


def _exact_product(s, b):
    c = s["c"]
    a = _exact_numbers(s["a"][b], s["a_scales"][b], c["group"])
    band = torch.arange(c["m"], device="cuda") // BLOCK
    w = _exact_numbers(s["w"], s["w_scales"][band], BLOCK)
    return {"out": torch.mm(a, w.t())}, {}


def _exact_product_grad(s, b):
    c = s["c"]
    a = _exact_numbers(s["a"][b], s["a_scales"][b], c["group"])
    dw = torch.mm(s["dz"][b].double().t(), a)
    if c["add"] and b.start == 0:
        dw += s["before"].double()
    return {}, {"dw": dw}
