"""The calls for layers in 8 bits together: a student with a layer norm, students whose
head runs on 8-bit rows, stage by stage against 64 bits; a captured layer replayed."""
import os
import textwrap

import pytest
import torch

from tests import helpers
from tests.op_util import BF16, E4M3, F16, F32, FLOOR, U, UNIT, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def lesson(n, N, dim, classes, k, seed=2):
    g = torch.Generator().manual_seed(seed)
    ids = torch.randint(0, N, (n,), generator=g)
    ids[n // 3: n // 2] = -1
    top_ids = torch.randint(0, classes, (n, k), generator=g)
    top_ids[::7, 2:] = -1
    return ids, top_ids, torch.randn(n, k, generator=g) * 2, torch.randn(n, dim, generator=g)


def numbers(codes, rows):
    """What 8-bit rows stand for, in 64 bits."""
    d = codes.shape[1]
    return codes.float().cpu().double() * rows.keep[1].cpu().double()[:, torch.arange(d) // 128]


def weights(codes, blocks):
    r, c = codes.shape
    sc = blocks.keep[1].cpu().double()
    return codes.float().cpu().double() * sc[torch.arange(r) // 128][:, torch.arange(c) // 128]


@pytest.mark.parametrize("n,dim,classes", [(1, 16, 5), (301, 100, 47), (2000, 33, 300)])
def test_a_step_with_a_layer_norm(n, dim, classes):
    """Against the same step in 64 bits, within a hundred roundings of fp32 of each
    gradient's largest entry: the products' sums add about as many."""
    from paper_2606_02916_amd import Student
    k, N = 4, 400
    st = Student(N, dim, classes, max_rows=2500, k=k, rate=0.5, device=DEV, generator=gen(n), norm="layer",
                 eps=1e-3)
    st.w.copy_(1 + 0.2 * torch.randn(dim, generator=gen(1), device=DEV))
    st.b.copy_(torch.randn(dim, generator=gen(2), device=DEV))
    ids, top_ids, top, x = lesson(n, N, dim, classes, k)
    names = ("table", "w", "b", "head")
    before = [getattr(st, a).clone() for a in names]
    p = [t.detach().cpu().double().requires_grad_(True) for t in before]
    e = torch.where((ids >= 0)[:, None], p[0][ids.clamp(min=0)], 0.0) * st.scale
    s = e + x.double()
    c = s - s.mean(1, keepdim=True)
    y = c * (c.square().mean(1, keepdim=True) + st.eps) ** -0.5 * p[1] + p[2]
    lq = torch.log_softmax(y @ p[3] / st.temperature, 1)
    hole = top_ids < 0
    lp = torch.log_softmax((top.double() / st.temperature).masked_fill(hole, -float("inf")), 1)
    q = lp.exp().masked_fill(hole, 0)
    lp = lp.masked_fill(hole, 0)
    want = (q * (lp - lq.gather(1, top_ids.clamp(min=0)))).sum(1) * st.temperature ** 2
    want = want * torch.tensor(1.0 / n, dtype=F32).double()
    want.sum().backward()
    loss = st.step(ids.to(DEV), n, top_ids.to(DEV), top.to(DEV), x.to(DEV)).cpu().double()
    assert int(st.status) == 0
    want = want.detach()
    assert float((loss - want).abs().max()) <= 100 * U * float(want.abs().max())
    tol = 100 + dim + classes + n
    for name, old, t in zip(names, before, p):
        moved = getattr(st, name).cpu().double() - (old.cpu().double() - st.rate * t.grad)
        bound = 2 * U * old.cpu().double().abs() + tol * U * st.rate * float(t.grad.abs().max())
        assert bool((moved.abs() <= bound).all()), name


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,dim,classes", [(1, 16, 5), (301, 100, 47), (1500, 260, 300)])
def test_a_step_on_8_bit_rows(n, dim, classes, t, norm):
    """Every stage against its formula in 64 bits on what the stage before gave: 8-bit
    rows, logits, their gradient, the gradients of head, norm and table."""
    from paper_2606_02916_amd import Student
    k, N = 4, 400
    st = Student(N, dim, classes, max_rows=1600, k=k, rate=0.5, dtype=t, device=DEV, generator=gen(n),
                 norm=norm, eight_bit=True, eps=1e-3)
    st.w.copy_(1 + 0.2 * torch.randn(dim, generator=gen(1), device=DEV))
    ids, top_ids, top, x = lesson(n, N, dim, classes, k)
    ids_d, x_d = ids.to(DEV), x.to(t).to(DEV)
    before = {a: getattr(st, a).clone() for a in ("table", "w", "head")}
    z = st.forward(ids_d, n, x_d).cpu().double()
    # the 8-bit rows are the normed ones, to a code's rounding
    keep = (ids >= 0)[:, None]
    s = torch.where(keep, before["table"].cpu().double()[ids.clamp(min=0)], 0.0) * st.scale
    s = s.to(t).double() + x_d.cpu().double()
    c = s - (s.mean(1, keepdim=True) if norm == "layer" else 0)
    rho = (c.square().mean(1, keepdim=True) + st.eps) ** -0.5
    y = c * rho * st.w.cpu().double()
    top_y = torch.cat([p.abs().amax(1, keepdim=True).expand_as(p) for p in y.split(128, 1)], 1)
    q, head8t = numbers(st.q, st._q)[:n], weights(st.head8t, st._head8t)
    size = s.abs().amax(1, keepdim=True) * rho * st.w.cpu().double().abs()
    bound = 1.02 * (UNIT[E4M3] * y.abs() + FLOOR[E4M3] * top_y / 448) + size * (UNIT[t] * 4 + (dim + 20) * U)
    assert bool(((q - y).abs() <= bound).all())
    # the head, and the logits
    h = before["head"].cpu().double()
    top_h = torch.cat([torch.cat([b.abs().max().expand_as(b) for b in a.split(128, 1)], 1)
                       for a in h.split(128, 0)], 0)
    assert bool(((head8t.t() - h).abs() <= 1.02 * (UNIT[E4M3] * h.abs() + FLOOR[E4M3] * top_h / 448)).all())
    assert torch.equal(weights(st.head8, st._head8), head8t.t())
    want, mag = q @ head8t.t(), q.abs() @ head8t.abs().t()
    coarse = 0 if t == F32 else 2.0 ** -10
    off = mag * (coarse + (dim + 4) * U) + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    assert bool(((z - want).abs() <= off).all())
    # a step, from the same logits
    loss = st.step(ids_d, n, top_ids.to(DEV), top.to(DEV), x_d).cpu().double()
    assert int(st.status) == 0
    zz, dz = z.requires_grad_(True), st.z[:n].cpu().double()
    lq = torch.log_softmax(zz / st.temperature, 1)
    hole = top_ids < 0
    lp = torch.log_softmax((top.double() / st.temperature).masked_fill(hole, -float("inf")), 1)
    p = lp.exp().masked_fill(hole, 0)
    ref = (p * (lp.masked_fill(hole, 0) - lq.gather(1, top_ids.clamp(min=0)))).sum(1)
    ref = ref * st.temperature ** 2 * torch.tensor(1.0 / n, dtype=F32).double()
    ref.sum().backward()
    ref = ref.detach()
    assert float((loss - ref).abs().max()) <= 100 * U * float(ref.abs().max())
    assert float((dz - zz.grad).abs().max()) <= (UNIT[t] + 200 * U) * float(zz.grad.abs().max()) + FLOOR[t]
    # the way back
    assert torch.equal(numbers(st.q, st._q)[:n], q)
    want, mag = dz.t() @ q, dz.abs().t() @ q.abs()
    assert bool(((st.dhead.cpu().double() - want).abs() <= (n + n / 256 + 5) * U * mag + FLOOR[F32]).all())
    dz8 = numbers(st.dz8, st._dz8)[:n]
    top_z = torch.cat([a.abs().amax(1, keepdim=True).expand_as(a) for a in dz.split(128, 1)], 1)
    assert bool(((dz8 - dz).abs() <= 1.02 * (UNIT[E4M3] * dz.abs() + FLOOR[E4M3] * top_z / 448) +
                 2.0 ** -136).all())
    dy, want, mag = st.dy[:n].cpu().double(), dz8 @ head8t, dz8.abs() @ head8t.abs()
    off = mag * (coarse + (classes + 4) * U) + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    assert bool(((dy - want).abs() <= off).all())
    kept = numbers(st.kept, st._kept)[:n]
    top_s = torch.cat([a.abs().amax(1, keepdim=True).expand_as(a) for a in s.split(128, 1)], 1)
    assert bool(((kept - s).abs() <= 1.02 * (UNIT[E4M3] * s.abs() + FLOOR[E4M3] * top_s / 448) +
                 2 * UNIT[t] * top_s).all())
    rho, mu = st.rstd[:n].cpu().double()[:, None], 0
    if norm == "layer":
        mu = st.mean[:n].cpu().double()[:, None]
    hh, g = (kept - mu) * rho, dy * before["w"].cpu().double()
    dx = rho * (g - hh * (g * hh).mean(1, keepdim=True) - (g.mean(1, keepdim=True) if norm == "layer" else 0))
    got = st.e[:n].cpu().double()
    rows = rho * (g.abs() + hh.abs() * (g * hh).abs().mean(1, keepdim=True) + g.abs().mean(1, keepdim=True) +
                  rho * (kept.abs() + abs(mu)) * g.abs().amax(1, keepdim=True) * (1 + hh.abs()))
    assert bool(((got - dx).abs() <= 1.01 * UNIT[t] * dx.abs() + (dim + 20) * U * rows + FLOOR[t]).all())
    dw = (dy * hh).sum(0)
    sizes = (dy.abs() * (hh.abs() + rho * (kept.abs() + abs(mu)))).sum(0)
    assert bool(((st.dw.cpu().double() - dw).abs() <= (n + 6) * U * sizes + FLOOR[F32]).all())
    for name, grad in (("w", st.dw), ("head", st.dhead.t())):
        want = before[name].cpu().double() - st.rate * grad.cpu().double()
        off = 2 * U * (before[name].cpu().double().abs() + st.rate * grad.cpu().double().abs())
        assert bool(((getattr(st, name).cpu().double() - want).abs() <= off).all())


@pytest.mark.parametrize("t", [F32, BF16])
def test_a_layer_in_a_replayed_graph(t):
    """A layer's forward and backward calls, captured once and replayed on new inputs,
    with other work and synchronisations between the replays; a second graph shares
    the workspace."""
    from paper_2606_02916_amd import gg
    n, d, m = 1500, 260, 400
    x, res, dz = (torch.empty(n, w, dtype=t, device=DEV) for w in (d, d, m))
    w, b, weights = (torch.empty(s, device=DEV) for s in (d, d, (m, d)))
    z, dy, dx, s = (torch.empty(n, c, dtype=t, device=DEV) for c in (m, d, d, d))
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dw, db, dweights = torch.empty(d, device=DEV), torch.empty(d, device=DEV), torch.empty(m, d, device=DEV)

    def rows8(c):
        return gg.make_rows(torch.empty(n, c, dtype=E4M3, device=DEV),
                            scales=torch.empty(n, -(-c // 128), device=DEV), group=128)

    q, kept, dz8 = rows8(d), rows8(d), rows8(m)
    w8, w8t = (gg.make_blocks(torch.empty(r, c, dtype=E4M3, device=DEV),
                              torch.empty(-(-r // 128), -(-c // 128), device=DEV)) for r, c in ((m, d), (d, m)))
    ws = torch.empty(max(gg.gg_ws_layernorm(n, d), gg.gg_ws_product(n, d, m)), dtype=torch.uint8, device=DEV)
    r = gg.make_rows

    def calls():
        gg.gg_layernorm_forward(r(x), r(res), n, d, w, b, 1e-5, r(s), None, q, kept, mean, rstd)
        gg.gg_quantise_blocks(r(weights), m, d, w8, w8t)
        gg.gg_product_forward(q, n, d, w8, m, r(z))
        gg.gg_product_backward(q, n, d, r(dz), m, r(dweights), gg.GG_PRODUCT_ADD, ws)
        gg.gg_quantise_rows(r(dz), n, m, dz8)
        gg.gg_product_forward(dz8, n, m, w8t, d, r(dy))
        gg.gg_layernorm_backward(r(dy), r(res), kept, mean, rstd, n, d, w, r(dx), dw, db, ws)

    def fill(seed):
        g = gen(seed)
        for v in (x, res, dz, w, b, weights, dweights):
            v.copy_(torch.randn(v.shape, generator=g, device=DEV))

    outs = (s, z, dweights, dy, dx, dw, db, q.keep[0], kept.keep[0], dz8.keep[0], w8.keep[0], w8t.keep[0])
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for graph in graphs:
        with torch.cuda.graph(graph):
            calls()
    for seed in range(1, 6):
        fill(seed)
        calls()
        want = [o.clone() for o in outs]
        fill(seed)
        for o in outs:
            if o is not dweights:
                o.view(torch.uint8).fill_(0x7F)
        torch.cuda.synchronize()
        graphs[seed % 2].replay()
        torch.cuda.synchronize()
        for i, (a, e) in enumerate(zip(outs, want)):
            assert torch.equal(a.view(torch.uint8), e.view(torch.uint8)), (seed, i)


def test_readme_example_of_a_product():
    """The README's lines on a layer's product, as they are written."""
    from paper_2606_02916_amd import gg
    text = open(os.path.join(helpers.ROOT, "README.md")).read()
    start = text.index("    a = gg.make_rows(codes, scales=scales, group=128)")
    code = textwrap.dedent(text[start:text.index("\n\n", start)])
    n, k, m, g = 200, 300, 140, torch.Generator().manual_seed(3)
    x, w, dout = (torch.randn(*s, generator=g).to(DEV) for s in ((n, k), (m, k), (n, m)))
    ns = {"gg": gg, "torch": torch, "n": n, "k": k, "m": m, "x": x, "w": w, "dout": dout,
          "codes": torch.empty(n, k, dtype=E4M3, device=DEV), "scales": torch.empty(n, 3, device=DEV),
          "w8": torch.empty(m, k, dtype=E4M3, device=DEV), "w_scales": torch.empty(2, 3, device=DEV),
          "w8t": torch.empty(k, m, dtype=E4M3, device=DEV), "wt_scales": torch.empty(3, 2, device=DEV),
          "out": torch.empty(n, m, device=DEV), "dw": torch.empty(m, k, device=DEV)}
    exec(code, ns)
    # a code is off by 2^-4 of its number at most, or by half the least code, 2^-10 of a scale
    # of at most max|x| / 448
    def off(v):
        return v.abs() / 16 + v.abs().max() / 448 / 1024
    x, w, dout = x.cpu().double(), w.cpu().double(), dout.cpu().double()
    bound = off(x) @ w.abs().t() + x.abs() @ off(w).t() + off(x) @ off(w).t()
    assert within(ns["out"], x @ w.t(), bound * 1.001) <= 0
    assert within(ns["dw"], dout.t() @ x, dout.abs().t() @ off(x) * 1.001) <= 0
