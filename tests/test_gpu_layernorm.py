"""Layer norm, its 8-bit rows and its gradient against their formulas in 64 bits."""
import zlib

import pytest
import torch

from tests.op_util import BF16, E4M3, F16, F32, FLOOR, U, UNIT, like, rows, untouched, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TINY = 2.0 ** -126
# one lane, odd pieces, whole waves, several pieces per lane, a block per row, blocks
# whose registers do not hold the weights
DIMS = [1, 3, 7, 8, 13, 100, 256, 511, 602, 1030, 2049, 4096, 8192, 8200, 16381]


def lib():
    from paper_2606_02916_amd import gg
    return gg


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def d64(x):
    return x.detach().cpu().double()


def forward(x, res, w, b, eps, tsum, ty, group=None, kept=None, lead=1, pad=1):
    """The call's outputs as 64-bit tensors on the CPU."""
    gg = lib()
    n, d = x.shape
    outs, made, sc = {}, {}, {}
    for name, t in (("sum", tsum), ("y", ty), ("q", E4M3 if group is not None else None),
                    ("kept", E4M3 if kept is not None else None)):
        if t is not None:
            made[name] = like(n, d, t, DEV, lead=lead, pad=pad)
    mean, rstd = (torch.full((n,), float("nan"), device=DEV) for _ in range(2))
    r = {}
    for name, m in made.items():
        more = {}
        if name in ("q", "kept"):
            gr = group if name == "q" else kept
            k = -(-d // gr) if gr else 1
            sc[name] = torch.full((n, k + 2), float("nan"), device=DEV)[:, 1:1 + k]
            more = dict(scales=sc[name], group=gr)
        r[name] = gg.make_rows(m[0], **more)
    gg.gg_layernorm_forward(gg.make_rows(x), None if res is None else gg.make_rows(res), n, d, w, b, eps,
                            r.get("sum"), r.get("y"), r.get("q"), r.get("kept"), mean, rstd)
    for name, (out, flat, own) in made.items():
        assert untouched(flat, own), name
        outs[name] = d64(out)
    for name, s in sc.items():
        outs[name + "_scales"] = d64(s)
    outs["mean"], outs["rstd"] = d64(mean), d64(rstd)
    return outs


def reference(x, res, w, b, eps):
    """s, mean, rstd and y, and how far fp32 may take them off.  A sum of d terms is
    off by d U of their magnitudes; s by U; c = s - mean by those and its own
    rounding; rstd by half of the variance's relative error and the 8 U of a sum,
    a root and a division; y by what h = c rstd and one fused operation add."""
    s = d64(x) if res is None else d64(x) + d64(res)
    d = s.shape[1]
    mean = s.mean(1, keepdim=True)
    c = s - mean
    es = U * s.abs() if res is not None else torch.zeros_like(s)
    em = (d + 2) * U * s.abs().mean(1, keepdim=True)
    ec = es + em + U * c.abs()
    var = c.square().mean(1, keepdim=True) + eps
    off = ((2 * c.abs() * ec + ec * ec).mean(1, keepdim=True) / var + (d + 4) * U)
    assert float(off.max()) < 0.1
    off = 0.6 * off + 8 * U
    rstd = var ** -0.5
    h = c * rstd
    eh = (ec + c.abs() * (off + 2 * U)) * rstd
    w = torch.ones(d).double() if w is None else d64(w)
    b = torch.zeros(d).double() if b is None else d64(b)
    y = h * w + b
    return s, es, mean, em, rstd, off, y, eh * w.abs() + U * y.abs()


def check_codes(codes, scales, y, ey, group):
    d = y.shape[1]
    g = group or d
    col = torch.arange(d) // g
    top = torch.stack([p.abs().amax(1) for p in y.split(g, 1)], 1)
    etop = torch.stack([p.amax(1) for p in ey.split(g, 1)], 1)
    scale = (top / 448).clamp(min=TINY)
    assert within(scales, scale, etop / 448 + scale * 2 * U) <= 0
    sc = scales[:, col]
    assert within(codes * sc, y, ey + y.abs() * (3 * U + 1.01 * UNIT[E4M3]) + FLOOR[E4M3] * sc * 1.01) <= 0


def check(outs, x, res, w, b, eps, tsum, ty, group, kept):
    s, es, mean, em, rstd, off, y, ey = reference(x, res, w, b, eps)
    assert within(outs["mean"], mean[:, 0], em[:, 0] + FLOOR[F32]) <= 0
    assert within(outs["rstd"], rstd[:, 0], (rstd * off)[:, 0]) <= 0
    if tsum is not None:
        assert within(outs["sum"], s, es + 1.01 * UNIT[tsum] * s.abs() + FLOOR[tsum]) <= 0
    if ty is not None:
        assert within(outs["y"], y, ey + 1.01 * UNIT[ty] * y.abs() + FLOOR[ty]) <= 0
    if group is not None:
        check_codes(outs["q"], outs["q_scales"], y, ey, group)
    if kept is not None:
        check_codes(outs["kept"], outs["kept_scales"], s, es, kept)


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("t,ts", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("res,q,kept", [(False, None, None), (True, 0, 32), (True, 128, 0)])
def test_norm(dim, t, ts, res, q, kept):
    g = gen(dim, str(t), str(ts), res)
    n = 7 if dim > 4000 else 67
    x = rows(torch.randn(n, dim, generator=g) * 3 + 1, t, DEV, lead=1, pad=2)
    r = rows(torch.randn(n, dim, generator=g), ts, DEV, lead=2, pad=1) if res else None
    tw = F32 if dim % 2 else t
    w = (1 + torch.randn(dim, generator=g) * 0.3).to(tw).to(DEV)
    b = None if dim == 256 else torch.randn(dim, generator=g).to(tw).to(DEV)
    outs = forward(x, r, w, b, 1e-5, ts if res else None, t, q, kept)
    check(outs, x, r, w, b, 1e-5, ts if res else None, t, q, kept)


@pytest.mark.parametrize("group,kept", [(16, 256), (64, 16), (256, 128)])
@pytest.mark.parametrize("dim", [16, 17, 130, 257, 602, 2050, 5000])
@pytest.mark.parametrize("t", [F32, BF16])
def test_scales_by_group(dim, group, kept, t):
    """Groups of very different size, a shorter last one, two groupings in one call."""
    g = gen(dim, group)
    x = torch.randn(5, dim, generator=g) * torch.exp2((torch.arange(dim) // group % 7 * 4).float())
    x = rows(x, t, DEV)
    outs = forward(x, None, None, None, 1e-6, None, None, group, kept)
    check(outs, x, None, None, None, 1e-6, None, None, group, kept)


@pytest.mark.parametrize("n", [0, 1, 2, 255, 256, 1000])
@pytest.mark.parametrize("dim", [33, 3000])
def test_numbers_of_rows(n, dim):
    x = rows(torch.randn(n, dim, generator=gen(n)), BF16, DEV)
    b = torch.rand(dim, generator=gen(dim)).to(BF16).to(DEV)
    outs = forward(x, None, None, b, 1e-5, None, BF16, 0, 64)
    if n:
        check(outs, x, None, None, b, 1e-5, None, BF16, 0, 64)


@pytest.mark.parametrize("dim", [9, 602, 4100, 16_000])
@pytest.mark.parametrize("t", [F32, BF16])
def test_outputs_may_lie_on_the_inputs(dim, t):
    gg, g = lib(), gen(dim)
    n = 33
    x, r = (torch.randn(n, dim, generator=g).to(t).to(DEV) for _ in range(2))
    want = forward(x, r, None, None, 1e-5, t, t)
    gg.gg_layernorm_forward(gg.make_rows(x), gg.make_rows(r), n, dim, None, None, 1e-5, gg.make_rows(r),
                            gg.make_rows(x), None, None, None, None)
    assert torch.equal(d64(r), want["sum"]) and torch.equal(d64(x), want["y"])


def test_rows_that_repeat_and_rows_of_equal_elements():
    """A residual of stride 0 (one row for all); equal elements leave the bias, or with eps
    0 NaNs, and nothing of a NaN or an infinity reaches another row."""
    gg, dim = lib(), 300
    x = torch.randn(9, dim, generator=gen(1)).to(DEV)
    r = torch.randn(1, dim, generator=gen(2)).to(DEV).expand(9, dim)
    outs = forward(x, r, None, None, 1e-5, F32, F32)
    check(outs, x, r, None, None, 1e-5, F32, F32, None, None)
    clean = d64(forward(x, None, None, None, 1e-5, None, F32)["y"])
    b = torch.randn(dim, generator=gen(3)).to(DEV)
    x[2] = 5.0
    x[4, 7] = float("nan")
    x[6, 9] = float("inf")
    y, q, k = (torch.empty(9, dim, device=DEV), *(torch.empty(9, dim, dtype=E4M3, device=DEV) for _ in "qk"))
    sq, sk = torch.empty(9, device=DEV), torch.empty(9, device=DEV)
    gg.gg_layernorm_forward(gg.make_rows(x), None, 9, dim, None, None, 1e-5, None, gg.make_rows(y),
                            gg.make_rows(q, scales=sq), gg.make_rows(k, scales=sk), None, None)
    y, good = y.cpu(), [0, 1, 3, 5, 7, 8]
    assert torch.equal(y[good].double(), clean[good])
    assert not y[2].any() and bool(torch.isnan(y[4]).all()) and bool(torch.isnan(y[6]).all())
    kf, sk = k.float().cpu(), sk.cpu()
    assert bool(torch.isnan(sk[4])) and float(sk[6]) == float("inf") and float(sq[2]) == TINY
    assert not kf[6, [j for j in range(dim) if j != 9]].any() and bool(torch.isnan(kf[6, 9]))
    gg.gg_layernorm_forward(gg.make_rows(x), None, 3, dim, None, b, 1e-5, None,
                            gg.make_rows(z := torch.empty(3, dim, device=DEV)), None, None, None, None)
    assert torch.equal(z[2], b)
    gg.gg_layernorm_forward(gg.make_rows(x), None, 3, dim, None, b, 0.0, None, gg.make_rows(z), None,
                            None, None, None)
    assert bool(torch.isnan(z[2]).all())


@pytest.mark.parametrize("n,dim,group", [(8192, 1030, 0), (8192, 1030, 64), (2048, 4100, 256)])
def test_codes_are_the_rounded_quotients(n, dim, group):
    """Scales and codes are functions of the fp32 y and s alone: equal to the last bit."""
    gg, g = lib(), torch.Generator(device=DEV).manual_seed(dim + group)
    x, r, b = (torch.randn(m, dim, generator=g, device=DEV) for m in (n, n, 1))
    x[6] *= 1e-20
    r[6] *= 1e-20
    k = -(-dim // group) if group else 1
    q, kept = (torch.empty(n, dim, dtype=E4M3, device=DEV) for _ in range(2))
    sq, sk = (torch.empty(n, k, device=DEV) for _ in range(2))
    s, y = torch.empty_like(x), torch.empty_like(x)
    gg.gg_layernorm_forward(gg.make_rows(x), gg.make_rows(r), n, dim, None, b[0], 1e-30, gg.make_rows(s),
                            gg.make_rows(y), gg.make_rows(q, scales=sq, group=group),
                            gg.make_rows(kept, scales=sk, group=group), None, None)
    for v, codes, sc in ((y, q, sq), (s, kept, sk)):
        v, sc = v.cpu(), sc.cpu()
        top = torch.stack([p.abs().amax(1) for p in v.split(group or dim, 1)], 1)
        assert torch.equal(sc, (top / 448).clamp(min=TINY))
        want = (v / sc[:, torch.arange(dim) // (group or dim)]).to(E4M3)
        assert torch.equal(codes.cpu().view(torch.uint8), want.view(torch.uint8))


# ---------------------------------------------------------------------------
# Backward.
# ---------------------------------------------------------------------------
def back_case(n, dim, t, ts, dsum, kept=None, layer=True, key=0):
    """Random inputs, the call's dx, dw and db, and those of the formula in 64 bits with their
    bounds.  kept: the group of 8-bit sums."""
    gg, g = lib(), gen(n, dim, str(t), str(ts), dsum, kept, key)
    x = torch.randn(n, dim, generator=g) * 2 + (0.5 if layer else 0)
    w = (1 + torch.randn(dim, generator=g) * 0.3).to(t).to(DEV)
    dy = rows(torch.randn(n, dim, generator=g), t, DEV, lead=1, pad=1)
    ds = rows(torch.randn(n, dim, generator=g), ts, DEV, lead=2, pad=2) if dsum else None
    mean = (x.mean(1) if layer else torch.zeros(n)).to(DEV)
    rstd = ((x - mean.cpu()[:, None]).square().mean(1) + 1e-5).rsqrt().to(DEV)
    if kept is None:
        s = rows(x, ts, DEV, lead=1, pad=3)
        s64, sr = d64(s), gg.make_rows(s)
    else:
        k = -(-dim // kept) if kept else 1
        col = torch.arange(dim) // (kept or dim)
        top = torch.stack([p.abs().amax(1) for p in x.split(kept or dim, 1)], 1) if n else torch.zeros(0, k)
        sc = (top / 448).clamp(min=TINY)
        s = rows((x / sc[:, col]).clamp(-448, 448), E4M3, DEV, lead=1, pad=3)
        scd = torch.full((n, k + 1), float("nan"), device=DEV)[:, 1:]
        scd.copy_(sc)
        s64, sr = d64(s.float()) * sc.double()[:, col], gg.make_rows(s, scales=scd, group=kept)
    dx, flat, own = like(n, dim, ts, DEV, lead=1, pad=1)
    dw, db = (torch.full((dim,), float("nan"), device=DEV) for _ in range(2))
    ws = torch.full((max(gg.gg_ws_layernorm(n, dim), 16),), 0xFF, dtype=torch.uint8, device=DEV)
    dsr = None if ds is None else gg.make_rows(ds)
    if layer:
        gg.gg_layernorm_backward(gg.make_rows(dy), dsr, sr, mean, rstd, n, dim, w, gg.make_rows(dx), dw,
                                 db, ws)
    else:
        gg.gg_rmsnorm_backward(gg.make_rows(dy), dsr, sr, rstd, n, dim, w, gg.make_rows(dx), dw, ws)
    assert untouched(flat, own)
    rho, mu = d64(rstd)[:, None], d64(mean)[:, None]
    dy, c = d64(dy), s64 - mu
    h, gw = c * rho, dy * d64(w)
    eh = rho * U * ((s64.abs() if kept is not None else 0) + 2 * c.abs() + c.abs())
    mg, mgh = gw.mean(1, keepdim=True) * layer, (gw * h).mean(1, keepdim=True)
    e_mg = (dim + 2) * U * gw.abs().mean(1, keepdim=True) * layer
    e_mgh = (dim + 4) * U * (gw * h).abs().mean(1, keepdim=True) + (gw.abs() * eh).mean(1, keepdim=True)
    want = rho * (gw - mg - h * mgh)
    bound = rho * (e_mg + h.abs() * e_mgh + eh * mgh.abs() +
                   4 * U * (gw.abs() + mg.abs() + (h * mgh).abs())) + U * want.abs()
    if ds is not None:
        want = want + d64(ds)
    bound = bound + want.abs() * (U + 1.01 * UNIT[ts]) + FLOOR[ts]
    results = [(dx, want, bound), (dw, (dy * h).sum(0), (n + 3) * U * (dy * h).abs().sum(0) +
                                   (dy.abs() * eh).sum(0) + FLOOR[F32])]
    if layer:
        results.append((db, dy.sum(0), (n + 1) * U * dy.abs().sum(0) + FLOOR[F32]))
    return results


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("t,ts", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("dsum", [False, True])
def test_gradient(dim, t, ts, dsum):
    for got, want, bound in back_case(9 if dim > 4000 else 131, dim, t, ts, dsum):
        assert within(got, want, bound) <= 0


@pytest.mark.parametrize("layer", [True, False])
@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("t,ts", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("group", [0, 16, 128])
def test_gradient_from_8_bit_sums(dim, t, ts, group, layer):
    for got, want, bound in back_case(9 if dim > 4000 else 131, dim, t, ts, dim % 2 == 0, group, layer):
        assert within(got, want, bound) <= 0


@pytest.mark.parametrize("n", [1, 2, 767, 3001])
@pytest.mark.parametrize("dim", [40, 2500])
@pytest.mark.parametrize("kept", [None, 32])
def test_gradient_of_rows(n, dim, kept):
    for got, want, bound in back_case(n, dim, BF16, BF16, True, kept):
        assert within(got, want, bound) <= 0


def test_gradient_of_no_rows_is_zero():
    gg = lib()
    r, none = gg.make_rows(torch.empty(0, 9, device=DEV)), torch.empty(0, device=DEV)
    dw, db = (torch.full((9,), float("nan"), device=DEV) for _ in range(2))
    ws = torch.empty(0, dtype=torch.uint8, device=DEV)
    gg.gg_layernorm_backward(r, None, r, none, none, 0, 9, None, r, dw, db, ws)
    assert not dw.cpu().any() and not db.cpu().any()


@pytest.mark.parametrize("which", ["dw", "db", "neither"])
def test_gradients_that_are_not_wanted(which):
    gg, n, dim = lib(), 50, 70
    dy, s = (torch.randn(n, dim, generator=gen(i)).to(DEV) for i in range(2))
    mean, rstd = s.mean(1), s.var(1).rsqrt()
    ws = torch.empty(gg.gg_ws_layernorm(n, dim), dtype=torch.uint8, device=DEV)
    got = []
    for a, b, w in ((True, True, ws), (which == "dw", which == "db", None if which == "neither" else ws)):
        dx, dw, db = torch.empty_like(s), torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
        gg.gg_layernorm_backward(gg.make_rows(dy), None, gg.make_rows(s), mean, rstd, n, dim, None,
                                 gg.make_rows(dx), dw if a else None, db if b else None, w)
        got.append((dx, dw, db))
    assert torch.equal(got[0][0], got[1][0])
    assert which != "dw" or torch.equal(got[0][1], got[1][1])
    assert which != "db" or torch.equal(got[0][2], got[1][2])


@pytest.mark.parametrize("dim", [100, 602, 5000, 16_000])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("on", ["dy", "dsum", "s"])
def test_dx_may_lie_on_an_input(dim, t, on):
    gg, n = lib(), 41
    dy, ds, s = (torch.randn(n, dim, generator=gen(i, dim)).to(t).to(DEV) for i in range(3))
    mean, rstd = s.float().mean(1), s.float().var(1).rsqrt()
    dx = torch.empty_like(s)
    m = gg.make_rows
    gg.gg_layernorm_backward(m(dy), m(ds), m(s), mean, rstd, n, dim, None, m(dx), None, None, None)
    to = {"dy": dy, "dsum": ds, "s": s}[on]
    gg.gg_layernorm_backward(m(dy), m(ds), m(s), mean, rstd, n, dim, None, m(to), None, None, None)
    assert torch.equal(to, dx)


def test_gradient_against_differences():
    """Along a direction, against central differences of the formula in 64
    bits.  Their own error is about h^2 of the third derivative and 2^-53 / h of
    the loss; the kernels' is a few roundings of fp32."""
    gg, g = lib(), gen(5)
    n, dim, eps, h = 20, 130, 1e-3, 1e-4
    x, r, way_x, c, cs = (torch.randn(n, dim, generator=g) for _ in range(5))
    w, way_w, b, way_b = (torch.rand(dim, generator=g) + 0.5 for _ in range(4))

    def loss(step):
        s = x.double() + r.double() + step * way_x.double()
        k = s - s.mean(1, keepdim=True)
        y = k * (k.square().mean(1, keepdim=True) + eps) ** -0.5 * (w.double() + step * way_w.double())
        y = y + b.double() + step * way_b.double()
        return float((c.double() * y).sum() + (cs.double() * s).sum())

    slope = (loss(h) - loss(-h)) / (2 * h)
    outs = {k: torch.empty(n, dim, device=DEV) for k in ("sum", "dx")}
    mean, rstd = torch.empty(n, device=DEV), torch.empty(n, device=DEV)
    dw, db = torch.empty(dim, device=DEV), torch.empty(dim, device=DEV)
    wd, m = w.to(DEV), gg.make_rows
    gg.gg_layernorm_forward(m(x.to(DEV)), m(r.to(DEV)), n, dim, wd, b.to(DEV), eps, m(outs["sum"]), None,
                            None, None, mean, rstd)
    ws = torch.empty(gg.gg_ws_layernorm(n, dim), dtype=torch.uint8, device=DEV)
    gg.gg_layernorm_backward(m(c.to(DEV)), m(cs.to(DEV)), m(outs["sum"]), mean, rstd, n, dim, wd,
                             m(outs["dx"]), dw, db, ws)
    parts = [d64(outs["dx"]) * way_x.double(), d64(dw) * way_w.double(), d64(db) * way_b.double()]
    got, size = sum(float(p.sum()) for p in parts), sum(float(p.abs().sum()) for p in parts)
    assert abs(got - slope) <= size * (dim + n + 16) * U + 1e-6 * size


@pytest.mark.parametrize("t,ts,n,dim,group", [(BF16, BF16, 9001, 1030, 64), (F32, F32, 1003, 8200, 0),
                                              (F16, F32, 120_001, 70, 32)])
def test_outputs_of_more_than_the_caches_take(t, ts, n, dim, group):
    """Of more than 32 MB together: the rows that calls of fewer give."""
    gg, g = lib(), torch.Generator(device=DEV).manual_seed(dim)
    x = torch.randn(n, dim, generator=g, device=DEV).to(t)
    res = torch.randn(n, dim, generator=g, device=DEV).to(ts)
    b = torch.rand(dim, generator=g, device=DEV)
    k = -(-dim // group) if group else 1

    def outputs():
        rows8 = [torch.full((n, dim), float("nan"), device=DEV).to(E4M3) for _ in range(2)]
        scales = [torch.full((n, k), float("nan"), device=DEV) for _ in range(2)]
        return (torch.full((n, dim), float("nan"), dtype=ts, device=DEV),
                torch.full((n, dim), float("nan"), dtype=t, device=DEV), *rows8, *scales,
                *(torch.full((n,), float("nan"), device=DEV) for _ in range(2)))

    def call(o, i, j):
        s, y, q, kept, sq, sk, mean, rstd = (p[i:j] for p in o)
        gg.gg_layernorm_forward(gg.make_rows(x[i:j]), gg.make_rows(res[i:j]), j - i, dim, None, b, 1e-6,
                                gg.make_rows(s), gg.make_rows(y),
                                gg.make_rows(q, scales=sq, group=group),
                                gg.make_rows(kept, scales=sk, group=group), mean, rstd)

    whole, parts = outputs(), outputs()
    call(whole, 0, n)
    step = (16 << 20) // (dim * 10)
    assert step >= 200          # (the waves of a wide row go by whether there are 256 rows)
    step = max(step, 256)
    cut = list(range(0, n, step))
    if n - cut[-1] < 256:
        cut.pop()
    for i, j in zip(cut, cut[1:] + [n]):
        call(parts, i, j)
    for p, q in zip(whole, parts):
        assert torch.equal(p.view(torch.uint8), q.view(torch.uint8))
