"""RMS norm, its 8-bit rows and its gradient against their formulas in 64 bits."""
import itertools
import zlib

import pytest
import torch

from tests.op_util import BF16, E4M3, F16, F32, FLOOR, U, UNIT, like, rows, untouched, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TINY = 2.0 ** -126
# one lane, odd pieces, whole waves, several pieces per lane, a block per row
DIMS = [1, 3, 7, 8, 13, 100, 256, 511, 602, 1030, 2049, 4096, 8192, 16381]


def lib():
    from paper_2606_02916_amd import gg
    return gg


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def forward(x, res, w, eps, tsum, ty, group=None, lead=1, pad=1):
    """The call's outputs as 64-bit tensors on the CPU."""
    gg = lib()
    n, d = x.shape
    outs, made = {}, {}
    for name, t in (("sum", tsum), ("y", ty), ("q", E4M3 if group is not None else None)):
        if t is not None:
            made[name] = like(n, d, t, DEV, lead=lead, pad=pad)
    rstd = torch.full((n,), float("nan"), device=DEV)
    k = -(-d // group) if group else 1
    scales = torch.full((n, k + 2), float("nan"), device=DEV)[:, 1:1 + k]
    r = {name: gg.make_rows(m[0], **(dict(scales=scales, group=group) if name == "q" else {}))
         for name, m in made.items()}
    gg.gg_rmsnorm_forward(gg.make_rows(x), None if res is None else gg.make_rows(res), n, d, w, eps,
                          r.get("sum"), r.get("y"), r.get("q"), rstd)
    for name, (out, flat, own) in made.items():
        assert untouched(flat, own), name
        outs[name] = out.cpu().double()
    outs["rstd"] = rstd.cpu().double()
    outs["scales"] = scales.cpu().double()
    return outs


def reference(x, res, w, eps):
    s = x.cpu().double()
    if res is not None:
        s = s + res.cpu().double()
    rstd = (s.square().mean(1, keepdim=True) + eps) ** -0.5
    y = s * rstd
    return s, rstd[:, 0], y if w is None else y * w.cpu().double()


def check(outs, x, res, w, eps, tsum, ty, group):
    d = x.shape[1]
    s, rstd, y = reference(x, res, w, eps)
    off = (d / 2 + 8) * U               # of rstd, and of y before it is rounded
    assert within(outs["rstd"], rstd, rstd * off) <= 0
    if tsum is not None:
        assert within(outs["sum"], s, s.abs() * (U + 1.01 * UNIT[tsum]) + FLOOR[tsum]) <= 0
    if ty is not None:
        assert within(outs["y"], y, y.abs() * (off + 1.01 * UNIT[ty]) + FLOOR[ty]) <= 0
    if group is not None:
        g = group or d
        col = torch.arange(d) // g
        top = torch.stack([p.abs().amax(1) for p in y.split(g, 1)], 1)
        scale = (top / 448).clamp(min=TINY)
        assert within(outs["scales"], scale, scale * (off + 2 * U)) <= 0
        sc = outs["scales"][:, col]
        bound = y.abs() * (off + 3 * U + 1.01 * UNIT[E4M3]) + FLOOR[E4M3] * sc * 1.01
        assert within(outs["q"] * sc, y, bound) <= 0
        most = torch.stack([p.abs().amax(1) for p in outs["q"].split(g, 1)], 1)
        assert torch.equal(most[top > 448 * TINY * 2],
                           torch.full_like(most, 448)[top > 448 * TINY * 2])


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("t,ts", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("res,q", [(False, None), (True, 0), (True, 32)])
def test_norm(dim, t, ts, res, q):
    g = gen(dim, str(t), str(ts), res)
    n = 7 if dim > 4000 else 67
    x = rows(torch.randn(n, dim, generator=g) * 3, t, DEV, lead=1, pad=2)
    r = rows(torch.randn(n, dim, generator=g), ts, DEV, lead=2, pad=1) if res else None
    w = (1 + torch.randn(dim, generator=g) * 0.3).to(F32 if dim % 2 else t).to(DEV)
    outs = forward(x, r, w, 1e-5, ts if res else None, t, q)
    check(outs, x, r, w, 1e-5, ts if res else None, t, q)


@pytest.mark.parametrize("group", [16, 64, 128, 256])
@pytest.mark.parametrize("dim", [16, 17, 130, 257, 602, 2050, 5000])
@pytest.mark.parametrize("t", [F32, BF16])
def test_scales_by_group(dim, group, t):
    """Groups of very different size, a shorter last one."""
    g = gen(dim, group)
    x = torch.randn(5, dim, generator=g) * torch.exp2((torch.arange(dim) // group % 7 * 4).float())
    x = rows(x, t, DEV)
    outs = forward(x, None, None, 1e-6, None, None, group)
    check(outs, x, None, None, 1e-6, None, None, group)


@pytest.mark.parametrize("n", [0, 1, 2, 255, 256, 1000])
@pytest.mark.parametrize("dim", [33, 3000])
def test_numbers_of_rows(n, dim):
    x = rows(torch.randn(n, dim, generator=gen(n)), BF16, DEV)
    w = torch.rand(dim, generator=gen(dim)).to(BF16).to(DEV)
    outs = forward(x, None, w, 1e-5, None, BF16, 0)
    if n:
        check(outs, x, None, w, 1e-5, None, BF16, 0)


@pytest.mark.parametrize("dim", [9, 602, 4100])
@pytest.mark.parametrize("t", [F32, BF16])
def test_outputs_may_lie_on_the_inputs(dim, t):
    gg, g = lib(), gen(dim)
    n = 33
    x = rows(torch.randn(n, dim, generator=g), t, DEV, pad=3)
    res = rows(torch.randn(n, dim, generator=g), t, DEV, lead=1)
    want = forward(x, res, None, 1e-5, t, t)
    rx, rr = gg.make_rows(x), gg.make_rows(res)
    gg.gg_rmsnorm_forward(rx, rr, n, dim, None, 1e-5, rr, rx, None, None)
    assert torch.equal(x.cpu().double(), want["y"]) and torch.equal(res.cpu().double(), want["sum"])
    dy, ds = (rows(torch.randn(n, dim, generator=g), t, DEV) for _ in range(2))
    rstd = want["rstd"].float().to(DEV)
    out, _, _ = like(n, dim, t, DEV)
    back = [gg.make_rows(dy), gg.make_rows(ds), rr, rstd, n, dim, None]
    gg.gg_rmsnorm_backward(*back, gg.make_rows(out), None, None)
    for i in (1, 0, 2):                # on dsum, then on dy and on s with the others as before
        old = (ds, dy, res)[(1, 0, 2).index(i)].clone()
        gg.gg_rmsnorm_backward(*back, back[i], None, None)
        got = (ds, dy, res)[(1, 0, 2).index(i)]
        assert torch.equal(got, out)
        got.copy_(old)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("dim", [40, 4100])
def test_zeros_infinities_and_nans(t, dim):
    x = torch.randn(6, dim, generator=gen(1))
    x[0] = 0                           # nothing: zeros, the smallest scale
    x[1, dim - 1] = float("inf")       # mean of squares infinite: zeros, NaN at the infinity
    x[2, 3] = float("nan")             # everything NaN
    x[3, :] = torch.finfo(t).tiny      # squares vanish beside eps
    x[4, 5] = -float("inf")
    gg = lib()
    xd = x.to(t).to(DEV)
    y = torch.empty(6, dim, dtype=t, device=DEV)
    q = torch.empty(6, dim, dtype=E4M3, device=DEV)
    sc, rstd = torch.empty(6, device=DEV), torch.empty(6, device=DEV)
    gg.gg_rmsnorm_forward(gg.make_rows(xd), None, 6, dim, None, 1e-6, None, gg.make_rows(y),
                          gg.make_rows(q, scales=sc), rstd)
    y, q, sc = y.cpu().float(), q.cpu().float(), sc.cpu()
    assert not y[0].any() and not q[0].any() and sc[0] == TINY
    for r, c in ((1, dim - 1), (4, 5)):
        other = torch.arange(dim) != c
        assert not y[r][other].any() and torch.isnan(y[r][c]) and rstd[r] == 0
        assert torch.isnan(sc[r]) and torch.isnan(q[r]).all()
    assert torch.isnan(y[2]).all() and torch.isnan(sc[2]) and torch.isnan(q[2]).all()
    assert torch.isfinite(y[3]).all() and torch.isfinite(y[5]).all() and torch.isfinite(sc[5])


def back_case(n, dim, t, ts, with_dsum, with_w, seed=0, scale=1.0):
    gg, g = lib(), gen(n, dim, str(t), str(ts), with_dsum, seed)
    dy = rows(torch.randn(n, dim, generator=g) * scale, t, DEV, lead=1, pad=1)
    s = rows(torch.randn(n, dim, generator=g) * 2 + 0.5, ts, DEV, lead=2, pad=1)
    dsum = rows(torch.randn(n, dim, generator=g), ts, DEV, pad=1) if with_dsum else None
    w = (1 + torch.randn(dim, generator=g) * 0.3).to(t).to(DEV) if with_w else None
    rstd = (s.cpu().double().square().mean(1) + 1e-5).rsqrt().float().to(DEV)
    dx, flat, own = like(n, dim, ts, DEV, lead=3, pad=2)
    dw = torch.full((dim,), float("nan"), device=DEV)
    ws = torch.full((gg.gg_ws_rmsnorm(n, dim),), 0xFF, dtype=torch.uint8, device=DEV)
    gg.gg_rmsnorm_backward(gg.make_rows(dy), None if dsum is None else gg.make_rows(dsum),
                           gg.make_rows(s), rstd, n, dim, w, gg.make_rows(dx), dw, ws)
    assert untouched(flat, own)
    return dy, dsum, s, rstd, w, dx, dw


@pytest.mark.parametrize("dim", DIMS)
@pytest.mark.parametrize("t,ts", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("n,with_dsum", [(1, True), (37, True), (301, False), (2600, True)])
def test_gradient(dim, t, ts, n, with_dsum):
    if n * dim > 3_000_000:
        n = 700
    with_w = dim != 100
    dy, dsum, s, rstd, w, dx, dw = back_case(n, dim, t, ts, with_dsum, with_w)
    d64 = lambda v: v.cpu().double()  # noqa: E731
    g = d64(dy) * (d64(w) if w is not None else 1.0)
    rho = d64(rstd)[:, None]
    h = d64(s) * rho
    mean, mags = (g * h).mean(1, keepdim=True), (g * h).abs().mean(1, keepdim=True)
    add = d64(dsum) if dsum is not None else torch.zeros_like(h)
    want = add + rho * (g - h * mean)
    bound = rho * (6 * U * (g.abs() + (h * mean).abs()) + (dim + 4) * U * h.abs() * mags) + \
        2 * U * add.abs() + 1.01 * UNIT[ts] * want.abs() + FLOOR[ts]
    assert within(dx, want, bound) <= 0
    want = (d64(dy) * h).sum(0)
    assert within(dw, want, (n + 3) * U * (d64(dy) * h).abs().sum(0) + FLOOR[F32]) <= 0


def test_gradient_of_no_rows_is_zero():
    gg = lib()
    e = torch.empty(0, 9, device=DEV)
    dw = torch.full((9,), float("nan"), device=DEV)
    ws = torch.empty(0, dtype=torch.uint8, device=DEV)
    r = gg.make_rows(e)
    gg.gg_rmsnorm_backward(r, None, r, torch.empty(0, device=DEV), 0, 9, None, r, dw, ws)
    assert not dw.cpu().any()


def test_gradient_against_differences():
    """Along a direction, against central differences of the formula in 64
    bits.  Their own error is about h^2 of the third derivative and 2^-53 / h of
    the loss; the kernels' is a few roundings of fp32."""
    gg, g = lib(), gen(5)
    n, dim, eps, h = 20, 130, 1e-3, 1e-4
    x, r, way_x, c = (torch.randn(n, dim, generator=g) for _ in range(4))
    w, way_w = torch.rand(dim, generator=g) + 0.5, torch.randn(dim, generator=g)
    cs = torch.randn(n, dim, generator=g)

    def loss(step):
        s = x.double() + r.double() + step * way_x.double()
        y = s * (s.square().mean(1, keepdim=True) + eps) ** -0.5 * (w.double() + step * way_w.double())
        return float((c.double() * y).sum() + (cs.double() * s).sum())

    slope = (loss(h) - loss(-h)) / (2 * h)
    outs = {k: torch.empty(n, dim, device=DEV) for k in ("sum", "dx")}
    rstd, dw = torch.empty(n, device=DEV), torch.empty(dim, device=DEV)
    wd, m = w.to(DEV), gg.make_rows
    gg.gg_rmsnorm_forward(m(x.to(DEV)), m(r.to(DEV)), n, dim, wd, eps, m(outs["sum"]), None, None, rstd)
    ws = torch.empty(gg.gg_ws_rmsnorm(n, dim), dtype=torch.uint8, device=DEV)
    gg.gg_rmsnorm_backward(m(c.to(DEV)), m(cs.to(DEV)), m(outs["sum"]), rstd, n, dim, wd,
                           m(outs["dx"]), dw, ws)
    dx, dw = outs["dx"].cpu().double(), dw.cpu().double()
    got = float((dx * way_x.double()).sum() + (dw * way_w.double()).sum())
    size = float((dx * way_x.double()).abs().sum() + (dw * way_w.double()).abs().sum())
    assert abs(got - slope) <= size * (dim + 16) * U + 1e-6 * size


def test_gradient_is_the_same_each_time_and_on_another_stream():
    side = torch.cuda.Stream()
    first = back_case(3000, 602, F32, F32, True, True)
    for _ in range(2):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = back_case(3000, 602, F32, F32, True, True)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(first[-1], again[-1]) and torch.equal(first[-2], again[-2])


def test_rows_of_8_bits_read_back():
    """The norm's 8-bit rows, codes and scales in one row, through the lookup:
    to within the code's rounding of the 32-bit norm."""
    gg, g = lib(), gen(9)
    n, dim, group = 50, 100, 32
    x = torch.randn(n, dim, generator=g).to(DEV)
    buf = torch.zeros(n, 100 + 16 + 4, dtype=torch.uint8, device=DEV)
    q = gg.make_rows(buf[:, :100].view(E4M3), scales=buf[:, 100:116].view(F32), group=group)
    y, out = torch.empty(n, dim, device=DEV), torch.empty(n, dim, device=DEV)
    gg.gg_rmsnorm_forward(gg.make_rows(x), None, n, dim, None, 1e-6, None, gg.make_rows(y), q, None)
    gg.gg_embed_forward(q, n, dim, None, n, 1.0, gg.make_rows(out),
                        torch.zeros(1, dtype=torch.int32, device=DEV))
    y = y.cpu().double()
    top = torch.cat([p.abs().amax(1, keepdim=True).expand(-1, p.shape[1]) for p in y.split(group, 1)], 1)
    assert within(out, y, y.abs() * UNIT[E4M3] * 1.01 + FLOOR[E4M3] * top / 448 * 1.01 + 4 * U * y.abs()) <= 0
    assert not buf[:, 116:].any()


@pytest.mark.parametrize("n,dim,group", [(8192, 1030, 0), (8192, 1030, 64), (2048, 4100, 0), (2048, 4100, 256)])
@pytest.mark.parametrize("with_w", [False, True])
def test_codes_are_the_rounded_quotients(n, dim, group, with_w):
    """Scales and codes are functions of the fp32 y alone, each by one division in
    fp32 and, for the codes, one rounding more: equal to the last bit."""
    gg, g = lib(), torch.Generator(device=DEV).manual_seed(dim + group)
    x = torch.randn(n, dim, generator=g, device=DEV)
    w = torch.rand(dim, generator=g, device=DEV) + 0.5 if with_w else None
    x[5] = 0
    x[6] *= 1e-20
    y, q = torch.empty_like(x), torch.empty(n, dim, dtype=E4M3, device=DEV)
    k = -(-dim // group) if group else 1
    sc = torch.empty(n, k, device=DEV)
    gg.gg_rmsnorm_forward(gg.make_rows(x), None, n, dim, w, 1e-30, None, gg.make_rows(y),
                          gg.make_rows(q, scales=sc, group=group), None)
    y, sc = y.cpu(), sc.cpu()
    top = torch.stack([p.abs().amax(1) for p in y.split(group or dim, 1)], 1)
    assert torch.equal(sc, (top / 448).clamp(min=TINY))
    want = (y / sc[:, torch.arange(dim) // (group or dim)]).to(E4M3)
    assert torch.equal(q.cpu().view(torch.uint8), want.view(torch.uint8))


def test_an_infinite_weight_leaves_zeros_beside_its_own_code():
    """The scale of a row with one infinity is infinite, the other codes are 0."""
    gg = lib()
    x = torch.randn(3, 70, generator=gen(2)).to(DEV)
    w = torch.ones(70, device=DEV)
    w[9] = float("inf")
    q, sc = torch.empty(3, 70, dtype=E4M3, device=DEV), torch.empty(3, device=DEV)
    gg.gg_rmsnorm_forward(gg.make_rows(x), None, 3, 70, w, 1e-6, None, None,
                          gg.make_rows(q, scales=sc), None)
    q, other = q.float().cpu(), torch.arange(70) != 9
    assert bool(torch.isinf(sc).all()) and not q[:, other].any() and bool(torch.isnan(q[:, 9]).all())


@pytest.mark.parametrize("t,ts,n,dim,group", [(BF16, BF16, 9001, 1030, 64), (F32, F32, 1003, 8200, 0),
                                              (F16, F32, 120_001, 70, 32)])
def test_outputs_of_more_than_the_caches_take(t, ts, n, dim, group):
    """Of more than 32 MB together: the rows that calls of fewer give."""
    gg, g = lib(), torch.Generator(device=DEV).manual_seed(dim)
    x = torch.randn(n, dim, generator=g, device=DEV).to(t)
    res = torch.randn(n, dim, generator=g, device=DEV).to(ts)
    w = torch.rand(dim, generator=g, device=DEV) + 0.5
    k = -(-dim // group) if group else 1

    def outputs():
        return (torch.full((n, dim), float("nan"), dtype=ts, device=DEV),
                torch.full((n, dim), float("nan"), dtype=t, device=DEV),
                torch.full((n, dim), float("nan"), device=DEV).to(E4M3),
                torch.full((n, k), float("nan"), device=DEV), torch.full((n,), float("nan"), device=DEV))

    def call(o, a, b):
        s, y, q, sc, r = (p[a:b] for p in o)
        gg.gg_rmsnorm_forward(gg.make_rows(x[a:b]), gg.make_rows(res[a:b]), b - a, dim, w, 1e-6,
                              gg.make_rows(s), gg.make_rows(y),
                              gg.make_rows(q, scales=sc, group=group), r)

    whole, parts = outputs(), outputs()
    assert sum(p[0].numel() * p.element_size() for p in whole[:3]) * n > 32 << 20
    call(whole, 0, n)
    step = (20 << 20) // (dim * 8)
    assert step >= 256          # (the waves of a wide row go by whether there are 256 rows)
    cut = list(range(0, n, step))
    if n - cut[-1] < 256:
        cut.pop()
    for a, b in zip(cut, cut[1:] + [n]):
        call(parts, a, b)
    for a, b in zip(whole, parts):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))
