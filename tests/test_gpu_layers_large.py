"""The calls for layers in 8 bits over as many rows as the default graph has nodes, and more."""
import pytest
import torch

from tests.op_util import BF16, E4M3, F16, F32, FLOOR, U, UNIT

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
N = 2_450_003


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def rows8(n, d, group, seed):
    """Rows in 8 bits, their description, and what they stand for, in 64 bits by pieces."""
    from paper_2606_02916_amd import gg
    x = torch.empty(n, d, device=DEV).normal_(generator=gen(seed))
    q, sc = torch.empty(n, d, dtype=E4M3, device=DEV), torch.empty(n, -(-d // group) if group else 1, device=DEV)
    r = gg.make_rows(q, scales=sc, group=group)
    gg.gg_quantise_rows(gg.make_rows(x), n, d, r)
    col = torch.arange(d, device=DEV) // (group or d)
    return r, lambda at: q[at].float().double() * sc[at].double()[:, col]


def close(got, want, bound):
    return bool(((got.double() - want).abs() <= bound).all())


PLACES = [slice(0, 300), slice(1_048_500, 1_048_700), slice(2_097_000, 2_097_400), slice(N - 300, N)]


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("group", [0, 128])
def test_product(t, group):
    from paper_2606_02916_amd import gg
    k, m = 200, 47
    a, num = rows8(N, k, group, 1)
    w = torch.empty(m, k, device=DEV).normal_(generator=gen(2))
    w8, ws = torch.empty(m, k, dtype=E4M3, device=DEV), torch.empty(1, 2, device=DEV)
    b = gg.make_blocks(w8, ws)
    gg.gg_quantise_blocks(gg.make_rows(w), m, k, b, None)
    wn = w8.float().double() * ws.double()[:, torch.arange(k, device=DEV) // 128]
    out = torch.full((N + 3, m), float("nan"), device=DEV).to(t)
    gg.gg_product_forward(a, N, k, b, m, gg.make_rows(out[:N]))
    assert bool(torch.isnan(out[N:]).all()) and bool(torch.isfinite(out[:N]).all())
    for at in PLACES:
        x = num(at)
        want, size = x @ wn.t(), x.abs() @ wn.abs().t()
        # (sums of eight in the 8-bit instructions are cut below 2^-13 of the largest of them)
        cut = 0 if t == F32 else 7 * 2.0 ** -13 * size
        assert close(out[at], want, (k + 4) * U * size + 1.01 * UNIT[t] * want.abs() + FLOOR[t] + cut)


@pytest.mark.parametrize("tz,t", [(F32, F32), (BF16, BF16), (F16, F32)])
@pytest.mark.parametrize("k,m", [(100, 47), (128, 136)])
def test_weight_gradient(k, m, tz, t):
    from paper_2606_02916_amd import gg
    a, num = rows8(N, k, 128, 3)
    dz = (torch.empty(N, m, device=DEV).normal_(generator=gen(4)) * 0.01).to(tz)
    dw = torch.empty(m, k, dtype=t, device=DEV)
    ws = torch.full((max(gg.gg_ws_product(N, k, m), 16),), 0xFF, dtype=torch.uint8, device=DEV)
    gg.gg_product_backward(a, N, k, gg.make_rows(dz), m, gg.make_rows(dw), 0, ws)
    want, size = torch.zeros(2, m, k, dtype=torch.float64, device=DEV)
    for i in range(0, N, 500_000):
        at = slice(i, min(N, i + 500_000))
        x, z = num(at), dz[at].double().t().contiguous()
        want += z @ x
        size += z.abs() @ x.abs()
    left = {F32: 0.0, BF16: 2.0 ** -8}[t]
    # (a lane adds a split's rows by 32, and the splits are joined: N / 32 + 1,000 roundings at most)
    bound = (N / 32 + 1000) * U * size + 1.01 * left * size + 1.01 * UNIT[t] * want.abs()
    assert close(dw, want, bound)


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("d", [33, 602])
def test_layer_norm_and_its_gradient(d, t):
    from paper_2606_02916_amd import gg
    x = torch.empty(N, d, device=DEV).normal_(generator=gen(5)).add_(0.5).to(t)
    dy = (torch.empty(N, d, device=DEV).normal_(generator=gen(6))).to(t)
    w, b = (torch.empty(d, device=DEV).normal_(generator=gen(s)) for s in (7, 8))
    y, mean, rstd = torch.empty_like(x), torch.empty(N, device=DEV), torch.empty(N, device=DEV)
    kept = gg.make_rows(torch.empty(N, d, dtype=E4M3, device=DEV),
                        scales=torch.empty(N, -(-d // 128), device=DEV), group=128)
    gg.gg_layernorm_forward(gg.make_rows(x), None, N, d, w, b, 1e-5, None, gg.make_rows(y), None, kept, mean, rstd)
    dx, dw, db = torch.empty_like(x), torch.empty(d, device=DEV), torch.empty(d, device=DEV)
    ws = torch.full((gg.gg_ws_layernorm(N, d),), 0xFF, dtype=torch.uint8, device=DEV)
    gg.gg_layernorm_backward(gg.make_rows(dy), None, gg.make_rows(x), mean, rstd, N, d, w, gg.make_rows(dx), dw, db, ws)
    sums, sizes = torch.zeros(2, 2, d, dtype=torch.float64, device=DEV)
    for i in range(0, N, 250_000):
        at = slice(i, min(N, i + 250_000))
        s, g = x[at].double(), dy[at].double()
        mu = s.mean(1, keepdim=True)
        rho = ((s - mu).square().mean(1, keepdim=True) + 1e-5) ** -0.5
        h = (s - mu) * rho
        sums += torch.stack([(g * h).sum(0), g.sum(0)])
        sizes += torch.stack([(g.abs() * (h.abs() + rho * (s.abs() + mu.abs()))).sum(0), g.abs().sum(0)])
        want = h * w.double() + b.double()
        # (mean and variance are sums of d, off by d U of their terms' size)
        size = (h.abs() + rho * (s.abs() + mu.abs())) * w.double().abs() + b.double().abs()
        assert close(y[at], want, (d + 10) * U * size * (1 + h.abs().amax(1, keepdim=True)) + 1.01 * UNIT[t] * want.abs())
        gw = g * w.double()
        want = rho * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
        size = rho * (gw.abs() + gw.abs().mean(1, keepdim=True) + h.abs() * (gw * h).abs().mean(1, keepdim=True))
        grow = 1 + rho * (s.abs() + mu.abs()).amax(1, keepdim=True)
        assert close(dx[at], want, (2 * d + 20) * U * size * grow + 1.01 * UNIT[t] * want.abs())
    # (a lane's share is of N / 768 rows at most, 1,024 shares at most are added)
    for got, want, size in ((dw, sums[0], sizes[0]), (db, sums[1], sizes[1])):
        assert close(got, want, (N / 768 + 1024 + d + 20) * U * size)
    assert bool(torch.isfinite(kept.keep[1]).all())
