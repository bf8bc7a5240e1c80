"""Rows and weights in 8 bits: the numbers are those of fp32's quotients, each one."""
import zlib

import pytest
import torch

from tests.op_util import BF16, E4M3, F16, F32, like, rows

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
TINY = 2.0 ** -126


def lib():
    from paper_2606_02916_amd import gg
    return gg


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def groups(d, g):
    return -(-d // g) if g else 1


def bits(t):
    return t.cpu().contiguous().view(torch.uint8)


def same(q, want):
    """Whether the codes stand for the same numbers (a zero of either sign is zero)."""
    return torch.equal(q.cpu().float(), want.float())


def quantise(x, group, lead=1, pad=3):
    """Codes and scales of x, with the bytes around both seen to be left alone."""
    gg = lib()
    n, d = x.shape
    q, flat, own = like(n, d, E4M3, DEV, lead=lead, pad=pad)
    k = groups(d, group)
    sc, sflat, sown = like(n, k, F32, DEV, lead=1, pad=2)
    gg.gg_quantise_rows(gg.make_rows(x), n, d, gg.make_rows(q, scales=sc, group=group))
    for f, o in ((flat, own), (sflat, sown)):
        assert bool(torch.isnan(f.cpu().float())[~o].all())
    return q.cpu(), sc.cpu()


def want_rows(x, group):
    x = x.cpu().float()
    d = x.shape[1]
    top = torch.stack([p.abs().amax(1) for p in x.split(group or d, 1)], 1)
    sc = (top / 448).clamp(min=TINY)
    return (x / sc[:, torch.arange(d) // (group or d)]).to(E4M3), sc


# widths of one lane, parts of a wave, whole waves, a block per row of every size, and
# rows of more than a block's registers
@pytest.mark.parametrize("dim", [1, 3, 7, 8, 16, 17, 31, 100, 255, 256, 602, 2049, 4100, 16_385, 40_003])
@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("group", [0, 16, 32, 128, 256])
def test_rows(dim, t, group):
    g = gen(dim, str(t), group)
    n = 3 if dim > 4000 else 37
    size = torch.exp2(torch.randint(-12, 6, (n, 1), generator=g).float())
    x = rows(torch.randn(n, dim, generator=g) * size, t, DEV, lead=1, pad=5)
    x[1] = 0
    q, sc = quantise(x, group)
    wq, wsc = want_rows(x, group)
    assert torch.equal(sc, wsc) and same(q, wq)


@pytest.mark.parametrize("n,dim", [(0, 40), (1, 16), (2000, 16), (5001, 40), (70_001, 24), (300, 8200)])
@pytest.mark.parametrize("group", [0, 32])
def test_numbers_of_rows(n, dim, group):
    x = torch.randn(n, dim, generator=gen(n, dim)).to(BF16).to(DEV)
    q, sc = quantise(x, group)
    if n:
        wq, wsc = want_rows(x, group)
        assert torch.equal(sc, wsc) and same(q, wq)


def test_outputs_of_more_than_the_caches_take():
    n, dim = 10_001, 4096
    x = torch.randn(n, dim, generator=torch.Generator(device=DEV).manual_seed(1), device=DEV).to(BF16)
    for group in (0, 128):
        q, sc = quantise(x, group)
        wq, wsc = want_rows(x, group)
        assert torch.equal(sc, wsc) and same(q, wq)


@pytest.mark.parametrize("group", [0, 16, 64])
@pytest.mark.parametrize("dim", [50, 700])
def test_numbers_at_the_ends(group, dim):
    """The largest and the smallest numbers of fp32, NaNs and infinities: the scale of
    a group with a NaN is NaN, with an infinity infinite, its other codes 0."""
    x = torch.randn(8, dim, generator=gen(dim)).to(DEV)
    x[0] *= 1e-38
    x[1] *= 2.0 ** -140
    x[2, 3] = 3.4e38
    x[3, 7] = float("nan")
    x[4, 9] = float("inf")
    x[5, 9] = -float("inf")
    x[6] = -0.0
    q, sc = quantise(x, group)
    wq, wsc = want_rows(x, group)
    assert torch.equal(bits(sc)[[0, 1, 2, 6, 7]], bits(wsc)[[0, 1, 2, 6, 7]])
    fq, fw, clean = q.float(), wq.float(), [0, 1, 2, 7]
    assert torch.equal(fq[clean], fw[clean]) and not fq[6].any()
    g = group or dim
    assert bool(torch.isnan(sc[3, 7 // g])) and bool(torch.isnan(fq[3, 7]))
    assert torch.equal(sc[3, 1:], wsc[3, 1:]) and torch.equal(fq[3, g:], fw[3, g:])
    for r in (4, 5):
        lo, hi = 9 // g * g, min(dim, 9 // g * g + g)
        assert float(sc[r, 9 // g]) == float("inf") and bool(torch.isnan(fq[r, 9]))
        assert not fq[r, [j for j in range(lo, hi) if j != 9]].any()
        assert torch.equal(fq[r, hi:], fw[r, hi:])


def test_rows_beyond_32_bits_of_bytes():
    """Rows whose places pass 2^32 bytes, in and out."""
    gg, n, dim, step = lib(), 4099, 200, 1 << 20
    x = torch.empty(n * step // 4 + 512, device=DEV).as_strided((n, dim), (step // 4, 1))
    x.copy_(torch.randn(n, dim, generator=gen(3)))
    q = torch.empty(n * step + 512, dtype=torch.uint8, device=DEV)
    qv, sc = q.as_strided((n, dim), (step, 1)).view(E4M3), torch.empty(n, 2, device=DEV)
    gg.gg_quantise_rows(gg.make_rows(x), n, dim, gg.make_rows(qv, scales=sc, group=128))
    wq, wsc = want_rows(x, 128)
    assert torch.equal(sc.cpu(), wsc) and same(qv, wq)


# ---------------------------------------------------------------------------
# Weights.
# ---------------------------------------------------------------------------
def want_blocks(w):
    w = w.cpu().float()
    r, c = w.shape
    sc = torch.stack([torch.stack([p.abs().max() for p in band.split(128, 1)]) for band in w.split(128, 0)])
    sc = (sc / 448).clamp(min=TINY)
    return (w / sc[torch.arange(r) // 128][:, torch.arange(c) // 128]).to(E4M3), sc


@pytest.mark.parametrize("r,c", [(1, 1), (1, 300), (300, 1), (47, 100), (100, 47), (127, 129), (128, 128),
                                 (256, 384), (130, 602), (602, 130), (1000, 515)])
@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("which", ["q", "qt", "both"])
def test_blocks(r, c, t, which):
    gg, g = lib(), gen(r, c)
    size = torch.exp2((torch.arange(r)[:, None] // 128 + torch.arange(c) // 128) % 9 - 4).float()
    w = rows(torch.randn(r, c, generator=g) * size, t, DEV, lead=1, pad=3)
    wq, wsc = want_blocks(w)
    made = {}
    for name, (a, b) in (("q", (r, c)), ("qt", (c, r))):
        if which in (name, "both"):
            made[name] = (like(a, b, E4M3, DEV, lead=3, pad=5),
                          like(groups(a, 128), groups(b, 128), F32, DEV, lead=1, pad=1))
    m = {k: gg.make_blocks(v[0][0], v[1][0]) for k, v in made.items()}
    gg.gg_quantise_blocks(gg.make_rows(w), r, c, m.get("q"), m.get("qt"))
    for name, parts in made.items():
        for _, flat, own in parts:
            assert bool(torch.isnan(flat.cpu().float())[~own].all())
        q, sc = parts[0][0].cpu(), parts[1][0].cpu()
        if name == "qt":
            q, sc = q.view(torch.uint8).t().contiguous().view(E4M3), sc.t()
        assert torch.equal(sc, wsc) and same(q, wq)


def test_blocks_with_nan_and_infinity_keep_to_their_block():
    gg, r, c = lib(), 300, 260
    w = torch.randn(r, c, generator=gen(9)).to(DEV)
    w[5, 200] = float("nan")
    w[290, 3] = float("inf")
    wq, wsc = want_blocks(w)
    q, sc = torch.empty(r, c, dtype=E4M3, device=DEV), torch.empty(3, 3, device=DEV)
    gg.gg_quantise_blocks(gg.make_rows(w), r, c, gg.make_blocks(q, sc), None)
    q, sc = q.cpu().float(), sc.cpu()
    assert bool(torch.isnan(sc[0, 1])) and float(sc[2, 0]) == float("inf")
    bad = torch.zeros(r, c, dtype=torch.bool)
    bad[:128, 128:256] = bad[256:, :128] = True
    assert torch.equal(q[~bad], wq.float()[~bad])
    assert bool(torch.isnan(q[5, 200])) and bool(torch.isnan(q[290, 3]))
    q[290, 3] = 0
    assert not q[256:, :128].any()


def test_more_rows_than_one_dimension_of_a_grid():
    """One scale to a wide row, a block each: 2^21 + 3 of them, and what lies behind left alone."""
    gg, n, dim, over = lib(), (1 << 21) + 3, 260, 4096
    x = torch.empty(n, dim, device=DEV)
    x.normal_(generator=torch.Generator(device=DEV).manual_seed(2))
    q = torch.full((n + over, dim), 0x7F, dtype=torch.uint8, device=DEV)
    sc = torch.full((n + over,), float("nan"), device=DEV)
    gg.gg_quantise_rows(gg.make_rows(x), n, dim, gg.make_rows(q[:n].view(E4M3), scales=sc[:n]))
    assert bool((q[n:] == 0x7F).all()) and bool(torch.isnan(sc[n:]).all())
    assert not bool(torch.isnan(sc[:n]).any())
    for at in (0, 1 << 20, (1 << 21) - 40, n - 40):
        wq, wsc = want_rows(x[at:at + 40], 0)
        assert torch.equal(sc[at:at + 40].cpu()[:, None], wsc) and same(q[at:at + 40].view(E4M3), wq)


def test_more_blocks_of_weights_than_one_dimension_of_a_grid():
    """2^24 rows (one, at a stride of 0) of 17 blocks: 2^21 + 131,072 blocks, and what lies behind
    codes and scales left alone."""
    gg, r, c, over = lib(), 1 << 24, 16 * 128 + 3, 4096
    one = torch.randn(1, c, generator=gen(c)).to(BF16)
    q = torch.full((r + over, c), 0x7F, dtype=torch.uint8, device=DEV)
    sc = torch.full((r // 128 + over, 17), float("nan"), device=DEV)
    gg.gg_quantise_blocks(gg.make_rows(one.to(DEV).expand(r, c)), r, c,
                          gg.make_blocks(q[:r].view(E4M3), sc[:r // 128]), None)
    wq, wsc = want_blocks(one)
    assert bool((q[r:] == 0x7F).all()) and bool(torch.isnan(sc[r // 128:]).all())
    assert bool((sc[:r // 128] == wsc.to(DEV)).all())
    for at in (0, 1 << 23, (1 << 21) // 17 * 128 - 64, r - 128):
        assert same(q[at:at + 128].view(E4M3), wq.expand(128, c))
    del q
    torch.cuda.empty_cache()
