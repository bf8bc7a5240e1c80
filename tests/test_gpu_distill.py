"""The distillation loss and its gradient against their formulas in 64 bits.

Bounds.  A term exp((z - m) / T) takes three roundings in its exponent x (a
relative error of 3 |x| U in the term) and the exponential's own two units; a
sum of such terms adds one rounding per addition along its longest chain,
which is a lane's elements and the tree after it.  Logarithms of p and of the
sum are off by a few U of their size."""
import math
import zlib

import pytest
import torch

from tests.op_util import BF16, F16, F32, FLOOR, U, UNIT, like, rows, untouched, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
INF = float("inf")


def lib():
    from paper_2606_02916_amd import gg
    return gg


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def make(n, v, k, t, seed=0, idt=torch.int32, spread=3.0, tt=None, pad=1):
    g = gen(n, v, k, str(t), seed)
    z = torch.randn(n, v, generator=g) * spread
    ids = torch.randint(0, v, (n, k), generator=g)
    top = torch.randn(n, k, generator=g) * 2 + 5
    ids[torch.rand(n, k, generator=g) < 0.1] = -1
    w = torch.rand(n, generator=g) + 0.5
    return (rows(z, t, DEV, lead=1, pad=pad), ids.to(idt).to(DEV), rows(top, tt or t, DEV, pad=pad),
            w.to(DEV))


def reference(z, ids, top, w, T, weight):
    """loss, lse, dz and the bounds of each, in 64 bits on the CPU (before dz
    is rounded to its type)."""
    z, ids, top, w = z.cpu().double(), ids.cpu().long(), top.cpu().double(), w.cpu().double()
    n, v = z.shape
    a = w * torch.tensor(weight, dtype=F32).double()
    T = torch.tensor(T, dtype=F32).double()
    x = z / T
    lse = torch.logsumexp(x, 1)
    q = torch.exp(x - lse[:, None])
    hole = ids < 0
    t = (top / T).masked_fill(hole, -INF)
    has = (t.amax(1) > -INF) & (a != 0) & (x.amax(1) > -INF)
    lp = torch.log_softmax(t, 1).masked_fill(t == -INF, 0.0)
    p = torch.exp(lp) * (t > -INF)
    at = ids.clamp(min=0)
    zx = x.gather(1, at)
    gap = lp - zx + lse[:, None]
    gap = torch.where(p > 0, gap, 0.0)
    loss = torch.where(has, a * T * T * (p * gap).sum(1), 0.0)
    dz = torch.where(has[:, None], q.scatter_add(1, at, -p) * (a * T)[:, None], 0.0)
    # bounds
    far = (x.amax(1, keepdim=True) - x)
    far = torch.where(q > 0, far, 0.0)
    chain = 200 + v / 256
    es = ((3 * far + 4) * q).sum(1) * U + chain * U          # of the sum, relative
    big = x.abs().masked_fill(x == -INF, 0).amax(1)
    el = es + 4 * U * (big + lse.abs()) + 4 * U * (lse - x.amax(1)).abs()
    ep = (6 * lp.abs() + 4 * (t.amax(1, keepdim=True) - t).masked_fill(t == -INF, 0) + ids.shape[1] +
          20) * U
    finite = torch.where(torch.isfinite(gap), gap, 0.0)
    eloss = (a * T * T).abs() * ((p * (ep * (1 + finite.abs()) + el[:, None] + 4 * U * zx.abs().masked_fill(
        zx == -INF, 0) + (ids.shape[1] + 6) * U * finite.abs())).sum(1))
    eq = q * ((3 * far + 12) * U + es[:, None] + el[:, None])
    edz = (a * T).abs()[:, None] * (eq + torch.zeros_like(q).scatter_add(1, at, p * (ep + 4 * U)))
    edz = edz + 4 * U * dz.abs()
    return (loss, lse, dz), (eloss, el, edz), has


def run(z, ids, top, w, T, weight, fused, dz=None):
    gg = lib()
    n, v = z.shape
    k = ids.shape[1]
    loss, lse = (torch.full((n,), float("nan"), device=DEV) for _ in range(2))
    out, flat, own = dz if dz is not None else like(n, v, z.dtype, DEV, lead=3, pad=2)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.full((gg.gg_ws_distill(n, v),), 0xFF, dtype=torch.uint8, device=DEV)
    rz, rt, rd = gg.make_rows(z), gg.make_rows(top), gg.make_rows(out)
    a = (rz, n, v, ids, rt, k, T, weight, w)
    gg.gg_distill_forward(*a, loss, lse, rd if fused else None, st, ws)
    if not fused:
        gg.gg_distill_backward(*a, lse, rd, st)
    if flat is not None:
        assert untouched(flat, own)
    return loss, lse, out, int(st)


def check(z, ids, top, w, T=2.0, weight=0.7, fused=True):
    print(f"distillation of {tuple(z.shape)} {z.dtype}, {ids.shape[1]} entries, fused {fused}",
          flush=True)
    loss, lse, dz, st = run(z, ids, top, w, T, weight, fused)
    (rl, rs, rd), (bl, bs, bd), has = reference(z, ids, top, w, T, weight)
    assert within(loss, rl, bl + FLOOR[F32]) <= 0
    assert within(lse, rs, bs) <= 0
    extra = 1.0 if fused else 2.0       # the backward call starts from the rounded lse
    assert within(dz, rd, extra * bd + 1.01 * UNIT[z.dtype] * rd.abs() + FLOOR[z.dtype]) <= 0
    assert not dz.cpu()[~has].any() and st == 0
    return loss, lse, dz


# part of a wave, a wave with 1, 2 and 4 pieces a lane, blocks of 256 to 1,024 lanes and 2 to
# 16 pieces, rows that no block holds; whole and odd vocabularies
@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("n,v,k", [(1, 1, 1), (5, 3, 2), (2, 7, 9), (9, 41, 8), (260, 47, 8),
                                   (33, 64, 1), (70, 255, 5), (31, 513, 16), (17, 1030, 64),
                                   (6, 2049, 20), (300, 2100, 20), (3, 5000, 256), (4, 16_385, 33),
                                   (260, 16_400, 10), (257, 33_003, 12), (258, 66_001, 5),
                                   (3, 131_072, 50), (2, 200_003, 32), (1, 300_000, 8)])
def test_loss_and_gradient(n, v, k, t, fused):
    check(*make(n, v, k, t, idt=torch.int64 if v % 2 else torch.int32), fused=fused)


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("n,v", [(259, 131_072), (260, 131_080)])
def test_many_rows_at_the_largest_that_a_block_holds(n, v, fused):
    check(*make(n, v, 20, BF16), fused=fused)


# Rows dealt to 4, 8, 16 and more lanes, of a few pieces each; rows of less than a
# piece; the longest rows that one wave has, and the next ones.
@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,v,k", [(66_001, 3, 3), (66_001, 7, 16), (70_003, 17, 5), (66_000, 47, 16),
                                   (33_001, 100, 17), (20_003, 172, 64), (9001, 601, 30),
                                   (4100, 1025, 3), (300, 2047, 64), (300, 2052, 64),
                                   (300, 4095, 9), (300, 4104, 256)])
def test_rows_of_a_part_of_a_wave(n, v, k, t, fused):
    check(*make(n, v, k, t, idt=torch.int32 if v % 2 else torch.int64, tt=BF16 if k % 2 else F32),
          fused=fused)


@pytest.mark.parametrize("tt", [F32, F16, BF16])
def test_the_teachers_logits_have_a_type_of_their_own(tt):
    check(*make(20, 300, 12, BF16, tt=tt))


@pytest.mark.parametrize("T", [0.25, 1.0, 3.7, 100.0])
@pytest.mark.parametrize("n,v", [(40, 47), (2, 70_000)])
def test_temperatures(T, n, v):
    for fused in (True, False):
        check(*make(n, v, 8, F32, seed=1), T=T, fused=fused)


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("n,v", [(64, 60), (40, 3000), (3, 40_000)])
def test_entries_that_recur_or_lack(n, v, fused):
    """All of a row's entries on one id, lists of one entry, empty lists, rows
    without a weight."""
    z, ids, top, w = make(n, v, 24, F32, seed=2)
    ids[0] = v - 1
    ids[1, 1:] = -1
    ids[1, 0] = 0
    ids[2] = -1
    ids[min(3, n - 1), 12:] = ids[min(3, n - 1), :12]
    if n > 8:
        w[5] = 0
        top[6] = -INF
        top[7, ::2] = -INF
    check(z, ids, top, w, fused=fused)


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("v", [50, 5000, 30_000])
def test_masked_logits(v, t, fused):
    """-infinity and the type's lowest value: in places, in long runs, and in
    all of a row."""
    n, k = 6, 10
    z, ids, top, w = make(n, v, k, t, seed=3)
    low = torch.finfo(t).min
    ids[:] = torch.randint(0, v // 2, (n, k), generator=gen(v)).to(DEV)
    z[0, v // 2:] = -INF
    z[1, v // 2:] = low
    z[2] = -INF                        # nothing to choose from: zeros
    z[3, v // 2 + 1:] = -INF
    z[3, 1:v // 2 - 1:2] = low
    top[3] = 1.0
    ids[3] = 0
    z[4, 1:] = -INF                    # one choice, and the teacher's
    ids[4] = 0
    loss, lse, dz, st = run(z, ids, top, w, 1.0, 1.0, fused)
    (rl, rs, rd), (bl, bs, bd), has = reference(z, ids, top, w, 1.0, 1.0)
    keep = torch.tensor([0, 1, 3, 4, 5])
    assert within(loss[keep], rl[keep], bl[keep] + FLOOR[F32]) <= 0
    assert within(lse[keep], rs[keep], bs[keep]) <= 0
    extra = 1.0 if fused else 2.0
    assert within(dz[keep], rd[keep],
                  (extra * bd + 1.01 * UNIT[t] * rd.abs())[keep] + FLOOR[t]) <= 0
    assert loss[2] == 0 and lse[2] == -INF and not dz[2].any() and not has[2]


@pytest.mark.parametrize("v", [50, 5000, 30_000])
def test_a_row_of_the_types_lowest_value_is_uniform(v):
    z, ids, top, w = make(3, v, 4, F32, seed=4)
    z[:] = torch.finfo(F32).min
    ids[:] = torch.arange(4)
    loss, lse, dz, st = run(z, ids, top, w, 1.0, 1.0, True)
    want = torch.full((3, v), 1.0 / v, dtype=torch.float64)
    p = torch.softmax(top.cpu().double(), 1)
    want[:, :4] -= p
    want = want * w.cpu().double()[:, None]
    assert within(dz, want, (want.abs() + w.cpu().double()[:, None]) * 40 * U) <= 0


def test_infinite_losses_and_nans_stay_in_their_rows():
    z, ids, top, w = make(6, 70, 5, F32, seed=5)
    ids[:] = torch.arange(5)
    z[0, 2] = -INF                     # the teacher's choice is masked
    z[1, 60] = float("nan")
    z[2, 60] = INF
    top[3, 1] = float("nan")
    for fused in (True, False):
        loss, lse, dz, st = run(z, ids, top, w, 1.0, 1.0, fused)
        loss, dz = loss.cpu(), dz.cpu()
        assert loss[0] == INF and torch.isfinite(dz[0]).all()
        assert torch.isnan(loss[1:4]).all() and torch.isnan(dz[1:3]).all()
        assert torch.isnan(dz[3, :5]).all() and torch.isfinite(dz[3, 5:]).all()
        assert torch.isfinite(loss[4:]).all() and torch.isfinite(dz[4:]).all()


@pytest.mark.parametrize("idt", [torch.int32, torch.int64])
@pytest.mark.parametrize("v", [50, 5000, 40_000])
def test_ids_out_of_range_are_no_entries_and_are_reported(v, idt):
    gg = lib()
    z, ids, top, w = make(4, v, 6, F32, idt=idt)
    ids[:, 2], ids[:, 4] = v, -2
    if idt == torch.int64:
        ids[:, 2] = 2 ** 33 + 1
    clean = ids.clone()
    clean[:, 2] = clean[:, 4] = -1
    for fused in (True, False):
        got, want = run(z, ids, top, w, 2.0, 1.0, fused), run(z, clean, top, w, 2.0, 1.0, fused)
        assert all(torch.equal(a, b) for a, b in zip(got[:3], want[:3]))
        assert got[3] == gg.DEV_BAD_ID and want[3] == 0


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,v", [(20, 47), (300, 3001), (3, 50_001), (260, 140_001)])
def test_the_gradient_may_take_the_logits_place(n, v, t):
    for fused in (True, False):
        z, ids, top, w = make(n, v, 9, t, seed=6)
        want = run(z, ids, top, w, 2.0, 1.0, fused)
        got = run(z, ids, top, w, 2.0, 1.0, fused, dz=(z, None, None))
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
        assert torch.equal(got[2], want[2])


def test_loss_alone_and_no_rows():
    gg = lib()
    z, ids, top, w = make(30, 100, 4, F32)
    whole = run(z, ids, top, w, 2.0, 1.0, True)
    loss = torch.full((30,), float("nan"), device=DEV)
    ws = torch.empty(gg.gg_ws_distill(30, 100), dtype=torch.uint8, device=DEV)
    st = torch.zeros(1, dtype=torch.int32, device=DEV)
    gg.gg_distill_forward(gg.make_rows(z), 30, 100, ids, gg.make_rows(top), 4, 2.0, 1.0, w, loss, None,
                          None, st, ws)
    assert torch.equal(loss, whole[0])
    e = torch.empty(0, 100, device=DEV)
    r = gg.make_rows(e)
    gg.gg_distill_forward(r, 0, 100, torch.empty(0, 4, dtype=torch.int32, device=DEV), r, 4, 2.0, 1.0,
                          None, torch.empty(0, device=DEV), None, r, st, ws)


def test_one_broadcast_row_and_shared_entries():
    """Rows, entries and ids of stride 0: every row the same."""
    z, ids, top, w = make(1, 300, 6, F32, seed=8)
    n = 40
    one = run(z, ids, top, w, 2.0, 1.0, True)
    many = run(z.expand(n, 300), ids.expand(n, 6), top.expand(n, 6), w.expand(n).contiguous(), 2.0,
               1.0, True)
    for a, b in zip(one[:3], many[:3]):
        assert torch.equal(a.expand_as(b), b)


@pytest.mark.parametrize("n,v", [(12, 61), (2, 40_000)])
def test_gradient_against_differences(n, v):
    """Along a direction, against central differences of the loss in 64 bits:
    their own error is about h^2 of the third derivative, far below fp32's."""
    z, ids, top, w = make(n, v, 7, F32, seed=9)
    way = torch.randn(n, v, generator=gen(10)).double()
    h = 1e-4
    f = lambda s: float(reference((z.cpu().double() + s * way), ids, top, w, 2.0, 1.0)[0][0].sum())  # noqa: E731
    slope = (f(h) - f(-h)) / (2 * h)
    for fused in (True, False):
        dz = run(z, ids, top, w, 2.0, 1.0, fused)[2].cpu().double()
        size = float((dz * way).abs().sum())
        bound = float((reference(z, ids, top, w, 2.0, 1.0)[1][2] * way.abs()).sum())
        assert abs(float((dz * way).sum()) - slope) <= 2 * bound + 1e-6 * size


def test_the_same_each_time_and_on_another_stream():
    z, ids, top, w = make(300, 9001, 12, BF16)
    first = run(z, ids, top, w, 2.0, 1.0, True)
    side = torch.cuda.Stream()
    for _ in range(2):
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            again = run(z, ids, top, w, 2.0, 1.0, True)
        torch.cuda.current_stream().wait_stream(side)
        assert all(torch.equal(a, b) for a, b in zip(first[:3], again[:3]))


# Rows of one value; of a value and two larger ones; and with one largest logit a few
# units above the rest: beyond |z| / T of 2^31 any difference leaves all to the largest.
def huge_rows(v, mask, T):
    z, ids, top, w = make(3, v, 4, F32, seed=11)
    z[:] = mask
    z[1, 1] = z[1, 3] = mask * (1.5 if mask > 0 else 0.5)
    z[2, 2] = mask * (1 - 2.0 ** -22 if mask < 0 else 1 + 2.0 ** -22)
    ids[:] = torch.arange(4)
    top[:] = 0.25
    q = torch.zeros(3, v, dtype=torch.float64)
    q[0] = 1.0 / v
    q[1, 1] = q[1, 3] = 0.5
    q[2, 2] = 1.0
    want = q.clone()
    want[:, :4] -= 0.25
    a = w.cpu().double()[:, None] * T
    return (z, ids, top, w), want * a, (q + 0.25) * a * 40 * U


HUGE = [(-1e30, 1.0), (-1e10, 0.1), (-1e37, 2.0), (3.3, 1e-30), (-1e20, 3.0)]


@pytest.mark.parametrize("v", [5, 50, 5000, 30_000, 40_000])
@pytest.mark.parametrize("mask,T", HUGE)
def test_the_largest_logit_may_be_a_masks_value(mask, T, v):
    args, want, bound = huge_rows(v, mask, T)
    loss, lse, dz, st = run(*args, T, 1.0, True)
    assert within(dz, want, bound) <= 0 and st == 0


@pytest.mark.parametrize("place", [False, True])
@pytest.mark.parametrize("v", [5, 50, 5000, 30_000, 40_000, 140_001])
@pytest.mark.parametrize("mask,T", HUGE + [(torch.finfo(F32).min, 1.0), (torch.finfo(F32).min, 3.0),
                                           (torch.finfo(F32).min / 4, 0.5), (-20_000.0, 1.0)])
def test_the_gradient_from_an_lse_that_holds_no_more_than_its_largest_logit(mask, T, v, place):
    args, want, bound = huge_rows(v, mask, T)
    z = args[0]
    if mask == -20_000.0:
        z[2] = mask
        z[2, 2] = 0.0
    loss, lse, dz, st = run(*args, T, 1.0, False, dz=(z, None, None) if place else None)
    assert within(dz, want, bound) <= 0 and st == 0


@pytest.mark.parametrize("v", [5, 50, 5000, 30_000, 40_000])
@pytest.mark.parametrize("mask,T", [(-1e30, 1.0), (-1e10, 0.1), (-3e5, 2.0), (torch.finfo(F32).min, 1.0)])
def test_the_loss_of_a_row_of_one_value(mask, T, v):
    """log p - log q = log v - log 4, whatever the value: a product and two
    logarithms of a sum that a lane's elements and the tree after it make."""
    (z, ids, top, w), _, _ = huge_rows(v, mask, T)
    z[:] = mask
    loss, lse, dz, st = run(z, ids, top, w, T, 1.0, False)
    a = w.cpu().double() * T * T
    want = a * (torch.log(torch.tensor(float(v)).double()) - math.log(4.0))
    assert within(loss, want, a * (200 + v / 256) * U + 8 * U * (want.abs() + a * math.log(4.0 * v))) <= 0


# Rows that are split, with elements behind the last whole piece, where |z| / T lies
# below 2^31 and m / T's own rounding is far above a unit of the exponent.  Rows of
# one value; its only largest logit at the end, at the front, and at both.
SPLIT_TAILS = [(40_001, F32), (40_002, F32), (40_003, F32), (70_001, BF16), (70_007, F16)]
LARGE = [(60_000.0, 6e-5), (-60_000.0, 6e-3), (60_000.0, 0.6), (-60_000.0, 0.06), (3.3, 1e-8)]


@pytest.mark.parametrize("mode", ["loss", "fused", "two", "in place"])
@pytest.mark.parametrize("v,t", SPLIT_TAILS)
@pytest.mark.parametrize("mask,T", LARGE)
def test_the_last_elements_of_split_rows_count_as_the_others(mask, T, v, t, mode):
    """q depends on differences, which are 0 or far too large to count here; the
    rounding of m / T, up to 64 units of the exponent, is in both of log q's terms."""
    gg = lib()
    z, ids, top, w = make(4, v, 4, t, seed=12)
    low, high = sorted((mask, mask / 2))
    z[:] = low
    z[1, v - 1] = z[2, 2] = z[3, 1] = z[3, v - 1] = high
    ids[:] = torch.tensor([0, 1, 2, v - 1])
    top[:] = 0.25
    (rl, rs, rd), (_, bs, _), _ = reference(z, ids, top, w, T, 1.0)
    a = w.cpu().double()
    Td = torch.tensor(T, dtype=F32).double()
    x = z.cpu().double() / Td
    q = torch.softmax(x, 1)
    far = (x.amax(1, keepdim=True) - x[:, [0, 1, 2, v - 1]]).mean(1)
    chain = (220 + v / 256) * U
    bl = a * Td * Td * (chain + 8 * U * (far + math.log(4.0 * v) + 70))
    at_ids = torch.zeros_like(q).scatter_(1, ids.cpu().long(), 0.25 * 40 * U)
    bd = (a * Td)[:, None] * (q * chain + at_ids) + 1.01 * UNIT[t] * rd.abs() + FLOOR[t]
    if mode == "loss":
        loss, lse = (torch.full((4,), float("nan"), device=DEV) for _ in range(2))
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        ws = torch.full((gg.gg_ws_distill(4, v),), 0xFF, dtype=torch.uint8, device=DEV)
        gg.gg_distill_forward(gg.make_rows(z), 4, v, ids, gg.make_rows(top), 4, T, 1.0, w, loss, lse,
                              None, st, ws)
        dz, st = None, int(st)
    else:
        loss, lse, dz, st = run(z, ids, top, w, T, 1.0, mode == "fused",
                                dz=(z, None, None) if mode == "in place" else None)
    assert st == 0
    assert within(loss, rl, bl + FLOOR[F32]) <= 0
    assert within(lse, rs, bs) <= 0
    if dz is not None:
        assert within(dz, rd, bd) <= 0


# All differences are far beyond 2^31 T, so the rows' largest logits take everything:
# the loss is a T times distances, finite although T^2 is not a number of fp32.
@pytest.mark.parametrize("v", [50, 5000, 40_000])
@pytest.mark.parametrize("T", [1e-20, 1e-25, 1e-30])
def test_the_loss_at_the_smallest_temperatures(T, v):
    z, ids, top, w = make(4, v, 4, F32, seed=13)
    ids[:] = torch.arange(4)
    z[:, 4:] = 0.0
    z[:, :4] = torch.tensor([-3.0, -1.0, 2.0, 5.0])
    top[:] = torch.tensor([1.0, 4.0, 2.0, 3.0])          # all of p at the second
    loss, lse, dz, st = run(z, ids, top, w, T, 1.0, True)
    want = w.cpu().double() * torch.tensor(T, dtype=F32).double() * 6.0
    assert st == 0 and within(loss, want, 16 * U * want + FLOOR[F32]) <= 0


@pytest.mark.parametrize("T", [1e20, 1e30])
def test_a_loss_of_zero_at_the_largest_temperatures(T):
    """Entries that cover the vocabulary, all logits equal: p = q exactly."""
    z, ids, top, w = make(3, 4, 4, F32, seed=14)
    ids[:] = torch.arange(4)
    z[:], top[:] = 0.5, 2.0
    loss, lse, dz, st = run(z, ids, top, w, T, 1.0, True)
    assert st == 0 and not loss.any() and not dz.any()


@pytest.mark.parametrize("mode", ["loss", "fused", "two"])
@pytest.mark.parametrize("v", [50, 5000, 40_000])
def test_a_teacher_of_nans_alone_shows(v, mode):
    """A row whose entries' logits are all NaN has a loss of NaN, and a gradient of NaN
    at its entries; one without entries has none, whatever lies at its -1."""
    gg = lib()
    z, ids, top, w = make(3, v, 4, F32, seed=15)
    ids[:] = torch.arange(4)
    top[0] = float("nan")
    ids[1, 1:], top[1, 0] = -1, float("nan")
    ids[2], top[2] = -1, float("nan")
    if mode == "loss":
        loss = torch.zeros(3, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        ws = torch.empty(gg.gg_ws_distill(3, v), dtype=torch.uint8, device=DEV)
        gg.gg_distill_forward(gg.make_rows(z), 3, v, ids, gg.make_rows(top), 4, 2.0, 1.0, w, loss,
                              None, None, st, ws)
    else:
        loss, _, dz, st = run(z, ids, top, w, 2.0, 1.0, mode == "fused")
        nan = torch.isnan(dz.cpu())
        assert nan[0, :4].all() and not nan[0, 4:].any()
        assert nan[1, 0] and not nan[1, 1:].any()
        assert not dz[2].any()
    loss = loss.cpu()
    assert torch.isnan(loss[:2]).all() and loss[2] == 0


@pytest.mark.parametrize("mode", ["loss", "fused", "two"])
@pytest.mark.parametrize("v", [50, 5000, 40_000])
@pytest.mark.parametrize("T", [0.25, 1.0, 1.5])
def test_the_loss_where_an_entry_is_masked_by_the_types_lowest_value(T, v, mode):
    """p times the distance, a number of fp32 although z log2(e) / T is none."""
    gg = lib()
    z, ids, top, w = make(3, v, 4, F32, seed=16)
    ids[:] = torch.arange(4)
    z[:, 2] = torch.finfo(F32).min
    top[:] = torch.tensor([8.0, 8.0, 8.0 - T, 8.0])
    if mode == "loss":
        loss = torch.zeros(3, device=DEV)
        st = torch.zeros(1, dtype=torch.int32, device=DEV)
        ws = torch.empty(gg.gg_ws_distill(3, v), dtype=torch.uint8, device=DEV)
        gg.gg_distill_forward(gg.make_rows(z), 3, v, ids, gg.make_rows(top), 4, T, 1.0, w, loss, None,
                              None, st, ws)
    else:
        loss = run(z, ids, top, w, T, 1.0, mode == "fused")[0]
    p = math.exp(-1) / (3 + math.exp(-1))
    want = w.cpu().double() * T * p * -torch.finfo(F32).min
    assert bool((want < torch.finfo(F32).max).all())
    assert within(loss, want, 40 * U * want) <= 0


@pytest.mark.parametrize("fused", [True, False])
@pytest.mark.parametrize("v", [50, 5000, 40_000, 140_001])
@pytest.mark.parametrize("rest,T", [(-3e38, 0.5), (3e38, 0.5), (-3e38, 2.0), (0.0, 1.0)])
def test_the_loss_is_infinite_where_all_entries_have_no_logit(rest, T, v, fused):
    z, ids, top, w = make(2, v, 4, F32, seed=17)
    ids[:] = torch.arange(4)
    z[:], z[:, :4] = rest, -INF
    loss, _, dz, st = run(z, ids, top, w, T, 1.0, fused)
    assert (loss == INF).all() and torch.isfinite(dz).all() and st == 0
