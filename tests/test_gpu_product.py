"""The product of 8-bit rows and 8-bit weights, and the weights' gradient, against the
same in 64 bits."""
import zlib

import pytest
import torch

from tests.op_util import BF16, E4M3, F16, F32, FLOOR, U, UNIT, like, untouched, within

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def lib():
    from paper_2606_02916_amd import gg
    return gg


def gen(*key):
    return torch.Generator().manual_seed(zlib.crc32(repr(key).encode()))


def blocks_of(d, g):
    return -(-d // g) if g else 1


def place8(codes, lead, pad):
    """e4m3 codes on the device at an odd place, NaNs around them."""
    n, d = codes.shape
    out, flat, _ = like(n, d, E4M3, DEV, lead=lead, pad=pad)
    out.view(torch.uint8).copy_(codes.view(torch.uint8))
    return out


def codes8(n, d, g):
    """Codes of all sizes, and some zeros."""
    x = torch.randn(n, d, generator=g) * torch.exp2(torch.randint(-6, 7, (n, d), generator=g).float())
    return x.clamp(-448, 448).to(E4M3)


def some_rows(n, k, group, g, lead=1, pad=3):
    """8-bit rows: the description, and their numbers and codes in 64 bits."""
    gg = lib()
    codes, kb = codes8(n, k, g), blocks_of(k, group)
    sc = torch.exp2(torch.rand(n, kb, generator=g) * 8 - 6)
    scd = torch.full((n, kb + 1), float("nan"), device=DEV)[:, 1:]
    scd.copy_(sc)
    num = codes.float().double() * sc.double()[:, torch.arange(k) // (group or k)]
    return gg.make_rows(place8(codes, lead, pad), scales=scd, group=group), num, codes.float().double()


def some_blocks(m, k, g, lead=3, pad=1):
    gg = lib()
    codes, mb, kb = codes8(m, k, g), blocks_of(m, 128), blocks_of(k, 128)
    sc = torch.exp2(torch.rand(mb, kb, generator=g) * 8 - 6)
    scd = torch.full((mb, kb + 2), float("nan"), device=DEV)[:, 1:1 + kb]
    scd.copy_(sc)
    num = codes.float().double() * sc.double()[torch.arange(m) // 128][:, torch.arange(k) // 128]
    return gg.make_blocks(place8(codes, lead, pad), scd), num, codes.float().double()


def coarse(an, ac, bn, bc):
    """What the 8-bit matrix instructions may drop: of each eight columns' products all
    but the largest lose less than 2^-13 of the largest, in which a code below 2^-6
    counts as 2^-6.  an, bn: the numbers, ac, bc: their codes."""
    def floor(num, codes):
        up = torch.where(codes == 0, 1.0, (2.0 ** -6 / codes.abs()).clamp(min=1.0))
        return torch.nn.functional.pad(num.abs() * up, (0, -num.shape[1] % 8))
    p, q = floor(an, ac).to(DEV), floor(bn, bc).to(DEV)
    lost = torch.zeros(len(p), len(q), dtype=torch.float64, device=DEV)
    for i in range(0, p.shape[1], 8):
        lost += (p[:, None, i:i + 8] * q[None, :, i:i + 8]).amax(2)
    return 7 * 2.0 ** -13 * lost.cpu()


def check(got, want, bound, t):
    """Within the bound; a result that rounds beyond fp16's largest number, 65504, is infinite."""
    got, over = got.detach().cpu().double(), torch.zeros_like(want, dtype=torch.bool)
    if t == F16:
        over = want.abs() + bound >= 65_520
        sure = want.abs() - bound >= 65_520
        assert torch.equal(got[sure], want[sure].sign() * float("inf"))
    assert within(got[~over], want[~over], bound[~over]) <= 0


def check_forward(n, k, m, t, group, lead=1, pad=3):
    """A sum of k products, in any order, is off by at most k U of their magnitudes, each
    block's scale by two roundings, the result by one."""
    gg, g = lib(), gen(n, k, m, group)
    a, an, ac = some_rows(n, k, group, g, lead, pad)
    b, bn, bc = some_blocks(m, k, g, lead + 2 if lead else 0, pad)
    out, flat, own = like(n, m, t, DEV, lead=lead, pad=pad)
    gg.gg_product_forward(a, n, k, b, m, gg.make_rows(out))
    assert untouched(flat, own)
    want, size = an @ bn.t(), an.abs() @ bn.abs().t()
    bound = (k + 4) * U * size + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    if t != F32:
        bound += coarse(an, ac, bn, bc) * 1.01
    check(out, want, bound, t)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 100, 129, 300])
@pytest.mark.parametrize("k", [1, 7, 16, 100, 127, 128, 129, 160, 255, 384, 602, 1200])
@pytest.mark.parametrize("m", [1, 5, 47, 128, 130, 333])
def test_product(n, k, m):
    t = (F32, F16, BF16)[(n + k + m) % 3]
    check_forward(n, k, m, t, 0 if (n + k) % 2 else 128)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n,k,m", [(1, 4096, 512), (16, 2048, 200), (40, 1024, 260), (100, 4096, 256),
                                   (200, 512, 512), (512, 256, 640), (1000, 1024, 700), (2500, 384, 1300),
                                   (47, 16_384, 33), (700, 128, 64), (3400, 400, 3700), (4097, 128, 3000), (20, 640, 700),
                                   (70, 900, 400), (600, 384, 900), (1400, 256, 2000), (2700, 272, 2500), (1500, 272, 1200),
                                   (6000, 144, 2900)])
def test_product_at_aligned_places(n, k, m, group, t):
    """Rows on 16-byte boundaries, and whole or partial tiles of them."""
    check_forward(n, k, m, t, group, 0, 0)


@pytest.mark.parametrize("n,k,m", [(10, 4104, 4100), (20, 4100, 2050), (50, 2104, 2100), (64, 2048, 2048),
                                   (90, 2000, 1500), (90, 1100, 9000), (200, 1304, 1000),
                                   (500, 520, 1000), (700, 520, 1000), (1000, 520, 1000), (700, 300, 1700), (700, 256, 1700),
                                   (2000, 300, 1900), (2000, 388, 1901), (2100, 260, 2200), (2100, 256, 2201), (2200, 700, 4000),
                                   (2200, 768, 4001)])
@pytest.mark.parametrize("a_at,b_at", [((1, 3), (2, 5)), ((4, 4), (8, 8)), ((0, 0), (1, 1)), ((3, 2), (0, 0)),
                                       ((4, 12), (0, 0))])
def test_product_wherever_rows_begin(n, k, m, a_at, b_at):
    """Tiles of every size, with rows that begin with a word, on a boundary of 16 bytes or at
    any byte, both matrices alike or not."""
    gg, g, t = lib(), gen(n, k, m), (F32, F16, BF16)[(n + k + m + a_at[0]) % 3]
    a, an, ac = some_rows(n, k, 128 if n % 4 else 0, g, *a_at)
    b, bn, bc = some_blocks(m, k, g, *b_at)
    out, flat, own = like(n, m, t, DEV, lead=1, pad=0)
    gg.gg_product_forward(a, n, k, b, m, gg.make_rows(out))
    assert untouched(flat, own)
    x, y = an.to(DEV), bn.to(DEV)
    want, size = (x @ y.t()).cpu(), (x.abs() @ y.abs().t()).cpu()
    bound = (k + 4) * U * size + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    if t != F32:
        bound += coarse(an, ac, bn, bc) * 1.01
    check(out, want, bound, t)


@pytest.mark.parametrize("n,k,m", [(3, 200, 140), (60, 300, 50), (400, 300, 300), (600, 256, 512)])
def test_nans_and_infinities_keep_to_their_row_and_column(n, k, m):
    gg, g = lib(), gen(n)
    acodes, bcodes = codes8(n, k, g), codes8(m, k, g)
    kb, mb = blocks_of(k, 128), blocks_of(m, 128)
    sa, sb = (torch.rand(n, kb, generator=g) + 0.5).to(DEV), (torch.rand(mb, kb, generator=g) + 0.5).to(DEV)
    a, b = place8(acodes, 0, 0), place8(bcodes, 0, 0)
    clean, out = torch.empty(n, m, device=DEV), torch.empty(n, m, device=DEV)

    def call(to):
        gg.gg_product_forward(gg.make_rows(a, scales=sa, group=128), n, k, gg.make_blocks(b, sb), m,
                              gg.make_rows(to))

    call(clean)
    a.view(torch.uint8)[1, k - 1] = 0x7F
    b.view(torch.uint8)[m - 2, 5] = 0xFF
    sa[2, kb - 1] = float("inf")
    call(out)
    out, clean = out.cpu(), clean.cpu()
    rest = torch.ones(n, m, dtype=torch.bool)
    rest[1:3] = False
    rest[:, m - 2] = False
    assert torch.equal(out[rest], clean[rest])
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isnan(out[:, m - 2]).all())
    assert not bool(torch.isfinite(out[2]).any())


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("k", [512, 640, 1536])
def test_scales_by_fours(k, offset):
    """Many tiles of rows whose scales lie on 16-byte boundaries, and beside them."""
    gg, g, n, m = lib(), gen(k), 3333, 4000
    ac, bc, kb = codes8(n, k, g), codes8(m, k, g), k // 128
    sa, sb = torch.exp2(torch.rand(n, kb, generator=g) * 8 - 6), torch.rand(32, kb, generator=g) + 0.5
    wide = -(-(kb + 1) // 4) * 4
    far = [torch.full((r, wide), float("nan"), device=DEV) for r in (n, 32)]
    sad, sbd = (f[:, offset:offset + kb] for f in far)
    sad.copy_(sa), sbd.copy_(sb)
    a, b, out = ac.to(DEV), bc.to(DEV), torch.empty(n, m, dtype=BF16, device=DEV)
    gg.gg_product_forward(gg.make_rows(a, scales=sad, group=128), n, k, gg.make_blocks(b, sbd), m,
                          gg.make_rows(out))
    col = torch.arange(k) // 128
    ac, bc = ac.float().double(), bc.float().double()
    an, bn = ac * sa.double()[:, col], bc * sb.double()[torch.arange(m) // 128][:, col]
    want, size = ((x.to(DEV) @ y.to(DEV).t()).cpu() for x, y in ((an, bn), (an.abs(), bn.abs())))
    check(out, want, (k + 4) * U * size + 1.01 * UNIT[BF16] * want.abs() + 1.01 * coarse(an, ac, bn, bc), BF16)


@pytest.mark.parametrize("k", [400, 1000, 1010, 4000])
def test_the_last_of_four_blocks_is_cut(k):
    """As many scales as whole fours of blocks have, aligned, and codes that end inside a block."""
    gg, g, n, m = lib(), gen(k), 2200, 4000
    ac, bc, kb = codes8(n, k, g), codes8(m, k, g), blocks_of(k, 128)
    assert kb % 4 == 0
    sa, sb = torch.exp2(torch.rand(n, kb, generator=g) * 8 - 6), torch.rand(32, kb, generator=g) + 0.5
    a, b = (torch.zeros(x, kb * 128, device=DEV).to(E4M3)[:, :k] for x in (n, m))
    a.view(torch.uint8).copy_(ac.view(torch.uint8)), b.view(torch.uint8).copy_(bc.view(torch.uint8))
    out = torch.empty(n, m, dtype=BF16, device=DEV)
    gg.gg_product_forward(gg.make_rows(a, scales=sa.to(DEV), group=128), n, k,
                          gg.make_blocks(b, sb.to(DEV)), m, gg.make_rows(out))
    col = torch.arange(k) // 128
    ac, bc = ac.float().double(), bc.float().double()
    an, bn = ac * sa.double()[:, col], bc * sb.double()[torch.arange(m) // 128][:, col]
    want, size = ((x.to(DEV) @ y.to(DEV).t()).cpu() for x, y in ((an, bn), (an.abs(), bn.abs())))
    check(out, want, (k + 4) * U * size + 1.01 * UNIT[BF16] * want.abs() + 1.01 * coarse(an, ac, bn, bc), BF16)


def test_product_of_no_rows():
    gg = lib()
    b = some_blocks(20, 30, gen(0))[0]
    a = gg.make_rows(torch.empty(0, 30, device=DEV).to(E4M3), scales=torch.empty(0, device=DEV))
    gg.gg_product_forward(a, 0, 30, b, 20, gg.make_rows(torch.empty(0, 20, device=DEV)))


@pytest.mark.parametrize("n", [5, 300])
def test_one_row_for_all_and_rows_beyond_32_bits_of_bytes(n):
    """Rows of stride 0; weights, rows and results whose places pass 2^32 bytes."""
    gg, g, k, m, step = lib(), gen(n), 300, 150, 1 << 25
    ac, bc = codes8(1, k, g), codes8(m, k, g)
    sc, sb = torch.rand(1, 3, generator=g) + 0.5, torch.rand(2, 3, generator=g) + 0.5
    big = torch.empty(m * step, dtype=torch.uint8, device=DEV)
    b = big.as_strided((m, k), (step, 1))
    b.copy_(bc.view(torch.uint8))
    a, sa = ac.to(DEV).expand(n, k), sc.to(DEV).expand(n, 3)
    out = torch.empty(n, m, device=DEV)
    gg.gg_product_forward(gg.make_rows(a, scales=sa, group=128), n, k,
                          gg.make_blocks(b.view(E4M3), sb.to(DEV)), m, gg.make_rows(out))
    an = ac.float().double() * sc.double()[:, torch.arange(k) // 128]
    bn = bc.float().double() * sb.double()[torch.arange(m) // 128][:, torch.arange(k) // 128]
    want, size = (an @ bn.t()).expand(n, m), (an.abs() @ bn.abs().t()).expand(n, m)
    assert within(out, want, (k + 5) * U * size) <= 0
    # the other operand and the result far apart
    step = (1 << 32) // n + 4096 & -4
    a = big[:n * step].as_strided((n, k), (step, 1))
    a.copy_(ac.view(torch.uint8).expand(n, k))
    far = torch.empty(n * step // 4, device=DEV).as_strided((n, m), (step // 4, 1))
    gg.gg_product_forward(gg.make_rows(a.view(E4M3), scales=sa, group=128), n, k,
                          gg.make_blocks(bc.to(DEV), sb.to(DEV)), m, gg.make_rows(far))
    assert within(far, want, (k + 5) * U * size) <= 0


def test_results_do_not_depend_on_the_stream_or_the_call():
    gg, g = lib(), gen(11)
    side = torch.cuda.Stream()
    for n, k, m in ((1, 2048, 300), (60, 4096, 200), (900, 640, 900)):
        a = some_rows(n, k, 128, g)[0]
        b = some_blocks(m, k, g)[0]
        outs = [torch.empty(n, m, device=DEV) for _ in range(3)]
        gg.gg_product_forward(a, n, k, b, m, gg.make_rows(outs[0]))
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            gg.gg_product_forward(a, n, k, b, m, gg.make_rows(outs[1]))
        gg.gg_product_forward(a, n, k, b, m, gg.make_rows(outs[2]), stream=side)
        torch.cuda.current_stream().wait_stream(side)
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])


# ---------------------------------------------------------------------------
# The weights' gradient.
# ---------------------------------------------------------------------------
PARTS = {F32: 0.0, F16: 2.0 ** -15, BF16: 2.0 ** -8}    # what is left off dz * scale


def grad_case(n, k, m, tz, t, group, add=False, lead=1, pad=3, dz=None):
    gg, g = lib(), gen(n, k, m, str(tz), group)
    a, an, _ = some_rows(n, k, group, g, lead, pad)
    z = (torch.randn(n, m, generator=g) * torch.exp2(torch.randint(-8, 3, (n, 1), generator=g).float())).to(tz)
    zd, _, _ = like(n, m, tz, DEV, lead=lead, pad=pad)
    zd.copy_(z)
    dw, flat, own = like(m, k, t, DEV, lead=lead, pad=pad)
    old = torch.randn(m, k, generator=g).to(t) * 8
    if add:
        dw.copy_(old)
    size = gg.gg_ws_product(n, k, m)
    ws = torch.full((size,), 0xFF, dtype=torch.uint8, device=DEV) if size else None
    gg.gg_product_backward(a, n, k, gg.make_rows(zd), m, gg.make_rows(dw),
                           gg.GG_PRODUCT_ADD if add else 0, ws)
    assert untouched(flat, own)
    z = z.double()
    want, size = z.t() @ an, z.abs().t() @ an.abs()
    if add:
        want = want + old.double()
        size = size + old.double().abs()
    # (splits add one rounding each, and their join)
    bound = (n + n / 256 + 4) * U * size + 1.01 * PARTS[t] * size + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    return dw, want, bound


def grad_on_device(n, k, m, tz, t, group, add, z_at):
    """The same of larger sizes, the 64-bit products on the device."""
    gg, g = lib(), gen(n, k, m)
    a, an, _ = some_rows(n, k, group, g)
    z = torch.randn(n, m, generator=g).to(tz)
    zd = like(n, m, tz, DEV, lead=z_at[0], pad=z_at[1])[0]
    zd.copy_(z)
    dw, flat, own = like(m, k, t, DEV, lead=1, pad=3)
    old = (torch.randn(m, k, generator=g) * 8).to(t)
    if add:
        dw.copy_(old)
    ws = torch.full((max(gg.gg_ws_product(n, k, m), 16),), 0xFF, dtype=torch.uint8, device=DEV)
    gg.gg_product_backward(a, n, k, gg.make_rows(zd), m, gg.make_rows(dw),
                           gg.GG_PRODUCT_ADD if add else 0, ws)
    assert untouched(flat, own)
    z, an, old = z.to(DEV).double(), an.to(DEV), (old.to(DEV).double() if add else 0)
    want, size = z.t().contiguous() @ an + old, z.abs().t().contiguous() @ an.abs() + abs(old)
    bound = (n + 4) * U * size + 1.01 * PARTS[t] * size + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    check(dw, want.cpu(), bound.cpu(), t)


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 100, 257, 1000])
@pytest.mark.parametrize("k", [1, 7, 100, 128, 129, 200, 602])
@pytest.mark.parametrize("m", [1, 5, 47, 64, 65, 130, 333])
def test_weight_gradient(n, k, m):
    tz, t = ((F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32))[(n + k + m) % 5]
    check(*grad_case(n, k, m, tz, t, 0 if (n + k) % 2 else 128, add=(n + m) % 3 == 0), t)


@pytest.mark.parametrize("tz,t", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n,k,m", [(64, 128, 64), (128, 256, 512), (3000, 128, 40), (5000, 512, 256),
                                   (1024, 1024, 1024), (520, 640, 2048), (40_001, 100, 47), (130, 130, 136),
                                   (2000, 700, 1000)])
@pytest.mark.parametrize("add", [False, True])
def test_weight_gradient_at_aligned_places(n, k, m, group, tz, t, add):
    check(*grad_case(n, k, m, tz, t, group, add, 0, 0), t)


@pytest.mark.parametrize("n,k,m", [(1100, 4090, 4088), (1088, 4096, 4096), (50_001, 1030, 1000),
                                   (33_000, 1024, 1032), (70_000, 130, 2000)])
@pytest.mark.parametrize("group,add", [(0, False), (128, True)])
def test_weight_gradient_with_work_for_every_cu(n, k, m, group, add):
    """bf16 gradients whose rows lie on 16-byte boundaries, and products enough for large
    tiles; codes and results at odd places."""
    grad_on_device(n, k, m, BF16, BF16, group, add, (8, 8))


@pytest.mark.parametrize("tz,t", [(F32, F32), (F16, F16), (BF16, BF16), (F16, F32), (BF16, F32)])
@pytest.mark.parametrize("n,k,m", [(9001, 1301, 1299), (20_001, 300, 1004), (1000, 2503, 2499), (257, 3001, 2999)])
@pytest.mark.parametrize("group,add", [(128, False), (0, True)])
def test_weight_gradient_with_work_for_tiles_of_128(n, k, m, tz, t, group, add):
    grad_on_device(n, k, m, tz, t, group, add, (1, 3))


@pytest.mark.parametrize("tz,t", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, F32)])
@pytest.mark.parametrize("n,k,m", [(40, 70, 50), (300, 260, 136)])
def test_weight_gradient_of_small_scales(n, k, m, tz, t):
    """Scales near the least one, whose products with gradients, and what those leave behind
    their upper bits, lie below the least normal number."""
    gg, g = lib(), gen(n)
    codes, z = codes8(n, k, g), torch.randn(n, m, generator=g).to(tz)
    sc = torch.exp2(-110 - 12 * torch.rand(n, generator=g))
    out = torch.empty(m, k, dtype=t, device=DEV)
    ws = torch.empty(max(gg.gg_ws_product(n, k, m), 16), dtype=torch.uint8, device=DEV)
    gg.gg_product_backward(gg.make_rows(codes.to(DEV), scales=sc.to(DEV)), n, k, gg.make_rows(z.to(DEV)), m,
                           gg.make_rows(out), 0, ws)
    an, z = codes.float().double() * sc.double()[:, None], z.double()
    want, size = z.t() @ an, z.abs().t() @ an.abs()
    # (bf16's least number, of which a term's other factor is a multiple, is 2^-133)
    least = (n + 4) * 2.0 ** -133 * 448 + FLOOR[t]
    check(out, want, (n + 4) * U * size + 1.01 * PARTS[t] * size + 1.01 * UNIT[t] * want.abs() + least, t)


def test_weight_gradient_of_no_rows():
    gg = lib()
    a = gg.make_rows(torch.empty(0, 30, device=DEV).to(E4M3), scales=torch.empty(0, device=DEV))
    dz = gg.make_rows(torch.empty(0, 20, device=DEV))
    dw = torch.full((20, 30), 3.0, device=DEV)
    gg.gg_product_backward(a, 0, 30, dz, 20, gg.make_rows(dw), gg.GG_PRODUCT_ADD, None)
    assert bool((dw == 3).all())
    gg.gg_product_backward(a, 0, 30, dz, 20, gg.make_rows(dw), 0, None)
    assert not dw.any()


@pytest.mark.parametrize("tz,t", [(F32, F32), (F16, F16), (BF16, BF16), (BF16, F32)])
def test_infinities_of_a_gradient(tz, t):
    """An infinite gradient makes its weights' row infinite (NaN where the code is zero),
    a NaN makes it NaN, a NaN code its column, and nothing else changes."""
    gg, g, n, k, m = lib(), gen(1), 300, 140, 70
    codes = codes8(n, k, g)
    codes.view(torch.uint8)[7] = torch.where(torch.arange(k) % 2 == 0, 0x38, 0xB8)   # 1, -1
    codes.view(torch.uint8)[9, 3] = 0
    z = torch.randn(n, m, generator=g).to(tz)
    a, zd, sc = place8(codes, 0, 0), z.to(DEV), torch.ones(n, device=DEV)
    size = gg.gg_ws_product(n, k, m)
    ws = torch.empty(size, dtype=torch.uint8, device=DEV)

    def call():
        dw = torch.empty(m, k, dtype=t, device=DEV)
        gg.gg_product_backward(gg.make_rows(a, scales=sc), n, k, gg.make_rows(zd), m, gg.make_rows(dw), 0,
                               ws)
        return dw.cpu().float()

    clean = call()
    zd[7, 5] = float("inf")
    zd[8, 6] = float("nan")
    zd[9, 7] = -float("inf")
    a.view(torch.uint8)[20, 100] = 0x7F
    dw, rest = call(), torch.ones(m, k, dtype=torch.bool)
    rest[5:8] = False
    rest[:, 100] = False
    assert torch.equal(dw[rest], clean[rest])
    sign = torch.where(torch.arange(k) % 2 == 0, 1.0, -1.0) * float("inf")
    here = torch.arange(k) != 100
    assert torch.equal(dw[5][here], sign[here])
    assert bool(torch.isnan(dw[6]).all()) and bool(torch.isnan(dw[:, 100]).all())
    assert bool(torch.isnan(dw[7, 3]))
    nonzero = (codes[9].float() != 0) & here
    assert torch.equal(dw[7][nonzero], -codes[9].float()[nonzero].sign() * float("inf"))


def test_weight_gradient_of_rows_beyond_32_bits_of_bytes():
    gg, g, n, k, m, step = lib(), gen(4), 300, 200, 70, 1 << 24
    codes, z = codes8(n, k, g), torch.randn(n, m, generator=g)
    sc = torch.rand(n, generator=g) + 0.5
    big = torch.empty(n * step, dtype=torch.uint8, device=DEV)
    a = big.as_strided((n, k), (step, 1))
    a.copy_(codes.view(torch.uint8))
    far = big[1024:].view(F32).as_strided((n, m), (step // 4, 1))
    far.copy_(z)
    out = big[4096:].view(F32).as_strided((m, k), (1 << 24, 1))
    ws = torch.empty(gg.gg_ws_product(n, k, m), dtype=torch.uint8, device=DEV)
    gg.gg_product_backward(gg.make_rows(a.view(E4M3), scales=sc.to(DEV)), n, k, gg.make_rows(far), m,
                           gg.make_rows(out), 0, ws)
    an = codes.float().double() * sc.double()[:, None]
    want, size = z.double().t() @ an, z.double().abs().t() @ an.abs()
    assert within(out, want, (n + 6) * U * size) <= 0


def test_gradients_against_differences():
    """The loss sum(c * (a b^T)) along directions of a and b, numbers in 8 bits: central
    differences of a bilinear form are exact but for their own roundings in 64 bits.  The
    way to a is the forward call on c in 8 bits and the transposed weights, whose own
    rounding to 8 bits the difference takes along."""
    gg, g, n, k, m = lib(), gen(21), 150, 200, 140
    w = torch.randn(m, k, generator=g).to(DEV)
    b, bt = (torch.empty(s, dtype=E4M3, device=DEV) for s in ((m, k), (k, m)))
    sb, sbt = (torch.empty(2, 2, device=DEV) for _ in range(2))
    blocks, back = gg.make_blocks(b, sb), gg.make_blocks(bt, sbt)
    gg.gg_quantise_blocks(gg.make_rows(w), m, k, blocks, back)
    x, c = torch.randn(n, k, generator=g).to(DEV), torch.randn(n, m, generator=g).to(DEV)
    a, c8 = (torch.empty(s, dtype=E4M3, device=DEV) for s in ((n, k), (n, m)))
    sa, sc = (torch.empty(n, 2, device=DEV) for _ in range(2))
    ar, cr = (gg.make_rows(t, scales=s, group=128) for t, s in ((a, sa), (c8, sc)))
    gg.gg_quantise_rows(gg.make_rows(x), n, k, ar)
    gg.gg_quantise_rows(gg.make_rows(c), n, m, cr)
    da, db = torch.empty(n, k, device=DEV), torch.empty(m, k, device=DEV)
    gg.gg_product_forward(cr, n, m, back, k, gg.make_rows(da))
    ws = torch.empty(gg.gg_ws_product(n, k, m), dtype=torch.uint8, device=DEV)
    gg.gg_product_backward(ar, n, k, gg.make_rows(c), m, gg.make_rows(db), 0, ws)
    num = lambda q, s: q.float().cpu().double() * s.cpu().double()[:, torch.arange(q.shape[1]) // 128]  # noqa: E731
    an, cn = num(a, sa), num(c8, sc)
    bn = num(b, sb[(torch.arange(m) // 128).to(DEV)])
    way_a, way_b = (torch.randn(s, generator=g).double() for s in ((n, k), (m, k)))
    for got, way, f in ((da, way_a, lambda h: (cn * ((an + h * way_a) @ bn.t())).sum()),
                        (db, way_b, lambda h: (c.cpu().double() * (an @ (bn + h * way_b).t())).sum())):
        slope = float(f(0.5) - f(-0.5))
        part = got.cpu().double() * way
        size = float((cn.abs() @ bn.abs() * way.abs()).sum() if got is da else
                     (c.cpu().double().abs().t() @ an.abs() * way.abs()).sum())
        assert abs(float(part.sum()) - slope) <= size * (max(n, m) + 8) * U


def test_gradients_are_the_same_each_time_and_on_another_stream():
    side = torch.cuda.Stream()
    for n, k, m in ((20_000, 200, 47), (700, 900, 1300)):
        first = grad_case(n, k, m, F32, F32, 128)[0]
        for _ in range(2):
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                again = grad_case(n, k, m, F32, F32, 128)[0]
            torch.cuda.current_stream().wait_stream(side)
            assert torch.equal(first, again)


# ---------------------------------------------------------------------------
# Scales at the ends of fp32's range: the product of two may lie beyond them.
# ---------------------------------------------------------------------------
def scaled(n, k, m, t, sa, sb, group, ac, bc, a_at=(0, 0), step=None):
    """The product of given codes and scales, and its value, its terms' magnitudes and what the
    8-bit instructions may drop, in 64 bits.  step: weights' rows so many bytes apart."""
    gg = lib()
    col, row = torch.arange(k) // 128, torch.arange(m) // 128
    if step:
        b = torch.empty(m * step, dtype=torch.uint8, device=DEV).as_strided((m, k), (step, 1))
        b.copy_(bc.view(torch.uint8))
        b = b.view(E4M3)
    else:
        b = bc.to(DEV)
    out = torch.full((n, m), float("nan"), device=DEV).to(t)
    sad = sa.to(DEV)
    gg.gg_product_forward(gg.make_rows(place8(ac, *a_at), scales=sad, group=group), n, k,
                          gg.make_blocks(b, sb.to(DEV)), m, gg.make_rows(out))
    ac, bc = ac.float().double(), bc.float().double()
    an = ac * (sa.double()[:, col] if group else sa.double()[:, :1])
    bn = bc * sb.double()[row][:, col]
    x, y = an.to(DEV), bn.to(DEV)
    want, size = (x @ y.t()).cpu(), (x.abs() @ y.abs().t()).cpu()
    return out, want, size, 0.0 if t == F32 else 1.01 * coarse(an, ac, bn, bc)


# few rows, of words and of bytes; tiles of 32, 128 and 256 rows; rows far apart
ENDS = [(3, 700, 140, (0, 0), None), (60, 300, 50, (1, 0), None), (64, 2048, 2048, (0, 0), None),
        (70, 2100, 1500, (1, 2), None), (2100, 260, 2200, (0, 0), None), (2200, 768, 4001, (0, 0), None),
        (2200, 700, 4001, (4, 0), None), (40, 300, 150, (0, 0), 1 << 24)]


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n,k,m,a_at,step", ENDS)
def test_scales_whose_product_is_no_normal_number(n, k, m, a_at, step, group, t):
    """Rows of tiny gradients with ordinary weights, and tiny weights with tiny rows: the
    product of scales lies below 2^-126, results do not."""
    g = gen(n, k, m, group)
    kb, mb = blocks_of(k, 128), blocks_of(m, 128)
    # codes from 32 to 448 of either sign, more of them positive, so that sums are large
    ac, bc = ((torch.rand(r, k, generator=g) * 416 + 32) * torch.where(torch.rand(r, k, generator=g) < 0.8, 1, -1)
              for r in (n, m))
    ac, bc = ac.to(E4M3), bc.to(E4M3)
    for ea, eb in ((-126, -14), (-70, -72), (-14, -126), (-20, -110)):
        sa = torch.exp2(ea + 4 * torch.rand(n, kb if group else 1, generator=g))
        sb = torch.exp2(eb + 2 * torch.rand(mb, kb, generator=g))
        out, want, size, cut = scaled(n, k, m, t, sa, sb, group, ac, bc, a_at, step)
        assert float(size.max()) > 2.0 ** -126
        # (below 2^-126 each block's sum is rounded to a multiple of 2^-149, bf16's results of 2^-133)
        least = (kb + 1) * 2.0 ** -150 + (2.0 ** -134 if t == BF16 else 0)
        check(out, want, (k + 4) * U * size + 1.01 * UNIT[t] * want.abs() + least + cut, t)


@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n,k,m,a_at,step", ENDS)
def test_scales_whose_product_is_beyond_the_largest_number(n, k, m, a_at, step, group, t):
    """Zeros stay zeros, and the least codes' products are finite, where the product of scales
    passes 2^128."""
    g = gen(n, k, m, group)
    kb, mb = blocks_of(k, 128), blocks_of(m, 128)
    ac, bc = (torch.where(torch.rand(r, k, generator=g) < 0.5, 2.0 ** -9, 0.0).to(E4M3) for r in (n, m))
    ac[n // 2], bc[m // 2] = torch.zeros(k).to(E4M3), torch.zeros(k).to(E4M3)
    for ea, eb in ((90, 40), (118, 11), (20, 110), (12, 118)):
        sa = torch.exp2(ea + torch.rand(n, kb if group else 1, generator=g))
        sb = torch.exp2(eb + torch.rand(mb, kb, generator=g))
        out, want, size, cut = scaled(n, k, m, t, sa, sb, group, ac, bc, a_at, step)
        assert float(size.max()) < 2.0 ** 127
        if t == F16:
            big = want >= 65_520
            assert torch.equal(out.cpu().double(), torch.where(big, float("inf"), 0.0).double())
        else:
            check(out, want, (k + 4) * U * size + 1.01 * UNIT[t] * want.abs() + cut, t)


@pytest.mark.parametrize("t", [F32, BF16])
@pytest.mark.parametrize("n,k,m,a_at,step", ENDS)
def test_scales_of_every_size(n, k, m, a_at, step, t):
    """Scales from 2^-126 to 2^119, each row's and block's of its own size."""
    g = gen(n, k, m)
    kb, mb = blocks_of(k, 128), blocks_of(m, 128)
    ac, bc = codes8(n, k, g), codes8(m, k, g)
    sa = torch.exp2(torch.randint(-126, 119, (n, 1), generator=g) + torch.rand(n, kb, generator=g))
    sb = torch.exp2(torch.randint(-126, 111, (mb, 1), generator=g) + torch.rand(mb, kb, generator=g))
    out, want, size, cut = scaled(n, k, m, t, sa, sb, 128, ac, bc, a_at, step)
    least = (kb + 1) * 2.0 ** -150 + (2.0 ** -134 if t == BF16 else 0)
    bound = (k + 4) * U * size + 1.01 * UNIT[t] * want.abs() + least + cut
    here = size < 2.0 ** 127
    assert 0.3 < float(here.double().mean()) and float((size[here] > 2.0 ** -126).double().mean()) > 0.3
    assert within(out.cpu()[here], want[here], bound[here]) <= 0
    # far beyond the range no result is finite (blocks' sums that overflow in both directions add
    # up to a NaN)
    assert not bool(torch.isfinite(out.cpu()[want.abs() - bound > 2.0 ** 129]).any())


# ---------------------------------------------------------------------------
# Kernels in every type and with both kinds of scales.
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("t", [F32, F16, BF16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n,k,m", [(5, 300, 150), (140, 260, 131), (130, 128, 40)])
def test_rows_far_apart(n, k, m, group, t):
    """Rows of both matrices, their scales and the results more than 2^23 bytes apart."""
    gg, g, step = lib(), gen(n, k, m, group), (1 << 23) + 4096
    ac, bc = codes8(n, k, g), codes8(m, k, g)
    ka, kb, mb = blocks_of(k, group), blocks_of(k, 128), blocks_of(m, 128)
    sa, sb = (torch.exp2(torch.rand(r, c, generator=g) * 8 - 6) for r, c in ((n, ka), (mb, kb)))
    size = torch.finfo(t).bits // 8
    big = torch.full((max(n, m) * step,), 0xFF, dtype=torch.uint8, device=DEV)

    def far(rows, cols, dtype, at):
        e = torch.finfo(dtype).bits // 8
        return big[at:].view(dtype).as_strided((rows, cols), (step // e, 1))

    a, b, out = far(n, k, E4M3, 0), far(m, k, E4M3, 4096), far(n, m, t, 8192)
    sad, sbd = far(n, ka, F32, 16_384), far(mb, kb, F32, 20_480)
    a.view(torch.uint8).copy_(ac.view(torch.uint8)), b.view(torch.uint8).copy_(bc.view(torch.uint8))
    sad.copy_(sa), sbd.copy_(sb)
    gg.gg_product_forward(gg.make_rows(a, scales=sad, group=group), n, k, gg.make_blocks(b, sbd), m,
                          gg.make_rows(out))
    # what lies before and behind a result's row is left alone
    around = torch.stack([big[i * step + 8192 - 64:i * step + 8192 + m * size + 64] for i in range(n)]).cpu()
    assert bool((around[:, :64] == 0xFF).all()) and bool((around[:, -64:] == 0xFF).all())
    col = torch.arange(k)
    ac, bc = ac.float().double(), bc.float().double()
    an = ac * sa.double()[:, col // (group or k)]
    bn = bc * sb.double()[torch.arange(m) // 128][:, col // 128]
    want, mag = an @ bn.t(), an.abs() @ bn.abs().t()
    bound = (k + 4) * U * mag + 1.01 * UNIT[t] * want.abs() + FLOOR[t]
    if t != F32:
        bound += 1.01 * coarse(an, ac, bn, bc)
    check(out, want, bound, t)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("group", [0, 128])
@pytest.mark.parametrize("n,k,m", [(2200, 1024, 4000), (2304, 1536, 4096), (2200, 644, 4001)])
def test_large_tiles_of_every_kind(n, k, m, group, t):
    """More than four blocks of k and a round of large tiles, rows on word or 16-byte boundaries:
    scales one by one, and one a row."""
    check_forward(n, k, m, t, group, 0, 0)


@pytest.mark.parametrize("offset", [0, 1])
@pytest.mark.parametrize("k", [1024, 2048])
def test_scales_by_fours_of_more_blocks(k, offset):
    """Fours of blocks, in the tiles that load scales so, on 16-byte boundaries and beside them."""
    test_scales_by_fours(k, offset)


@pytest.mark.parametrize("t", [F16, BF16])
@pytest.mark.parametrize("n,k,m", [(3, 200, 140), (60, 300, 50), (600, 256, 512), (2200, 900, 4000)])
def test_nans_of_8_bit_instructions_keep_to_their_row_and_column(n, k, m, t):
    """A NaN code and infinite and NaN scales, of a row and of a block of weights."""
    gg, g = lib(), gen(n)
    acodes, bcodes = codes8(n, k, g), codes8(m, k, g)
    kb, mb = blocks_of(k, 128), blocks_of(m, 128)
    sa, sb = (torch.rand(n, kb, generator=g) + 0.5).to(DEV), (torch.rand(mb, kb, generator=g) + 0.5).to(DEV)
    a, b = place8(acodes, 0, 0), place8(bcodes, 0, 0)
    clean, out = (torch.empty(n, m, dtype=t, device=DEV) for _ in range(2))

    def call(to):
        gg.gg_product_forward(gg.make_rows(a, scales=sa, group=128), n, k, gg.make_blocks(b, sb), m,
                              gg.make_rows(to))

    call(clean)
    a.view(torch.uint8)[1, k - 1] = 0x7F
    b.view(torch.uint8)[m - 2, 5] = 0xFF
    sa[2, kb - 1] = float("inf")
    last = (mb - 1) * 128 if mb > 1 else m
    if mb > 1:
        sb[mb - 1, 0] = float("nan")
    call(out)
    out, clean = out.cpu(), clean.cpu()
    rest = torch.ones(n, m, dtype=torch.bool)
    rest[1:3] = False
    rest[:, m - 2] = False
    rest[:, last:] = False
    assert torch.equal(out[rest], clean[rest])
    assert bool(torch.isnan(out[1]).all()) and bool(torch.isnan(out[:, m - 2]).all())
    assert bool(torch.isnan(out[:, last:]).all())
    assert not bool(torch.isfinite(out[2]).any())
