"""The student: one step against the same step in 64 bits, its lessons from a
window's GraphSAGE answers, its 8-bit rows through the fetch path, and the
operators in a replayed graph."""
import numpy as np
import pytest
import torch

import synth
from tests.gpu_util import World
from tests.op_util import BF16, E4M3, F16, F32, U, UNIT

pytestmark = pytest.mark.gpu
DEV = "cuda:0"


def gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def step64(table, w, head, ids, top_ids, top, x, scale, T, eps, weight):
    """Loss per row and the gradients of table, w and head in 64 bits."""
    p = [t.detach().cpu().double().requires_grad_(True) for t in (table, w, head)]
    here = (ids >= 0)[:, None]
    e = torch.where(here, p[0][ids.clamp(min=0)], 0.0) * scale
    s = e + (0 if x is None else x.cpu().double())
    y = s * (s.square().mean(1, keepdim=True) + eps) ** -0.5 * p[1]
    lq = torch.log_softmax(y @ p[2] / T, 1)
    hole = top_ids < 0
    lp = torch.log_softmax((top.double() / T).masked_fill(hole, -float("inf")), 1).masked_fill(hole, 0)
    q = lp.exp().masked_fill(hole, 0)
    loss = (q * (lp - lq.gather(1, top_ids.clamp(min=0)))).sum(1) * T * T * weight
    loss.sum().backward()
    return loss.detach(), [t.grad for t in p]


@pytest.mark.parametrize("with_x", [False, True])
@pytest.mark.parametrize("n,dim,classes", [(1, 16, 5), (301, 100, 47), (2000, 33, 300)])
def test_step_against_64_bits(n, dim, classes, with_x):
    """Differences stay within a hundred roundings of fp32 of each gradient's
    largest entry: the products' sums of `dim`, `classes` and `n` terms add
    about as many."""
    from paper_2606_02916_amd import Student
    k, N = 4, 400
    st = Student(N, dim, classes, max_rows=2500, k=k, rate=0.5, device=DEV, generator=gen(n))
    st.w.copy_(1 + 0.2 * torch.randn(dim, generator=gen(1), device=DEV))
    g = torch.Generator().manual_seed(2)
    ids = torch.randint(0, N, (n,), generator=g)
    ids[n // 3: n // 2] = -1
    top_ids = torch.randint(0, classes, (n, k), generator=g)
    top_ids[::7, 2:] = -1
    top = torch.randn(n, k, generator=g) * 2
    x = torch.randn(n, dim, generator=g) if with_x else None
    before = [t.clone() for t in (st.table, st.w, st.head)]
    want, grads = step64(*before, ids, top_ids, top, x, st.scale, st.temperature, st.eps,
                         torch.tensor(1.0 / n, dtype=F32).double())
    loss = st.step(ids.to(DEV), n, top_ids.to(DEV), top.to(DEV),
                   None if x is None else x.to(DEV)).cpu().double()
    assert int(st.status) == 0
    assert float((loss - want).abs().max()) <= 100 * U * float(want.abs().max())
    tol = 100 + dim + classes + n
    for new, old, grad in zip((st.table, st.w, st.head), before, grads):
        moved = new.cpu().double() - (old.cpu().double() - st.rate * grad)
        # the step's own rounding, and the gradient's error
        bound = 2 * U * old.cpu().double().abs() + tol * U * st.rate * float(grad.abs().max())
        assert bool((moved.abs() <= bound).all())


def test_the_student_learns_a_windows_answers():
    """GraphSAGE answers a window's seeds; the student, given their rows and its
    own table, comes closer to the best eight classes with every few steps."""
    from paper_2606_02916_amd import SageConsumer, Student
    inst = synth.instance("tiny")
    w = World(inst)
    rng = np.random.default_rng(3)
    d, classes, k = inst.wl.row_bytes // 4, 47, 8
    layers = [(torch.from_numpy(rng.standard_normal((a, b)).astype(np.float32) / a ** 0.5).to(DEV),
               torch.from_numpy(rng.standard_normal((a, b)).astype(np.float32) / a ** 0.5).to(DEV),
               torch.zeros(b, device=DEV), r) for a, b, r in ((d, 32, True), (32, classes, False))]
    cons = SageConsumer(w.pipe.geo, layers, device=DEV)
    seeds, so, b0 = w.window_inputs(0)
    Wk = w.pipe.window(torch.from_numpy(seeds).to(DEV), so, b0, consumer=cons)
    n = int(w.pipe.frontier_off[Wk])               # the window's distinct seeds, batch by batch
    ids = w.pipe.frontier_ids[:n]
    top = torch.topk(cons.out[:n], k)
    feats = torch.from_numpy(np.concatenate(inst.shards)).to(DEV)
    row = (ids % inst.wl.num_parts).long() * inst.shards[0].shape[0] + ids.long() // inst.wl.num_parts
    x = feats[row][:, :4 * d].contiguous().view(F32).view(n, d)
    st = Student(inst.wl.num_nodes, d, classes, max_rows=cons.out_cap, k=k, rate=2.0, device=DEV,
                 generator=gen(4))
    losses = [float(st.step(ids, n, top.indices, top.values, x).sum()) for _ in range(30)]
    assert w.pipe.read_status() == 0 and int(st.status) == 0
    assert all(np.isfinite(losses))
    assert losses[-1] < 0.7 * losses[0] and losses[10] < losses[0] and losses[20] < losses[10]


def test_8bit_rows_through_the_fetch_path():
    """A student's rows as the shards of a fetch pipeline: every gathered row is
    its shard's, byte for byte, and reads back as code * scale."""
    from paper_2606_02916_amd import Student, student
    inst = synth.instance("tiny")
    wl = inst.wl
    dim, group = 70, 32
    st = Student(wl.num_nodes, dim, 5, max_rows=2500, device=DEV, generator=gen(5))
    rb = student.row_bytes_8bit(dim, group)
    assert rb == 72 + 12
    shards = []
    for m in range(wl.num_parts):                   # owner = node mod parts
        ids = torch.arange(m, wl.num_nodes, wl.num_parts, device=DEV)
        buf = torch.zeros(len(ids), rb, dtype=torch.uint8, device=DEV)
        for i in range(0, len(ids), 2000):
            part = ids[i:i + 2000]
            st.write_rows(buf[i:i + 2000], part, len(part), group)
        shards.append(buf)
    assert int(st.status) == 0
    w = World(inst, shards=[s.cpu().numpy() for s in shards], row_bytes=rb, stride=rb)
    r = w.run_and_compare(0)                        # gathered rows against the oracle's
    Wk, foff = r["Wk"], r["foff"]
    L = len(w.fanout)
    n = int(foff[(L + 1) * Wk] - foff[L * Wk])
    rows = w.pipe.win_out[:n]
    out = torch.full((n, dim), float("nan"), device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    student.read_rows(rows, n, dim, group, out, status)
    codes = rows[:, :dim].view(E4M3).float()
    sc = rows[:, 72:84].contiguous().view(F32)[:, torch.arange(dim, device=DEV) // group]
    assert torch.equal(out, codes * sc) and int(status) == 0
    # and the numbers are the table's normed rows to within a code's rounding
    ids = torch.from_numpy(r["fids"][int(foff[L * Wk]):int(foff[(L + 1) * Wk])].astype(np.int64))
    t = st.table.cpu().double()[ids]
    y = t / (t.square().mean(1, keepdim=True) + st.eps / st.scale ** 2) ** 0.5
    top = torch.cat([p.abs().amax(1, keepdim=True).expand(-1, p.shape[1]) for p in y.split(group, 1)], 1)
    off = (out.cpu().double() - y).abs()
    assert bool((off <= y.abs() * 2.0 ** -4 * 1.01 + top / 448 * 2.0 ** -10 * 1.01 +
                 100 * U * y.abs()).all())


def test_operators_in_a_replayed_graph():
    """The calls of a step, captured once and replayed on new inputs, with other
    work and synchronisations between the replays."""
    from paper_2606_02916_amd import gg
    n, N, d, V, k = 20_000, 3000, 64, 70, 4
    g = gen(6)
    table, w = torch.randn(N, d, generator=g, device=DEV), torch.rand(d, generator=g, device=DEV)
    ids = torch.empty(n, dtype=torch.int64, device=DEV)
    z, tl = torch.empty(n, V, device=DEV), torch.empty(n, k, device=DEV)
    ti = torch.empty(n, k, dtype=torch.int32, device=DEV)
    e, y, dx = (torch.empty(n, d, device=DEV) for _ in range(3))
    rstd, loss, lse = (torch.empty(n, device=DEV) for _ in range(3))
    dz, dw, grad = torch.empty(n, V, device=DEV), torch.empty(d, device=DEV), torch.empty(N, d, device=DEV)
    status = torch.zeros(1, dtype=torch.int32, device=DEV)
    ws = torch.empty(max(gg.gg_ws_embed(n, N, d), gg.gg_ws_rmsnorm(n, d), gg.gg_ws_distill(n, V)),
                     dtype=torch.uint8, device=DEV)
    m = gg.make_rows

    def calls():
        gg.gg_embed_forward(m(table), N, d, ids, n, 2.0, m(e), status)
        gg.gg_rmsnorm_forward(m(e), None, n, d, w, 1e-6, m(e), m(y), None, rstd)
        gg.gg_distill_forward(m(z), n, V, ti, m(tl), k, 2.0, 1.0, None, loss, lse, m(dz), status, ws)
        gg.gg_rmsnorm_backward(m(y), None, m(e), rstd, n, d, w, m(dx), dw, ws)
        gg.gg_embed_backward(m(dx), ids, n, N, d, 2.0, m(grad), 0, status, ws)

    def fill(seed):
        g = gen(seed)
        ids.copy_(torch.randint(-1, N, (n,), generator=g, device=DEV))
        z.copy_(torch.randn(n, V, generator=g, device=DEV))
        tl.copy_(torch.randn(n, k, generator=g, device=DEV))
        ti.copy_(torch.randint(-1, V, (n, k), generator=g, device=DEV))

    outs = (y, loss, lse, dz, dx, dw, grad)
    fill(0)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        calls()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for seed in range(1, 5):
        fill(seed)
        calls()
        want = [o.clone() for o in outs]
        for o in outs:
            o.fill_(float("nan"))
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(outs, want):
            assert torch.equal(a, b), seed
    assert int(status) == 0


@pytest.mark.parametrize("t", [F16, BF16])
def test_a_step_with_16_bit_activations_lands_whole(t):
    """The parameters move by what the step's own gradients ask for, to a rounding of
    fp32.  Those gradients, after some 64 roundings to 16 bits that a logit's products
    and the softmax add up at most, are the 64-bit step's."""
    from paper_2606_02916_amd import Student
    n, N, dim, classes, k = 1024, 2000, 100, 47, 8
    st = Student(N, dim, classes, max_rows=n, k=k, dtype=t, device=DEV, generator=gen(7))
    g = torch.Generator().manual_seed(8)
    ids = torch.randint(0, N, (n,), generator=g)
    ids[5:9] = -1
    top_ids = torch.stack([torch.randperm(classes, generator=g)[:k] for _ in range(n)])
    top = (torch.randn(n, k, generator=g) * 2 + 5).to(t)
    before = [p.clone() for p in (st.table, st.w, st.head)]
    want, grads = step64(*before, ids, top_ids, top, None, st.scale, st.temperature, st.eps, 1 / n)
    st.step(ids.to(DEV), n, top_ids.to(DEV), top.to(DEV))
    assert int(st.status) == 0
    moved = [p.cpu().double() - b.cpu().double() for p, b in zip((st.table, st.w, st.head), before)]
    # the buffer of the looked-up rows holds their gradient after a step
    de, keep = st.e[:n].cpu().double(), ids >= 0
    asked, size = torch.zeros(2, N, dim, dtype=torch.float64)
    asked.index_add_(0, ids[keep], de[keep])
    size.index_add_(0, ids[keep], de[keep].abs())
    bound = 2 * U * before[0].cpu().double().abs() + 40 * U * st.rate * st.scale * size
    assert bool(((moved[0] + st.rate * st.scale * asked).abs() <= bound).all())
    bound = 2 * U * (before[2].cpu().double().abs() + st.rate * st.dhead.cpu().double().abs())
    assert bool(((moved[2] + st.rate * st.dhead.cpu().double()).abs() <= bound).all())
    for m, grad in zip(moved, grads):
        assert float((m + st.rate * grad).norm()) <= 64 * UNIT[t] * st.rate * float(grad.norm())
    assert float((st.loss[:n].cpu().double() - want).norm()) <= 64 * UNIT[t] * float(want.norm())
