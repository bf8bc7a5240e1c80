"""Students with a layer norm and with 8-bit rows: no rows, rows that are all skipped, and a step
that is captured and replayed."""
import pytest
import torch

from tests.op_util import BF16, F32

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
KINDS = [(norm, eight, t) for norm in ("rms", "layer") for eight in (False, True) for t in (F32, BF16)]


def student(norm, eight, t, rows=300, seed=3):
    from paper_2606_02916_amd import Student
    return Student(500, 100, 47, max_rows=rows, k=4, rate=0.5, dtype=t, device=DEV, norm=norm, eight_bit=eight,
                   eps=1e-3, generator=torch.Generator(device=DEV).manual_seed(seed))


def params(s):
    return [p.clone() for p in (s.table, s.w, s.head, s.b) if p is not None]


def lesson(n, seed):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return (torch.randint(-1, 500, (n,), generator=g, device=DEV),
            torch.randint(0, 47, (n, 4), generator=g, device=DEV), torch.randn(n, 4, generator=g, device=DEV),
            torch.randn(n, 100, generator=g, device=DEV))


@pytest.mark.parametrize("norm,eight,t", KINDS)
def test_a_step_of_no_rows_changes_nothing(norm, eight, t):
    s = student(norm, eight, t)
    before = params(s)
    ids, top_ids, top, x = lesson(0, 1)
    assert s.step(ids, 0, top_ids, top, x.to(t)).numel() == 0
    assert int(s.status) == 0
    assert all(torch.equal(a, b) for a, b in zip(before, params(s)))


@pytest.mark.parametrize("norm,eight,t", KINDS)
def test_rows_without_a_lesson_leave_no_gradient(norm, eight, t):
    """Rows whose weights are zero, and ids that the table skips: the table stays."""
    s = student(norm, eight, t)
    ids, top_ids, top, x = lesson(200, 2)
    table, head = s.table.clone(), s.head.clone()
    loss = s.step(ids, 200, top_ids, top, x.to(t), torch.zeros(200, device=DEV))
    assert not loss.any() and torch.equal(s.table, table) and torch.equal(s.head, head)
    s.step(torch.full_like(ids, -1), 200, top_ids, top, x.to(t))
    assert torch.equal(s.table, table) and bool(torch.isfinite(s.head).all())
    assert not torch.equal(s.head, head) and int(s.status) == 0


@pytest.mark.parametrize("norm,eight,t", [k for k in KINDS if k[1]])
def test_a_captured_step_is_the_eager_one(norm, eight, t):
    """Five replays on new lessons, with eager work and synchronisations between them."""
    n = 257
    a, b = student(norm, eight, t), student(norm, eight, t)
    ids, top_ids, top, x = lesson(n, 10)
    x = x.to(t)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        b.step(ids, n, top_ids, top, x)
    torch.cuda.current_stream().wait_stream(side)
    a.step(ids, n, top_ids, top, x)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step(ids, n, top_ids, top, x)
    for seed in range(11, 16):
        for to, new in zip((ids, top_ids, top, x), lesson(n, seed)):
            to.copy_(new)
        want = a.step(ids, n, top_ids, top, x).clone()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(b.loss[:n], want)
        for p, q in zip(params(a), params(b)):
            assert torch.equal(p, q), seed
