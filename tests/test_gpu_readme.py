"""The README's example of driving the look-ahead pipeline, executed as
written on the large_sparse workload: in every window, every gathered row of
the first and the last batch must equal its node's row of the feature
matrix."""
import os
import textwrap

import numpy as np
import pytest

import synth
from tests import helpers

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def _example():
    """The README's code block, from its imports to its status check, with
    a call to _check after the line that takes the window's rows."""
    text = open(os.path.join(helpers.ROOT, "README.md")).read()
    start = text.index("    import torch\n    from paper_2606_02916_amd import LookaheadPipeline")
    end = text.index("\n", text.index("look.read_status() == 0", start))
    lines = textwrap.dedent(text[start:end]).split("\n")
    at = next(i for i, ln in enumerate(lines) if ln.lstrip().startswith("x = bufs.win_out"))
    indent = lines[at][:len(lines[at]) - len(lines[at].lstrip())]
    lines.insert(at + 1, indent + "_check(k, Wk, bufs, off, x)")
    return "\n".join(lines)


def test_readme_example_runs_as_written():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print("large_sparse: the README's look-ahead example", flush=True)
    dev = torch.device("cuda:0")
    inst, row_ptr, col_idx, shards = synth.torch_instance("large_sparse", dev)
    wl = inst.wl
    assert (wl.num_parts, wl.local_owner, wl.row_bytes, wl.row_stride, wl.W, wl.batch_size) == \
        (4, 0, 400, 400, 16, 1024) and list(wl.fanout) == [15, 10, 5]
    seeds_d = torch.from_numpy(inst.seeds).to(dev)
    boff = inst.batch_off
    windows = []
    for k in range(synth.n_windows(boff, wl.W)):
        b0, b1 = synth.window_batches(boff, wl.W, k)
        windows.append((seeds_d[boff[b0]:boff[b1]], boff[b0:b1 + 1] - boff[b0], b0))
    feats = np.concatenate(inst.shards)          # the range book's owners in id order
    seen = []

    def _check(k, Wk, bufs, off, x):
        fid = bufs.frontier_ids.cpu().numpy()
        for b in (0, Wk - 1):
            lo, hi = int(off[b] - off[0]), int(off[b + 1] - off[0])
            ids = fid[int(off[b]):int(off[b + 1])]
            assert hi > lo
            assert np.array_equal(x[lo:hi, :wl.row_bytes].cpu().numpy(),
                                  feats[ids, :wl.row_bytes]), (k, b)
        seen.append(k)

    ns = {"row_ptr": row_ptr, "col_idx": col_idx, "range_start": inst.range_start,
          "shards": shards, "windows": windows, "_check": _check}
    exec(compile(_example(), "README.md", "exec"), ns)
    assert seen == list(range(len(windows)))


def _student_example():
    text = open(os.path.join(helpers.ROOT, "README.md")).read()
    start = text.index("    from paper_2606_02916_amd import Student\n")
    end = text.index("\n", text.index("    read_rows(", start))
    return textwrap.dedent(text[start:end])


def test_the_students_example_runs_as_written():
    if not torch.cuda.is_available():
        pytest.skip("no GPU")
    print("the README's example of teaching a student", flush=True)
    dev = torch.device("cuda:0")
    g = torch.Generator(device=dev).manual_seed(1)
    num_nodes, n, m = 5000, 900, 700
    seeds = torch.randint(0, num_nodes, (800,), generator=g, device=dev)
    logits = torch.randn(900, 47, generator=g, device=dev)      # a consumer's buffer, seeds first
    nodes = torch.randint(0, num_nodes, (n,), generator=g, device=dev, dtype=torch.int32)
    out = torch.empty(m, 100, device=dev)
    ns = {"torch": torch, "num_nodes": num_nodes, "seeds": seeds, "logits": logits, "nodes": nodes,
          "n": n, "m": m, "out": out}
    lines = _student_example().split("\n")
    at = next(i for i, ln in enumerate(lines) if ln.startswith("read_rows("))
    lines.insert(at, "gathered = rows[:m]")
    exec(compile("\n".join(lines), "README.md", "exec"), ns)
    s, rows = ns["s"], ns["rows"]
    assert int(s.status) == 0
    assert ns["loss"].shape == (800,) and bool(torch.isfinite(ns["loss"]).all())
    assert ns["z"].shape == (n, 47)
    # the 8-bit rows are the nodes' normed rows to within a code's rounding
    t = s.table[nodes[:m].long()].double()
    y = t / (t.square().mean(1, keepdim=True) + s.eps / s.scale ** 2) ** 0.5 * s.w.double()
    off = (out.double() - y).abs()
    top = y.abs().amax(1, keepdim=True)
    assert bool((off <= y.abs() * 2.0 ** -4 * 1.01 + top / 448 * 2.0 ** -10 * 1.01 +
                 1e-5 * y.abs()).all())
