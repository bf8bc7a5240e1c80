"""Host-side argument checks of the calls for layers in 8 bits: a bad call is refused
with a message before anything is enqueued, so no GPU is needed.  Addresses here are
numbers that nothing reads."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2606_02916_amd import gg
from tests.test_operator_args import P, ROOT, refused, rows


def blocks(data=P, stride=400, scales=P, scales_stride=64):
    b = gg.gg_blocks_t()
    b.data, b.stride, b.scales, b.scales_stride = data, stride, scales, scales_stride
    return b


def test_blocks_layout_matches_the_header():
    src = r"""
#include <stddef.h>
#include <stdio.h>
#include "gg.h"
int main() {
  printf("%zu %zu %zu %zu %zu %d\n", sizeof(gg_blocks_t), offsetof(gg_blocks_t, data),
         offsetof(gg_blocks_t, stride), offsetof(gg_blocks_t, scales),
         offsetof(gg_blocks_t, scales_stride), GG_SCALE_BLOCK);
}
"""
    d = tempfile.mkdtemp(prefix="ggblocks_")
    with open(os.path.join(d, "p.cpp"), "w") as f:
        f.write(src)
    subprocess.run(["g++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), os.path.join(d, "p.cpp"), "-o",
                    os.path.join(d, "p")], check=True)
    got = [int(x) for x in subprocess.run([os.path.join(d, "p")], capture_output=True,
                                          text=True).stdout.split()]
    B = gg.gg_blocks_t
    assert got == [C.sizeof(B), B.data.offset, B.stride.offset, B.scales.offset,
                   B.scales_stride.offset, gg.GG_SCALE_BLOCK]


NORM = dict(x=rows(), res=None, n=7, dim=100, w=P, b=P, w_dtype=gg.GG_F32, eps=1e-6, sum=None,
            y=rows(), q=None, kept=None, mean=P, rstd=P, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(dim=0), "dim"), (dict(dim=16385), "dim"), (dict(n=-1), "n = -1"), (dict(n=1 << 28), "n = "),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"),
    (dict(y=None, rstd=None, mean=None), "output"), (dict(x=None), "x: "),
    (dict(x=rows(gg.GG_E4M3)), "x: dtype"), (dict(w_dtype=gg.GG_F16), "weights"),
    (dict(w=None, w_dtype=gg.GG_F16), "weights"), (dict(w=P + 2), "weights"), (dict(b=P + 2), "bias"),
    (dict(rstd=P + 2), "rstd"), (dict(mean=P + 2), "mean"), (dict(y=rows(gg.GG_BF16)), "y: dtype"),
    (dict(y=rows(stride=200)), "y: stride"), (dict(res=rows(gg.GG_F16)), "res: dtype"),
    (dict(q=rows()), "q: dtype"), (dict(kept=rows()), "kept: dtype"),
    (dict(kept=rows(gg.GG_E4M3, group=512)), "kept: group"),
    (dict(kept=rows(gg.GG_E4M3, group=16, scales_stride=24)), "kept: scales"),
    (dict(kept=rows(gg.GG_E4M3, stride=99)), "kept: stride"),
    (dict(x=rows(gg.GG_BF16), y=rows(gg.GG_BF16), res=rows(gg.GG_BF16), sum=rows()), "differ")])
def test_norm_refuses(change, word):
    refused(gg.lib.gg_layernorm_forward, NORM, change, word)


NORM_BACK = dict(dy=rows(), dsum=None, s=rows(), mean=P, rstd=P, n=7, dim=100, w=P, w_dtype=gg.GG_F32,
                 dx=rows(), dw=P, db=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(dim=0), "dim"), (dict(n=-1), "n = -1"), (dict(dy=None), "dy"), (dict(s=None), "s: "),
    (dict(s=rows(gg.GG_F16)), "s: dtype"), (dict(dx=rows(gg.GG_F16)), "dx: dtype"),
    (dict(s=rows(gg.GG_E4M3), dx=rows(gg.GG_F16)), "dx: dtype"),
    (dict(s=rows(gg.GG_E4M3), dx=rows(gg.GG_E4M3)), "dx: dtype"),
    (dict(s=rows(gg.GG_E4M3, group=8)), "s: group"), (dict(s=rows(gg.GG_E4M3, scales=None)), "s: "),
    (dict(dsum=rows(gg.GG_BF16)), "dsum: dtype"), (dict(rstd=None), "rstd"), (dict(mean=None), "mean"),
    (dict(mean=P + 1), "mean"), (dict(dw=P + 1), "dw"), (dict(db=P + 1), "db"),
    (dict(w_dtype=gg.GG_BF16), "weights"), (dict(w=P + 1), "weights"), (dict(ws=None), "workspace"),
    (dict(ws=P + 8), "workspace"), (dict(ws_bytes=16), "workspace"),
    (dict(dw=None, ws=None), "workspace"),
    (dict(ws_bytes=gg.gg_ws_rmsnorm(7, 100)), "workspace"), (dict(dx=rows(stride=4)), "dx: stride")])
def test_norm_gradient_refuses(change, word):
    refused(gg.lib.gg_layernorm_backward, NORM_BACK, change, word)


Q8 = rows(gg.GG_E4M3, group=16)
ROWS = dict(x=rows(), n=7, dim=100, q=Q8, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(dim=0), "dim"), (dict(dim=(1 << 24) + 1), "dim"), (dict(n=-1), "n = -1"),
    (dict(n=1 << 28), "n = "), (dict(x=None), "x: "), (dict(q=None), "q: "),
    (dict(x=rows(gg.GG_E4M3)), "x: dtype"), (dict(q=rows()), "q: dtype"),
    (dict(x=rows(data=P + 2)), "x: not aligned"), (dict(q=rows(gg.GG_E4M3, stride=99)), "q: stride"),
    (dict(q=rows(gg.GG_E4M3, group=24)), "q: group"), (dict(q=rows(gg.GG_E4M3, scales=None)), "q: "),
    (dict(q=rows(gg.GG_E4M3, group=16, scales_stride=24)), "q: scales")])
def test_rows_refuse(change, word):
    refused(gg.lib.gg_quantise_rows, ROWS, change, word)


BLOCKS = dict(w=rows(stride=1200), rows=200, cols=300, q=blocks(), qt=blocks(), stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(rows=0), "rows 0"), (dict(cols=0), "cols 0"), (dict(rows=(1 << 24) + 1), "rows"),
    (dict(cols=(1 << 24) + 1), "cols"), (dict(q=None, qt=None), "output"), (dict(w=None), "w: "),
    (dict(w=rows(gg.GG_E4M3)), "w: dtype"), (dict(q=blocks(data=None)), "q: data"),
    (dict(q=blocks(scales=None)), "q: data or scales"), (dict(q=blocks(stride=299)), "q: stride"),
    (dict(qt=blocks(stride=199)), "qt: stride"), (dict(q=blocks(scales=P + 2)), "q: scales"),
    (dict(q=blocks(scales_stride=8)), "q: scales"), (dict(qt=blocks(scales_stride=4)), "qt: scales"),
    (dict(q=blocks(scales_stride=14)), "q: scales"), (dict(q=blocks(stride=-400)), "q: stride")])
def test_blocks_refuse(change, word):
    refused(gg.lib.gg_quantise_blocks, BLOCKS, change, word)


PRODUCT = dict(a=rows(gg.GG_E4M3, group=128), n=7, k=300, b=blocks(), m=200, out=rows(stride=800),
               stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(n=-1), "n = -1"), (dict(n=1 << 28), "n = "), (dict(k=0), "k 0"), (dict(m=0), "m 0"),
    (dict(k=(1 << 24) + 1), "k "), (dict(m=(1 << 24) + 1), "m "), (dict(a=None), "a: "),
    (dict(a=rows()), "a: dtype"), (dict(a=rows(gg.GG_E4M3, group=64)), "a: group 64"),
    (dict(a=rows(gg.GG_E4M3, group=256)), "a: group 256"),
    (dict(a=rows(gg.GG_E4M3, scales=None)), "a: "), (dict(a=rows(gg.GG_E4M3, stride=-304)), "a: stride"),
    (dict(b=None), "b: "), (dict(b=blocks(data=None)), "b: data"), (dict(b=blocks(stride=-1)), "b: stride"),
    (dict(b=blocks(scales_stride=-64)), "b: scales"), (dict(b=blocks(scales_stride=30)), "b: scales"),
    (dict(b=blocks(scales=P + 1)), "b: scales"), (dict(out=None), "out"),
    (dict(out=rows(gg.GG_E4M3)), "out: dtype"), (dict(out=rows(stride=796)), "out: stride"),
    (dict(out=rows(data=P + 2)), "out: not aligned"),
    (dict(n=1 << 27, m=1 << 24, out=rows(stride=1 << 26)), "too many")])
def test_product_refuses(change, word):
    refused(gg.lib.gg_product_forward, PRODUCT, change, word)


PRODUCT_BACK = dict(a=rows(gg.GG_E4M3, group=128), n=700, k=300, dz=rows(stride=800), m=200,
                    dw=rows(stride=1200), flags=0, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(n=-1), "n = -1"), (dict(n=1 << 28), "n = "), (dict(k=0), "k 0"), (dict(m=0), "m 0"),
    (dict(k=(1 << 24) + 1), "k "), (dict(m=(1 << 24) + 1), "m "), (dict(a=None), "a: "),
    (dict(a=rows()), "a: dtype"), (dict(a=rows(gg.GG_E4M3, group=64)), "a: group 64"),
    (dict(a=rows(gg.GG_E4M3, scales=None)), "a: "), (dict(dz=None), "dz: "),
    (dict(dz=rows(gg.GG_E4M3)), "dz: dtype"), (dict(dz=rows(data=P + 2)), "dz: not aligned"),
    (dict(dw=None), "dw: "), (dict(dw=rows(gg.GG_BF16, stride=600)), "dw: dtype"),
    (dict(dw=rows(stride=1196)), "dw: stride"),
    (dict(dz=rows(gg.GG_F16), dw=rows(gg.GG_BF16, stride=600)), "dw: dtype"), (dict(flags=2), "flags"),
    (dict(flags=-1), "flags"), (dict(ws=None), "workspace"), (dict(ws=P + 8), "workspace"),
    (dict(ws_bytes=gg.gg_ws_product(700, 300, 200) - 1), "workspace"),
    (dict(k=1 << 24, m=1 << 24, dw=rows(stride=1 << 26)), "too many")])
def test_weight_gradient_refuses(change, word):
    refused(gg.lib.gg_product_backward, PRODUCT_BACK, change, word)


def test_make_blocks_refuses_what_it_cannot_describe():
    q, sc = torch.zeros(130, 300, dtype=torch.float8_e4m3fn), torch.zeros(2, 3)
    b = gg.make_blocks(q[:, 4:260], torch.zeros(2, 9)[:, 3:5])
    assert (b.stride, b.scales_stride, b.rows, b.cols) == (300, 36, 130, 256)
    for bad in (lambda: gg.make_blocks(q.view(torch.uint8), sc), lambda: gg.make_blocks(q[0], sc),
                lambda: gg.make_blocks(q[:, ::2], sc), lambda: gg.make_blocks(q.t(), sc.t()),
                lambda: gg.make_blocks(q, sc.double()), lambda: gg.make_blocks(q, torch.zeros(3, 2).t()),
                lambda: gg.make_blocks(q, torch.zeros(2, 2)), lambda: gg.make_blocks(q, torch.zeros(130, 3))):
        with pytest.raises(gg.GGError):
            bad()


def test_workspaces():
    assert gg.gg_ws_layernorm(-1, 9) == gg.gg_ws_layernorm(9, 0) == gg.gg_ws_layernorm(9, 16_385) == 0
    got = [gg.gg_ws_layernorm(n, 100) for n in (0, 1, 7, 700, 1023, 1024, 5000, 1 << 27)]
    assert got == sorted(got) and got[-1] == 2 * 1024 * 400
    assert gg.gg_ws_product(-1, 9, 9) == gg.gg_ws_product(9, 0, 9) == gg.gg_ws_product(9, 9, 0) == 0
    for k, m in ((1, 1), (100, 47), (602, 41), (4096, 4096), (9, 1 << 24)):
        got = [gg.gg_ws_product(n, k, m) for n in (0, 1, 64, 65, 256, 257, 512, 513, 5000, 100_000, 1 << 27)]
        # (rows are split 64 at least to a part)
        assert got == sorted(got) and got[2] == 0 and all(x % (4 * k * m) < 256 for x in got)


def test_bindings_check_shapes():
    """No description of fewer rows or narrower ones than the call goes over, of other
    weights, or of another kind: refused before the stream is asked for."""
    r = lambda *shape: gg.make_rows(torch.zeros(*shape))  # noqa: E731
    r8 = lambda n, d: gg.make_rows(torch.zeros(n, d, dtype=torch.float8_e4m3fn),  # noqa: E731
                                   scales=torch.zeros(n))
    b = lambda n, d: gg.make_blocks(torch.zeros(n, d, dtype=torch.float8_e4m3fn),  # noqa: E731
                                    torch.zeros(-(-n // 128), -(-d // 128)))
    good, vec, w = r(7, 20), torch.zeros(7), torch.zeros(20)
    for name in ("short", "narrow"):
        bad, bad8 = (r(6, 20), r8(6, 20)) if name == "short" else (r(7, 19), r8(7, 19))
        for call in (
                lambda: gg.gg_layernorm_forward(bad, good, 7, 20, None, None, 1e-6, good, good, None,
                                                None, None, None),
                lambda: gg.gg_layernorm_forward(good, bad, 7, 20, None, None, 1e-6, good, good, None,
                                                None, None, None),
                lambda: gg.gg_layernorm_forward(good, good, 7, 20, None, None, 1e-6, bad, good, None,
                                                None, None, None),
                lambda: gg.gg_layernorm_forward(good, good, 7, 20, None, None, 1e-6, good, bad, None,
                                                None, None, None),
                lambda: gg.gg_layernorm_forward(good, good, 7, 20, None, None, 1e-6, good, good, bad8,
                                                None, None, None),
                lambda: gg.gg_layernorm_forward(good, good, 7, 20, None, None, 1e-6, good, good, None,
                                                bad8, None, None),
                lambda: gg.gg_layernorm_backward(bad, None, good, vec, vec, 7, 20, None, good, None, None,
                                                 None),
                lambda: gg.gg_layernorm_backward(good, bad, good, vec, vec, 7, 20, None, good, None, None,
                                                 None),
                lambda: gg.gg_layernorm_backward(good, None, bad8, vec, vec, 7, 20, None, good, None,
                                                 None, None),
                lambda: gg.gg_layernorm_backward(good, None, good, vec, vec, 7, 20, None, bad, None, None,
                                                 None),
                lambda: gg.gg_quantise_rows(bad, 7, 20, r8(7, 20)),
                lambda: gg.gg_quantise_rows(good, 7, 20, bad8),
                lambda: gg.gg_quantise_blocks(bad, 7, 20, b(7, 20), None),
                lambda: gg.gg_product_forward(bad8, 7, 20, b(20, 20), 20, good),
                lambda: gg.gg_product_forward(r8(7, 20), 7, 20, b(20, 20), 20, bad),
                lambda: gg.gg_product_backward(bad8, 7, 20, good, 20, r(20, 20), 0, None),
                lambda: gg.gg_product_backward(r8(7, 20), 7, 20, bad, 20, r(20, 20), 0, None),
                lambda: gg.gg_product_backward(r8(7, 20), 7, 20, r(7, 7), 7, bad, 0, None)):
            with pytest.raises(gg.GGError, match="rows of"):
                call()
    for call, word in (
            (lambda: gg.gg_layernorm_forward(good, None, 7, 20, w, w.half(), 1e-6, good, None, None, None,
                                             None, None), "biases of"),
            (lambda: gg.gg_layernorm_forward(good, None, 7, 20, w[:19], None, 1e-6, good, None, None,
                                             None, None, None), "weights must"),
            (lambda: gg.gg_layernorm_forward(good, None, 7, 20, None, w[:19], 1e-6, good, None, None,
                                             None, None, None), "weights must"),
            (lambda: gg.gg_layernorm_forward(good, None, 7, 20, None, None, 1e-6, good, None, None, None,
                                             vec[:6], None), "mean"),
            (lambda: gg.gg_layernorm_backward(good, None, good, vec[:6], vec, 7, 20, None, good, None,
                                              None, None), "mean"),
            (lambda: gg.gg_layernorm_backward(good, None, good, vec, vec, 7, 20, None, good, None, vec,
                                              None), "db"),
            (lambda: gg.gg_quantise_blocks(good, 7, 20, b(7, 21), None), "q: weights of"),
            (lambda: gg.gg_quantise_blocks(good, 7, 20, None, b(7, 20)), "qt: weights of"),
            (lambda: gg.gg_quantise_blocks(good, 7, 20, r8(7, 20), None), "make_blocks"),
            (lambda: gg.gg_product_forward(r8(7, 20), 7, 20, b(20, 21), 20, good), "b: weights of"),
            (lambda: gg.gg_product_forward(r8(7, 20), 7, 20, r8(20, 20), 20, good), "make_blocks"),
            (lambda: gg.gg_product_forward(b(7, 20), 7, 20, b(20, 20), 20, good), "make_rows"),
            (lambda: gg.gg_quantise_rows(good, 7, 20, b(7, 20)), "make_rows")):
        with pytest.raises(gg.GGError, match=word):
            call()


def test_the_student_checks_its_norm_and_tensors():
    from paper_2606_02916_amd import Student
    with pytest.raises(gg.GGError, match="neither"):
        Student(50, 20, 9, max_rows=7, device="cpu", norm="batch")
    s = Student(50, 20, 9, max_rows=7, k=3, device="cpu", norm="layer", eight_bit=True)
    ids, top = torch.zeros(8, dtype=torch.int64), torch.zeros(7, 3)
    for call, word in ((lambda: s.forward(ids, 8), "student of 7"),
                       (lambda: s.forward(ids, 7, torch.zeros(7, 19)), "x of shape"),
                       (lambda: s.step(ids, 7, top[:, :2].long(), top), "top_ids of shape"),
                       (lambda: s.step(ids, 8, torch.zeros(8, 3).long(), torch.zeros(8, 3)), "student of 7")):
        with pytest.raises(gg.GGError, match=word):
            call()


@pytest.mark.parametrize("norm", ["rms", "layer"])
@pytest.mark.parametrize("eight_bit", [False, True])
def test_a_step_stores_the_sums_that_its_way_back_reads(norm, eight_bit, monkeypatch):
    """The forward norm's outputs are what the norm's gradient (or the call that puts sums into 8
    bits) reads, no sums are stored beside them."""
    from paper_2606_02916_amd import Student, student
    s = Student(50, 20, 9, max_rows=7, k=3, device="cpu", norm=norm, eight_bit=eight_bit)
    seen = []
    for name in [x for x in dir(gg) if x.startswith("gg_") and not x.startswith("gg_ws")]:
        if callable(getattr(gg, name)) and not isinstance(getattr(gg, name), type):
            monkeypatch.setattr(student.gg, name, lambda *a, call=name, **k: seen.append((call, a)))
    s.step(torch.zeros(7, dtype=torch.int64), 7, torch.zeros(7, 3).long(), torch.zeros(7, 3))
    calls = dict(reversed(seen))
    if norm == "layer":
        forward, back = calls["gg_layernorm_forward"], calls["gg_layernorm_backward"]
        stored, kept = forward[7], forward[10]
    else:
        forward, back = calls["gg_rmsnorm_forward"], calls["gg_rmsnorm_backward"]
        stored, kept = forward[6], None
        if eight_bit:
            read, kept = [(a[0], a[3]) for c, a in seen if c == "gg_quantise_rows"][0]
            assert read is stored
    assert back[2] is (kept if eight_bit else stored)
    assert (stored is None) == (norm == "layer" and eight_bit)
