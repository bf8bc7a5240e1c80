"""Host-side argument checks of the operator calls: a bad call is refused with
a message before anything is enqueued, so no GPU is needed.  Addresses here
are numbers that nothing reads."""
import ctypes as C
import os
import subprocess
import tempfile

import pytest
import torch

from paper_2606_02916_amd import gg

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
P = 1 << 20


def rows(dtype=gg.GG_F32, data=P, stride=400, group=0, scales=P, scales_stride=64):
    r = gg.gg_rows_t()
    r.data, r.stride, r.dtype, r.group, r.scales, r.scales_stride = (data, stride, dtype, group,
                                                                     scales, scales_stride)
    return r


def refused(call, args, change, word):
    args = {**args, **change}
    ref = [C.byref(v) if isinstance(v, C.Structure) else v for v in args.values()]
    assert call(*ref) == gg.GG_ERR_ARG, change
    assert word in gg.gg_last_error(), (change, gg.gg_last_error())


def test_rows_layout_matches_the_header():
    src = r"""
#include <stddef.h>
#include <stdio.h>
#include "gg.h"
int main() {
  printf("%zu %zu %zu %zu %zu %zu %zu\n", sizeof(gg_rows_t), offsetof(gg_rows_t, stride),
         offsetof(gg_rows_t, dtype), offsetof(gg_rows_t, group), offsetof(gg_rows_t, scales),
         offsetof(gg_rows_t, scales_stride), offsetof(gg_rows_t, data));
  printf("%d %d %d %d %d\n", GG_F32, GG_F16, GG_BF16, GG_E4M3, GG_EMBED_ADD);
}
"""
    d = tempfile.mkdtemp(prefix="ggrows_")
    with open(os.path.join(d, "p.cpp"), "w") as f:
        f.write(src)
    subprocess.run(["g++", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                    "-I" + os.path.join(ROOT, "include"), os.path.join(d, "p.cpp"), "-o",
                    os.path.join(d, "p")], check=True)
    a, b = subprocess.run([os.path.join(d, "p")], capture_output=True,
                          text=True).stdout.split("\n")[:2]
    R = gg.gg_rows_t
    assert [int(x) for x in a.split()] == [C.sizeof(R), R.stride.offset, R.dtype.offset,
                                           R.group.offset, R.scales.offset, R.scales_stride.offset,
                                           R.data.offset]
    assert [int(x) for x in b.split()] == [gg.GG_F32, gg.GG_F16, gg.GG_BF16, gg.GG_E4M3,
                                           gg.GG_EMBED_ADD]


def test_make_rows_refuses_what_it_cannot_describe():
    x = torch.zeros(6, 40)
    assert gg.make_rows(x[:, 3:9]).stride == 160
    assert gg.make_rows(x[:1].expand(9, 40)).stride == 0
    q = torch.zeros(6, 40, dtype=torch.float8_e4m3fn)
    assert gg.make_rows(q, scales=torch.zeros(6, 3), group=16).group == 16
    assert gg.make_rows(q, scales=torch.zeros(6)).scales_stride == 4
    for bad in (lambda: gg.make_rows(x.t()), lambda: gg.make_rows(x[0]),
                lambda: gg.make_rows(x.double()), lambda: gg.make_rows(x[:, ::2]),
                lambda: gg.make_rows(q), lambda: gg.make_rows(q, scales=torch.zeros(6, 2), group=16),
                lambda: gg.make_rows(q, scales=torch.zeros(6).double()),
                lambda: gg.make_rows(q, scales=torch.zeros(3, 6).t(), group=16),
                lambda: gg.make_rows(x, scales=torch.zeros(6))):
        with pytest.raises(gg.GGError):
            bad()


LOOKUP = dict(table=rows(), num_rows=50, dim=100, ids=P, bits=64, n=7, scale=1.0, out=rows(),
              status=P, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(status=None), "status"), (dict(dim=0), "dim"), (dict(dim=32769), "dim"),
    (dict(n=-1), "n -1"), (dict(num_rows=-1), "num_rows"), (dict(bits=16), "16 bits"),
    (dict(ids=P + 4), "aligned"), (dict(table=None), "table"), (dict(out=None), "out"),
    (dict(table=rows(data=None)), "table: data"), (dict(table=rows(data=P + 2)), "table: not aligned"),
    (dict(out=rows(stride=396)), "out: stride"), (dict(out=rows(gg.GG_E4M3)), "out: dtype"),
    (dict(table=rows(7)), "table: dtype"), (dict(table=rows(stride=-400)), "table: stride"),
    (dict(table=rows(gg.GG_E4M3, group=8)), "group"), (dict(table=rows(gg.GG_E4M3, group=48)), "group"),
    (dict(table=rows(gg.GG_E4M3, scales=None)), "scales"),
    (dict(table=rows(gg.GG_E4M3, scales=P + 2)), "scales"), (dict(n=1 << 33), "too many")])
def test_lookup_refuses(change, word):
    refused(gg.lib.gg_embed_forward, LOOKUP, change, word)


GRAD = dict(dy=rows(), ids=P, bits=64, n=7, num_rows=50, dim=100, scale=1.0, grad=rows(), flags=0,
            status=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(status=None), "status"), (dict(dim=0), "dim"), (dict(n=-1), "n = -1"),
    (dict(n=(1 << 31) - 1), "n = "), (dict(num_rows=(1 << 31) - 1), "num_rows"),
    (dict(bits=8), "8 bits"), (dict(ids=None), "ids are NULL"), (dict(ids=P + 2), "aligned"),
    (dict(flags=2), "flags"), (dict(dy=None), "dy"), (dict(dy=rows(gg.GG_E4M3)), "dy: dtype"),
    (dict(grad=rows(stride=0)), "grad: stride"), (dict(grad=rows(data=P + 1)), "grad: not aligned"),
    (dict(ws=None), "workspace"), (dict(ws_bytes=64), "workspace")])
def test_gradient_refuses(change, word):
    refused(gg.lib.gg_embed_backward, GRAD, change, word)


def test_workspace_sizes():
    assert gg.gg_ws_embed(0, 10, 4) == 0 or gg.gg_ws_embed(0, 10, 4) % 256 == 0
    assert gg.gg_ws_embed(1000, 10, 4) >= 4 * 4 * 1000
    assert gg.gg_ws_embed(-1, 10, 4) == gg.gg_ws_embed(1 << 31, 10, 4) == gg.gg_ws_embed(9, 9, 0) == 0


def test_workspaces_serve_smaller_calls():
    sizes = [1, 2, 15, 16, 17, 63, 64, 65, 1000, 1023, 1024, 1025, 2048, 2049, 16_384, 16_385, 65_536,
             65_537, 131_072, 131_073, 524_288, 524_289, 1_048_576, 1_048_577, 1_500_000, 5_000_000]
    for f in (lambda n: gg.gg_ws_embed(n, 1000, 100), lambda n: gg.gg_ws_rmsnorm(n, 100),
              lambda n: gg.gg_ws_distill(n, 50_000)):
        got = [f(n) for n in sizes]
        assert got == sorted(got) and got[0] > 0


def test_bindings_check_the_ids():
    with pytest.raises(gg.GGError, match="ids"):
        gg._ids(torch.zeros(3), 3, "x")
    with pytest.raises(gg.GGError, match="ids"):
        gg._ids(torch.zeros(3, dtype=torch.int32), 4, "x")
    with pytest.raises(gg.GGError, match="ids"):
        gg._ids(torch.zeros(8, dtype=torch.int64)[::2], 4, "x")


NORM = dict(x=rows(), res=None, n=7, dim=100, w=P, w_dtype=gg.GG_F32, eps=1e-6, sum=None, y=rows(),
            q=None, rstd=P, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(dim=0), "dim"), (dict(dim=16385), "dim"), (dict(n=-1), "n = -1"), (dict(n=1 << 28), "n = "),
    (dict(eps=-1.0), "eps"), (dict(eps=float("nan")), "eps"), (dict(y=None, rstd=None), "output"),
    (dict(x=None), "x: "), (dict(x=rows(gg.GG_E4M3)), "x: dtype"), (dict(w_dtype=gg.GG_F16), "weights"),
    (dict(w=P + 2), "weights"), (dict(rstd=P + 2), "rstd"), (dict(y=rows(gg.GG_BF16)), "y: dtype"),
    (dict(y=rows(stride=200)), "y: stride"), (dict(res=rows(gg.GG_F16)), "res: dtype"),
    (dict(q=rows()), "q: dtype"), (dict(q=rows(gg.GG_E4M3, group=512)), "q: group"),
    (dict(q=rows(gg.GG_E4M3, group=16, scales_stride=24)), "q: scales"),
    (dict(q=rows(gg.GG_E4M3, stride=99)), "q: stride"),
    (dict(x=rows(gg.GG_BF16), y=rows(gg.GG_BF16), res=rows(gg.GG_BF16), sum=rows()), "differ")])
def test_norm_refuses(change, word):
    refused(gg.lib.gg_rmsnorm_forward, NORM, change, word)


NORM_BACK = dict(dy=rows(), dsum=None, s=rows(), rstd=P, n=7, dim=100, w=P, w_dtype=gg.GG_F32,
                 dx=rows(), dw=P, ws=P, ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(dim=0), "dim"), (dict(n=-1), "n = -1"), (dict(dy=None), "dy"), (dict(s=None), "s: "),
    (dict(s=rows(gg.GG_F16)), "s: dtype"), (dict(dx=rows(gg.GG_F16)), "dx: dtype"),
    (dict(dsum=rows(gg.GG_BF16)), "dsum: dtype"), (dict(rstd=None), "rstd"), (dict(dw=P + 1), "dw"),
    (dict(w_dtype=gg.GG_BF16), "weights"), (dict(w=P + 1), "weights"), (dict(ws=None), "workspace"),
    (dict(ws=P + 8), "workspace"), (dict(ws_bytes=16), "workspace"), (dict(dx=rows(stride=4)), "dx: stride")])
def test_norm_gradient_refuses(change, word):
    refused(gg.lib.gg_rmsnorm_backward, NORM_BACK, change, word)


DISTILL = dict(z=rows(), n=7, vocab=100, ids=P, bits=64, ids_stride=64, top=rows(), k=8,
               temperature=2.0, weight=1.0, row_w=None, loss=P, lse=P, dz=rows(), status=P, ws=P,
               ws_bytes=1 << 30, stream=None)


@pytest.mark.parametrize("change,word", [
    (dict(status=None), "status"), (dict(n=-1), "n = -1"), (dict(n=1 << 28), "n = "),
    (dict(vocab=0), "vocab"), (dict(vocab=(1 << 24) + 1), "vocab"), (dict(k=0), "k = 0"),
    (dict(k=257), "k = 257"), (dict(temperature=0.0), "temperature"),
    (dict(temperature=-1.0), "temperature"), (dict(temperature=float("inf")), "temperature"),
    (dict(temperature=float("nan")), "temperature"), (dict(z=None), "z: "), (dict(top=None), "top: "),
    (dict(z=rows(gg.GG_E4M3)), "z: dtype"), (dict(dz=rows(gg.GG_F16)), "dz: dtype"),
    (dict(dz=rows(stride=0)), "dz: stride"), (dict(bits=31), "31 bits"), (dict(ids=None), "ids are NULL"),
    (dict(ids=P + 4), "aligned"), (dict(ids_stride=4), "aligned"), (dict(ids_stride=-64), "aligned"),
    (dict(row_w=P + 2), "row_w"), (dict(loss=None), "loss"), (dict(lse=P + 2), "lse"),
    (dict(ws=None), "workspace"), (dict(ws_bytes=8), "workspace")])
def test_distill_refuses(change, word):
    refused(gg.lib.gg_distill_forward, DISTILL, change, word)


@pytest.mark.parametrize("change,word", [
    (dict(dz=None), "dz"), (dict(lse=None), "lse"), (dict(lse=P + 1), "lse"), (dict(n=-1), "n = -1"),
    (dict(status=None), "status"), (dict(k=0), "k = 0")])
def test_distill_gradient_refuses(change, word):
    args = {k: v for k, v in DISTILL.items() if k not in ("loss", "ws", "ws_bytes")}
    refused(gg.lib.gg_distill_backward, args, change, word)


def test_bindings_check_shapes_of_lists_and_vectors():
    ids = torch.zeros(5, 8, dtype=torch.int64)
    assert gg._top_ids(ids[:, :4], 5, 4)[1:] == (64, 64)
    for bad in (lambda: gg._top_ids(ids, 5, 7), lambda: gg._top_ids(ids.float(), 5, 8),
                lambda: gg._top_ids(ids.t(), 8, 5), lambda: gg._fp32(torch.zeros(4), 5, "x"),
                lambda: gg._fp32(torch.zeros(8)[::2], 4, "x"),
                lambda: gg._weight(torch.zeros(4), 5, "x"), lambda: gg._weight(ids[0], 8, "x")):
        with pytest.raises(gg.GGError):
            bad()


def test_bindings_check_the_rows():
    """No description of fewer rows or narrower ones than the call goes over: refused
    before the stream is asked for, so without a GPU."""
    st, ws = torch.zeros(1, dtype=torch.int32), torch.zeros(1 << 16, dtype=torch.uint8)
    ids, top_ids = torch.zeros(7, dtype=torch.int64), torch.zeros(7, 3, dtype=torch.int64)
    r = lambda *shape: gg.make_rows(torch.zeros(*shape))  # noqa: E731
    good, vec = r(7, 20), torch.zeros(20)
    for name in ("short", "narrow"):
        bad = r(6, 20) if name == "short" else r(7, 19)
        k = r(6, 3) if name == "short" else r(7, 2)
        for call in (
                lambda: gg.gg_embed_forward(bad, 7, 20, ids, 7, 1.0, good, st),
                lambda: gg.gg_embed_forward(good, 7, 20, ids, 7, 1.0, bad, st),
                lambda: gg.gg_embed_backward(bad, ids, 7, 7, 20, 1.0, good, 0, st, ws),
                lambda: gg.gg_embed_backward(good, ids, 7, 7, 20, 1.0, bad, 0, st, ws),
                lambda: gg.gg_rmsnorm_forward(bad, good, 7, 20, None, 1e-6, good, good, None, None),
                lambda: gg.gg_rmsnorm_forward(good, bad, 7, 20, None, 1e-6, good, good, None, None),
                lambda: gg.gg_rmsnorm_forward(good, good, 7, 20, None, 1e-6, bad, good, None, None),
                lambda: gg.gg_rmsnorm_forward(good, good, 7, 20, None, 1e-6, good, bad, None, None),
                lambda: gg.gg_rmsnorm_backward(bad, None, good, vec, 7, 20, None, good, None, None),
                lambda: gg.gg_rmsnorm_backward(good, bad, good, vec, 7, 20, None, good, None, None),
                lambda: gg.gg_rmsnorm_backward(good, None, bad, vec, 7, 20, None, good, None, None),
                lambda: gg.gg_rmsnorm_backward(good, None, good, vec, 7, 20, None, bad, None, None),
                lambda: gg.gg_distill_forward(bad, 7, 20, top_ids, r(7, 3), 3, 1.0, 1.0, None, vec, vec,
                                              good, st, ws),
                lambda: gg.gg_distill_forward(good, 7, 20, top_ids, k, 3, 1.0, 1.0, None, vec, vec,
                                              good, st, ws),
                lambda: gg.gg_distill_forward(good, 7, 20, top_ids, r(7, 3), 3, 1.0, 1.0, None, vec,
                                              vec, bad, st, ws),
                lambda: gg.gg_distill_backward(bad, 7, 20, top_ids, r(7, 3), 3, 1.0, 1.0, None, vec,
                                               good, st),
                lambda: gg.gg_distill_backward(good, 7, 20, top_ids, k, 3, 1.0, 1.0, None, vec, good,
                                               st),
                lambda: gg.gg_distill_backward(good, 7, 20, top_ids, r(7, 3), 3, 1.0, 1.0, None, vec,
                                               bad, st)):
            with pytest.raises(gg.GGError, match="rows of"):
                call()
    q = torch.zeros(6, 20, dtype=torch.float8_e4m3fn)
    with pytest.raises(gg.GGError, match="rows of"):
        gg.gg_rmsnorm_forward(good, None, 7, 20, None, 1e-6, None, None,
                              gg.make_rows(q, scales=torch.zeros(6)), None)


def test_the_student_checks_its_tensors():
    from paper_2606_02916_amd import Student, student
    s = Student(50, 20, 9, max_rows=7, k=3, device="cpu")
    ids = torch.zeros(7, dtype=torch.int64)
    top_ids, top = torch.zeros(7, 3, dtype=torch.int64), torch.zeros(7, 3)
    buf = torch.zeros(6, student.row_bytes_8bit(20), dtype=torch.uint8)
    for call, word in (
            (lambda: s.forward(ids, 8), "student of 7"),
            (lambda: s.forward(ids, 7, torch.zeros(6, 20)), "x of shape"),
            (lambda: s.forward(ids, 7, torch.zeros(7, 19)), "x of shape"),
            (lambda: s.forward(ids[:6], 7), "ids"),
            (lambda: s.step(ids, 7, top_ids, top[:6]), "top of shape"),
            (lambda: s.step(ids, 7, top_ids, top[:, :2]), "top of shape"),
            (lambda: s.step(ids, 7, top_ids[:, :2], top), "top_ids of shape"),
            (lambda: s.step(ids, 7, top_ids, top, torch.zeros(7, 21)), "x of shape"),
            (lambda: s.write_rows(buf, ids, 7), "buffer of 6"),
            (lambda: s.write_rows(buf[:, :20], ids, 6), "8-bit rows"),
            (lambda: s.write_rows(buf, ids, 6, x=torch.zeros(5, 20)), "x of shape"),
            (lambda: student.read_rows(buf, 7, 20, 0, torch.zeros(7, 20), s.status), "buffer of 6"),
            (lambda: student.read_rows(buf, 6, 20, 0, torch.zeros(5, 20), s.status), "out: 5 rows"),
            (lambda: student.read_rows(buf, 6, 20, 0, torch.zeros(6, 18), s.status), "out: 6 rows")):
        with pytest.raises(gg.GGError, match=word):
            call()


@pytest.mark.parametrize("off", [1, 2, 4])
def test_gradient_refuses_a_workspace_off_its_alignment(off):
    """Pairs of 32-bit counters are read from it."""
    refused(gg.lib.gg_embed_backward, GRAD, dict(ws=P + off), "workspace")
