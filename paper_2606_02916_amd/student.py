"""A graph-free student of the GraphSAGE consumer: learned rows for every node,
an RMS norm and a linear head, trained on the consumer's best classes.  It
answers from a node's own row, without sampling or fetching neighbours, and
its normed rows in 8 bits are feature rows that the fetch path moves at a
quarter of their fp32 size.  Buffers and argument marshalling; lookups, norms,
the loss and their gradients run in libgg, the head's products in torch.

    e = sqrt(dim) * table[ids];  s = e + x;  y = s / rms(s) * w;  z = y @ head
    loss = T^2 sum_k p_k (log p_k - log softmax(z / T)[class_k])
"""
from __future__ import annotations

import math

import torch

from . import gg


def row_bytes_8bit(dim, group=0):
    """Bytes of a row in 8 bits: the codes, then at the next multiple of 4 one
    fp32 scale per `group` elements (per row with group 0)."""
    return (dim + 3) // 4 * 4 + 4 * (-(-dim // group) if group else 1)


def rows_8bit(buf, dim, group=0):
    """The rows of `buf` (uint8, [n, at least row_bytes_8bit(dim, group)]; a
    shard, a cache or a window's gathered rows) as 8-bit rows for the gg_*
    calls."""
    at, end = (dim + 3) // 4 * 4, row_bytes_8bit(dim, group)
    if buf.dtype != torch.uint8 or buf.dim() != 2 or buf.shape[1] < end:
        raise gg.GGError(f"8-bit rows of {dim} elements need uint8 rows of {end} bytes")
    return gg.make_rows(buf[:, :dim].view(torch.float8_e4m3fn),
                        scales=buf[:, at:end].view(torch.float32), group=group)


def _shaped(t, n, cols, what):
    """t, of at least n rows of just cols elements."""
    if t.dim() != 2 or t.shape[0] < n or t.shape[1] != cols:
        raise gg.GGError(f"{what} of shape {tuple(t.shape)} for {n} rows of {cols}")
    return t


class Student:
    """table [num_nodes, dim], norm weights w [dim] and head [dim, classes] on
    the device, with the buffers of steps of up to max_rows rows and k teacher
    entries each.  What is trained is fp32: most of a step of a mean loss is less
    than half a unit of a 16-bit number and would be rounded away.  dtype: fp32,
    fp16 or bf16, of the activations, their gradients and the copy of the head
    that they are multiplied with."""

    def __init__(self, num_nodes, dim, classes, max_rows, k=8, temperature=2.0, rate=0.05,
                 dtype=torch.float32, eps=1e-6, device=None, generator=None):
        self.device = dev = torch.device(device if device is not None else "cuda")
        self.N, self.dim, self.classes, self.k = int(num_nodes), int(dim), int(classes), int(k)
        self.max_rows, self.dtype = int(max_rows), dtype
        self.temperature, self.rate, self.eps = float(temperature), float(rate), float(eps)
        self.scale = math.sqrt(dim)

        def normal(*shape, std):
            return torch.randn(*shape, generator=generator, device=dev) * std

        self.table = normal(self.N, self.dim, std=1 / self.scale)
        self.w = torch.ones(self.dim, device=dev)
        self.head = normal(self.dim, self.classes, std=1 / self.scale)
        self.status = torch.zeros(1, dtype=torch.int32, device=dev)
        rows = lambda d: torch.empty((self.max_rows, d), dtype=dtype, device=dev)  # noqa: E731
        vec = lambda: torch.empty(self.max_rows, device=dev)  # noqa: E731
        # e becomes the sum with x, and in a step its gradient; z its gradient
        self.e, self.y, self.dy, self.z = rows(dim), rows(dim), rows(dim), rows(classes)
        self.rstd, self.loss, self.lse = vec(), vec(), vec()
        self.dw, self.dhead = torch.empty_like(self.w), torch.empty_like(self.head, dtype=dtype)
        self._head = torch.empty_like(self.dhead) if dtype != torch.float32 else self.head
        self._table = gg.make_rows(self.table)
        self._e, self._y, self._dy, self._z = (gg.make_rows(t)
                                               for t in (self.e, self.y, self.dy, self.z))
        ws = max(gg.gg_ws_embed(self.max_rows, self.N, self.dim),
                 gg.gg_ws_rmsnorm(self.max_rows, self.dim),
                 gg.gg_ws_distill(self.max_rows, self.classes))
        self.ws = torch.empty(max(ws, 16), dtype=torch.uint8, device=dev)

    def _normed(self, ids, n, x, q=None, y=True, stream=None):
        """The normed rows of ids[:n] (None: the nodes 0 .. n-1), with x [n, dim]
        added to the looked-up rows if given; into self.y, and in 8 bits into q."""
        if n > self.max_rows:
            raise gg.GGError(f"{n} rows for a student of {self.max_rows}")
        if x is not None:
            x = gg.make_rows(_shaped(x, n, self.dim, "x"))
        gg.gg_embed_forward(self._table, self.N, self.dim, ids, n, self.scale, self._e,
                            self.status, stream=stream)
        gg.gg_rmsnorm_forward(self._e, x, n, self.dim, self.w, self.eps, self._e,
                              self._y if y else None, q, self.rstd, stream=stream)

    def forward(self, ids, n, x=None):
        """Logits [n, classes] of the nodes ids[:n] on the current stream: a view of
        self.z, which the next forward overwrites and a step turns into the gradient."""
        self._normed(ids, n, x)
        if self._head is not self.head:
            self._head.copy_(self.head)
        return torch.mm(self.y[:n], self._head, out=self.z[:n])

    def step(self, ids, n, top_ids, top, x=None, row_w=None):
        """One step of gradient descent on the nodes ids[:n] (int32 or int64,
        nodes may recur; -1 is skipped by the table) against the teacher's top
        classes top_ids [n, k] and their logits top [n, k]; row_w [n]: fp32
        weights of the rows (mean loss by default).  On the current stream;
        returns the rows' weighted losses, a view of self.loss, which the next step
        overwrites."""
        _shaped(top_ids, n, self.k, "top_ids"), _shaped(top, n, self.k, "top")
        self.forward(ids, n, x)
        weight = 1.0 if row_w is not None else 1.0 / max(n, 1)
        gg.gg_distill_forward(self._z, n, self.classes, top_ids, gg.make_rows(top), self.k,
                              self.temperature, weight, row_w, self.loss, self.lse, self._z,
                              self.status, self.ws)
        dz = self.z[:n]
        torch.mm(self.y[:n].t(), dz, out=self.dhead)
        torch.mm(dz, self._head.t(), out=self.dy[:n])
        gg.gg_rmsnorm_backward(self._dy, None, self._e, self.rstd, n, self.dim, self.w, self._e,
                               self.dw, self.ws)
        # the step on the table, in place: only rows that occur are touched
        gg.gg_embed_backward(self._e, ids, n, self.N, self.dim, -self.rate * self.scale,
                             self._table, gg.GG_EMBED_ADD, self.status, self.ws)
        self.head.add_(self.dhead, alpha=-self.rate)
        self.w.add_(self.dw, alpha=-self.rate)
        return self.loss[:n]

    def write_rows(self, buf, ids, n, group=0, x=None):
        """The normed rows of ids[:n] in 8 bits into buf (uint8 rows, see
        rows_8bit): feature rows for a fetch pipeline."""
        q = rows_8bit(buf, self.dim, group)
        if n > buf.shape[0]:
            raise gg.GGError(f"{n} rows for a buffer of {buf.shape[0]}")
        self._normed(ids, n, x, q=q, y=False)
        return buf


def read_rows(buf, n, dim, group, out, status):
    """8-bit rows buf[:n] (gathered by a fetch pipeline, say) as numbers in
    out [n, dim], on the current stream."""
    rows = rows_8bit(buf, dim, group)
    if n > buf.shape[0]:
        raise gg.GGError(f"{n} rows of a buffer of {buf.shape[0]}")
    gg.gg_embed_forward(rows, buf.shape[0], dim, None, n, 1.0,
                        gg.make_rows(out), status)
    return out
