"""What the operator tests share: types, rounding bounds, rows at odd places.

Bounds are derived, not tuned.  U is the unit roundoff of fp32; a result
rounded once to type t adds UNIT[t] of itself, or FLOOR[t] (half of the
smallest subnormal).  A sum of m fp32 terms, in any order, is off by at most
m U times the sum of the terms' magnitudes."""
import torch

U = 2.0 ** -24
F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
E4M3 = torch.float8_e4m3fn
UNIT = {F32: U, F16: 2.0 ** -11, BF16: 2.0 ** -8, E4M3: 2.0 ** -4}
FLOOR = {F32: 2.0 ** -126, F16: 2.0 ** -25, BF16: 2.0 ** -126, E4M3: 2.0 ** -10}


def rows(x, dtype, device, lead=0, pad=0):
    """x (2-d, on the CPU) as dtype on the device, rows `pad` elements apart
    and the first `lead` elements into its buffer; NaN in between."""
    n, d = x.shape
    flat = torch.full((lead + n * (d + pad) + 1,), float("nan")).to(dtype).to(device)
    out = flat[lead:lead + n * (d + pad)].view(n, d + pad)[:, :d]
    out.copy_(x.to(dtype).to(device))
    return out


def like(n, d, dtype, device, lead=0, pad=0):
    """An output of NaNs, its buffer, and the mask of the buffer's elements that belong to
    the output."""
    flat = torch.full((lead + n * (d + pad) + 8,), float("nan")).to(dtype).to(device)
    out = flat[lead:lead + n * (d + pad)].view(n, d + pad)[:, :d]
    own = torch.zeros(flat.numel(), dtype=torch.bool)
    own[lead:lead + n * (d + pad)].view(n, d + pad)[:, :d] = True
    return out, flat, own


def untouched(flat, own):
    """Whether the elements outside the output still hold NaN."""
    return bool(torch.isnan(flat.cpu().float())[~own].all())


def within(got, want, bound):
    """Largest excess of |got - want| over its bound; got and want finite."""
    got = got.detach().cpu().double()
    assert torch.isfinite(got).all()
    return float(((got - want).abs() - bound).max()) if got.numel() else 0.0
