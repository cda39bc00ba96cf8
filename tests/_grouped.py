"""Plain forms of the operators on groups and on gradients, in 64 bits, and what their results may be off by."""
import torch

from _util import dev

TYPES = [torch.float32, torch.bfloat16, torch.float16]
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}  # half the smallest step


def offsets_of(sizes, first=0):
    return torch.tensor([first, *(first + torch.tensor(sizes).cumsum(0)).tolist()], dtype=torch.int32, device=dev())


def randn(*shape, seed, dtype=torch.float32):
    return torch.randn(shape, device=dev(), generator=torch.Generator(dev()).manual_seed(seed)).to(dtype)


def rows_of(x, rows, m):
    """Rows of the entries, zeros where there is no such row."""
    if rows is None:
        return x[:m].double()
    r = rows.long()
    there = (r >= 0) & (r < x.shape[0])
    return torch.where(there[:, None], x[r.clamp(0, x.shape[0] - 1)].double(), 0.0)


def spans(offsets):
    o = offsets.tolist()
    return [(g, o[g], o[g + 1]) for g in range(len(o) - 1) if o[g + 1] > o[g]]


def product(x, W, offsets, m, rows=None, transposed=False):
    """(results of the m entries, sums of the terms' magnitudes, additions of one result); entries of no group: NaN."""
    x, W = rows_of(x, rows, m), W.double()
    W = W.transpose(1, 2).contiguous() if transposed else W
    y = torch.full((m, W.shape[2]), float("nan"), dtype=torch.float64, device=x.device)
    size = y.clone()
    for g, a, b in spans(offsets):
        y[a:b], size[a:b] = x[a:b] @ W[g], x[a:b].abs() @ W[g].abs()
    return y, size, W.shape[1]


def weight_gradient(x, d, offsets, m, x_rows=None, d_rows=None):
    x, d = rows_of(x, x_rows, m), rows_of(d, d_rows, m)
    w = torch.zeros(offsets.numel() - 1, x.shape[1], d.shape[1], dtype=torch.float64, device=x.device)
    size = w.clone()
    for g, a, b in spans(offsets):
        w[g], size[g] = x[a:b].T.contiguous() @ d[a:b], x[a:b].abs().T.contiguous() @ d[a:b].abs()
    return w, size, max([b - a for _, a, b in spans(offsets)], default=0)


def assert_sums(got, want, size, terms, what=""):
    """A sum of `terms` products in fp32, in any order: every addition (and, of floats, the product in it) rounds once, by half a step of
    2^-23 of a partial sum, which `size` bounds; zero partial sums that a tile adds are exact.  Then the result is rounded to its type.
    (Twice that: 2^-23, for matrix instructions that cut off what they shift out.)"""
    off = terms * 2.0 ** -23 * size
    half = torch.finfo(got.dtype).eps / 2 if got.dtype != torch.float32 else 0.0
    off = off + half * (want.abs() + off) + TINY[got.dtype]
    err = (got.double() - want).abs()
    assert torch.isfinite(got).all(), what
    assert (err <= off).all(), f"{what}: {(err - off).max().item()} beyond, {int((err > off).sum())} of {err.numel()}"
