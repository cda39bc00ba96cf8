"""The norm of many gradients and their clipping against plain ones in 64 bits."""
import math

import pytest
import torch

import paper_2204_02662_amd as epp
from _grouped import TINY, TYPES, randn
from _util import dev

pytestmark = pytest.mark.gpu


def plain_norm(grads):
    return math.sqrt(math.fsum(g.double().square().sum().item() for g in grads))


def workspace(n):
    return torch.full((epp.epp_gradient_norm_workspace(n),), 255, dtype=torch.uint8, device=dev())


def assert_norm(got, want):
    # a rounding to fp32, and sums of squares in 64 bits, whose errors are far below a step of fp32.  (A norm below 2^-126 is a
    # denormal float: their steps are 2^-149, so a rounding is off by up to 2^-150 whatever the norm is.)
    assert abs(got.item() - want) <= 1.001 * 2.0 ** -24 * want + 2.0 ** -150, (got.item(), want)


def assert_scaled(got, g, norm, max_norm):
    want = g.double() * (1.0 if norm <= max_norm else max_norm / norm)
    # rounded to fp32 and then to the type; the norm in 64 bits
    off = (torch.finfo(got.dtype).eps / 2 * (1 + 2.0 ** -20) + (2.0 ** -24 if got.dtype != torch.float32 else 0)) * want.abs() + 1.01 * TINY[got.dtype]
    assert ((got.double() - want).abs() <= off).all()


def check(grads, max_norm):
    norm, ws = torch.full((3,), 7.0, device=dev()), workspace(len(grads))
    want = plain_norm(grads)
    epp.epp_gradient_norm(grads, norm[1:2], ws)
    assert_norm(norm[1], want)
    out = [torch.empty_like(g) for g in grads]
    norm.fill_(7.0)
    epp.epp_clip_gradients(grads, max_norm, norm[1:2], ws, out=out)
    assert_norm(norm[1], want)
    assert norm[0] == 7.0 and norm[2] == 7.0
    for g, o in zip(grads, out):
        assert_scaled(o, g, want, max_norm)
    own = [g.clone() for g in grads]
    epp.epp_clip_gradients(own, max_norm, norm[1:2], ws)
    for g, o, x in zip(grads, out, own):
        assert torch.equal(x, o)
        if want <= max_norm:
            assert torch.equal(x, g)


@pytest.mark.parametrize("max_norm", [0.0, 1.0, 1e9])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("count", [0, 1, 2, 7, 8, 9, 255, 2048, 8191, 8192, 8193, 100_003])
def test_sizes(count, dtype, max_norm):
    check([randn(count, seed=count, dtype=dtype)], max_norm)


@pytest.mark.parametrize("n", [0, 1, 2, 95, 96, 97, 200])
def test_many_of_all_types_and_shapes(n):
    shapes = [(3,), (128, 16), (0,), (33, 7, 5), (), (1, 1), (5000,), (64, 128)]
    grads = [randn(*shapes[i % len(shapes)], seed=i, dtype=TYPES[i % 3]) for i in range(n)]
    check(grads, 0.25)
    check([g.transpose(0, 1).contiguous().transpose(0, 1) if g.dim() == 2 else g for g in grads], 1e6)


@pytest.mark.parametrize("dtype", TYPES)
def test_places_in_a_larger_buffer(dtype):
    """Gradients one after another in one buffer, beginning anywhere: their neighbours keep their bits."""
    buf = randn(60_000, seed=9, dtype=dtype)
    was = buf.clone()
    views, at = [], 1
    for i, size in enumerate((1, 2, 3, 5, 8, 13, 4000, 21, 9000, 34, 17_000)):
        views.append(buf[at:at + size])
        at += size + i % 3
    want = plain_norm(views)
    norm = torch.empty(1, device=dev())
    epp.epp_clip_gradients(views, 1.0, norm, workspace(len(views)))
    assert_norm(norm, want)
    inside = torch.zeros_like(buf, dtype=torch.bool)
    at = 1
    for i, v in enumerate(views):
        inside[at:at + v.numel()] = True
        assert_scaled(v, was[at:at + v.numel()], want, 1.0)
        at += v.numel() + i % 3
    assert torch.equal(buf[~inside], was[~inside])
    # into a buffer at other distances from 16 bytes than the gradients'
    other = torch.zeros(60_003, dtype=dtype, device=dev())
    out = [other[3:][v.storage_offset():v.storage_offset() + v.numel()] for v in views]
    copies = [v.clone() for v in views]
    epp.epp_clip_gradients(views, 0.5, norm, workspace(len(views)), out=out)
    for v, c, o in zip(views, copies, out):
        assert torch.equal(v, c)
        assert_scaled(o, c, plain_norm(copies), 0.5)


def test_bounds_that_the_norm_meets():
    """Exactly the bound: the bits stay.  A bound next to it: scaled."""
    g = torch.zeros(1000, device=dev())
    g[3], g[800] = 3.0, 4.0
    norm, ws = torch.empty(1, device=dev()), workspace(1)
    for bound, want in ((5.0, [3.0, 4.0]), (math.nextafter(5.0, 0), [3.0, 4.0]), (2.5, [1.5, 2.0]), (0.0, [0.0, 0.0]), (math.inf, [3.0, 4.0])):
        out = torch.full_like(g, 7.0)
        epp.epp_clip_gradients([g], bound, norm, ws, out=[out])
        assert norm.item() == 5.0 and out[[3, 800]].tolist() == want and out.count_nonzero() <= 2


def test_large_small_and_no_numbers():
    norm, ws = torch.empty(1, device=dev()), workspace(2)
    huge = torch.full((1000,), 2.0 ** 120, device=dev())  # (squares beyond fp32)
    check([huge, huge.clone()], 1.0)
    check([torch.full((77,), 2.0 ** -140, device=dev())], 2.0 ** -142)  # (squares below fp32, elements denormal)
    top = torch.full((4096,), torch.finfo(torch.float32).max, device=dev())
    out = torch.empty_like(top)
    epp.epp_clip_gradients([top], 64.0, norm, ws, out=[out])  # (the norm is beyond fp32, its factor is not lost)
    assert math.isinf(norm.item()) and (out - 1.0).abs().max().item() <= 2.0 ** -23
    for dtype in TYPES:
        g = randn(5000, seed=3, dtype=dtype)
        g[4001] = float("inf")
        epp.epp_clip_gradients([g, top], 1.0, norm, ws, out=[torch.empty_like(g), out])
        assert math.isinf(norm.item()) and (out == 0).all()
        own = g.clone()
        epp.epp_clip_gradients([own], 1.0, norm, ws)
        assert torch.isnan(own[4001]) and (own[:4001] == 0).all() and (own[4002:] == 0).all()
        g[17] = float("nan")
        epp.epp_gradient_norm([top, g], norm, ws)
        assert math.isnan(norm.item())
        epp.epp_clip_gradients([g], 1.0, norm, ws)
        assert math.isnan(norm.item()) and torch.isnan(g).all()


def test_an_infinite_bound_leaves_everything():
    """Infinities as well: nothing is scaled, in place or not."""
    for n in (300, 100_000):
        g = randn(n, seed=n)
        g[7], g[-1] = float("inf"), float("-inf")
        norm, ws, out = torch.empty(1, device=dev()), workspace(1), torch.empty_like(g)
        epp.epp_clip_gradients([g], math.inf, norm, ws, out=[out])
        assert math.isinf(norm.item()) and torch.equal(out, g)


def test_a_gradient_twice():
    """Counts twice in the norm; scaling it twice has no meaning and is refused, as is an output on another's memory."""
    g, h = randn(100, seed=1), randn(100, seed=2)
    norm, ws = torch.empty(1, device=dev()), workspace(3)
    epp.epp_gradient_norm([g, h, g], norm, ws)
    assert_norm(norm, plain_norm([g, h, g]))
    outs = [torch.empty_like(g) for _ in range(2)]
    epp.epp_clip_gradients([g, g], 1.0, norm, ws, out=outs)
    assert torch.equal(outs[0], outs[1])
    for grads, out in (([g, g], None), ([g, h], [h, g]), ([g, h], [outs[0], outs[0]]), ([g, g[10:20]], None), ([g], [h[:100]]), ([g, h], [outs[0], g])):
        if out is not None and len(grads) == 1:
            epp.epp_clip_gradients(grads, 1.0, norm, ws, out=out)  # (another tensor of the same kind: nothing wrong with it)
            continue
        with pytest.raises(epp.EppError):
            epp.epp_clip_gradients(grads, 1.0, norm, ws, out=out)


def test_past_32_bits():
    g = torch.full(((1 << 32) // 2 + 4099,), 2.0 ** -3, dtype=torch.bfloat16, device=dev())  # (more than 2^32 bytes)
    want = math.sqrt(g.numel()) / 8
    norm, ws = torch.empty(1, device=dev()), workspace(1)
    epp.epp_clip_gradients([g], want / 4, norm, ws)
    assert_norm(norm, want)
    assert (g == 2.0 ** -5).all()
