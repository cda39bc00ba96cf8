"""Tensors that share or reinterpret memory, at the entry points of the operators on groups and on gradients."""
import pytest
import torch

import paper_2204_02662_amd as epp
from _util import dev

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m", [100, 20_000])
def test_group_rows_writes_to_its_own_copy(m):
    """Offsets and order that share their memory with other tensors until they are written: the others keep their bits."""
    G = 5
    group_of = torch.randint(0, G, (m,), generator=torch.Generator().manual_seed(1)).int().to(dev())
    ws = torch.empty(epp.epp_group_rows_workspace(m, G), dtype=torch.uint8, device=dev())
    offsets, order = torch.full((G + 1,), -9, dtype=torch.int32, device=dev()), torch.full((m,), -9, dtype=torch.int32, device=dev())
    lazy = torch._lazy_clone(offsets), torch._lazy_clone(order)
    assert lazy[0]._is_view() is False and torch._C._is_cow_tensor(lazy[0]) and torch._C._is_cow_tensor(lazy[1])
    epp.epp_group_rows(group_of, G, lazy[0], lazy[1], ws)
    assert (offsets == -9).all() and (order == -9).all()
    assert torch.equal(lazy[1], torch.sort(group_of, stable=True).indices.int())
    assert torch.equal(lazy[0][1:], torch.bincount(group_of, minlength=G).cumsum(0).int()) and lazy[0][0] == 0


def test_views_that_only_change_the_sign_are_refused():
    """A tensor that stands for the negative of its memory: its numbers are not what lies there."""
    def t(*shape, dtype=torch.float32):
        return torch.ones(*shape, dtype=dtype, device=dev())
    x, W, y, s = t(6, 4), t(2, 4, 4), t(6, 4), t(1)
    offsets = torch.tensor([0, 3, 6], dtype=torch.int32, device=dev())
    b = torch.empty(1 << 16, dtype=torch.uint8, device=dev())
    neg = torch._neg_view
    assert neg(x).is_neg() and neg(x).is_contiguous()
    for call in (lambda: epp.epp_grouped_product(neg(x), W, offsets, y), lambda: epp.epp_grouped_product(x, neg(W), offsets, y),
                 lambda: epp.epp_grouped_product(x, W, offsets, neg(y)), lambda: epp.epp_grouped_input_gradient(neg(x), W, offsets, y),
                 lambda: epp.epp_grouped_weight_gradient(neg(x), y, offsets, W, b), lambda: epp.epp_grouped_weight_gradient(x, neg(y), offsets, W, b),
                 lambda: epp.epp_grouped_weight_gradient(x, y, offsets, neg(W), b), lambda: epp.epp_gradient_norm([x], neg(s), b),
                 lambda: epp.epp_clip_gradients([neg(x)], 1.0, s, b, out=[y]), lambda: epp.epp_clip_gradients([x], 1.0, s, b, out=[neg(y)])):
        with pytest.raises(ValueError, match="negative"):
            call()
    # (a norm has no sign, and what is scaled in place keeps it)
    epp.epp_gradient_norm([neg(x)], s, b)
    assert abs(s.item() - 24 ** 0.5) <= 2.0 ** -24 * 5
    g = neg(torch.full((8, 2), 2.0, device=dev()))
    epp.epp_clip_gradients([g], 4.0, s, b)
    assert s.item() == 8.0 and (g == -1.0).all()
    # (what such a program has in hand: the imaginary part of a conjugate)
    z = torch.full((6, 1), 1 + 2j, dtype=torch.complex64, device=dev()).conj().imag
    assert z.is_neg()
    with pytest.raises(ValueError, match="negative"):
        epp.epp_grouped_product(z, t(2, 1, 4), offsets, y)
    epp.epp_grouped_product(z.resolve_neg(), t(2, 1, 4), offsets, y)
    assert (y == -2.0).all()


def test_a_row_beside_the_results():
    """The only row of the input, and every second row, in other columns of the matrix that the results are columns of."""
    F, n = 24, 10
    W = torch.randint(-2, 3, (2, F, F), generator=torch.Generator().manual_seed(2)).float().to(dev())
    offsets = torch.tensor([0, 4, n], dtype=torch.int32, device=dev())
    wide = torch.randint(-2, 3, (n, 2 * F), generator=torch.Generator().manual_seed(3)).float().to(dev())
    for part, rows in ((slice(3, 4), [0] * n), (slice(0, n, 2), [i // 2 for i in range(n)])):
        was, x = wide.clone(), wide[part, :F]
        picked = was[part, :F][rows]
        epp.epp_grouped_product(x, W, offsets, wide[:, F:], in_rows=torch.tensor(rows, dtype=torch.int32, device=dev()))
        assert torch.equal(wide[:, :F], was[:, :F])
        assert torch.equal(wide[:, F:], torch.cat([picked[:4] @ W[0], picked[4:] @ W[1]]))
