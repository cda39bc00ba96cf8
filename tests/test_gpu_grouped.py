"""Products of rows that belong to groups against plain ones in 64 bits: sizes at the tiles' edges, empty groups, lists of rows, strides,
types, and what must not be touched."""
import pytest
import torch

import paper_2204_02662_amd as epp
from _grouped import TYPES, assert_sums, offsets_of, product, randn, spans, weight_gradient
from _util import dev

pytestmark = pytest.mark.gpu

SIZES = {"none": [0], "one": [1], "empty": [0, 0, 0], "edges": [1, 0, 31, 32, 33, 0, 127, 128, 129], "first": [300, 0, 0], "last": [0, 0, 257],
         "many": [(7 * i) % 5 for i in range(131)], "long": [5, 1400, 0, 700]}
WIDTHS = [(1, 1), (3, 5), (16, 41), (64, 64), (65, 127), (128, 256), (257, 72), (777, 130), (1024, 264)]


def run_rows(sizes, Fi, Fo, dtype, transposed, seed=1):
    m, G = sum(sizes), len(sizes)
    offsets, W = offsets_of(sizes), randn(G, Fi, Fo, seed=seed, dtype=dtype)
    x = randn(m, Fo if transposed else Fi, seed=seed + 1, dtype=dtype)
    got = torch.full((m, Fi if transposed else Fo), 7.0, dtype=dtype, device=dev())
    (epp.epp_grouped_input_gradient if transposed else epp.epp_grouped_product)(x, W, offsets, got)
    assert_sums(got, *product(x, W, offsets, m, transposed=transposed), f"{sizes[:9]} {Fi}x{Fo} {dtype}")


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Fi,Fo", WIDTHS)
@pytest.mark.parametrize("sizes", SIZES)
def test_rows(sizes, Fi, Fo, dtype):
    run_rows(SIZES[sizes], Fi, Fo, dtype, False)
    run_rows(SIZES[sizes], Fi, Fo, dtype, True)


@pytest.mark.parametrize("to32", [False, True])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Fi,Fo", WIDTHS)
@pytest.mark.parametrize("sizes", SIZES)
def test_weight_gradient(sizes, Fi, Fo, dtype, to32):
    if to32 and dtype == torch.float32:
        return
    sizes = SIZES[sizes]
    m, G = sum(sizes), len(sizes)
    offsets, x, d = offsets_of(sizes), randn(m, Fi, seed=3, dtype=dtype), randn(m, Fo, seed=4, dtype=dtype)
    need = epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo)
    held = torch.full((need + 256,), 255, dtype=torch.uint8, device=dev())
    got = torch.full((G, Fi, Fo), 7.0, dtype=torch.float32 if to32 else dtype, device=dev())
    again = torch.full_like(got, 8.0)
    epp.epp_grouped_weight_gradient(x, d, offsets, got, held[:need])
    epp.epp_grouped_weight_gradient(x, d, offsets, again, held[:need])
    want, size, terms = weight_gradient(x, d, offsets, m)
    assert_sums(got, want, size, terms + 520, f"{sizes[:9]} {Fi}x{Fo} {dtype}")  # (at most 512 partial sums and the zeros before)
    assert torch.equal(got, again)
    assert (held[need:] == 255).all()


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("Fi,Fo", [(24, 40), (33, 130), (136, 200)])
def test_lists_strides_and_what_is_left(Fi, Fo, dtype):
    """Rows through lists (inputs' rows twice and rows that do not exist, outputs' in any order), columns of wider matrices, entries before
    the first and behind the last group; rows that nobody names hold NaN and infinity, and what is not written keeps its bits."""
    sizes, first, tail = [40, 0, 150, 3], 7, 11
    m, G, n = first + sum(sizes) + tail, len(sizes), 400
    gen = torch.Generator("cpu").manual_seed(Fi)
    offsets = offsets_of(sizes, first)
    named = torch.randperm(n, generator=gen)[:120].int()
    in_rows = named[torch.randint(0, 120, (m,), generator=gen)]
    in_rows[[first + 3, first + 60, first + 190]] = torch.tensor([-1, n, 2 ** 31 - 1], dtype=torch.int32)
    in_rows[:first] = 2 ** 30
    out_rows = torch.randperm(n, generator=gen)[:m].int()
    out_rows[[first + 5, first + 100]] = torch.tensor([-5, n], dtype=torch.int32)
    in_rows, out_rows = in_rows.to(dev()), out_rows.to(dev())
    outside = torch.ones(n, dtype=torch.bool)
    outside[named.long()] = False
    for step in (8, 3):  # (a stride and a first column that are multiples of 16 bytes with any type, and ones that are not)
        for transposed in (False, True):
            wi, wo = (Fo, Fi) if transposed else (Fi, Fo)
            wide = randn(n, wi + 4 * step, seed=5, dtype=dtype)
            wide[:, :step], wide[:, step + wi:] = float("nan"), float("inf")
            x = wide[:, step:step + wi]
            x[outside.to(dev())] = float("nan")
            W = randn(G, Fi, Fo, seed=6, dtype=dtype)
            held = torch.full((n, wo + 3 * step), 3.0, dtype=dtype, device=dev())
            call = epp.epp_grouped_input_gradient if transposed else epp.epp_grouped_product
            call(x, W, offsets, held[:, step:step + wo], in_rows=in_rows, out_rows=out_rows)
            want, size, terms = product(x, W, offsets, m, in_rows, transposed)
            inside = torch.zeros(m, dtype=torch.bool, device=dev())
            inside[first:m - tail] = True
            inside &= (out_rows >= 0) & (out_rows < n)
            at = out_rows[inside].long()
            assert_sums(held[at, step:step + wo], want[inside], size[inside], terms, f"{step} {transposed}")
            held[at, step:step + wo] = 3.0
            assert (held == 3.0).all()
    x, d = randn(n, Fi, seed=7, dtype=dtype), randn(m, Fo + 8, seed=8, dtype=dtype)[:, 8:]
    x[outside.to(dev())] = float("inf")
    d[:first] = float("nan")
    d[m - tail:] = float("nan")
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo), dtype=torch.uint8, device=dev())
    got = torch.empty(G, Fi, Fo, dtype=dtype, device=dev())
    epp.epp_grouped_weight_gradient(x, d, offsets, got, ws, x_rows=in_rows)
    want, size, terms = weight_gradient(x, d, offsets, m, in_rows)
    assert_sums(got, want, size, terms + 8)
    rows = torch.randperm(n, generator=gen)[:m].int().to(dev())
    y = randn(n, Fo, seed=9, dtype=dtype)
    epp.epp_grouped_weight_gradient(x, y, offsets, got, ws, x_rows=in_rows, grad_rows=rows)
    want, size, terms = weight_gradient(x, y, offsets, m, in_rows, rows)
    assert_sums(got, want, size, terms + 8)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("m,G,Fi,Fo", [(1, 8, 512, 768), (2, 8, 1000, 1016), (16, 16, 777, 520), (17, 3, 2048, 256), (64, 64, 520, 1024),
                                       (200, 32, 640, 512), (1, 4, 1777, 1333), (30, 8, 8, 9), (60, 4, 9, 801), (90, 4, 801, 33), (100, 4, 130, 1021)])
def test_few_rows(m, G, Fi, Fo, dtype):
    """A handful of rows to a group and wide matrices, as single tokens are served."""
    gen = torch.Generator("cpu").manual_seed(m)
    sizes = torch.bincount(torch.randint(0, G, (m,), generator=gen), minlength=G).tolist()
    run_rows(sizes, Fi, Fo, dtype, False, 11)
    run_rows(sizes, Fi, Fo, dtype, True, 12)


@pytest.mark.parametrize("Fi", [1, 4, 30, 32, 33, 40, 64, 72, 95, 96, 97, 128])
@pytest.mark.parametrize("Fo", [2, 16, 32, 35, 56, 64, 66, 96, 100, 128])
def test_narrow_floats(Fi, Fo):
    """Widths of up to 128, at the edges of the blocks of 32 and of the pieces of 16 bytes; few entries and many."""
    for sizes in ([70, 0, 50, 1], [40_000, 31, 9_001, 700], [500_000, 24_300])[:2 if Fi > 40 or Fo in (2, 35, 66) else 3]:
        run_rows(sizes, Fi, Fo, torch.float32, False, Fi)
        run_rows(sizes, Fi, Fo, torch.float32, True, Fo)
        m, offsets = sum(sizes), offsets_of(sizes)
        x, d = randn(m, Fi, seed=13), randn(m, Fo, seed=14)
        ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, len(sizes), Fi, Fo), dtype=torch.uint8, device=dev())
        got = torch.empty(len(sizes), Fi, Fo, device=dev())
        epp.epp_grouped_weight_gradient(x, d, offsets, got, ws)
        want, size, terms = weight_gradient(x, d, offsets, m)
        assert_sums(got, want, size, terms + 1_100)  # (up to 1,024 chunks)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows(dtype):
    sizes = [3000, 0, 1111, 5000]
    run_rows(sizes, 520, 384, dtype, False, 21)
    run_rows(sizes, 520, 384, dtype, True, 22)
    m = sum(sizes)
    offsets, x, d = offsets_of(sizes), randn(m, 264, seed=23, dtype=dtype), randn(m, 520, seed=24, dtype=dtype)
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, 4, 264, 520), dtype=torch.uint8, device=dev())
    got = torch.empty(4, 264, 520, dtype=dtype, device=dev())
    epp.epp_grouped_weight_gradient(x, d, offsets, got, ws)
    want, size, terms = weight_gradient(x, d, offsets, m)
    assert_sums(got, want, size, terms + 520)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_tiles(dtype):
    """Enough tiles of 256 x 256 for the chip, the last ones in quarters or not; contractions that end inside a tile of operands, rows that
    end inside a tile of the result; weights of large matrices, the longest groups first."""
    for sizes in ([700, 0, 300, 1, 255, 257, 600, 900], [2_000, 2_100, 0, 1_900], [513] * 9):
        run_rows(sizes, 200, 4_096, dtype, False, 25)
        run_rows(sizes, 4_104, 328, dtype, True, 26)
    sizes, Fi, Fo = [100, 0, 31, 300, 64, 1, 65, 100], 1_544, 4_096
    m, offsets = sum(sizes), offsets_of(sizes)
    x, d = randn(m + 20, Fi, seed=27, dtype=dtype), randn(m, Fo, seed=28, dtype=dtype)
    rows = torch.randperm(m + 20, generator=torch.Generator().manual_seed(3))[:m].int().to(dev())
    rows[50] = -1
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, 8, Fi, Fo), dtype=torch.uint8, device=dev())
    got = torch.empty(8, Fi, Fo, dtype=dtype, device=dev())
    for x_rows in (None, rows):
        epp.epp_grouped_weight_gradient(x[:m] if x_rows is None else x, d, offsets, got, ws, x_rows=x_rows)
        want, size, terms = weight_gradient(x, d, offsets, m, x_rows)
        assert_sums(got, want, size, terms)


@pytest.mark.parametrize("dtype", TYPES)
def test_large_tiles_of_any_alignment(dtype):
    """The same with rows that are no multiples of 16 bytes, and widths that all but fill their tiles."""
    for sizes in ([700, 0, 300, 1, 255, 257, 600, 900], [513] * 9):
        run_rows(sizes, 3_329, 131, dtype, True, 35)
        run_rows(sizes, 3_329, 7, dtype, True, 36)  # (less than a piece)
        run_rows(sizes, 131, 3_329, dtype, False, 37)
        run_rows(sizes, 72, 3_320, dtype, False, 38)
    sizes, Fi, Fo = [100, 0, 31, 300, 64, 1, 65, 100, 129, 0, 33], 1_537, 2_047
    m, G, offsets = sum(sizes), len(sizes), offsets_of(sizes)
    x, d = randn(m + 20, Fi, seed=39, dtype=dtype), randn(m + 7, Fo, seed=40, dtype=dtype)
    x_rows = torch.randperm(m + 20, generator=torch.Generator().manual_seed(4))[:m].int().to(dev())
    d_rows = torch.randint(0, m + 7, (m,), generator=torch.Generator().manual_seed(5)).int().to(dev())
    x_rows[50], d_rows[60] = -1, 2 ** 31 - 1
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo), dtype=torch.uint8, device=dev())
    for to in {dtype, torch.float32}:
        held = torch.full((G * Fi * Fo + 2,), 5.0, dtype=to, device=dev())
        got = held[1:-1].view(G, Fi, Fo)
        for lists in (dict(), dict(x_rows=x_rows), dict(x_rows=x_rows, grad_rows=d_rows)):
            epp.epp_grouped_weight_gradient(x if lists else x[:m], d if len(lists) == 2 else d[:m], offsets, got, ws, **lists)
            want, size, terms = weight_gradient(x, d, offsets, m, lists.get("x_rows"), lists.get("grad_rows"))
            assert_sums(got, want, size, terms)
        assert held[0] == 5.0 and held[-1] == 5.0


def test_offsets_that_are_not_as_they_should_be():
    """Falling, negative and too large ones: unspecified results in the rows, nothing outside them."""
    x, W = randn(100, 24, seed=31, dtype=torch.bfloat16), randn(4, 24, 40, seed=32, dtype=torch.bfloat16)
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(100, 4, 24, 40), dtype=torch.uint8, device=dev())
    for bad in ([0, 50, 20, 90, 100], [-7, 10, 20, 30, 2 ** 31 - 1], [2 ** 31 - 1, 0, -2 ** 31, 5, 5], [100, 0, 100, 0, 100]):
        offsets = torch.tensor(bad, dtype=torch.int32, device=dev())
        held = torch.full((140, 40), 3.0, dtype=torch.bfloat16, device=dev())
        epp.epp_grouped_product(x, W, offsets, held[20:120])
        assert (held[:20] == 3.0).all() and (held[120:] == 3.0).all()
        gw = torch.full((6, 24, 40), 3.0, device=dev())
        epp.epp_grouped_weight_gradient(x, held[20:120], offsets, gw[1:5], ws)
        assert (gw[0] == 3.0).all() and (gw[5] == 3.0).all()


@pytest.mark.parametrize("dtype,Fi,Fo", [(torch.float32, 16, 40), (torch.float32, 40, 40), (torch.bfloat16, 40, 72)])
def test_falling_offsets_and_partial_sums(dtype, Fi, Fo):
    """Groups that overlap name more partial sums than the workspace holds: nothing behind it is read or written."""
    m, G = 60_000, 4
    x, d = randn(m, Fi, seed=33, dtype=dtype), randn(m, Fo, seed=34, dtype=dtype)
    need = epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo)
    assert need > 4 * 8 * G * Fi * Fo  # (the entries are cut)
    for bad in ([0, m, 0, m, m], [0, m, 0, m, 0], [0, m, 0, 2 ** 31 - 1, 7]):
        held = torch.full((4 * need,), 255, dtype=torch.uint8, device=dev())
        got = torch.full((G + 2, Fi, Fo), 3.0, dtype=dtype, device=dev())
        epp.epp_grouped_weight_gradient(x, d, torch.tensor(bad, dtype=torch.int32, device=dev()), got[1:-1], held[:need])
        assert (held[need:] == 255).all() and (got[0] == 3.0).all() and (got[-1] == 3.0).all()
        assert torch.isfinite(got).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_places_past_32_bits(dtype):
    """Rows that lie more than 2^32 bytes behind the first."""
    width, n = 64, (1 << 32) // 128 + 1000
    x = torch.empty(n, width, dtype=dtype, device=dev())
    rows = torch.tensor([n - 1, 0, n - 500, n // 2, 3], dtype=torch.int32, device=dev())
    x[rows.long()] = randn(5, width, seed=41, dtype=dtype)
    W, offsets = randn(2, width, width, seed=42, dtype=dtype), offsets_of([3, 2])
    want, size, terms = product(x[rows.long()], W, offsets, 5)
    got = torch.empty(5, width, dtype=dtype, device=dev())
    epp.epp_grouped_product(x, W, offsets, got, in_rows=rows)
    assert_sums(got, want, size, terms)
    y = torch.empty(n, width, dtype=dtype, device=dev())
    epp.epp_grouped_product(got, W, offsets, y, out_rows=rows)
    want, size, terms = product(got, W, offsets, 5)
    assert_sums(y[rows.long()], want, size, terms)
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(5, 2, width, width), dtype=torch.uint8, device=dev())
    gw = torch.empty(2, width, width, dtype=dtype, device=dev())
    epp.epp_grouped_weight_gradient(x, y, offsets, gw, ws, x_rows=rows, grad_rows=rows)
    want, size, terms = weight_gradient(x[rows.long()], y[rows.long()], offsets, 5)
    assert_sums(gw, want, size, terms + 8)


def test_gradients_are_the_products_derivatives():
    """<grad_out, product(X, W)> changes with X and W as the two gradients say: it is linear in each, so differences are exact but for
    rounding."""
    sizes, Fi, Fo = [9, 0, 30, 4], 20, 28
    m, offsets = sum(sizes), offsets_of(sizes)
    X, W, D = randn(m, Fi, seed=51), randn(4, Fi, Fo, seed=52), randn(m, Fo, seed=53)
    dX, dW, y = torch.empty_like(X), torch.empty_like(W), torch.empty_like(D)
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, 4, Fi, Fo), dtype=torch.uint8, device=dev())
    epp.epp_grouped_input_gradient(D, W, offsets, dX)
    epp.epp_grouped_weight_gradient(X, D, offsets, dW, ws)

    def value(x, w):
        epp.epp_grouped_product(x, w, offsets, y)
        return (y.double() * D.double()).sum().item(), (y.double().abs() * D.double().abs()).sum().item()
    for seed in range(3):
        u, v = randn(m, Fi, seed=60 + seed), randn(4, Fi, Fo, seed=70 + seed)
        for (a, sa), (b, sb), slope in ((value(X + u, W), value(X - u, W), (dX.double() * u.double()).sum().item()),
                                        (value(X, W + v), value(X, W - v), (dW.double() * v.double()).sum().item())):
            # (sums of 28 or 30 products, and one rounding of X +- u: 64 half steps of every term are more than all of it)
            assert abs((a - b) / 2 - slope) <= 64 * 2.0 ** -24 * 64 * (sa + sb), seed


def test_infinities_and_nan_stay_in_their_rows():
    sizes, Fi, Fo = [70, 50], 72, 56
    m, offsets = sum(sizes), offsets_of(sizes)
    for dtype in TYPES:
        x, W = randn(m, Fi, seed=81, dtype=dtype), randn(2, Fi, Fo, seed=82, dtype=dtype)
        x[5, 3], x[69, 71], x[70, 0] = float("nan"), float("inf"), float("-inf")
        got = torch.empty(m, Fo, dtype=dtype, device=dev())
        epp.epp_grouped_product(x, W, offsets, got)
        assert torch.isnan(got[5]).all()
        assert torch.equal(got[69], torch.where(W[0, 71] > 0, float("inf"), float("-inf")).to(dtype))
        assert torch.equal(got[70], torch.where(W[1, 0] > 0, float("-inf"), float("inf")).to(dtype))
        assert torch.isfinite(got[[i for i in range(m) if i not in (5, 69, 70)]]).all()
        W[0, 0, 0] = float("nan")  # (the other group's rows, and the other columns, do not see it)
        x[5, 3], x[69, 71], x[70, 0] = 0, 0, 0
        epp.epp_grouped_product(x, W, offsets, got)
        assert torch.isnan(got[:70, 0]).all() and torch.isfinite(got[70:]).all() and torch.isfinite(got[:, 1:]).all()
