"""Products of rows that belong to groups with lists of rows, row strides and rows that do not exist, at the sizes that the larger tiles,
the kernels of narrow floats and the cut weight gradients are for.

All numbers are whole ones from -2 to 2: every sum in fp32 is exact whatever the order of its additions (fewer than 2^22 terms of at most 4:
below 2^24), and a result is its exact value rounded to the type once, to the nearest (ties to even).  So results are equal, bit for bit, and a
term that is left out, doubled or taken from another row shows."""
import pytest
import torch

import paper_2204_02662_amd as epp
from _grouped import TYPES, offsets_of, product, weight_gradient
from _util import dev

pytestmark = pytest.mark.gpu
HALVES = [torch.bfloat16, torch.float16]
FIRST, TAIL = 7, 11  # entries before the first group and behind the last


def ints(*shape, seed, dtype=torch.float32):
    return torch.randint(-2, 3, shape, device=dev(), generator=torch.Generator(dev()).manual_seed(seed), dtype=torch.int8).to(dtype)


def named_rows(m, n, seed, once):
    """A list of m of n rows, each at most once or some of them often, and three that do not exist."""
    gen = torch.Generator(dev()).manual_seed(seed)
    if once:
        rows = torch.randperm(n, generator=gen, device=dev())[:m]
    else:
        rows = torch.randint(0, n, (m,), generator=gen, device=dev()) // 2 * 2  # (odd rows: nobody's)
    rows = rows.int()
    at = torch.randperm(m - FIRST - TAIL, generator=gen, device=dev())[:3] + FIRST
    rows[at] = torch.tensor([-1, n, 2 ** 31 - 1], dtype=torch.int32, device=dev())[:at.numel()]
    rows[:FIRST] = 2 ** 30
    return rows


def matrix(n, width, seed, dtype, step, rows=None):
    """Columns of a wider matrix whose other columns are NaN, and so are the rows that the list does not name."""
    wide = torch.full((n, width + 4 * step), float("nan"), dtype=dtype, device=dev())
    x = wide[:, step:step + width]
    x.copy_(ints(n, width, seed=seed, dtype=dtype))
    if rows is not None:
        named = torch.zeros(n, dtype=torch.bool, device=dev())
        named[rows[(rows >= 0) & (rows < n)].long()] = True
        x[~named] = float("nan")
    return x


def run_rows(sizes, Fi, Fo, dtype, transposed, seed, step=8, in_list=True, out_list=True):
    m, G = FIRST + sum(sizes) + TAIL, len(sizes)
    wi, wo = (Fo, Fi) if transposed else (Fi, Fo)
    offsets, W = offsets_of(sizes, FIRST), ints(G, Fi, Fo, seed=seed, dtype=dtype)
    n_in, n_out = m + 101 if in_list else m, m + 77 if out_list else m
    in_rows = named_rows(m, n_in, seed + 1, False) if in_list else None
    out_rows = named_rows(m, n_out, seed + 2, True) if out_list else None
    x = matrix(n_in, wi, seed + 3, dtype, step, in_rows)
    held = torch.full((n_out, wo + 3 * step), 3.0, dtype=dtype, device=dev())
    call = epp.epp_grouped_input_gradient if transposed else epp.epp_grouped_product
    call(x, W, offsets, held[:, step:step + wo], in_rows=in_rows, out_rows=out_rows)
    want, _, _ = product(x, W, offsets, m, in_rows, transposed)
    expected = torch.full_like(held, 3.0)
    inside = torch.zeros(m, dtype=torch.bool, device=dev())
    inside[FIRST:m - TAIL] = True
    if out_list:
        inside &= (out_rows >= 0) & (out_rows < n_out)
    to = out_rows[inside].long() if out_list else inside.nonzero().flatten()
    expected[to, step:step + wo] = want[inside].to(dtype)
    assert torch.equal(held, expected), (sizes[:9], Fi, Fo, dtype, transposed, step)


LISTS = [(True, True), (True, False), (False, True)]


@pytest.mark.parametrize("lists", LISTS)
@pytest.mark.parametrize("step", [8, 3])
@pytest.mark.parametrize("dtype", HALVES)
def test_tiles_of_256(dtype, step, lists):
    """Whole tiles, and (17 tiles of rows times 16 or 17 of columns: 272 or 289 for 256 compute units) the last ones in quarters.  A step of 3:
    rows of any alignment, which the gradient has tiles of 256 for, and the product of 128."""
    for sizes in ([700, 0, 300, 1, 255, 257, 600, 900, 30], [2_000, 2_100, 0, 1_900]):
        run_rows(sizes, 200, 4_096, dtype, False, 1, step, *lists)
        run_rows(sizes, 4_104, 136, dtype, True, 2, step, *lists)
    run_rows([700, 0, 300, 1, 255, 257, 600, 900, 30], 4_099, 131, dtype, True, 3, step, *lists)


@pytest.mark.parametrize("lists", LISTS)
@pytest.mark.parametrize("step", [8, 3])
@pytest.mark.parametrize("dtype", HALVES)
def test_tiles_of_128(dtype, step, lists):
    """More than 256 tiles of 128 x 128, of widths that waste too much of tiles of 256."""
    sizes = [3_000, 0, 1_111, 5_000]
    run_rows(sizes, 520, 640, dtype, False, 11, step, *lists)
    run_rows(sizes, 640, 520, dtype, True, 12, step, *lists)
    run_rows(sizes, 133, 645, dtype, False, 13, step, *lists)
    run_rows(sizes, 645, 133, dtype, True, 14, step, *lists)


@pytest.mark.parametrize("lists", LISTS)
@pytest.mark.parametrize("step", [8, 3])
@pytest.mark.parametrize("dtype", TYPES)
def test_tiles_of_64(dtype, step, lists):
    for sizes in ([70, 0, 50, 1, 200], [900, 1_200, 0, 300]):
        run_rows(sizes, 264, 392, dtype, False, 21, step, *lists)
        run_rows(sizes, 392, 264, dtype, True, 22, step, *lists)


@pytest.mark.parametrize("lists", LISTS)
@pytest.mark.parametrize("step", [8, 3])
@pytest.mark.parametrize("dtype", TYPES)
def test_few_rows(dtype, step, lists):
    for sizes in ([1, 0, 0, 2, 0, 1, 0, 0, 0, 0, 0, 0], [20, 0, 33, 5], [90, 4, 0, 9, 1]):
        run_rows(sizes, 520, 1_032, dtype, False, 31, step, *lists)
        run_rows(sizes, 777, 1_001, dtype, False, 32, step, *lists)
        run_rows(sizes, 1_032, 520, dtype, True, 33, step, *lists)
        run_rows(sizes, 1_001, 777, dtype, True, 34, step, *lists)


@pytest.mark.parametrize("lists", LISTS)
@pytest.mark.parametrize("step", [8, 3])
def test_few_rows_of_many_groups(step, lists):
    """Floats: 72 groups times 17 blocks of 64 columns."""
    for per in (5, 17):
        sizes = [(per * i) % (2 * per) + i % 3 for i in range(72)]
        run_rows(sizes, 264, 1_032, torch.float32, False, 35, step, *lists)
        run_rows(sizes, 1_032, 264, torch.float32, True, 36, step, *lists)
        run_rows(sizes, 133, 1_025, torch.float32, False, 37, step, *lists)


@pytest.mark.parametrize("lists", LISTS)
@pytest.mark.parametrize("Fi,Fo", [(16, 41), (41, 16), (128, 30), (7, 100), (32, 32), (1, 128), (64, 47), (97, 66)])
def test_narrow_floats(Fi, Fo, lists):
    """From 49,152 entries on where a side is at most 32, else from 2^19."""
    sizes = [40_000, 31, 0, 12_001, 700] if min(Fi, Fo) <= 32 else [500_000, 1, 24_400]
    for step in (8, 3):
        run_rows(sizes, Fi, Fo, torch.float32, False, 41, step, *lists)
        run_rows(sizes, Fi, Fo, torch.float32, True, 42, step, *lists)


def run_weight(sizes, Fi, Fo, dtype, seed, step, x_list, d_list):
    m, G = FIRST + sum(sizes) + TAIL, len(sizes)
    offsets = offsets_of(sizes, FIRST)
    rows, mats = [], []
    for k, (width, listed) in enumerate(((Fi, x_list), (Fo, d_list))):
        n = m + 101 if listed else m
        rows.append(named_rows(m, n, seed + k, False) if listed else None)
        mats.append(matrix(n, width, seed + 2 + k, dtype, step, rows[k]))
        if not listed:  # (entries of no group)
            mats[k][:FIRST] = float("nan")
            mats[k][m - TAIL:] = float("nan")
    need = epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo)
    held = torch.full((need + 256,), 255, dtype=torch.uint8, device=dev())
    # (what the list of the one does not reach in a group is NaN in neither)
    want, _, _ = weight_gradient(*mats, offsets, m, *rows)
    assert torch.isfinite(want).all()
    for to in {dtype, torch.float32}:
        got = torch.full((G + 2, Fi, Fo), 3.0, dtype=to, device=dev())
        epp.epp_grouped_weight_gradient(*mats, offsets, got[1:-1], held[:need], x_rows=rows[0], grad_rows=rows[1])
        assert torch.equal(got[1:-1], want.to(to)), (sizes[:9], Fi, Fo, dtype, to, step)
        assert (got[0] == 3.0).all() and (got[-1] == 3.0).all() and (held[need:] == 255).all()
    return need


WEIGHT_LISTS = [(True, True), (True, False), (False, True), (False, False)]


@pytest.mark.parametrize("lists", WEIGHT_LISTS)
@pytest.mark.parametrize("Fi,Fo", [(16, 41), (41, 16), (128, 30), (3, 100), (32, 64), (1, 1)])
def test_narrow_weight_gradients(Fi, Fo, lists):
    """Chunks of 256 entries, of 1,024, and of more, whose rows are looked up 1,024 at a time."""
    for sizes in ([40_000, 31, 0, 12_001, 700], [700_001, 0, 340_000, 8_500, 77], [1_500_003]):
        for step in (8, 3) if sum(sizes) < 10 ** 6 else (8,):
            run_weight(sizes, Fi, Fo, torch.float32, 51, step, *lists)


@pytest.mark.parametrize("lists", WEIGHT_LISTS)
@pytest.mark.parametrize("step", [8, 3])
@pytest.mark.parametrize("dtype", TYPES)
def test_cut_weight_gradients(dtype, step, lists):
    for sizes, Fi, Fo in (([30_000, 0, 22_001, 8_000], 40, 72), ([5_003, 1, 0, 9_000], 136, 200), ([90_001], 65, 64), ([30, 0, 40_000, 700], 33, 131)):
        need = run_weight(sizes, Fi, Fo, dtype, 61, step, *lists)
        assert need >= 2 * 4 * len(sizes) * Fi * Fo  # (the entries are cut)


@pytest.mark.parametrize("lists", WEIGHT_LISTS)
@pytest.mark.parametrize("step", [8, 3])
@pytest.mark.parametrize("dtype", HALVES)
def test_weight_gradients_in_tiles_of_128_and_256(dtype, step, lists):
    """16 groups of 25 tiles of 128 x 128; 64 tiles of 128 x 128 to each of a few chunks; 8 groups of 112 tiles of 256 x 256."""
    run_weight([(37 * i) % 260 for i in range(16)], 640, 640, dtype, 71, step, *lists)
    run_weight([9_000, 14_001, 0, 7_000], 1_024, 1_024, dtype, 72, step, *lists)
    run_weight([100, 0, 31, 300, 64, 1, 65, 100], 1_544, 4_096, dtype, 73, step, *lists)


@pytest.mark.parametrize("Fi", [1, 30, 33, 64, 97, 128])
@pytest.mark.parametrize("Fo", [2, 32, 35, 66, 128])
def test_long_sums_without_lists(Fi, Fo):
    """Half a million entries and a few, narrow floats: nothing is left out of a sum."""
    for sizes in ([40_000, 31, 9_001, 700], [500_000, 24_300]):
        run_weight(sizes, Fi, Fo, torch.float32, 81, 0, False, False)
