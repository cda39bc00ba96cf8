"""Products of rows that belong to groups on numbers below the smallest normal one: neither operands nor results are taken for zero.

The numbers are whole ones from -2 to 2 times the smallest step of the type (2^-149, 2^-133, 2^-24), so that sums are exact in fp32 (where
2^-149 is the smallest step as well) and results are the exact sums, rounded to the type once."""
import pytest
import torch

import paper_2204_02662_amd as epp
from _grouped import TYPES, offsets_of, product, weight_gradient
from _util import dev
from test_gpu_grouped_lists import ints

pytestmark = pytest.mark.gpu
STEP = {torch.float32: 2.0 ** -149, torch.bfloat16: 2.0 ** -133, torch.float16: 2.0 ** -24}


def small(*shape, seed, dtype):
    x = (ints(*shape, seed=seed).double() * STEP[dtype]).to(dtype)
    assert x.count_nonzero() > 0 and (x.double() / STEP[dtype]).abs().max() == 2
    return x


SHAPES = [([1, 0, 2], 264, 520), ([70, 0, 50], 64, 136), ([700, 0, 300, 1, 255, 257, 600, 900, 30], 72, 4_096), ([3_000, 0, 1_111, 5_000], 72, 640),
          ([40_000, 31, 0, 12_001], 16, 41), ([60, 31], 33, 47)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,Fi,Fo", SHAPES)
def test_rows(sizes, Fi, Fo, dtype):
    m, G, offsets = sum(sizes), len(sizes), offsets_of(sizes)
    for transposed in (False, True):
        wi, wo = (Fo, Fi) if transposed else (Fi, Fo)
        call = epp.epp_grouped_input_gradient if transposed else epp.epp_grouped_product
        for x, W in ((small(m, wi, seed=1, dtype=dtype), ints(G, Fi, Fo, seed=2, dtype=dtype)), (ints(m, wi, seed=3, dtype=dtype), small(G, Fi, Fo, seed=4, dtype=dtype))):
            got = torch.full((m, wo), 7.0, dtype=dtype, device=dev())
            call(x, W, offsets, got)
            assert torch.equal(got, product(x, W, offsets, m, transposed=transposed)[0].to(dtype)), transposed


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("sizes,Fi,Fo", SHAPES + [([30_000, 0, 22_001, 8_000], 40, 72), ([(37 * i) % 260 for i in range(16)], 640, 640)])
def test_weight_gradient(sizes, Fi, Fo, dtype):
    m, G, offsets = sum(sizes), len(sizes), offsets_of(sizes)
    ws = torch.empty(epp.epp_grouped_weight_gradient_workspace(m, G, Fi, Fo), dtype=torch.uint8, device=dev())
    for x, d in ((small(m, Fi, seed=5, dtype=dtype), ints(m, Fo, seed=6, dtype=dtype)), (ints(m, Fi, seed=7, dtype=dtype), small(m, Fo, seed=8, dtype=dtype))):
        want = weight_gradient(x, d, offsets, m)[0]
        for to in {dtype, torch.float32}:
            got = torch.full((G, Fi, Fo), 7.0, dtype=to, device=dev())
            epp.epp_grouped_weight_gradient(x, d, offsets, got, ws)
            assert torch.equal(got, want.to(to)), to
