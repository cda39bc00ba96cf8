"""Narrow floats at the largest widths that have kernels of their own, from 2^19 entries on: every pair of blocks of 32."""
import pytest
import torch

from test_gpu_grouped_lists import run_rows

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lists", [(True, True), (False, False)])
@pytest.mark.parametrize("Fi,Fo", [(33, 64), (40, 90), (64, 128), (72, 37), (65, 96), (96, 72), (90, 127), (100, 64), (97, 95), (128, 128), (97, 125)])
def test_widths(Fi, Fo, lists):
    for step in (8, 3):
        run_rows([400_000, 1, 0, 124_400], Fi, Fo, torch.float32, False, 91, step, *lists)
        run_rows([400_000, 1, 0, 124_400], Fi, Fo, torch.float32, True, 92, step, *lists)
