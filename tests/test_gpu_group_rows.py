"""Entries in the order of their groups, against a stable sort on the host: the one-workgroup and the three-launch way, lists, no group."""
import numpy as np
import pytest
import torch

import paper_2204_02662_amd as epp
from _util import dev

pytestmark = pytest.mark.gpu


def oracle(group_of, G, rows):
    rows = np.arange(group_of.size) if rows is None else rows
    inside = (rows >= 0) & (rows < group_of.size)
    g = np.full(rows.size, G)
    g[inside] = group_of[rows[inside]]
    g[(g < 0) | (g > G)] = G
    at = np.argsort(g, kind="stable")
    return np.searchsorted(g[at], np.arange(G + 1)), rows[at]


def check(group_of, G, rows=None):
    m = group_of.size if rows is None else rows.size
    need = epp.epp_group_rows_workspace(m, G)
    held = torch.full((need + 64,), 255, dtype=torch.uint8, device=dev())
    offsets = torch.full((G + 3,), -9, dtype=torch.int32, device=dev())
    order = torch.full((m + 2,), -9, dtype=torch.int32, device=dev())
    on_gpu = [None if a is None else torch.from_numpy(a.astype(np.int32)).to(dev()) for a in (group_of, rows)]
    epp.epp_group_rows(on_gpu[0], G, offsets[1:G + 2], order[1:m + 1], held[:need], rows=on_gpu[1])
    want_offsets, want_order = oracle(group_of, G, rows)
    assert np.array_equal(offsets[1:G + 2].cpu().numpy(), want_offsets)
    assert np.array_equal(order[1:m + 1].cpu().numpy(), want_order)
    assert offsets[0] == -9 and offsets[G + 2] == -9 and order[0] == -9 and order[m + 1] == -9 and (held[need:] == 255).all()


@pytest.mark.parametrize("G", [1, 2, 8, 63, 64, 65, 512, 513, 2048])
@pytest.mark.parametrize("m", [0, 1, 2, 63, 64, 65, 1023, 1025, 4097, 8191, 8192, 8193, 50_000])
def test_sizes(m, G):
    rng = np.random.default_rng(m + G)
    check(rng.integers(-1, G + 1, size=m), G)
    check(np.sort(rng.integers(0, G, size=m)), G)
    check(np.full(m, G - 1), G)


@pytest.mark.parametrize("m", [5, 8192, 70_001])
def test_lists(m):
    """Rows of a larger array, out of order and twice, rows that do not exist, numbers that are no group's."""
    rng = np.random.default_rng(m)
    group_of = rng.integers(-3, 20, size=100_000)
    group_of[::17] = -2 ** 31
    group_of[1::19] = 2 ** 31 - 1
    rows = rng.integers(-2, 100_003, size=m)
    rows[0] = 2 ** 31 - 1
    check(group_of, 13, rows)
    check(group_of, 13, np.sort(rng.choice(100_000, size=m, replace=False)))
    check(np.zeros(0, np.int64), 13, rows)  # (no rows at all: every entry is in no group)


def test_many():
    rng = np.random.default_rng(5)
    check(rng.integers(0, 300, size=3_000_001), 300)
    check(rng.integers(0, 2048, size=2_500_000), 2048)
