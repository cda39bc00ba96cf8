"""Entries in the order of their groups at the numbers of groups and entries where another kernel, or another way through one, begins."""
import numpy as np
import pytest

from test_gpu_group_rows import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("G", [31, 32, 33, 255, 256, 257])
@pytest.mark.parametrize("m", [1, 8_192, 8_193, 20_000])
def test_groups(m, G):
    """Up to 32 groups every block adds the counts up itself; up to 256 the single workgroup keeps a short table."""
    rng = np.random.default_rng(m + G)
    check(rng.integers(-1, G + 1, size=m), G)
    check(rng.integers(0, G, size=m), G, rng.integers(-1, m + 1, size=m))


@pytest.mark.parametrize("G", [1, 7, 32, 33])
@pytest.mark.parametrize("m", [2_097_152, 2_097_153, 3_000_001])
def test_more_entries_than_blocks_hold(m, G):
    """1,024 blocks of 2,048 entries are held in registers from their counting to their placing; larger blocks are looked up again."""
    rng = np.random.default_rng(m + G)
    check(rng.integers(-1, G + 1, size=m), G)
    check(rng.integers(-1, G + 1, size=m + 5), G, rng.integers(-1, m + 6, size=m))
