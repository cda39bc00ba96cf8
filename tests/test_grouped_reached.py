"""Kernels of few rows to a group that the library holds: those that some call launches (CPU only)."""
import re
import subprocess

import pytest


def test_wide_columns_of_few_rows():
    """64 columns to a workgroup from 512 of these on.  Numbers of 16 bits, and input gradients of floats of any alignment, take the larger tiles
    from 256 pairs of such column blocks on, so that they have none."""
    from paper_2204_02662_amd import build
    if not build.SO.exists():
        pytest.skip("library not built")
    out = subprocess.run(["nm", str(build.SO)], capture_output=True, text=True, timeout=60)
    assert out.returncode == 0, out.stderr
    few = set(re.findall(r"k_grouped_fewI(f|DF16_|DF16b)Li([01])ELi(\d)ELi(32|64)ELb([01])E", out.stdout))
    kinds = {(t, mode, rows, direct) for t in ("f", "DF16_", "DF16b") for mode in "01" for rows in ("124" if t != "f" else "12") for direct in "01"}
    assert {(t, mode, rows, direct) for t, mode, rows, wide, direct in few if wide == "32"} == kinds
    assert {(t, mode, rows, direct) for t, mode, rows, wide, direct in few if wide == "64"} == {
        k for k in kinds if k[0] == "f" and not (k[1] == "1" and k[3] == "0")}
