"""The kernels of the operators on groups and on gradients, from the compiler's report (CPU only), and their entry points with tensors that
PyTorch cannot give sizes for."""
import re
import subprocess
import sys
from concurrent.futures import ThreadPoolExecutor
from pathlib import Path

import pytest

ROOT = Path(__file__).resolve().parent.parent
CSRC = ROOT / "paper_2204_02662_amd" / "csrc"
FILES = ("epp_grouped", "epp_grouped_narrow", "epp_grouped_few", "epp_group_rows", "epp_gradients")


@pytest.fixture(scope="module")
def compiled(tmp_path_factory):
    """{file: (remarks, assembly)}"""
    d = tmp_path_factory.mktemp("grouped")

    def one(f):
        out = subprocess.run(
            ["hipcc", "--offload-arch=gfx950", "-O3", "-std=c++17", "-fPIC", "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops",
             f"-I{ROOT / 'include'}", f"-I{CSRC}", "--cuda-device-only", "-S", str(CSRC / (f + ".hip")), "-o", f"{f}.s",
             "-Rpass-analysis=kernel-resource-usage"], cwd=d, capture_output=True, text=True, timeout=900)
        assert out.returncode == 0, out.stderr[-3000:]
        return f, (out.stderr, (d / f"{f}.s").read_text())

    with ThreadPoolExecutor(4) as pool:
        return dict(pool.map(one, FILES))


def test_no_scratch_memory(compiled):
    for f, (remarks, _) in compiled.items():
        found = [int(x) for x in re.findall(r"ScratchSize \[bytes/lane\]: (\d+)", remarks)]
        assert found and max(found) == 0, (f, found)


def test_no_waits_for_operand_loads_within_a_tile(compiled):
    """The loop over a tile of 256 x 256: the only wait for vector memory is the one where the wavefronts meet, and nothing that the
    compiler loads itself is in it.  (Its transposing LDS reads wait for loads to LDS that it knows of: these are written out.)"""
    _, asm = compiled["epp_grouped"]
    checked = 0
    for m in re.finditer(r"^(_ZN\S*k_grouped_rowsI(?:DF16b|DF16_)Li[01]ELi2ELi4ELi4ELi2ELb1ELb1E\S*):(.*?)^\.Lfunc_end", asm, re.S | re.M):
        lines, labels, loops = [x.strip() for x in m.group(2).split("\n")], {}, []
        for i, x in enumerate(lines):
            if k := re.match(r"(\.LBB\S+):", x):
                labels[k.group(1)] = i
            elif (k := re.match(r"s_c?branch\S* (\.LBB\S+)", x)) and k.group(1) in labels:
                loops.append(lines[labels[k.group(1)]:i])
        loops = [b for b in loops if sum("v_mfma" in x for x in b) == 32 and sum("global_load_lds" in x for x in b) == 8
                 and not any(re.match(r"\.LBB", x) for x in b[1:])]
        assert loops, m.group(1)
        for b in loops:
            assert sum("vmcnt" in x for x in b) == 1 and sum("s_barrier" in x for x in b) == 1, m.group(1)
            assert not any(re.match(r"(global|flat|scratch|buffer)_load_(?!lds)", x) for x in b), m.group(1)
            checked += 1
    assert checked >= 4


def test_scalar_loads_from_tables_have_whole_addresses(compiled):
    """Scalar loads drop the lowest bits of their base and of their offset, each for itself: both have to be multiples of four.  Every
    base that the compiler adds up is the arguments' address plus a multiple of a record's size (or nothing to do with the tables)."""
    _, asm = compiled["epp_gradients"]
    for m in re.finditer(r"^(_ZN\S*(?:k_few|k_squares|k_scale)\S*):(.*?)^\.Lfunc_end", asm, re.S | re.M):
        lines = [x.strip() for x in m.group(2).split("\n")]
        # numbers that are a table's place: products with a record's size
        sizes = {int(k.group(1), 0) for x in lines if (k := re.match(r"s_mul_i32 s\d+, s\d+, (0x[0-9a-f]+|\d+)", x))}
        assert sizes and all(s % 8 == 0 for s in sizes), (m.group(1), sizes)


SCRIPT = """
import torch
from torch._subclasses.fake_tensor import FakeTensorMode
from torch.fx.experimental.symbolic_shapes import ShapeEnv
import paper_2204_02662_amd as epp

env = ShapeEnv()
with FakeTensorMode(shape_env=env):
    n = env.create_unbacked_symint()
    t, W = torch.empty((n, 3), device="cuda"), torch.empty((2, 3, 3), device="cuda")
    i, o = torch.empty((n,), dtype=torch.int32, device="cuda"), torch.empty(3, dtype=torch.int32, device="cuda")
    b, s = torch.empty(1 << 20, dtype=torch.uint8, device="cuda"), torch.empty(1, device="cuda")
for call in (lambda: epp.epp_group_rows(i, 2, o, i, b), lambda: epp.epp_grouped_product(t, W, o, t), lambda: epp.epp_grouped_input_gradient(t, W, o, t),
             lambda: epp.epp_grouped_weight_gradient(t, t, o, W, b), lambda: epp.epp_gradient_norm([t], s, b), lambda: epp.epp_clip_gradients([t], 1.0, s, b),
             lambda: epp.epp_clip_gradients([W], 1.0, s, b, out=[t])):
    try:
        call()
    except Exception:
        continue
    raise SystemExit("a tensor without sizes was accepted")
print("all refused")
"""


def test_tensors_of_unknown_shape_are_refused():
    from paper_2204_02662_amd import build
    if not build.BINDING.exists():
        pytest.skip("binding not built")
    out = subprocess.run([sys.executable, "-c", SCRIPT], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert out.returncode == 0 and "all refused" in out.stdout, out.stdout[-500:] + out.stderr[-2000:]
