"""Instructions written out in the sources (CPU only)."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2204_02662_amd" / "csrc"


def statements():
    for f in sorted(CSRC.glob("*")):
        if f.suffix in (".hip", ".h"):
            for m in re.finditer(r"\basm\b[^(;]*\(((?:\"(?:\\.|[^\"\\])*\"|[^\";])*)\)\s*;", f.read_text()):
                yield f.name, m.group(1)


def test_registers_that_are_written_are_named():
    """A register that a statement writes by its own name is among those that the compiler is told of: it may hold something there."""
    found = 0
    for name, text in statements():
        code, *lists = re.split(r":(?=(?:[^\"]*\"[^\"]*\")*[^\"]*$)", text)
        written = set(re.findall(r"\b[sv]_\w+ (m0|vcc|exec|[sv]\d+)\b", code))
        told = set(re.findall(r"\"([^\"]+)\"", lists[2])) if len(lists) > 2 else set()
        assert written <= told, (name, text)
        found += bool(written)
    assert found >= 3
