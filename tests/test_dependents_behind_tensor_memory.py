"""A kernel lets the next one's blocks in when it has its tensor memory: a dependent block beside it that came first would hold the memory and
wait for this kernel's end, which would wait for the memory."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2608_24070_b200" / "csrc"


def _allocations():
    """(file, what a function does in front of its allocation, what behind it)."""
    for path in sorted(CSRC.glob("*.cuh")):
        if path.name == "ptx.cuh":                             # (the instructions themselves)
            continue
        code = re.sub(r"//[^\n]*", "", path.read_text())
        for m in re.finditer(r"\btmem_alloc(_pair)?\(", code):
            begin, end = code.rfind("\n}\n", 0, m.start()), code.find("\n}\n", m.end())
            yield path.name, code[begin:m.start()], code[m.end():end]


def test_allocation_first():
    seen = 0
    for name, before, behind in _allocations():
        # (blocks that leave before they allocate may let others in at any time)
        early = re.sub(r"griddep_launch_dependents\(\);[^{}]*\breturn;", "", before)
        assert "griddep_launch_dependents" not in early, name
        assert "griddep_launch_dependents" in behind, name
        seen += 1
    assert seen >= 9
