"""Kernels that may start before their predecessors have ended (programmatic launches) must not read what those write
by read-only loads: lengths, block tables and row lists change between two calls of one stream, and the pool calls
and the sparse chain write them with the next kernel already waiting."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2409_04992_b200" / "csrc"
# The transposed key pool is written by ordinary launches only, which the next kernel does not overlap.
ALLOWED = {("sparf_kernels.cuh", "__ldg(reinterpret_cast<const uint4 *>(kt + (int64_t)ss.dim[t] * T))")}


def test_only_what_no_overlapped_kernel_writes_is_read_as_constant():
    found = set()
    for path in sorted(CSRC.iterdir()):
        text = re.sub(r"//[^\n]*", "", path.read_text())
        for line in text.splitlines():
            if "__ldg" in line or re.search(r"ld\.global[.\w]*\.nc", line) or "__restrict__" in line:
                found.add((path.name, line.strip()))
    stray = {(name, line) for name, line in found if not any(name == n and part in line for n, part in ALLOWED)}
    assert not stray, stray
