"""Dynamic shared memory starts where the static part ends, aligned as its array is declared and no further: kernels that read it 16 bytes
at a time, or copy into it asynchronously, have to say so, or to round the address up themselves."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2409_04992_b200" / "csrc"
ONE_AT_A_TIME = {("kv_pages_kernels.cuh", "plan_smem")}          # 32-bit counters, read and written singly


def test_every_dynamic_array_is_aligned():
    seen = 0
    for path in sorted(CSRC.iterdir()):
        text = path.read_text()
        for found in re.finditer(r"extern __shared__ (__align__\((\d+)\) )?[\w ]+ (\w+)\[\];", text):
            seen += 1
            aligned = found.group(2) is not None and int(found.group(2)) >= 16
            rounded = re.search(r"__cvta_generic_to_shared\(%s\)\);\s*const unsigned \w+ = \(raw \+ \d+u\) & ~\d+u;" % found.group(3), text)
            assert aligned or rounded or (path.name, found.group(3)) in ONE_AT_A_TIME, (path.name, found.group(0))
    assert seen >= 12
