"""A warp that copies meets at full-warp barriers inside every copy.  Its waits are bounded by the clock and may run out for some lanes and
not for others, so each wait's answer has to be the warp's before a copy: lanes that went on alone would wait there for the others."""
import re
from pathlib import Path

CSRC = Path(__file__).resolve().parent.parent / "paper_2409_04992_b200" / "csrc"


def copying_parts(text):
    """From each heading of a copying warp to the next warp's."""
    headings = [(m.start(), m.group(1)) for m in re.finditer(r"// =+ ([^=\n]*) =+\n", text)]
    ends = [at for at, _ in headings[1:]] + [len(text)]
    return [text[at:end] for (at, title), end in zip(headings, ends) if title.startswith("copies")]


def test_every_wait_before_a_copy_is_decided_by_the_warp():
    for name, parts in (("latent_pair_kernels.cuh", 2), ("latent_kernels.cuh", 1)):
        found = copying_parts((CSRC / name).read_text())
        assert len(found) == parts
        for part in found:
            waits = [m.start() for m in re.finditer(r"tree_wait\(", part)]
            assert waits
            for at in waits:
                before = part[:at].rstrip()
                # (void: a warp that has given up waits for its copies in flight and copies no more)
                assert before.endswith("__all_sync(0xffffffffu,") or before.endswith("(void)"), (name, part[at - 60:at + 60])
