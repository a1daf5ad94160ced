"""Loads that go straight into LDS take their base from M0, which has to be
written a wait state before them.  The compiler sees to that for its own, not
inside an asm statement: there the sources have to."""
import glob
import os
import re

from paper_2609_00865_amd import build

WRITES = re.compile(r"^s_\w+\s+m0\s*,")
LOADS = re.compile(r"^(global_load_lds_|buffer_load_\w+ .*\blds\b|scratch_load_lds_)")


def statements(text):
    """The instructions of every asm statement of a source."""
    for m in re.finditer(r"\basm\b\s*(?:volatile)?\s*\(", text):
        at, parts = m.end(), []
        while True:
            s = re.compile(r'\s*"((?:[^"\\]|\\.)*)"').match(text, at)
            if s is None:
                break
            parts.append(s.group(1))
            at = s.end()
        yield [x.strip() for x in re.split(r"(?:\\n|\\t|;)+", "".join(parts)) if x.strip()]


def test_m0_is_written_a_state_before_it_is_used():
    loads = 0
    for path in sorted(glob.glob(os.path.join(build.CSRC, "*"))):
        for insts in statements(open(path).read()):
            for i, x in enumerate(insts):
                if LOADS.match(x):
                    loads += 1
                    assert i == 0 or not WRITES.match(insts[i - 1]), (path, insts)
    assert loads > 6
