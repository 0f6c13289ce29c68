"""Inline assembly names the registers it writes itself."""

import glob
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2608_28003_amd", "csrc")


def statements():
    for path in sorted(glob.glob(os.path.join(CSRC, "**", "*"), recursive=True)):
        if path.endswith((".hip", ".h")):
            text = open(path).read()
            for m in re.finditer(r"\basm\s+volatile\s*\((.*?)\);", text, re.S):
                yield os.path.basename(path), m.group(1)


def test_assembly_that_writes_m0_says_so():
    """s_mov_b32 m0 without "m0" among the clobbered registers would let the
    compiler keep a value of its own there."""
    wrote = [(f, s) for f, s in statements() if re.search(r"s_\w+\s+m0\b", s)]
    assert wrote
    for f, s in wrote:
        assert '"m0"' in s.rsplit(":", 1)[1], (f, s)
