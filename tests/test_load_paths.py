"""No kernel reads through the non-coherent path: a chained kernel's lifetime overlaps the one that writes what it reads."""
import os
import re

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2609_32999_b200", "csrc")


def test_no_non_coherent_loads():
    found = []
    for name in sorted(os.listdir(CSRC)):
        if name.endswith((".cu", ".cuh", ".h")):
            for n, line in enumerate(open(os.path.join(CSRC, name)), 1):
                code = line.split("//")[0]
                if re.search(r"\b__ldg\s*\(", code) or re.search(r"\bld\.global(\.\w+)*\.nc\b", code):
                    found.append("%s:%d" % (name, n))
    assert not found
