"""What the HIP sources have to keep as one program (CPU)."""
import os
import re

import paper_2502_00340_amd as P

CSRC = os.path.join(os.path.dirname(P.__file__), "csrc")


def test_types_have_one_definition():
    """The sources share a namespace: a type of one name is one type, or the program has none."""
    where = {}
    for f in sorted(os.listdir(CSRC)):
        with open(os.path.join(CSRC, f)) as src:
            for m in re.finditer(r"^(?:struct|class|union|enum(?: class)?) (\w+)(?: final)?(?: : [^;{]+)? \{", src.read(), re.M):
                where.setdefault(m[1], set()).add(f)
    assert len(where) > 20
    assert {n: sorted(fs) for n, fs in where.items() if len(fs) > 1} == {}
