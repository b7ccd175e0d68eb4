"""Loads from tensor memory, and the wait for them, are executed by a whole warp at once. Lanes come to them out of polls, stores by
one lane and loads under a condition of their own, so each reconverges the warp itself. Read from the sources (what a warp does
that has not reconverged is not defined)."""
import os
import re

import pytest

from paper_2604_23996_gb300.build import CSRC


def source(name):
    with open(os.path.join(CSRC, name)) as f:
        return re.sub(r"//[^\n]*", "", f.read())


def functions(text):
    """(name, body) of the inline functions."""
    for m in re.finditer(r"__forceinline__ [\w<>]+ (\w+)\([^{;]*\{", text):
        depth, i = 1, m.end()
        while depth:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
        yield m.group(1), text[m.end():i - 1]


LOADS = {(f, name): body for f in sorted(os.listdir(CSRC)) for name, body in functions(source(f))
         if "tcgen05.ld.sync.aligned" in body or "tcgen05.wait::ld.sync.aligned" in body}
WAIT = ("ptx.cuh", "tmem_ld_wait")                      # the wait alone: behind a load of the same function


def test_the_loads_are_found():
    names = {name for _, name in LOADS}
    assert {"tmem_ld_wait", "tmem_ld32", "tmem_ld16", "tmem_ld_16x256b_x4", "tmem_ld_16x256b_x8", "tmem_ld_ready"} <= names
    for f in os.listdir(CSRC):                          # none outside these functions
        inside = sum(len(re.findall("tcgen05.ld|wait::ld", body)) for (g, _), body in LOADS.items() if g == f)
        assert len(re.findall("tcgen05.ld|wait::ld", source(f))) == inside, f
        assert f == WAIT[0] or "tmem_ld_wait(" not in source(f), f


@pytest.mark.parametrize("at", sorted(set(LOADS) - {WAIT}), ids="-".join)
def test_every_load_reconverges_the_warp_first(at):
    body, (f, name) = LOADS[at], at
    if "__syncwarp();" in body[:body.index("asm volatile")]:
        return
    assert f != WAIT[0]                                 # a file's own: each call may do it, in the statements before
    text = source(f)
    calls = [m.start() for m in re.finditer(rf"(?<!void ){name}\(", text)]
    assert calls and all("__syncwarp();" in text[i - 120:i] for i in calls)
