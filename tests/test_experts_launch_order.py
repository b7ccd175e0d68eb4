"""Kernels of the expert layer are scheduled while the kernel before them still runs. What that one and those before it wrote is
promised to be visible only behind a kernel's own wait, so every kernel makes it always, once, and before it touches global
memory. Read from the sources: a kernel that breaks this gives wrong results now and then at most."""
import os
import re

import pytest

from paper_2604_23996_gb300.build import CSRC

SOURCES = sorted(f for f in os.listdir(CSRC) if f.startswith("expert_") and f.endswith(".cu"))
GLOBAL = re.compile(r"__ldg\(|__ldcg\(|tma_load|tma_store|tma_add|count_row_tiles\(|expert_begin\(|zero_rows\(|atomic\w+\(p\.")


def kernels(text):
    """(name, body) of every kernel."""
    for m in re.finditer(r"__global__[^;{]*?(k_\w+)\(", text):
        at = text.index("{", m.end())
        depth, i = 0, at
        while True:
            depth += {"{": 1, "}": -1}.get(text[i], 0)
            i += 1
            if depth == 0:
                break
        yield m.group(1), text[at:i]


@pytest.mark.parametrize("source", SOURCES)
def test_every_kernel_waits_for_the_one_before_it_first(source):
    with open(os.path.join(CSRC, source)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    found = list(kernels(text))
    assert found
    for name, body in found:
        waits = [m.start() for m in re.finditer(r"\bpdl_wait\(\);", body)]
        assert len(waits) == 1, name
        before = body[:waits[0]]
        assert before.count("{") - before.count("}") == 1, f"{name}: a wait under a condition"
        assert not GLOBAL.search(before), f"{name}: {GLOBAL.search(before).group()} before the wait"
