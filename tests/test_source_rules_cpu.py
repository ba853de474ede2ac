"""Rules of the kernel sources that no run can show safely: what a broken one costs is a hung GPU."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2405_14366_b200", "csrc")


def kernels(text):
    """(name, body) of every __global__ function of a source file, comments removed."""
    text = re.sub(r"//[^\n]*", "", re.sub(r"/\*.*?\*/", "", text, flags=re.S))
    for m in re.finditer(r"__global__\s+void\b", text):
        at = text.index("{", m.end())
        name = [x for x in re.findall(r"(\w+)\s*\(", text[m.end():at]) if x != "__launch_bounds__"][0]
        depth, end = 1, at + 1
        while depth:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
        yield name, text[at:end]


def users():
    for f in sorted(os.listdir(CSRC)):
        if f.endswith(".cu"):
            with open(os.path.join(CSRC, f)) as src:
                for name, body in kernels(src.read()):
                    if "tmem_alloc(" in body:
                        yield pytest.param(body, id=name)


def test_the_kernels_are_found():
    assert {p.id for p in users()} >= {"prefill_merge_kernel", "layer_observe_kernel", "layer_observe_short_kernel"}


@pytest.mark.parametrize("body", list(users()))
def test_tensor_memory_is_taken_behind_the_wait(body):
    """A grid that held tensor memory while it waits for the grid ahead could keep it from a CTA of that grid which has
    let dependents start but not allocated yet: neither would ever go on."""
    assert body.count("tmem_alloc(") == 1 and body.count("grid_dep_wait()") == 1
    assert body.index("grid_dep_wait()") < body.index("tmem_alloc(")
