"""Asynchronous copies into shared memory and the waits for them, read from the kernels' sources:
a wait for groups waits for copies that were committed to one, and for no others."""
import glob
import os
import re

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
COPY = r"(?<!void )\b(?:copy16|copy4|cp_async16)\("
COMMIT = r"(?<!void )\bcommit\(\);|cp\.async\.commit_group"
WAIT = r"(?<!void )\bwait_all_but<[^>]*>\(\);|cp\.async\.wait_group "


def _code(path):
    return re.sub(r"//[^\n]*", "", open(path).read())


SOURCES = [p for p in sorted(glob.glob(os.path.join(ROOT, "paper_2605_06892_gb300", "csrc", "*.cu")))
           if re.search(COPY, _code(p))]


def test_the_sources_with_copies_are_found():
    names = {os.path.basename(p) for p in SOURCES}
    assert {"hsa_paged_attention.cu", "hsa_paged_attention4.cu", "hsa_attention_f32.cu"} <= names


@pytest.mark.parametrize("path", SOURCES, ids=os.path.basename)
def test_copies_are_committed_before_a_wait(path):
    """In the order of the source: the commits that follow copies come before the next wait."""
    open_copy = None
    waits = 0
    for m in re.finditer(f"(?P<copy>{COPY})|(?P<commit>{COMMIT})|(?P<wait>{WAIT})", _code(path)):
        if m.lastgroup == "copy":
            open_copy = m.start()
        elif m.lastgroup == "commit":
            open_copy = None
        else:
            waits += 1
            assert open_copy is None, "a wait for groups after copies that are in none"
    assert waits and open_copy is None
