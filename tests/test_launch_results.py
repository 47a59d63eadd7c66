"""A kernel that takes its work list from the one before it is launched only if that one was."""
import os
import re

import pytest

from paper_2605_16928_b200 import build


@pytest.mark.parametrize("name", ["attn_chunks.cu", "beam.cu", "pages.cu", "rope_append.cu"])
def test_every_launch_is_asked_for_its_result(name):
    """The statement behind a launch takes its error; the one behind that returns it, unless the first has."""
    with open(os.path.join(build.CSRC, name)) as f:
        text = re.sub(r"//[^\n]*", "", f.read())
    launches = list(re.finditer(r"\(void\)launch_chained\([^;]*;", text))
    assert launches
    for m in launches:
        rest = re.sub(r"\s+", " ", text[m.end():m.end() + 200]).strip()
        assert re.match(r"(return cudaGetLastError\(\);|(cudaError_t )?e = cudaGetLastError\(\); if \(e != cudaSuccess)", rest), (name, m.group(0)[:80], rest[:80])
