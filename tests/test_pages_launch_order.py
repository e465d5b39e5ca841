"""The kernels on pages and drafts are launched while their predecessors drain, so each waits for its predecessor in every
thread before it touches memory, and nothing leaves before (see test_kv_launch_order.py).  Checked in the sources."""
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_15763_b200", "csrc")


def kernels(name):
    text = re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())
    assert "<<<" not in text
    found = {}
    for m in re.finditer(r"__global__[^{]*?\b(k_[a-z_]+)\s*\(", text):
        at = text.index("{", m.end())
        depth, end = 0, at
        while True:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
            if depth == 0:
                break
        found[m.group(1)] = text[at + 1:end - 1]
    return found


ALL = {k: body for f in ("hos_pages.cu", "hos_drafts.cu") for k, body in kernels(f).items()}


def test_the_kernels_are_found():
    assert sorted(ALL) == ["k_kv_compact", "k_kv_copy_pages", "k_kv_fork", "k_kv_resize", "k_verify_drafts"]


@pytest.mark.parametrize("kernel", sorted(ALL))
def test_a_kernel_waits_before_anything_else(kernel):
    before, found, after = ALL[kernel].partition("\n    pdl_wait();\n")
    assert found and "pdl_wait" not in after
    assert not re.search(r"p\.|\bc\.|\bd\.|\breturn\b|cp_async|atomic|__ldg|cluster_sync", before)
