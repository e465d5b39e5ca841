"""The files of the calls on pages and drafts do not count for the recorded counters of the scheduling kernels; a new source of those would."""
import os
import re
import shutil

import pytest

from paper_2502_15763_b200 import _build


@pytest.mark.parametrize("name,counts", [("hos_pages.cu", False), ("hos_pages_api.cu", False), ("hos_pages_kernels.h", False), ("hos_drafts.cu", False),
                                         ("hos_cluster.cuh", False), ("hos_another.cu", True), ("hos_another.cuh", True)])
def test_which_files_count(name, counts, tmp_path, monkeypatch):
    shutil.copytree(_build.CSRC, tmp_path / "csrc")
    monkeypatch.setattr(_build, "CSRC", str(tmp_path / "csrc"))
    before = _build.source_hash()
    assert os.path.exists(tmp_path / "csrc" / name) != name.startswith("hos_another")
    with open(tmp_path / "csrc" / name, "a") as fh:
        fh.write("\n// another line\n")
    assert (_build.source_hash() != before) == counts


def test_no_file_that_does_not_count_has_a_scheduling_kernel():
    """What is left out by name launches and declares none of the kernels that the counters are of."""
    import json
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    kernels = json.load(open(os.path.join(root, "profiles", "ncu_counters_c4x296.json")))["kernels"]
    assert len(kernels) > 5
    for name in os.listdir(_build.CSRC):
        if name.startswith(("hos_kv", "hos_attn", "hos_pages", "hos_drafts", "hos_cluster")):
            text = open(os.path.join(_build.CSRC, name)).read()
            assert not [k for k in kernels if k in text], name
        else:                                                    # and what counts takes nothing from there
            text = open(os.path.join(_build.CSRC, name)).read()
            assert not re.search(r'#include "hos_(kv|attn|pages|drafts|cluster)', text), name
