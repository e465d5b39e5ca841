"""What a set of recorded profiler counters is held to: every source of the scheduling kernels, their headers included."""
import os
import shutil

import pytest

from paper_2502_15763_b200 import _build


@pytest.mark.parametrize("name,counts", [("include/hos.h", True), ("csrc/hos_common.cuh", True), ("csrc/hos_kernels.h", True),
                                         ("csrc/hos_online.cu", True), ("csrc/hos_api.cu", True), ("csrc/hos_kv_cache.cu", False),
                                         ("csrc/hos_attn_rows.cu", False), ("csrc/hos_kv.cuh", False), ("csrc/hos_kv_kernels.h", False)])
def test_which_files_count(name, counts, tmp_path, monkeypatch):
    shutil.copytree(_build.CSRC, tmp_path / "csrc")
    shutil.copytree(_build.INCLUDE, tmp_path / "include")
    monkeypatch.setattr(_build, "CSRC", str(tmp_path / "csrc"))
    monkeypatch.setattr(_build, "INCLUDE", str(tmp_path / "include"))
    before = _build.source_hash()
    assert os.path.exists(tmp_path / name)
    with open(tmp_path / name, "a") as fh:
        fh.write("\n// another line\n")
    assert (_build.source_hash() != before) == counts
