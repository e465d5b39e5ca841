"""The compiled half of kv_cache.py belongs to one torch and one interpreter."""
import importlib.metadata
import os
import sysconfig

import torch

import paper_2502_15763_b200 as hos
from paper_2502_15763_b200 import _build


def test_the_module_is_the_one_of_this_torch_and_interpreter():
    path = _build.build_binding()
    assert torch.__version__ in os.path.basename(path) and path.endswith(sysconfig.get_config_var("EXT_SUFFIX"))
    assert os.path.samefile(hos.kv_cache.binding().__file__, path)


def test_a_module_of_another_torch_is_not_taken(monkeypatch):
    mine = _build.build_binding()
    monkeypatch.setattr(importlib.metadata, "version", lambda name: "0.0.1")
    assert _build.binding_path() != mine and not os.path.exists(_build.binding_path())
