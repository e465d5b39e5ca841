"""The smoke pass runs every kernel of an iteration: scheduling, cache, attention."""
import pytest

pytestmark = pytest.mark.gpu


def test_smoke_launches_every_kind_of_kernel(capsys):
    import torch
    import __graft_entry__ as entry
    import paper_2502_15763_b200 as hos
    names = set()
    keep = hos.hos_set_launch_hook(lambda name, phase, stream, user: names.add(name.decode()))
    try:
        entry.smoke()
        torch.cuda.synchronize()
    finally:
        hos.hos_set_launch_hook(None)
    del keep
    assert {"k_lpt", "k_local_search", "k_simulate", "k_kv_append", "k_kv_read", "k_attn_rows", "k_attn_chunk", "k_attn_combine"} <= names
    assert capsys.readouterr().out.count("smoke ok") == 2
