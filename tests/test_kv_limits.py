"""Limits of the KV-cache calls that are checked on the host, before any CUDA call."""
import ctypes as C

import pytest

import paper_2502_15763_b200 as hos
from paper_2502_15763_b200.kv_cache import _KvBatch, _KvCache
from tests.test_kv_abi import BATCH, GOOD


@pytest.mark.parametrize("heads,code", [(65535 * 16 + 1, -4), (1 << 20, -4), (1 << 26, -4)])
def test_more_kv_heads_than_a_launch_grid_holds(heads, code):
    """Append and read give 16 heads to a block and have 65,535 blocks for that."""
    c, b = _KvCache(**{**GOOD, "n_kv_heads": heads}), _KvBatch(**BATCH)
    assert hos.lib().hos_kv_append(C.byref(c), C.byref(b), 4096, 4096, 64, 64, 64, 64, None, None) == code
    assert hos.lib().hos_kv_read(C.byref(c), C.byref(b), 4096, 4096, None, None) == code
