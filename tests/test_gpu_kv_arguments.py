"""Tensors of unusual strides, sizes and origins as arguments of the KV-cache calls."""
import math

import pytest
import torch

from tests import kv_reference as R
from tests.test_gpu_kv_cache import make_cache

pytestmark = pytest.mark.gpu


def hos():
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    import paper_2502_15763_b200 as h
    return h


def test_pages_that_overlap_are_refused():
    """An expanded page has the stride 0, which the C interface takes for densely packed pages: memory past the tensor."""
    h = hos()
    k, v, ks, vs = make_cache(4, 2, 16, 64, torch.bfloat16, "int8", 1)
    same, same_v = (torch.zeros((4, 2, 16, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for bad, bad_v in ((same[:1].expand(4, -1, -1, -1), same_v[:1].expand(4, -1, -1, -1)),
                       (same.as_strided((4, 2, 16, 64), (1024, 1024, 64, 1)), same_v.as_strided((4, 2, 16, 64), (1024, 1024, 64, 1)))):
        with pytest.raises(ValueError, match="overlap"):
            h.hos_kv_cache(bad, bad_v)
    with pytest.raises(ValueError, match="overlap"):
        h.hos_kv_cache(k, v, ks[:1].expand(4, -1, -1), vs[:1].expand(4, -1, -1), dtype=torch.bfloat16)
    # one page has no neighbour to overlap with
    h.hos_kv_cache(same[:1].expand(1, -1, -1, -1), same_v[:1])
