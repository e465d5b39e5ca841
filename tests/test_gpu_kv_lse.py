"""lse of rows whose scores are next to nothing, on 8-bit caches: the scales in the weights' exponents leave no rounding behind.  Every way
that a row may end: a whole tile or a split one, of few rows or many."""
import pytest

from tests.test_gpu_kv_cache import check_attention

pytestmark = pytest.mark.gpu

SHAPES = {"rows": [(1, 1), (1, 25), (3, 180), (1, 300), (2, 900)], "split rows": [(1, 12709), (1, 9000)],
          "tiles": [(60, 60), (130, 700), (33, 33), (200, 215)], "split tiles": [(300, 9000)], "mixed": [(1, 2000), (1, 9), (30, 411), (81, 85)]}


@pytest.mark.parametrize("shape", SHAPES)
@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
@pytest.mark.parametrize("dt,d", [("f16", 64), ("bf16", 128)])
@pytest.mark.parametrize("window", [0, 1, 43])
def test_lse_of_flat_scores(shape, fmt, dt, d, window):
    check_attention(SHAPES[shape], 24, 8, d, dt, fmt, 32, window=window, sm_scale=0.0, seed=61)
    check_attention(SHAPES[shape], 24, 8, d, dt, fmt, 16, window=window, q_gain=0.01, seed=62)
