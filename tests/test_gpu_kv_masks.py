"""Masks at the ends of their ranges."""
import pytest

from tests.test_gpu_kv_cache import ODD, check_attention

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("window", [2**31 - 1, 2**31 - 2, 2**30])
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_a_window_that_hides_nothing(window, causal, fmt):
    """The largest windows, also with rows before the sequence's first token (more new tokens than the cache holds)."""
    check_attention(ODD + [(9, 2), (300, 290), (40, 3)], 4, 2, 64, "bf16", fmt, 16, causal=causal, window=window, seed=31)
    check_attention([(5, 2)], 2, 2, 128, "f16", fmt, 32, causal=causal, window=window, seed=32)
