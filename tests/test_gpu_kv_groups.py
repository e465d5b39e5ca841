"""One KV head for many query heads: groups above the row kernel's 16 rows, whose queries and outputs are boxes of up to 128 heads (where
the group divides, or is divided by, what a box holds) or come and go row by row (where not); and the batches of serving and prefill
that have no other test at size: whole prompts on 8-bit caches, chunks behind a long context on a 16-bit cache, grouped decodes."""
import pytest

from tests.test_gpu_kv_cache import check_attention

pytestmark = pytest.mark.gpu

GROUPS = [17, 20, 24, 32, 48, 64, 96, 100, 128, 192, 256]


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("fmt", ["same", "e4m3", "int8"])
def test_single_tokens_of_large_groups(group, fmt):
    check_attention([(1, 1 + 173 * s) for s in range(9)], group, 1, 128, "bf16", fmt, 16, seed=group)
    check_attention([(1, 4000), (1, 0), (1, 65)], 2 * group, 2, 64, "f16", fmt, 64, window=900, seed=group + 1)


@pytest.mark.parametrize("group", GROUPS)
@pytest.mark.parametrize("fmt", ["same", "int8"])
def test_prompts_of_large_groups(group, fmt):
    check_attention([(130, 130), (5, 700), (1, 300), (0, 4), (33, 33), (7, 2)], group, 1, 128, "f16", fmt, 32, seed=group)
    check_attention([(40, 90), (2, 500), (3, 3)], 2 * group, 2, 64, "bf16", fmt, 16, strided=True, interleaved=True, seed=group + 1)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_whole_prompts_on_8_bit_caches(fmt):
    check_attention([(2048, 2048), (1500, 1500), (33, 33)], 16, 2, 128, "bf16", fmt, 128, seed=41)
    check_attention([(1024, 1024)] * 3, 8, 8, 64, "f16", fmt, 16, seed=42)


@pytest.mark.parametrize("dt,d", [("bf16", 128), ("f16", 64)])
def test_chunks_behind_a_long_context_on_a_16_bit_cache(dt, d):
    check_attention([(509, 16500), (64, 9000)], 16, 2, d, dt, "same", 64, seed=43)
    check_attention([(509, 16500), (64, 9000)], 16, 2, d, dt, "same", 32, window=4000, seed=44)


@pytest.mark.parametrize("group", [2, 4, 5, 8, 16])
def test_grouped_decodes_on_a_16_bit_cache(group):
    check_attention([(1, 200 + 211 * s) for s in range(32)], 4 * group, 4, 128, "bf16", "same", 16, seed=group)
