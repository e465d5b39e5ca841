"""The KV-cache kernels are launched while their predecessors drain.  What keeps them in order is that each waits for its
predecessor in every thread before it touches memory and on every way out: then the end of a kernel implies the end of all
before it, whatever fits on the device beside what.  The row kernel beside the chunk kernel waits at its end only, so the
chunk kernel may let it start only after its own wait.  Checked in the sources; what a missing wait does depends on timing."""
import glob
import os
import re

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2502_15763_b200", "csrc")
FILES = sorted(os.path.basename(f) for f in glob.glob(os.path.join(CSRC, "hos_kv*.cu")) + glob.glob(os.path.join(CSRC, "hos_attn*.cu")))


def source(name):
    return re.sub(r"//[^\n]*", "", open(os.path.join(CSRC, name)).read())


def kernels(name):
    text = source(name)
    for m in re.finditer(r"__global__[^{]*?\b(k_[a-z_]+)\s*\(", text):
        at = text.index("{", m.end())
        depth, end = 0, at
        while True:
            depth += {"{": 1, "}": -1}.get(text[end], 0)
            end += 1
            if depth == 0:
                break
        yield m.group(1), text[at + 1:end - 1]


ALL = {k: (f, body) for f in FILES for k, body in kernels(f)}
MEMORY = r"__ldg|\blds<|load_seq|find_place|load16|\.total\(|\.locate\(|\bmeta\[|\bstate\[|cp_async|bar_init|atomic|\breturn\s*;"


def test_the_kernels_are_found():
    assert sorted(ALL) == ["k_attn_chunk", "k_attn_combine", "k_attn_rows", "k_kv_append", "k_kv_read"]


@pytest.mark.parametrize("kernel", ["k_attn_chunk", "k_attn_combine", "k_kv_append", "k_kv_read"])
def test_a_kernel_waits_before_anything_else(kernel):
    before, found, after = ALL[kernel][1].partition("\n    pdl_wait();\n")
    assert found and "pdl_wait" not in after
    assert not re.search(MEMORY, before)


def test_the_chunk_kernel_signals_after_its_wait():
    body = ALL["k_attn_chunk"][1]
    assert body.count("pdl_launch_dependents();") == 1 and body.index("\n    pdl_wait();\n") < body.index("pdl_launch_dependents();")


def test_the_row_kernel_waits_first_or_beside_the_chunk_kernel_last():
    body = ALL["k_attn_rows"][1]
    before, found, after = body.partition("\n    if (beside) __threadfence();\n    else pdl_wait();\n")
    assert found and not re.search(MEMORY, before.replace("warp_state[", ""))
    # the early way out, and the end
    way_out = re.search(r"if \(w >= active\) \{(.*?)return;", after, re.S).group(1)
    assert way_out.rstrip().endswith("pdl_wait();")
    assert after.rstrip().endswith("pdl_wait();")
    assert len(re.findall(r"\breturn;", after.split("auto begin")[0])) == 1


def test_beside_means_right_after_the_chunk_kernel():
    api = source("hos_kv_api.cu")
    chunk, rows = api.index("launch_attn_chunk(a,"), api.index("launch_attn_rows(a,")
    assert chunk < rows and not re.search(r"launch_(?!attn_rows)\w+\(", api[chunk + 10:rows])
    # `beside` is `chunks`, under which the chunk kernel was launched
    assert re.search(r"if \(chunks && \(rc = cuda_rc\(launch_attn_chunk", api)
    assert re.search(r"launch_attn_rows\(a, c->type, c->format, tile, chunks \? tile : 0x7FFFFFFF, chunks, w\.rows", api)


def test_no_other_kind_of_launch():
    for name in FILES:
        assert "<<<" not in source(name), name
