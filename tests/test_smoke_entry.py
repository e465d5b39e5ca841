"""What the smoke pass takes from the tests, and that it runs the kernels on pages and drafts."""
import ast
import os

import pytest

ENTRY = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "__graft_entry__.py")


def test_smoke_takes_no_expected_values_of_pages_and_drafts_from_the_tests():
    """The entry states them itself; all that it takes is the harness and the attention formulas."""
    taken = set()
    for node in ast.walk(ast.parse(open(ENTRY).read())):
        if isinstance(node, ast.ImportFrom) and (node.module or "").split(".")[0] == "tests":
            taken |= {a.name for a in node.names} if node.module == "tests" else {node.module.split(".")[1]}
        elif isinstance(node, ast.Import):
            taken |= {a.name for a in node.names if a.name.split(".")[0] == "tests"}
    assert taken == {"gpu_harness", "kv_reference"}


def test_the_smoke_pass_states_what_drafts_come_to():
    """Its own few lines against the statement that the other tests use."""
    import torch
    import __graft_entry__ as entry
    from tests import pages_reference as P
    for seed in range(20):
        g = torch.Generator().manual_seed(seed)
        target, draft = (torch.softmax(2.0 * torch.randn((8, 203), generator=g), -1).double() for _ in range(2))
        draft = 0.3 * target + 0.7 * draft
        tokens = [0] + torch.multinomial(draft, 1, generator=g)[:-1, 0].tolist()
        off, ua, us = [0, 4, 5, 8], torch.rand(8, generator=g).tolist(), torch.rand(3, generator=g).tolist()
        accepted, nxt, out, _ = P.verify(tokens, target, draft, off, ua, us, 203)
        assert entry.verified(tokens, target.tolist(), draft.tolist(), off, ua, us) == (accepted, nxt, out)


@pytest.mark.gpu
def test_smoke_launches_the_kernels_on_pages_and_drafts():
    import torch
    import __graft_entry__ as entry
    import paper_2502_15763_b200 as hos
    names = set()
    keep = hos.hos_set_launch_hook(lambda name, phase, stream, user: names.add(name.decode()))
    try:
        entry.smoke_pages()
        torch.cuda.synchronize()
    finally:
        hos.hos_set_launch_hook(None)
    del keep
    assert names == {"k_kv_resize", "k_kv_fork", "k_kv_compact", "k_kv_copy_pages", "k_verify_drafts"}
