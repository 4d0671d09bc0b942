"""Calls of the paged window memory at the edges of what its header promises."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


@pytest.mark.parametrize("rope", [False, True])
def test_insertion_of_another_step_writes_nothing(rope):
    """A replayed insertion after a plan of the same rows whose longest sequence is another: its keys and values are
    another step's, and stay out of this one's pages."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    from paper_2606_10671_amd.rotary import Rotary
    c = PagedCache(seqs=2, pages=60, page_tokens=16, heads=4, kv_heads=2, head_dim=64, max_tokens=400, max_rows=100)
    c.pages().zero_()
    k, v = (torch.randn((100, 2, 64), device="cuda").bfloat16() for _ in range(2))
    rot = Rotary(64, (12, 10, 10)) if rope else None
    c.plan(i32([0, 0]), i32([60, 40]), rows=100, max_new=60)
    c.insert(k, v, rotary=rot)
    want = c.pages().clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.insert(k, v, rotary=rot)
    for new, most in (([1, 2], 2), ([99, 1], 99), ([60, 40], 61), ([60, 40], 100)):
        c.plan(i32([0, 0]), i32(new), rows=100, max_new=most)
        c.pages().zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert int(torch.count_nonzero(c.pages())) == 0, (new, most)
    c.plan(i32([0, 0]), i32([0, 0]), rows=0, max_new=0)
    c.plan(i32([0, 0]), i32([60, 40]), rows=100, max_new=60)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(c.pages(), want)
