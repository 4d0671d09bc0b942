"""The paged window memory at the largest lengths that the header allows and the
card holds."""
import math

import pytest

pytestmark = pytest.mark.gpu


def i32(x):
    import torch
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def test_a_sequence_of_more_than_two_to_the_28_tokens():
    """Keys of zero, so that every visible key weighs exactly 1: the output's elements are the shares of the keys whose
    value is 1 there, among them the newest and the oldest half million.  Sums of ones are exact below 2^24, which the
    about 2^19 keys of a workgroup stay; joining at most 1024 parts rounds numerator and denominator by 2^-24 each time,
    2^-13 together, and the output is rounded to bf16 by 2^-8."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    base, P, D = 1 << 28, 65536, 64
    c = PagedCache(seqs=2, pages=base // P + 3, page_tokens=P, heads=1, head_dim=D, max_tokens=base + 1000, max_rows=1 << 23)
    held, news = 0, 1 << 19
    while held < base:
        c.plan(i32([held, 0]), i32([1 << 23, 0]), rows=1 << 23, max_new=1 << 23)
        held += 1 << 23
    pages = c.pages()
    pages.zero_()
    v = pages[:, 1, 0]  # page t // P holds token t: the sequence took the lowest ones, in order
    assert c.table[0, :base // P].tolist() == list(range(base // P))
    v[(base - news) // P: base // P, :, 0] = 1.0
    v[:news // P, :, 1] = 1.0
    v[(base >> 1) // P: (base >> 1) // P + 16, :, 2] = 1.0
    v[..., 3] = 1.0
    for new, what in (([40, 0], "one tile, shared by every workgroup"), ([50, 60], "a short sequence beside it"),
                      ([1, 0], "one token"), ([1, 1], "one token of both")):
        print("long", what, flush=True)
        before = [int(x) for x in c.held]
        rows = sum(new)
        c.plan(i32(before), i32(new), rows=rows, max_new=max(new))
        assert c.status.tolist() == [0, 0]
        k = torch.zeros((rows, 1, D), device="cuda", dtype=torch.bfloat16)
        x = torch.zeros_like(k)
        x[..., 0] = x[..., 3] = 1.0
        c.insert(k, x)
        lse = torch.zeros((1, rows), device="cuda")
        out = c.attend(torch.ones_like(k), lse=lse).double()[:, 0]
        n = torch.arange(before[0] + 1, before[0] + new[0] + 1, device="cuda", dtype=torch.float64)
        want = torch.zeros((new[0], D), device="cuda", dtype=torch.float64)
        want[:, 0], want[:, 1], want[:, 2], want[:, 3] = (n - (base - news)) / n, news / n, 16 * P / n, 1.0
        assert bool(((out[:new[0]] - want).abs() <= want * (2.0**-8 + 2.0**-12)).all()), (out[0, :4], want[0, :4])
        assert bool(((lse[0, :new[0]].double() - n.log()).abs() <= 2.0**-12 + 2.0**-22 * math.log(base)).all())
        assert bool((out[new[0]:, [0, 3]] == 1.0).all()) and bool((out[new[0]:, 1:3] == 0.0).all())
