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


def filled(dtype, D, heads, kv_heads, P, lens, news, spoil, block=1, window=0, sinks=0, lse=True, seed=0):
    """A store whose sequences hold `lens` tokens and get `news`, with spoil(k, v, s, held before the step) applied to
    every sequence's keys and values; returns it with the queries and the sequences' keys and values."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    seqs = len(lens)
    c = PagedCache(seqs=seqs, pages=sum(-(-(a + b) // P) for a, b in zip(lens, news)) + 3, page_tokens=P, heads=heads,
                   kv_heads=kv_heads, head_dim=D, dtype=td, max_tokens=max(a + b for a, b in zip(lens, news)),
                   max_rows=max(sum(lens), sum(news)), block_tokens=block, window=window, sinks=sinks)
    torch.manual_seed(seed)
    kv = [[torch.randn((a + b, kv_heads, D), device="cuda").to(td) for _ in range(2)] for a, b in zip(lens, news)]
    for s in range(seqs):
        spoil(*kv[s], s, lens[s])
    if sum(lens):
        c.plan(i32([0] * seqs), i32(lens), rows=sum(lens), max_new=max(lens))
        c.insert(*(torch.cat([kv[s][w][:lens[s]] for s in range(seqs)]) for w in (0, 1)))
    c.plan(i32(lens), i32(news), rows=sum(news), max_new=max(news))
    c.insert(*(torch.cat([kv[s][w][lens[s]:] for s in range(seqs)]) for w in (0, 1)))
    assert c.status.tolist() == [0] * seqs
    return c, torch.randn((sum(news), heads, D), device="cuda").to(td), kv


def check_spoiled(c, q, kv, lens, news, block, window, sinks, lse=True):
    """Against torch in fp64: an element is NaN or infinite where a key that its row sees makes it so, and within the
    bounds of paged_parity elsewhere (A: the weighted mean of |V|; d: the error of a score)."""
    import torch
    rows, heads, D = q.shape
    bf16 = q.dtype == torch.bfloat16
    L = torch.full((heads, rows), 7.0, device="cuda") if lse else None
    out = c.attend(q, lse=L).double().transpose(0, 1)
    at = 0
    for s, (have, n) in enumerate(zip(lens, news)):
        held = have + n
        if n == 0:
            continue
        k, v = (x.double().transpose(0, 1).repeat_interleave(heads // x.shape[1], 0).contiguous() for x in kv[s])
        p, j = torch.arange(have, held, device="cuda")[:, None] // block, torch.arange(held, device="cuda")[None] // block
        seen = j <= p
        if window:
            seen &= (j > p - window) | (j < sinks)
        w = torch.matmul(q[at:at + n].double().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / D ** 0.5
        size = float(w[torch.isfinite(w)].abs().max()) * D ** 0.5
        w = w.masked_fill(~seen, float("-inf"))
        ref_l = torch.logsumexp(w, 2)
        ref_l = torch.where(torch.isposinf(ref_l), ref_l * float("nan"), ref_l)  # the maximum minus itself
        w = torch.softmax(w, 2)
        vf = torch.where(torch.isfinite(v), v, torch.zeros_like(v))
        ref, A = torch.matmul(w, vf), torch.matmul(w, vf.abs())
        sees = (w > 0).double()
        hit = [torch.matmul(sees, f(v).double()) > 0 for f in (torch.isposinf, torch.isneginf, torch.isnan)]
        ref = torch.where(hit[0], float("inf"), ref)
        ref = torch.where(hit[1], float("-inf"), ref)
        ref = torch.where(hit[2] | (hit[0] & hit[1]), float("nan"), ref)
        d = 2 * (D + 2) * 2.0**-24 * size
        step = 2.0**-8 if bf16 else 2.0**-24
        tol = step * ref.abs() + ((2.0**-8 if bf16 else 0.0) + 2 * d + (held + 16) * 2.0**-24) * A
        got = out[:, at:at + n]
        assert torch.equal(torch.isnan(got), torch.isnan(ref)), s
        inf = torch.isinf(ref)
        assert torch.equal(torch.isinf(got), inf) and torch.equal(got[inf], ref[inf]), s
        fin = torch.isfinite(ref)
        assert bool(((got - ref).abs() <= tol)[fin].all()), s
        if lse:
            got = L[:, at:at + n].double()
            assert torch.equal(torch.isnan(got), torch.isnan(ref_l)), s
            fin = torch.isfinite(ref_l)
            assert bool(((got - ref_l).abs() <= d + (held + 16) * 2.0**-24 + 2.0**-22 * ref_l.abs())[fin].all()), s
        at += n
    return out


# Whole tiles; equal ones in parts with tails; unequal ones that workgroups share; single tokens, whole and in parts.
SHAPES = [("whole", 64, 128, 128, 16, [300], [256], 256, 0, 0), ("parts", 64, 6, 3, 16, [1500], [300], 300, 3, 1),
          ("parts", 128, 5, 5, 64, [900], [300], 300, 0, 0), ("shared", 64, 8, 2, 30, [700, 20, 0], [90, 200, 33], 1, 300, 4),
          ("shared", 128, 4, 4, 64, [1000, 3], [70, 100], 1, 0, 0), ("tokens", 128, 8, 2, 16, [900, 5, 64], [1, 1, 1], 1, 0, 0),
          ("tokens", 64, 2, 1, 48, [9000], [3], 1, 0, 0), ("tokens", 64, 40, 40, 16, [20] * 40, [1] * 40, 1, 0, 0)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("what", ["seen by all", "of later tokens", "a row of NaN", "keys"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}-{s[1]}-{s[2]}")
def test_values_that_are_not_finite(dtype, what, shape):
    """Infinities and NaN that every row sees, that some rows see, that fill a row of V, and in keys: in tiles of one
    workgroup, in tiles that several share, and in single tokens' ones."""
    _, D, heads, kv_heads, P, lens, news, block, window, sinks = shape
    print("not finite", dtype, what, shape, flush=True)

    def spoil(k, v, s, have):
        new = v.shape[0] - have
        if what == "seen by all":
            v[0, 0, 3], v[0, -1, 7], v[0, 0, 9] = float("inf"), float("nan"), float("-inf")
        elif what == "of later tokens":
            v[have + new // 2, 0, 5], v[-1, -1, 6] = float("-inf"), float("nan")
        elif what == "a row of NaN":
            v[0, 0, :] = float("nan")
        else:
            k[0, 0, 1], k[have + new // 2, -1, 2], k[-1, 0, 2] = float("inf"), float("-inf"), float("nan")

    c, q, kv = filled(dtype, D, heads, kv_heads, P, lens, news, spoil, block, window, sinks)
    a = check_spoiled(c, q, kv, lens, news, block, window, sinks)
    b = check_spoiled(c, q, kv, lens, news, block, window, sinks, lse=False)
    assert np.array_equal(a.cpu().numpy(), b.cpu().numpy(), equal_nan=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_value_that_every_row_sees_does_not_stall_the_call(dtype):
    """Whole tiles, one for each workgroup, with an infinity in a value that all of their rows see: the rows that are worked out again are
    spread over the GPU.  By one workgroup they would take hundreds of milliseconds; they take a few."""
    import torch
    heads, rows = (128, 256) if dtype == "f32" else (512, 128)

    def spoil(k, v, s, have):
        v[0, :, 3] = float("inf")

    c, q, kv = filled(dtype, 64, heads, heads, 64, [512], [rows], spoil, block=512)
    q = q.contiguous()
    a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
    out = c.attend(q)
    a.record()
    c.attend(q, out=out)
    b.record()
    torch.cuda.synchronize()
    print("again", dtype, a.elapsed_time(b), "ms", flush=True)
    assert bool(torch.isposinf(out[..., 3]).all()) and bool(torch.isfinite(out[..., 4:]).all())
    assert a.elapsed_time(b) < 50.0


def test_going_back_and_on_deals_the_same_pages():
    """A step planned again changes nothing; gone back from and planned again, it gives its pages back and gets the same."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    c = PagedCache(seqs=5, pages=80, page_tokens=4, heads=2, head_dim=64, max_tokens=100, max_rows=200, window=20, sinks=2)
    kept, new, zero = i32([40, 33, 7, 0, 16]), i32([1, 9, 1, 30, 0]), i32([0] * 5)
    c.plan(zero, kept, rows=200, max_new=40)
    c.plan(kept, new, rows=41, max_new=30)
    want = [x.clone() for x in (c.table, c.slots[:41], c.pos[:41], c.held, c.status, c.free)]
    for back in (False, True, True):
        if back:
            c.plan(kept, zero, rows=0, max_new=0)
            assert c.held.tolist() == kept.tolist() and int(c.free[0]) > int(want[5][0])
        c.plan(kept, new, rows=41, max_new=30)
        assert all(torch.equal(a, b) for a, b in zip(want, (c.table, c.slots[:41], c.pos[:41], c.held, c.status, c.free)))


def test_a_store_of_more_tokens_than_a_step_may_have():
    """Without max_tokens and max_rows: all that the pages hold, in steps of the most rows that the library takes."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    c = PagedCache(seqs=1, pages=1 << 18, page_tokens=64, heads=1, head_dim=64)
    assert c.cfg.max_tokens == 1 << 24 and c.cfg.max_rows == 1 << 23
    c.plan(i32([0]), i32([1 << 23]), rows=1 << 23, max_new=1 << 23)
    c.plan(i32([1 << 23]), i32([1 << 23]), rows=1 << 23, max_new=1 << 23)
    assert c.status.tolist() == [0] and c.held.tolist() == [1 << 24] and int(c.free[0]) == 0
    assert torch.equal(c.slots, torch.arange(1 << 23, 1 << 24, device="cuda"))
    c = PagedCache(seqs=1, pages=1 << 16, page_tokens=64, heads=1024, kv_heads=1, head_dim=64)
    assert c.cfg.max_rows == 1 << 20
