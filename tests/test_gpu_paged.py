"""The paged window memory on the GPU against its oracle: plans element by
element, pages bit for bit, attention within bounds derived in paged_parity."""
import numpy as np
import pytest

from paged_parity import Pair

pytestmark = pytest.mark.gpu


def say(*args):
    print("paged", *args, flush=True)


# -- plans ---------------------------------------------------------------------

@pytest.mark.parametrize("seqs,P,window,sinks,block", [(1, 16, 0, 0, 1), (5, 7, 0, 0, 1), (5, 16, 40, 3, 1),
                                                       (3, 64, 2, 1, 90), (37, 1, 9, 2, 1), (300, 3, 5, 1, 2),
                                                       (4, 5, 1, 4, 11), (2, 1000, 3, 1, 50)])
def test_random_steps(seqs, P, window, sinks, block):
    """Steps that append, go back, start again, end, run out of pages, and name lengths that are refused."""
    say("plan", seqs, P, window, sinks, block)
    rng = np.random.default_rng(seqs * 100 + P)
    p = Pair(seqs, pages=max(8, 60 // P * seqs), P=P, heads=2, D=64, max_tokens=400, max_rows=40 * seqs, block=block,
             window=window, sinks=sinks, grid=(3, 4))
    seen = set()
    for step in range(40):
        held = p.oracle.held
        kept, added = [], []
        for s in range(seqs):
            r = rng.random()
            k = held[s] if r < 0.6 else 0 if r < 0.7 else int(rng.integers(0, held[s] + 1)) if r < 0.97 else held[s] + 1
            n = int(rng.integers(0, 30)) if rng.random() < 0.9 else 0
            kept.append(k if rng.random() < 0.99 else -1)
            added.append(n if rng.random() < 0.99 else -2)
        rows = min(40 * seqs, sum(max(a, 0) for a in added) + int(rng.integers(0, 5)))
        ref = p.plan(kept, added, rows=rows, max_new=min(rows, 29 if rng.random() < 0.9 else 20))
        seen |= set(ref["status"])
        again = p.cache.table.clone(), p.cache.slots[:rows].clone()
        if all(c == 0 for c in ref["status"]):  # the same step again changes nothing
            p.plan(kept, added, rows=rows, max_new=29 if rows >= 29 else rows)
            if all(c == 0 for c in p.step["status"]):
                assert p.torch.equal(again[0], p.cache.table) and p.torch.equal(again[1], p.cache.slots[:rows])
    assert 0 in seen and -1 in seen


def test_out_of_pages_in_order():
    p = Pair(4, pages=10, P=8, heads=2, D=64, max_tokens=200, max_rows=200)
    ref = p.plan([0, 0, 0, 0], [40, 41, 8, 0])        # 5 + 6 > 10: the second and the third get none
    assert ref["status"] == [0, -3, -3, 0] and ref["free"] == 5
    ref = p.plan([40, 0, 0, 0], [1, 30, 0, 8])        # 1 + 4 + 1 > 5
    assert ref["status"] == [0, 0, 0, -3]
    ref = p.plan([0, 30, 0, 0], [0, 2, 0, 40])        # the first leaves: its pages go out in the same step
    assert ref["status"] == [0, 0, 0, 0]


def test_window_gives_pages_back_and_going_back_behind_it_is_refused():
    p = Pair(1, pages=12, P=4, heads=2, D=64, max_tokens=4000, max_rows=8, window=10, sinks=2)
    held = 0
    for _ in range(60):                               # 480 tokens through 48 tokens of pages
        assert p.plan([held], [8])["status"] == [0]
        held += 8
    assert p.plan([held - 40], [1])["status"] == [-2]  # its window lies behind pages given back
    assert p.plan([held - 8], [8])["status"] == [0]    # the last step again
    assert p.plan([3], [8])["status"] == [0]           # all that is kept lies in the sinks' page
    assert p.plan([0], [0])["free"] == 12


def test_many_pages_and_rows():
    say("many pages")
    p = Pair(3, pages=40000, P=1, heads=2, D=64, max_tokens=30000, max_rows=40000)
    p.plan([0, 0, 0], [5, 20001, 3000], rows=30000)
    p.plan([5, 0, 3000], [1, 0, 29], rows=30)
    p.plan([6, 0, 3029], [0, 29999, 1], rows=30001)


def test_zero_rows_and_empty_steps():
    p = Pair(3, pages=10, P=8, heads=2, D=64, max_tokens=50, max_rows=20)
    p.plan([0, 0, 0], [0, 0, 0], rows=0, max_new=0)
    p.insert()
    p.attend()
    p.plan([0, 0, 0], [0, 0, 0], rows=7, max_new=0)
    p.insert()
    p.attend()


# -- insertion -----------------------------------------------------------------

@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,pairs,layout", [(64, None, "interleaved"), (128, (22, 21, 21), "interleaved"),
                                            (64, (8, 10, 10), "halves"), (128, (30, 0, 1), "halves")])
def test_insert(dtype, D, pairs, layout):
    say("insert", dtype, D, pairs, layout)
    p = Pair(3, pages=60, P=11, heads=6, kv_heads=3, D=D, dtype=dtype, layers=2, max_tokens=200, max_rows=150, grid=(3, 5),
             pairs=pairs, layout=layout)
    p.plan([0, 0, 0], [70, 1, 33], rows=110)
    p.insert(0)
    p.insert(1, pitch=3)
    p.plan([70, 1, 20], [1, 1, 1])
    p.insert(1)
    p.insert(0, pitch=2)
    p.check_pages(1)


# -- attention -----------------------------------------------------------------

HEADS = [(2, 2), (8, 2), (5, 1)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("heads,kv_heads", HEADS)
@pytest.mark.parametrize("P", [16, 48, 64])
def test_decode(dtype, D, heads, kv_heads, P):
    """One token of sequences of 1 to 700 tokens, and of none."""
    say("decode", dtype, D, heads, kv_heads, P)
    lens = [1, 63, 64, 65, 129, 256, 257, 700, 31, 2]
    p = Pair(10, pages=-(-2000 // P) + 40, P=P, heads=heads, kv_heads=kv_heads, D=D, dtype=dtype, max_tokens=800, max_rows=1800)
    p.plan([0] * 10, lens)
    p.insert()
    p.plan(lens, [1, 1, 1, 1, 1, 1, 1, 1, 0, 1])
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(0, 0), (0, 5), (50, 0), (50, 3), (1, 0), (1, 1), (200, 70), (64, 64)])
def test_causal_window(dtype, window, sinks):
    """Token by token causal chunks of odd lengths; windows and sinks that begin and end inside tiles and pages."""
    say("causal", dtype, window, sinks)
    p = Pair(4, pages=120, P=20, heads=4, kv_heads=2, D=64, dtype=dtype, max_tokens=900, max_rows=600, window=window, sinks=sinks)
    p.plan([0, 0, 0, 0], [150, 1, 17, 300])
    p.insert()
    p.attend()
    p.plan([150, 1, 17, 300], [33, 0, 200, 100], rows=350)
    p.insert()
    p.attend()
    p.plan([183, 1, 217, 400], [1, 1, 1, 1], rows=9)
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("block,window,sinks", [(70, 0, 0), (70, 2, 0), (70, 2, 1), (96, 3, 1), (64, 1, 2)])
def test_chunks(dtype, D, block, window, sinks):
    """Chunks whose tokens see each other, over a window of chunks and sink chunks; a partial last chunk."""
    say("chunks", dtype, D, block, window, sinks)
    p = Pair(2, pages=60, P=32, heads=3, D=D, dtype=dtype, max_tokens=1000, max_rows=500, block=block, window=window, sinks=sinks,
             grid=(5, 7))
    held = 0
    for n in (block, block, block, 2 * block, block, 13):
        p.plan([held, held], [n, max(1, n - 9)] if held == 0 and n == 13 else [n, n])
        p.insert()
        p.attend()
        held += n


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows", [1, 31, 32, 33, 127, 128, 129, 255, 256, 257, 300])
def test_rows_at_tile_edges(dtype, rows):
    say("rows", dtype, rows)
    p = Pair(1, pages=40, P=64, heads=2, D=128, dtype=dtype, max_tokens=2000, max_rows=700, block=2000)
    p.plan([0], [rows + 70])
    p.insert()
    p.plan([70], [rows])
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("window", [0, 77])
@pytest.mark.parametrize("P", [1, 3, 5, 8, 24, 31, 33, 96, 100, 300])
def test_page_sizes(dtype, D, window, P):
    """Tiles that begin and end anywhere in a page, one page under a tile or thirty-two: prompts, a chunk, single tokens."""
    say("pages", dtype, D, window, P)
    p = Pair(3, pages=3 * (-(-330 // P) + 2), P=P, heads=4, kv_heads=2, D=D, dtype=dtype, max_tokens=400, max_rows=500,
             window=window, sinks=5 if window else 0)
    for kept, new in (([0, 0, 0], [201, 70, 1]), ([201, 70, 1], [40, 97, 130]), ([241, 167, 131], [3, 1, 16]),
                      ([244, 168, 147], [1, 1, 0])):
        p.plan(kept, new)
        p.insert()
        p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,heads,kv_heads", [(64, 96, 1), (128, 40, 1), (64, 33, 1), (128, 66, 2)])
def test_more_heads_than_a_narrow_tile(dtype, D, heads, kv_heads):
    """One token's heads of a key head fill a wide tile, or more than one."""
    say("heads", dtype, D, heads, kv_heads)
    p = Pair(3, pages=60, P=32, heads=heads, kv_heads=kv_heads, D=D, dtype=dtype, max_tokens=700, max_rows=800)
    p.plan([0, 0, 0], [1, 130, 500])
    p.insert()
    p.plan([1, 130, 500], [1, 1, 1])
    p.insert()
    p.attend()
    p.plan([2, 131, 501], [7, 0, 4])
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_as_many_sequences_as_there_may_be(dtype):
    """1024 sequences that begin with one token: each sees itself."""
    say("1024", dtype)
    p = Pair(1024, pages=2048, P=16, heads=2, D=64, dtype=dtype, max_tokens=64, max_rows=4096)
    p.plan([0] * 1024, [1] * 1024)
    p.insert()
    p.attend()
    p.plan([1] * 1024, [i % 3 for i in range(1024)])
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_long_memory_is_split(dtype):
    """Few rows over many keys: the keys are shared out among workgroups and joined."""
    say("long", dtype)
    p = Pair(2, pages=400, P=64, heads=2, kv_heads=1, D=128, dtype=dtype, max_tokens=12000, max_rows=12000)
    p.plan([0, 0], [9001, 2500])
    p.insert()
    p.plan([9001, 2500], [1, 1])
    p.insert()
    p.attend()
    p.plan([9002, 2501], [20, 3])
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_scores_far_apart(dtype):
    say("peaked", dtype)
    p = Pair(2, pages=60, P=16, heads=2, D=64, dtype=dtype, max_tokens=400, max_rows=600, window=90, sinks=2)
    p.plan([0, 0], [290, 100])
    p.insert()
    p.attend(q_scale=30.0)
    p.attend(scale=3.0)
    p.attend(scale=1e-4)


def test_rows_of_joint_projections_and_layers():
    p = Pair(2, pages=60, P=16, heads=4, kv_heads=2, D=64, layers=3, max_tokens=400, max_rows=300)
    p.plan([0, 0], [100, 57], rows=160)
    for layer in (2, 0, 1):
        p.insert(layer, pitch=2)
    for layer in (0, 1, 2):
        p.attend(layer, pitch=3, lse=layer != 1)


def test_rows_of_refused_sequences_are_zero():
    p = Pair(5, pages=12, P=8, heads=2, D=64, max_tokens=60, max_rows=100)
    # 61 tokens are more than max_tokens; with it, 20 + 61 + 30 rows are more than 99: no row for what follows.
    ref = p.plan([0, 0, 0, 0, 0], [20, 61, 30, 10, 50], rows=99, max_new=70)
    assert ref["status"] == [0, -1, -1, -1, -1]
    p.insert()
    p.attend()
    ref = p.plan([20, 0, 31, 10, 0], [1, 41, 1, 1, 0])
    assert ref["status"] == [0, 0, -1, -1, 0]
    p.insert()
    p.attend()
    ref = p.plan([21, 41, 0, 0, 0], [1, 1, 20, 20, 0])  # 3 + 6 + 3 of 12 pages
    assert ref["status"] == [0, 0, 0, -3, 0]
    p.insert()
    p.attend()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_values_that_a_row_does_not_see_do_not_reach_it(dtype, bad):
    """Infinities and NaN in a later token, in a key or a value, reach that token's own row and later ones only."""
    say("hidden", dtype, bad)

    def spoil(k, v):
        k[40, 0, 3] = bad
        v[57, 1, 5] = bad
        v[58, 0, :] = bad

    p = Pair(1, pages=30, P=16, heads=4, kv_heads=2, D=64, dtype=dtype, max_tokens=300, max_rows=200)
    p.plan([0], [100])
    p.insert(edit=spoil)
    p.attend(finite=False)
    p = Pair(1, pages=30, P=16, heads=2, D=64, dtype=dtype, max_tokens=300, max_rows=200, window=30, sinks=2)
    p.plan([0], [100])
    p.insert(edit=spoil)
    p.attend(finite=False)
    p.plan([100], [1])                                 # the window has left them behind
    p.insert()
    p.attend()


# -- larger ones, against fp64 on the GPU ---------------------------------------

def large(dtype, D, heads, kv_heads, P, lens, news, block=1, window=0, sinks=0, pages=None, lse=True):
    """One step of sequences that hold `lens` tokens and get `news`; the reference is torch in fp64, from the
    same keys and values (bounds as in paged_parity: A, the weighted mean of |V|, carries the weights' error)."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    seqs, G = len(lens), heads // kv_heads
    need = sum(-(-(a + b) // P) for a, b in zip(lens, news))
    c = PagedCache(seqs=seqs, pages=pages or need + 3, page_tokens=P, heads=heads, kv_heads=kv_heads, head_dim=D, dtype=td,
                   max_tokens=max(a + b for a, b in zip(lens, news)), max_rows=max(sum(lens), sum(news), 1), block_tokens=block,
                   window=window, sinks=sinks)
    c.pages().fill_(float("nan"))
    torch.manual_seed(sum(lens) + D)
    kv = [[torch.randn((a + b, kv_heads, D), device="cuda").to(td) for _ in range(2)] for a, b in zip(lens, news)]
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    if sum(lens):
        c.plan(i32([0] * seqs), i32(lens), rows=sum(lens), max_new=max(lens))
        c.insert(*(torch.cat([kv[s][w][:lens[s]] for s in range(seqs)]) for w in (0, 1)))
    rows = sum(news)
    c.plan(i32(lens), i32(news), rows=rows, max_new=max(news))
    c.insert(*(torch.cat([kv[s][w][lens[s]:] for s in range(seqs)]) for w in (0, 1)))
    assert c.status.tolist() == [0] * seqs
    q = torch.randn((rows, heads, D), device="cuda").to(td)
    L = torch.full((heads, rows), 7.0, device="cuda") if lse else None
    out = c.attend(q, lse=L).double()
    at = 0
    for s in range(seqs):
        n, held = news[s], lens[s] + news[s]
        if n == 0:
            continue
        p, j = torch.arange(lens[s], held, device="cuda")[:, None] // block, torch.arange(held, device="cuda")[None] // block
        seen = j <= p
        if window:
            seen &= (j > p - window) | (j < sinks)
        k, v = (x.double().transpose(0, 1).repeat_interleave(G, 0).contiguous() for x in kv[s])  # [heads][held][D]
        w = torch.matmul(q[at:at + n].double().transpose(0, 1).contiguous(), k.transpose(1, 2).contiguous()) / D ** 0.5
        size = float(w.abs().max()) * D ** 0.5  # the products' sizes sum to at most the root of D times |q| |k| here
        w = w.masked_fill(~seen, float("-inf"))
        ref_l = torch.logsumexp(w, 2)
        w = torch.softmax(w, 2)
        ref, A = torch.matmul(w, v), torch.matmul(w, v.abs())
        d = 2 * (D + 2) * 2.0**-24 * size
        step = 2.0**-8 if dtype == "bf16" else 2.0**-24
        tol = step * ref.abs() + ((2.0**-8 if dtype == "bf16" else 0.0) + 2 * d + (held + 16) * 2.0**-24) * A
        err = (out[at:at + n].transpose(0, 1) - ref).abs()
        assert bool((err <= tol).all()), (s, float((err - tol).max()))
        if lse:
            assert bool(((L[:, at:at + n].double() - ref_l).abs() <= d + (held + 16) * 2.0**-24 + 2.0**-22 * ref_l.abs()).all()), s
        at += n
    return c, q, out


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_equal_tiles_are_dealt_evenly(dtype):
    """More tiles than workgroups, and a few left over that are cut into parts and tails."""
    say("even", dtype)
    large(dtype, 64, 130, 130, 64, [900], [300], block=300)
    large(dtype, 128, 50, 10, 64, [600, 600], [300, 300], block=300, window=2, sinks=1)
    large(dtype, 128, 9, 9, 64, [2000], [1000], block=1000)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_unequal_tiles_share_workgroups(dtype):
    say("uneven", dtype)
    large(dtype, 64, 16, 4, 48, [0, 2000, 31, 700, 5, 0], [513, 100, 1, 300, 0, 65], window=600, sinks=4)
    large(dtype, 128, 8, 1, 16, [3000, 10, 0], [40, 333, 1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_one_tile_shared_by_every_workgroup(dtype):
    say("long", dtype)
    large(dtype, 128, 1, 1, 64, [70000], [1])
    large(dtype, 64, 2, 1, 30, [40000], [150], block=1000)


def test_more_segments_than_one_list_holds():
    """A workgroup's segments are described 64 at a time: many short sequences and heads."""
    say("many segments")
    large("bf16", 64, 48, 48, 16, [3] * 500, [1] * 500)
    large("bf16", 64, 40, 40, 16, [20] * 600, [40] * 599 + [41])


def test_pages_beyond_32_bit_offsets():
    """Sequences whose pages lie more than 2^32 bytes and 2^31 elements into the pool."""
    say("far pages")
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    c = PagedCache(seqs=2, pages=24000, page_tokens=64, heads=8, kv_heads=8, head_dim=128, max_tokens=64 * 23990, max_rows=1 << 21)
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    held = 0
    while held < 64 * 23900:  # the first sequence takes the low pages
        n = min(1 << 20, 64 * 23900 - held)
        c.plan(i32([held, 0]), i32([n, 0]), rows=n, max_new=n)
        held += n
    k, v = (torch.randn((600, 8, 128), device="cuda").bfloat16() for _ in range(2))
    c.plan(i32([held, 0]), i32([0, 600]), rows=600, max_new=600)
    assert int(c.table[1, 0]) == 23900 and int(c.slots[0]) == 23900 * 64
    c.insert(k, v)
    assert torch.equal(c.pages()[23900, 0].transpose(0, 1), k[:64]) and torch.equal(c.pages()[23909, 1, :, 23], v[599])
    q = torch.randn((600, 8, 128), device="cuda").bfloat16()
    near = PagedCache(seqs=2, pages=20, page_tokens=64, heads=8, kv_heads=8, head_dim=128, max_tokens=1000, max_rows=1000)
    near.plan(i32([0, 0]), i32([0, 600]), rows=600, max_new=600)
    near.insert(k, v)
    assert torch.equal(c.attend(q), near.attend(q))
    for store, first in ((c, held), (near, 0)):
        store.plan(i32([first, 600]), i32([0, 1]), rows=1, max_new=1)
        store.insert(k[:1], v[:1])
    assert torch.equal(c.attend(q[:1]), near.attend(q[:1]))


def test_calls_of_another_step_do_nothing():
    """A graph of insertion and attention alone, replayed after a plan with other rows or for another kernel."""
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    c = PagedCache(seqs=2, pages=60, page_tokens=16, heads=4, kv_heads=2, head_dim=64, max_tokens=400, max_rows=300)
    c.pages().zero_()
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    q, k, v = (torch.randn((100, h, 64), device="cuda").bfloat16() for h in (4, 2, 2))
    out, lse = torch.zeros_like(q), torch.zeros((4, 100), device="cuda")

    def calls():
        c.insert(k, v)
        c.attend(q, out=out, lse=lse)

    c.plan(i32([0, 0]), i32([60, 40]), rows=100, max_new=60)
    calls()
    want = out.clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        calls()
    for kept, new, rows, most in (([0, 0], [200, 100], 300, 200), ([0, 0], [1, 2], 100, 2), ([0, 0], [99, 1], 100, 99),
                                  ([0, 0], [0, 0], 0, 0)):
        c.plan(i32(kept), i32(new), rows=rows, max_new=most)
        c.pages().zero_()
        out.fill_(7.0)
        lse.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert bool((out == 7.0).all()) and bool((lse == 7.0).all())
        if rows != 100:
            assert int(torch.count_nonzero(c.pages())) == 0
    c.plan(i32([0, 0]), i32([60, 40]), rows=100, max_new=60)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, want)


# -- together --------------------------------------------------------------------

def test_streams_generate_together():
    """Two videos chunk by chunk over three layers, four denoising passes a chunk that plan the same step again, keys
    rotated on three axes; a third joins late, the first leaves."""
    say("streams")
    chunk, grid = 2 * 4 * 6, (4, 6)
    p = Pair(3, pages=40, P=16, heads=4, kv_heads=4, D=64, layers=3, max_tokens=2000, max_rows=3 * chunk, block=chunk,
             window=3, sinks=1, grid=grid, pairs=(12, 10, 10))
    held = [0, 0, 0]
    for c in range(7):
        new = [chunk if c < 5 else 0, chunk, chunk if c >= 3 else 0]
        kept = [held[0] if c < 5 else 0, held[1], held[2]]
        for denoise in range(2):
            assert p.plan(kept, new)["status"] == [0, 0, 0]
            for layer in range(3):
                p.insert(layer)
                p.attend(layer, lse=denoise == 1)
        held = [k + n for k, n in zip(kept, new)]


def test_a_captured_step_replays_with_other_lengths():
    import torch
    from paper_2606_10671_amd.paged import PagedCache
    from paper_2606_10671_amd.rotary import Rotary
    rot = Rotary(64, (12, 10, 10))

    def store():
        return PagedCache(seqs=3, pages=200, page_tokens=16, heads=4, kv_heads=2, head_dim=64, max_tokens=900, max_rows=120,
                          window=100, sinks=4)

    torch.manual_seed(1)
    a, b = store(), store()
    a.pages().zero_()
    b.pages().zero_()
    kept, added = (torch.zeros(3, dtype=torch.int32, device="cuda") for _ in range(2))
    q, k, v = (torch.randn((120, h, 64), device="cuda").bfloat16() for h in (4, 2, 2))
    outs = [torch.zeros((120, 4, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2)]

    def step(cache, out):
        cache.plan(kept, added, rows=120, max_new=60)
        cache.insert(k, v, rotary=rot)
        cache.attend(rot.apply(q, cache.pos[:120]), out=out)

    step(a, outs[0])
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(a, outs[0])
    held = [0, 0, 0]
    for new in ([60, 1, 30], [3, 0, 60], [1, 1, 1], [60, 60, 0], [0, 7, 9]):
        kept.copy_(torch.tensor(held, dtype=torch.int32))
        added.copy_(torch.tensor(new, dtype=torch.int32))
        for t in (q, k, v):
            t.copy_(torch.randn(t.shape, device="cuda"))
        outs[0].zero_()
        outs[1].zero_()
        graph.replay()
        torch.cuda.synchronize()
        step(b, outs[1])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(a.table, b.table) and torch.equal(a.pages(), b.pages())
        assert a.status.tolist() == [0, 0, 0]
        held = [h + n for h, n in zip(held, new)]


def test_calls_repeat_bit_for_bit_on_another_stream():
    import torch
    p = Pair(2, pages=300, P=64, heads=2, D=128, max_tokens=9000, max_rows=9000)
    p.plan([0, 0], [5000, 900])
    p.insert()
    p.plan([5000, 900], [60, 7])
    p.insert()
    q = torch.randn((67, 2, 128), device="cuda").bfloat16()
    first = p.cache.attend(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = p.cache.attend(q, stream=side)
    side.synchronize()
    assert torch.equal(first, again)


def test_a_result_on_another_stream_takes_no_memory_that_this_stream_let_go():
    import torch
    p = Pair(1, pages=100, P=64, heads=12, D=128, max_tokens=6000, max_rows=6000)
    p.plan([0], [5000])
    p.insert()
    q = torch.randn((5000, 12, 128), device="cuda").bfloat16()
    first = p.cache.attend(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gone = torch.empty_like(q)  # work of the current stream may still read it
    at = gone.data_ptr()
    del gone
    again = p.cache.attend(q, stream=side)
    assert again.data_ptr() != at
    side.synchronize()
    assert torch.equal(first, again)


def test_refusals():
    import torch
    from paper_2606_10671_amd import fademem as fm
    from paper_2606_10671_amd.paged import PagedCache
    from paper_2606_10671_amd.rotary import Rotary
    c = PagedCache(seqs=2, pages=10, page_tokens=8, heads=4, kv_heads=2, head_dim=64, max_tokens=80, max_rows=40)
    i = torch.zeros(2, dtype=torch.int32, device="cuda")
    kv = torch.zeros((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    with pytest.raises(fm.FademError) as e:
        c.insert(kv, kv)
    assert e.value.code == fm.FADEMEM_ESTATE
    with pytest.raises(fm.FademError) as e:
        c.attend(torch.zeros((0, 4, 64), dtype=torch.bfloat16, device="cuda"))
    assert e.value.code == fm.FADEMEM_ESTATE
    for rows, most in ((41, 1), (-1, 0), (5, 6), (5, -1)):
        with pytest.raises(fm.FademError) as e:
            c.plan(i, i, rows=rows, max_new=most)
        assert e.value.code == fm.FADEMEM_EINVAL
    for bad in (i[:1], i.long(), i.cpu(), torch.zeros((2, 1), dtype=torch.int32, device="cuda")):
        with pytest.raises(ValueError):
            c.plan(bad, i, rows=4, max_new=2)
    c.plan(i, i + 3, rows=6, max_new=3)
    k, q = (torch.zeros((6, h, 64), dtype=torch.bfloat16, device="cuda") for h in (2, 4))
    for bad in (k[:5], k.float(), q, k[..., :32], k.transpose(0, 1)):
        with pytest.raises(ValueError):
            c.insert(bad, k)
        with pytest.raises(ValueError):
            c.insert(k, bad)
    for bad in (q[:5], q.float(), k):
        with pytest.raises(ValueError):
            c.attend(bad)
    for kw in (dict(layer=1), dict(layer=-1), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(out=q)):
        with pytest.raises(fm.FademError) as e:
            c.attend(q, **kw)
        assert e.value.code == fm.FADEMEM_EINVAL
    with pytest.raises(fm.FademError):
        c.insert(k, k, layer=1)
    with pytest.raises(fm.FademError):
        c.insert(k, k, rotary=Rotary(128, (1, 1, 1)))
    with pytest.raises(ValueError):
        c.attend(q, lse=torch.zeros((4, 5), device="cuda"))
    with pytest.raises(fm.FademError):
        fm.fademem_paged_array(c.handle, 8)
    with pytest.raises(fm.FademError):
        fm.fademem_paged_array(c.handle, fm.FADEMEM_PAGED_PAGES, 1)
