"""Rotary positions with three axes on the GPU against the fp64 oracle.

The library evaluates angle, cos, sin and rotation in fp64 and rounds once, so
an element is off by half a step of its type (eps/2 relative) plus the fp64
errors of both sides: 2^-50 of |x0| + |x1| covers a cos or sin that is off by
two units in fp64's last place on each side."""
import numpy as np
import pytest

from oracle.paged_oracle import rotary_apply

pytestmark = pytest.mark.gpu

THETA = 10000.0


def check(rows, heads, D, pairs, layout, dtype, inverse=False, pitch=1, in_place=False, far=False, seed=0):
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    print(f"rotary rows={rows} heads={heads} D={D} pairs={pairs} {layout} {dtype} inverse={inverse} pitch={pitch}", flush=True)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator().manual_seed(seed)
    base = torch.randn((rows, pitch, heads, D), generator=g).to(td).cuda()
    x = base[:, pitch // 2]
    before = x.double().cpu().numpy()
    hi = 2**31 - 1 if far else 1000
    pos = torch.randint(-hi if far else 0, hi, (rows, 3), generator=g, dtype=torch.int64).to(torch.int32)
    rot = Rotary(D, pairs, THETA, layout)
    others = base.clone()
    y = rot.apply(x, pos.cuda(), out=x if in_place else None, inverse=inverse)
    got = y.double().cpu().numpy()
    ref = rotary_apply(before, pos.numpy(), pairs, THETA, layout, inverse)
    size = np.abs(rotary_apply(np.abs(before), np.zeros((rows, 3)), pairs, THETA, layout))
    half = D // 2
    partner = np.empty_like(size)
    if layout == "interleaved":
        partner[..., 0::2], partner[..., 1::2] = size[..., 1::2], size[..., 0::2]
    else:
        partner[..., :half], partner[..., half:] = size[..., half:], size[..., :half]
    tol = torch.finfo(td).eps / 2 * np.abs(ref) + 2.0**-50 * (size + partner)
    assert (np.abs(got - ref) <= tol).all(), float((np.abs(got - ref) - tol).max())
    if in_place:  # the other slices of the rows are as they were
        for p in range(pitch):
            if p != pitch // 2:
                assert torch.equal(base[:, p], others[:, p])
    return x, y


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("layout", ["interleaved", "halves"])
@pytest.mark.parametrize("D,pairs", [(128, (22, 21, 21)), (64, (8, 10, 10)), (64, (0, 5, 0)), (64, (32, 0, 0)),
                                     (48, (7, 1, 9)), (16, (1, 0, 0)), (256, (44, 42, 42)), (128, (1, 30, 32))])
def test_shapes(D, pairs, layout, dtype):
    check(37, 3, D, pairs, layout, dtype)


@pytest.mark.parametrize("rows,heads", [(1, 1), (1, 40), (3, 1), (511, 12), (1025, 5), (5000, 1), (16, 12), (700, 160)])
def test_rows_and_heads(rows, heads):
    check(rows, heads, 128, (22, 21, 21), "interleaved", "bf16")
    check(rows, heads, 64, (8, 10, 10), "halves", "f32", inverse=True)


@pytest.mark.parametrize("layout", ["interleaved", "halves"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_inside_a_joint_projection(layout, dtype):
    check(129, 6, 64, (8, 10, 10), layout, dtype, pitch=3)
    check(129, 6, 64, (8, 10, 10), layout, dtype, pitch=3, in_place=True)
    check(130, 2, 128, (20, 20, 20), layout, dtype, pitch=2, in_place=True, inverse=True)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_far_positions(dtype):
    check(64, 2, 128, (22, 21, 21), "interleaved", dtype, far=True)


def test_elements_without_a_pair_keep_their_bits():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    x = torch.full((5, 2, 64), float("nan"), dtype=torch.bfloat16, device="cuda")
    x[..., :14] = 1.0
    x[..., 20] = float("inf")
    y = Rotary(64, (3, 2, 2)).apply(x, torch.ones((5, 3), dtype=torch.int32, device="cuda"))
    assert torch.equal(y.view(torch.int16)[..., 14:], x.view(torch.int16)[..., 14:])
    assert torch.isfinite(y[..., :14].float()).all()


def test_time_axis_has_the_bits_of_the_memory_views():
    """The caller's rotation and the library's re-indexed views are the same: both within one rounding of fp64, and
    equal to the oracle's rounded values except where fp64 cos and sin of two libraries differ by an ulp next to a tie."""
    import torch
    from oracle import rope_rotate
    from paper_2606_10671_amd.rotary import Rotary
    x = np.random.default_rng(5).standard_normal((300, 4, 128)).astype(np.float32)
    t = torch.from_numpy(x).to("cuda", torch.bfloat16)
    pos = torch.zeros((300, 3), dtype=torch.int32, device="cuda")
    pos[:, 0] = 17
    y = Rotary(128, (22, 0, 0)).apply(t, pos).float().cpu().numpy()
    ref = rope_rotate(t.float().cpu().numpy(), 17, 22, 10000.0, "bf16").astype(np.float32)
    assert (y != ref).mean() <= 1e-6


def test_inverse_undoes_and_is_the_gradient():
    """<g, R x> has the gradient R^T g = R^-1 g, by the formula and by differences (the rotation is linear, so a
    difference quotient is exact up to fp64 rounding of the sums)."""
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    torch.manual_seed(3)
    x = torch.randn((9, 2, 64), device="cuda")
    g = torch.randn((9, 2, 64), device="cuda")
    pos = torch.randint(0, 500, (9, 3), dtype=torch.int32, device="cuda")
    for layout in ("interleaved", "halves"):
        rot = Rotary(64, (8, 10, 10), THETA, layout)
        back = rot.apply(rot.apply(x, pos), pos, inverse=True)
        # Two roundings of half a step (2^-24) relative to the pair's length.
        assert float((back - x).abs().max()) <= 2 * 2.0**-24 * float(x.abs().max()) * 2.0
        grad = rot.apply(g, pos, inverse=True)
        for d in (0, 5, 33, 63):
            e = torch.zeros_like(x)
            e[:, :, d] = 1.0
            diff = ((rot.apply(x + e, pos).double() - rot.apply(x, pos).double()) * g.double()).sum(-1)
            # With M the row's largest |x|: two results, each rounded at 2^-24 of at most sqrt(2) (M + 1), and x + e
            # rounded at 2^-24 (M + 1), all times |g|.
            bound = 4 * 2.0**-24 * (x.abs().amax(-1).double() + 1.0) * g.abs().double().sum(-1)
            assert ((grad[:, :, d].double() - diff).abs() <= bound).all()


def test_given_frequencies_and_streams():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    x = torch.randn((33, 2, 64), device="cuda")
    pos = torch.randint(0, 90, (33, 3), dtype=torch.int32, device="cuda")
    freq = [0.5 / (i + 1) for i in range(10)]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = Rotary(64, (4, 3, 3), freq=freq).apply(x, pos, stream=side)
    side.synchronize()
    ang = pos.double()[:, [0] * 4 + [1] * 3 + [2] * 3] * torch.tensor(freq, dtype=torch.float64, device="cuda")
    c, s = torch.cos(ang)[:, None], torch.sin(ang)[:, None]
    a, b = x[..., 0:20:2].double(), x[..., 1:20:2].double()
    assert float((y[..., 0:20:2].double() - (a * c - b * s)).abs().max()) <= 2.0**-24 * 8
    assert torch.equal(y[..., 20:], x[..., 20:])


def test_a_result_on_another_stream_takes_no_memory_that_this_stream_let_go():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    x = torch.randn((5000, 12, 64), device="cuda")
    pos = torch.zeros((5000, 3), dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    gone = torch.empty_like(x)  # work of the current stream may still read it
    at = gone.data_ptr()
    del gone
    y = Rotary(64, (32, 0, 0)).apply(x, pos, stream=side)
    assert y.data_ptr() != at
    side.synchronize()
    assert torch.equal(x, y)


def test_a_captured_call_replays_with_other_positions():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    rot = Rotary(128, (22, 21, 21))
    x = torch.randn((100, 3, 128), device="cuda").bfloat16()
    pos = torch.zeros((100, 3), dtype=torch.int32, device="cuda")
    out = torch.empty_like(x)
    rot.apply(x, pos, out=out)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        rot.apply(x, pos, out=out)
    for i in range(3):
        pos.copy_(torch.randint(0, 999, (100, 3), dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, rot.apply(x, pos))


def test_refusals_of_the_binding():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    rot = Rotary(64, (8, 8, 8))
    x = torch.zeros((4, 2, 64), device="cuda")
    pos = torch.zeros((4, 3), dtype=torch.int32, device="cuda")
    for bad_x, bad_pos in ((x.half(), pos), (x[..., :32], pos), (x, pos[:3]), (x, pos.long()), (x.cpu(), pos),
                           (x.transpose(0, 1), pos), (x[:, :, ::2], pos), (x, pos.cpu())):
        with pytest.raises(ValueError):
            rot.apply(bad_x, bad_pos)
    with pytest.raises(ValueError):
        rot.apply(x, pos, out=torch.zeros((4, 2, 64), dtype=torch.bfloat16, device="cuda"))
    assert rot.apply(x[:0], pos[:0]).shape == (0, 2, 64)
