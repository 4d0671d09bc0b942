"""Rotary positions under torch's autograd: the gradient is the inverse rotation."""
import numpy as np
import pytest

from oracle.paged_oracle import rotary_apply

pytestmark = pytest.mark.gpu

THETA = 10000.0


def inputs(dtype, rows, heads, D, pitch=1, seed=0):
    import torch
    g = torch.Generator().manual_seed(seed)
    x = torch.randn((rows, pitch, heads, D), generator=g).to(dtype).cuda()
    pos = torch.randint(0, 900, (rows, 3), generator=g, dtype=torch.int32).cuda()
    return x, pos, torch.randn((rows, heads, D), generator=g).to(dtype).cuda()


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
@pytest.mark.parametrize("layout", ["interleaved", "halves"])
@pytest.mark.parametrize("inverse", [False, True])
@pytest.mark.parametrize("rows,heads,D,pairs,pitch", [(1, 1, 16, (1, 0, 0), 1), (37, 3, 64, (8, 10, 10), 3), (300, 2, 128, (22, 20, 21), 1)])
def test_gradient(dtype, layout, inverse, rows, heads, D, pairs, pitch):
    """An element of the gradient is off by half a step of its type and the fp64 errors of both sides (2^-50 of the
    pair, as for the rotation itself); what has no pair keeps its bits."""
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    td = getattr(torch, dtype)
    base, pos, g = inputs(td, rows, heads, D, pitch)
    base.requires_grad_()
    rot = Rotary(D, pairs, THETA, layout)
    y = rot.apply(base[:, pitch // 2], pos, inverse=inverse)
    assert y.requires_grad and torch.equal(y.detach(), rot.apply(base.detach()[:, pitch // 2], pos, inverse=inverse))
    y.backward(g)
    got = base.grad[:, pitch // 2]
    assert torch.equal(got, rot.apply(g, pos, inverse=not inverse))
    ref = rotary_apply(g.double().cpu().numpy(), pos.cpu().numpy(), pairs, THETA, layout, not inverse)
    size = np.abs(g.double().cpu().numpy())
    pair = size + (size.reshape(rows, heads, -1, 2)[..., ::-1].reshape(size.shape) if layout == "interleaved"
                   else np.roll(size, D // 2, -1))
    tol = torch.finfo(td).eps / 2 * np.abs(ref) + 2.0**-50 * pair
    assert (np.abs(got.double().cpu().numpy() - ref) <= tol).all()
    for p in range(pitch):
        assert p == pitch // 2 or int(torch.count_nonzero(base.grad[:, p])) == 0


def test_gradient_against_differences():
    """The rotation is linear: a difference quotient of <g, R x> is exact up to the roundings of two results (2^-24 of
    at most sqrt(2) (M + 1) each, M the row's largest |x|) and of x + e (2^-24 (M + 1)), times |g|."""
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    base, pos, g = inputs(torch.float32, 9, 2, 64)
    x = base[:, 0].clone().requires_grad_()
    rot = Rotary(64, (8, 10, 10), THETA)
    (rot.apply(x, pos) * g).sum().backward()
    with torch.no_grad():
        for d in (0, 5, 33, 63):
            e = torch.zeros_like(x)
            e[:, :, d] = 1.0
            diff = ((rot.apply(x + e, pos).double() - rot.apply(x, pos).double()) * g.double()).sum(-1)
            bound = 4 * 2.0**-24 * (x.abs().amax(-1).double() + 1.0) * g.abs().double().sum(-1)
            assert bool(((x.grad[:, :, d].double() - diff).abs() <= bound).all())


def test_positions_that_change_before_the_backward_pass():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    base, pos, g = inputs(torch.float32, 33, 2, 64)
    x, kept = base[:, 0].clone().requires_grad_(), pos.clone()
    rot = Rotary(64, (8, 10, 10), THETA)
    y = rot.apply(x, pos)
    pos.zero_()
    y.backward(g)
    assert torch.equal(x.grad, rot.apply(g, kept, inverse=True))


def test_gradients_of_other_shapes_and_of_the_gradient():
    """A broadcast gradient, a transposed one, one that begins off a 16-byte border, and the gradient's own gradient."""
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    base, pos, g = inputs(torch.float32, 20, 3, 64)
    rot = Rotary(64, (8, 10, 10), THETA)
    odd = torch.empty(g.numel() + 1, device="cuda")[1:].view(g.shape).copy_(g)
    for grad in (torch.ones((), device="cuda").expand(20, 3, 64), g.transpose(0, 1).contiguous().transpose(0, 1), odd):
        x = base[:, 0].clone().requires_grad_()
        rot.apply(x, pos).backward(grad)
        assert torch.equal(x.grad, rot.apply(grad.clone(memory_format=torch.contiguous_format), pos, inverse=True))
    x, g = base[:, 0].clone().requires_grad_(), g.clone().requires_grad_()
    dx, = torch.autograd.grad(rot.apply(x, pos), x, g, create_graph=True)
    w = torch.randn_like(dx)
    dg, = torch.autograd.grad(dx, g, w)
    assert torch.equal(dg, rot.apply(w, pos))
    x = base[:0, 0].clone().requires_grad_()
    rot.apply(x, pos[:0]).sum().backward()
    assert x.grad.shape == (0, 3, 64)


def test_gradient_on_another_stream():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    base, pos, g = inputs(torch.float32, 3000, 6, 128)
    rot = Rotary(128, (22, 21, 21), THETA)
    x = base[:, 0].clone().requires_grad_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    y = rot.apply(x, pos, stream=side)
    torch.cuda.current_stream().wait_stream(side)
    (y * g).sum().backward()
    torch.cuda.synchronize()
    assert torch.equal(x.grad, rot.apply(g, pos, inverse=True))


def test_without_a_gradient_and_into_given_memory():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    base, pos, _ = inputs(torch.float32, 8, 2, 64)
    rot = Rotary(64, (8, 10, 10), THETA)
    x = base[:, 0].clone().requires_grad_()
    for out in (torch.empty_like(x), x, x * 1.0):
        with pytest.raises(ValueError):
            rot.apply(x, pos, out=out)
    with pytest.raises(ValueError):
        rot.apply(x.detach(), pos, out=x * 1.0)
    with torch.no_grad():
        want = rot.apply(base[:, 0], pos)
        assert not rot.apply(x, pos).requires_grad and torch.equal(rot.apply(x, pos, out=torch.empty_like(x)), want)
    assert not rot.apply(x.detach(), pos).requires_grad


def test_a_captured_forward_and_backward_pass_replays():
    import torch
    from paper_2606_10671_amd.rotary import Rotary
    base, pos, g = inputs(torch.bfloat16, 40, 3, 128)
    rot = Rotary(128, (22, 21, 21), THETA)
    x = base[:, 0].clone().requires_grad_()

    def both():
        y = rot.apply(x, pos)
        return y.detach(), torch.autograd.grad(y, x, g)[0]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        both()
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx = both()
    for i in range(4):
        with torch.no_grad():
            x.copy_(torch.randn(x.shape, device="cuda"))
            pos.copy_(torch.randint(0, 500, (40, 3), dtype=torch.int32))
            g.copy_(torch.randn(g.shape, device="cuda"))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, rot.apply(x.detach(), pos)) and torch.equal(dx, rot.apply(g, pos, inverse=True))
