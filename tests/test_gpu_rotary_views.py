"""The rotation of a caller's keys beside the memory's own re-indexed views of its keys."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("D,pairs,theta", [(64, 8, 1e4), (128, 64, 1e4), (128, 22, 256.0), (128, 63, 17.3)])
def test_time_axis_and_the_views_of_the_memory(dtype, D, pairs, theta):
    """The memory's re-indexed keys, read from the views at the end of its pool, and the caller's rotation to the same
    index: fp64 both, so that an element is the same or its neighbour (a step of its type, where the two fp64 values,
    2^-48 of the pair apart at most, lie on both sides of a border)."""
    import torch
    from paper_2606_10671_amd.fademem import Cache
    from paper_2606_10671_amd.rotary import Rotary
    torch.manual_seed(D + pairs)
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    M, N, H = 12, 64, 3
    c = Cache(budget=M, heads=H, head_dim=D, tokens_per_block=N, beta=0.3, anchor=True, dtype=td, rope_pairs=pairs,
              rope_theta=theta)
    frames = [torch.randn((N, H, D), device="cuda").to(td) for _ in range(M)]
    for i, k in enumerate(frames):
        c.insert(k, k, i)
    q = torch.randn((N, H, D), device="cuda").to(td)
    c.attend(q, q, q)
    block = frames[0].numel() * frames[0].element_size()  # a multiple of 256, as blocks are
    views = c.pool[c.pool.numel() - (M + 1) * block:].view(td).view(M + 1, N, H, D)
    rot = Rotary(D, (pairs, 0, 0), theta)
    for i, k in enumerate(frames):
        pos = torch.zeros((N, 3), dtype=torch.int32, device="cuda")
        pos[:, 0] = i
        y = rot.apply(k, pos)
        view = views[int((views != y).flatten(1).sum(1).argmin())]  # of the slot that holds the entry
        a, b, x = y.double(), view.double(), k.double().abs()
        assert torch.equal(y[..., 2 * pairs:], view[..., 2 * pairs:])
        pair = (x[..., 0::2] + x[..., 1::2]).repeat_interleave(2, -1)
        assert bool(((a - b).abs() <= torch.finfo(td).eps * torch.maximum(a.abs(), b.abs()) + 2.0**-48 * pair).all()), i
        assert float((y != view).double().mean()) <= 1e-4
