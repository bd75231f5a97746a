"""How far a value kept in 8 bits may be off.  Codes from 2^-6 on have three bits behind the first, so the nearest is within 2^-4 of a value; below they
are 2^-9 apart, and what would become 0 becomes 2^-9, so it is less than 2^-9 off.  A scale is the smallest power of two that leaves a block's largest at
most 448, so that one is above 224 = 2^7.8 of it (or the scale is 2^-126).  So from 2^-13 of the largest and from 2^-132 on a value is above 2^-6 of the
scale, and all others are off by less than 2^-9 / 224 < 2^-16 of the largest, or 2^-135.  2^-4 also holds for what is next to the type's largest number
and held as 240 of the scale: less than 256, it is less than 16 off."""
import pytest

from tests.test_gpu_dense import dense  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
def test_what_is_kept_is_as_near_as_is_said(dense, dtype):
    import torch
    t = getattr(torch, dtype)
    info, g = torch.finfo(t), torch.Generator(device="cuda")
    g.manual_seed(1)
    # a block's largest: next to 224, 448 and powers of two, over the type's range; the others from it down to 2^-20 of it
    m = torch.tensor([224.0, 224.9, 225.0, 240.0, 255.0, 256.0, 320.0, 447.0, 448.0], device="cuda", dtype=torch.float64)
    low, high = {"float32": (-140, 119), "bfloat16": (-133, 119), "float16": (-24, 7)}[dtype]
    top = (m[:, None] * torch.exp2(torch.arange(low, high, device="cuda", dtype=torch.float64) - 1)).flatten().clamp(max=info.max)
    top = torch.cat([top, torch.tensor([info.max, info.max * (1 - info.eps)], device="cuda", dtype=torch.float64)])
    below = torch.exp2(-20 * torch.rand(len(top), 64, 31, device="cuda", generator=g, dtype=torch.float64))
    x = torch.cat([top[:, None, None].expand(-1, 64, 1), top[:, None, None] * below], 2).to(t)
    rows = x.flatten(0, 1)
    c = dense.ps_checkpoint_encode(rows)
    held = (c.codes.double() * c.scales.double()).view(x.shape)
    x, biggest = x.double(), x.double().amax(2, keepdim=True)
    off = (held - x).abs()
    near = (x >= biggest * 2.0 ** -13) & (x >= 2.0 ** -132)
    assert bool(near.any()) and bool((~near).any())
    assert bool((off <= x / 16)[near].all())
    assert bool((off < torch.maximum(biggest * 2.0 ** -16, torch.full_like(biggest, 2.0 ** -135)))[~near & (x > 0)].all())
    assert torch.equal(dense.ps_checkpoint_decode(c, t).double().view(x.shape), held)
