"""Dense layers that keep their pre-activations in 8 bits, for groups whose offsets do not ascend: a group that ends before it begins is empty, and the
rows that are kept are those that any group has, as for pre-activations in the layer's type, whichever kernel does it."""
import pytest

from tests.test_gpu_checkpoint import bits
from tests.test_gpu_dense import dense, gen, randn  # noqa: F401

pytestmark = pytest.mark.gpu

CUTS = [[20, 30, 5, 10], [0, 30, 5, 10], [10, 12, 3, 4, 39, 2, 2, 38], [30, 20, 10], [35, 40, 0, 5, 100, -7, 20], [0, 0, 16, 3, 7, 1, 40]]


# few rows of a group, and so many columns that tiles take them
@pytest.mark.parametrize("fin,fout", [(64, 40), (48, 100), (33, 255), (16, 16384)])
@pytest.mark.parametrize("cuts", CUTS)
def test_the_same_rows_are_kept(dense, cuts, fin, fout):
    import torch
    rows, n, t = 40, len(cuts) - 1, torch.bfloat16
    g = gen(fin)
    offsets, index = torch.tensor(cuts, dtype=torch.int32).cuda(), torch.zeros(n, dtype=torch.int32, device="cuda")
    x, w = randn(g, t, rows, fin), randn(g, t, 1, fout, fin, scale=fin ** -0.5)
    pre, kept = torch.full((rows, fout), 7.0, device="cuda", dtype=t), dense.ps_checkpoint_empty(rows, fout, "cuda:0")
    kept.codes.view(torch.uint8).fill_(55)
    kept.scales.view(torch.uint8).fill_(66)
    dense.ps_grouped_linear_forward(x, offsets, w, None, None, "gelu", index, pre=pre)
    dense.ps_grouped_linear_forward(x, offsets, w, None, None, "gelu", index, pre=kept)
    there = torch.zeros(rows, dtype=torch.bool)
    for lo, hi in zip(cuts, cuts[1:]):
        there[max(lo, 0):max(hi, 0)] = True
    assert torch.equal((pre != 7).any(1).cpu(), there)
    code, scale = bits(kept)
    want = bits(dense.ps_checkpoint_encode(pre))
    assert torch.equal(code[there], want[0][there]) and torch.equal(scale[there], want[1][there])
    assert bool((code[~there] == 55).all()) and bool((scale[~there] == 66).all())


@pytest.mark.parametrize("groups,rows", [(1, 3), (64, 64), (65, 200), (3000, 4000), (200, 50)])
def test_many_small_groups(dense, groups, rows):
    import torch
    g, t = gen(groups), torch.float16
    cuts = sorted(torch.randint(0, rows + 1, (groups + 1,), generator=torch.Generator().manual_seed(rows)).tolist())
    offsets, index = torch.tensor(cuts, dtype=torch.int32).cuda(), (torch.arange(groups, device="cuda") % 3).int()
    x, w, b = randn(g, t, rows, 40), randn(g, t, 3, 72, 40), randn(g, t, 3, 72)
    pre, kept = torch.full((rows, 72), 7.0, device="cuda", dtype=t), dense.ps_checkpoint_empty(rows, 72, "cuda:0")
    kept.codes.view(torch.uint8).fill_(55)
    kept.scales.view(torch.uint8).fill_(66)
    y = dense.ps_grouped_linear_forward(x, offsets, w, b, None, "silu", index, pre=pre)
    y8 = dense.ps_grouped_linear_forward(x, offsets, w, b, None, "silu", index, pre=kept)
    inside = slice(cuts[0], cuts[-1])
    assert torch.equal(y[inside], y8[inside])
    code, scale = bits(kept)
    want = bits(dense.ps_checkpoint_encode(pre))
    assert torch.equal(code[inside], want[0][inside]) and torch.equal(scale[inside], want[1][inside])
    outside = torch.cat([torch.arange(cuts[0]), torch.arange(cuts[-1], rows)])
    assert bool((code[outside] == 55).all()) and bool((scale[outside] == 66).all())
