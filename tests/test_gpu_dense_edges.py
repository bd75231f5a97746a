"""Dense layers and AdamW on the GPU at their edges.  Tolerances are those of test_gpu_dense."""
import pytest

from tests.test_gpu_dense import dense, gen, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("bad", ["nan", "inf"])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("count", [257, 300, 504, 2049, 4099, 5000])
def test_adamw_what_is_not_finite_stays_in_its_block(dense, bad, dtype, rows, count):  # noqa: F811
    """A gradient that is not finite in the first block of a tensor, whose last block is not whole: all other blocks are, step after step, what they
    are without it."""
    import torch
    t, g = getattr(torch, dtype), gen(count + rows)
    start, steps = randn(g, t, count), randn(g, t, 4, rows, count, scale=0.1)
    runs = []
    for value in (None, float(bad)):
        p, grad = start.clone(), torch.empty(rows, count, device="cuda", dtype=t)
        opt = dense.ps_adamw_create([p], [grad], state_bits=8, weight_decay=0.1)
        seen = []
        for k in range(4):
            grad.copy_(steps[k])
            if k == 0 and value is not None:
                grad[rows - 1, 5] = value
            dense.ps_adamw_step(opt, k + 1, 0.01)
            seen.append([s.clone() for s in (p, opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0])])
        runs.append(seen)
        dense.ps_adamw_destroy(opt)
    for fine, hurt in zip(*runs):
        for a, b, first in zip(fine, hurt, (256, 256, 256, 1, 1)):
            assert torch.equal(a[first:], b[first:])
            assert a.dtype == torch.uint8 or bool(a.isfinite().all())
        assert bool(hurt[3][0].isnan() | hurt[3][0].isinf()) and bool(hurt[4][0].isnan() | hurt[4][0].isinf())
