"""Input gradients of few rows, whose kernel reads the weights straight to registers: few and odd columns, contractions
in parts, strides, and what is not finite.  Tolerances are those of test_gpu_dense."""
import pytest

from tests.test_gpu_dense import TYPES, check_backward, check_forward, dense, gen, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", [(1, 3, 300), (1, 7, 300), (1, 8, 1000), (3, 9, 2000), (9, 4, 5000), (16, 130, 4500), (17, 129, 1031), (32, 2056, 2000), (2, 3001, 37),
                                           (31, 64, 16), (5, 1024, 33)])
def test_sizes(dense, dtype, rows, fin, fout):  # noqa: F811
    import torch
    t = getattr(torch, dtype)
    g = gen(rows * fin + fout)
    x, w, dy, z = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, rows, fout), randn(g, t, rows, fout, scale=2.0)
    for act in ("none", "gelu"):
        dx, _, _ = dense.ps_linear_backward(dy, x, w, act, pre=z if act != "none" else None, need_dw=False, need_db=False)
        check_backward((dx, None, None), dy, x, w, act, z)
        again, _, _ = dense.ps_linear_backward(dy, x, w, act, pre=z if act != "none" else None, need_dw=False, need_db=False)
        assert torch.equal(dx, again)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,extra", [(8, 16), (1, 3), (3, 5)])
def test_rows_apart_and_at_any_alignment(dense, dtype, first, extra):  # noqa: F811
    import torch
    t = getattr(torch, dtype)
    g = gen(first)
    rows, fin, fout = 11, 77, 530
    part = lambda r, c: randn(g, t, r, first + c + extra)[:, first:first + c]  # noqa: E731
    x, w, dy = part(rows, fin), part(fout, fin), part(rows, fout)
    room = torch.full((rows, first + fin + extra), 7.0, device="cuda", dtype=t)
    dense.ps_linear_backward(dy, x, w, need_dw=False, need_db=False, dx=room[:, first:first + fin])
    check_backward((room[:, first:first + fin], None, None), dy, x, w, "none", None)
    assert bool((room[:, :first] == 7).all()) and bool((room[:, first + fin:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fin,fout", [(70, 33), (264, 4099)])
def test_what_is_not_finite_stays_in_its_row_and_column(dense, dtype, fin, fout):  # noqa: F811
    import torch
    t = getattr(torch, dtype)
    g = gen(fin)
    w, dy, x = randn(g, t, fout, fin), randn(g, t, 4, fout), randn(g, t, 4, fin)
    w[fout - 1, 5], w[0, fin - 1] = float("inf"), float("nan")
    dy[2, fout - 1], dy[3, 7] = 0, float("inf")
    dx, _, _ = dense.ps_linear_backward(dy, x, w, need_dw=False, need_db=False)
    want = dy.double() @ w.double()
    assert torch.equal(dx.isfinite(), want.isfinite()) and torch.equal(dx.isnan(), want.isnan())
    assert int(dx[:3].isfinite().sum()) == 3 * (fin - 2)


def test_groups_whose_sizes_are_far_from_their_mean(dense):  # noqa: F811
    import torch
    t, g = torch.bfloat16, gen(4)
    sizes = [1, 0, 90, 2, 33, 0, 1, 1]
    edges = [sum(sizes[:i]) for i in range(len(sizes) + 1)]
    offsets = torch.tensor(edges, dtype=torch.int32, device="cuda")
    fin, fout = 200, 700
    x, w, dy = randn(g, t, edges[-1] + 5, fin), randn(g, t, len(sizes), fout, fin, scale=fin ** -0.5), randn(g, t, edges[-1] + 5, fout)
    dx = torch.full_like(x, 7.0)
    dense.ps_grouped_linear_backward(dy, x, offsets, w, need_dw=False, need_db=False, dx=dx)
    for i, n in enumerate(sizes):
        if n:
            s = slice(edges[i], edges[i + 1])
            check_backward((dx[s], None, None), dy[s], x[s], w[i], "none", None)
    assert bool((dx[edges[-1]:] == 7).all())


def test_more_groups_than_one_launch_of_the_small_blocks_holds(dense):  # noqa: F811
    """32768 groups, most of them empty, and 4608 columns: 9.4 million blocks of 16 columns would pass 2^32 threads."""
    import torch
    t, g = torch.bfloat16, gen(6)
    groups, rows, fin, fout = 32768, 40, 16, 4608
    edges = torch.zeros(groups + 1, dtype=torch.int32)
    edges[7:] = 9
    edges[20000:] = rows
    x, w, b = randn(g, t, rows, fin), randn(g, t, 2, fout, fin, scale=0.25), randn(g, t, 2, fout)
    index = torch.zeros(groups, dtype=torch.int32)
    index[19999] = 1
    y = dense.ps_grouped_linear_forward(x, edges.cuda(), w, b, weight_of_group=index.cuda())
    check_forward(y[:9], x[:9], w[0], b[0], None, "none")
    check_forward(y[9:], x[9:], w[1], b[1], None, "none")
