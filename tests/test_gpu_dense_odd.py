"""Layers whose rows are no multiples of 16 bytes and large enough for their operands to be copied to rows that are.
Tolerances are those of test_gpu_dense."""
import pytest

from tests.test_gpu_dense import TYPES, check_backward, check_forward, dense, gen, randn  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", [(3001, 1111, 777), (2049, 1025, 2050), (4096, 1023, 1024), (2500, 1024, 1025), (300, 1000, 77)])
def test_sizes(dense, dtype, rows, fin, fout):  # noqa: F811
    import torch
    t = getattr(torch, dtype)
    g = gen(rows + fin + fout)
    x, w, dy, z = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, rows, fout), randn(g, t, rows, fout, scale=2.0)
    b, r = randn(g, t, fout), randn(g, t, rows, fout)
    for act in ("none", "gelu"):
        pre = torch.empty_like(r)
        y = dense.ps_linear_forward(x, w, b, r, act, pre=pre)
        check_forward(y, x, w, b, r, act, pre)
        check_backward(dense.ps_linear_backward(dy, x, w, act, pre=z if act != "none" else None), dy, x, w, act, z)
    only = dense.ps_linear_backward(dy, x, w, need_dx=False, need_db=False)[1]
    assert torch.equal(only, dense.ps_linear_backward(dy, x, w, need_db=False)[1])


@pytest.mark.parametrize("dtype", TYPES)
def test_groups_and_rows_apart(dense, dtype):  # noqa: F811
    import torch
    t, g = getattr(torch, dtype), gen(8)
    sizes = [900, 0, 1300, 1, 700]
    edges = [3 + sum(sizes[:i]) for i in range(len(sizes) + 1)]
    rows, fin, fout = edges[-1] + 4, 1029, 515
    part = lambda *s: randn(g, t, *s[:-1], s[-1] + 4)[..., 1:s[-1] + 1]  # noqa: E731
    x, dy, w = part(rows, fin), part(rows, fout), randn(g, t, 3, fout + 2, fin + 5, scale=fin ** -0.5)[:, 1:-1, 3:-2]
    x[:3], x[-4:], dy[:3], dy[-4:] = 4 * [float("nan")]  # in no group
    offsets, index = torch.tensor(edges, dtype=torch.int32, device="cuda"), torch.tensor([2, 0, 0, 1, 2], dtype=torch.int32, device="cuda")
    y, dx = (torch.full((rows, n), 7.0, device="cuda", dtype=t) for n in (fout, fin))
    dense.ps_grouped_linear_forward(x, offsets, w, weight_of_group=index, out=y)
    _, dw, db = dense.ps_grouped_linear_backward(dy, x, offsets, w, weight_of_group=index, dx=dx)
    for i, k in enumerate(index.tolist()):
        s = slice(edges[i], edges[i + 1])
        if sizes[i]:
            check_forward(y[s], x[s], w[k], None, None, "none")
            check_backward((dx[s], dw[i], db[i]), dy[s], x[s], w[k], "none", None)
        else:
            assert bool((dw[i] == 0).all()) and bool((db[i] == 0).all())
    for o in (y, dx):
        assert bool((o[:3] == 7).all()) and bool((o[-4:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_what_is_not_finite_stays_in_its_row_and_column(dense, dtype):  # noqa: F811
    import torch
    t, g = getattr(torch, dtype), gen(9)
    rows, fin, fout = 2001, 1111, 1001
    x, w, dy = randn(g, t, rows, fin, scale=0.1), randn(g, t, fout, fin, scale=0.1), randn(g, t, rows, fout, scale=0.1)
    x[rows - 1, fin - 1], w[fout - 1, fin - 1], dy[rows - 1, fout - 1] = float("inf"), float("nan"), float("-inf")
    y = dense.ps_linear_forward(x, w)
    assert bool(y[:-1, :-1].isfinite().all()) and not bool(y[-1].isfinite().any()) and bool(y[:, -1].isnan().all())
    dx, dw, db = dense.ps_linear_backward(dy, x, w)
    assert bool(dx[:-1, :-1].isfinite().all()) and not bool(dx[-1].isfinite().any()) and bool(dx[:, -1].isnan().all())
    assert bool(dw[:-1, :-1].isfinite().all()) and not bool(dw[-1].isfinite().any()) and not bool(dw[:, -1].isfinite().any())
    assert bool(db[:-1].isfinite().all()) and float(db[-1]) == float("-inf")


@pytest.mark.parametrize("rows,fin,fout", [(2049, 1025, 1111), (5, 520, 4099)])
def test_captured_into_a_graph(dense, rows, fin, fout):  # noqa: F811
    """Copies, parts and the products of them, replayed on new values, with eager calls between the replays."""
    import torch
    t, g = torch.bfloat16, gen(rows)
    x, w, dy = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, rows, fout)
    call = lambda: (dense.ps_linear_forward(x, w), *dense.ps_linear_backward(dy, x, w))  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = call()
    for _ in range(4):
        for v in (x, w, dy):
            v.copy_(randn(g, t, *v.shape, scale=fin ** -0.5))
        want = [v.clone() for v in call()]
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))
