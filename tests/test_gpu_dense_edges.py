"""Dense layers and AdamW on the GPU at their edges.  Tolerances are those of test_gpu_dense."""
import pytest

from tests.test_gpu_dense import TYPES, check_backward, check_forward, dense, gen, randn  # noqa: F401

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


def matrix(dense, t):  # noqa: F811
    return dense.ps_matrix(t.data_ptr(), t.stride(-2) if t.dim() > 1 else t.numel(), t.stride(0) if t.dim() > 1 else 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", [(5, 4096, 200), (128, 4096, 256), (100, 2048, 77), (300, 64, 80)])
def test_one_group_of_all_rows_on_any_of_several_matrices(dense, dtype, rows, fin, fout):  # noqa: F811
    """Without offsets, and with the number of the matrix: W and the bias are that matrix's, also where the contraction is cut into parts
    (the second and third size, in dx the first too)."""
    import ctypes

    import torch
    t, g = getattr(torch, dtype), gen(rows + fin)
    x, w, b = randn(g, t, rows, fin), randn(g, t, 3, fout, fin, scale=fin ** -0.5), randn(g, t, 3, fout)
    y, z = torch.empty(rows, fout, device="cuda", dtype=t), torch.empty(rows, fout, device="cuda", dtype=t)
    dy, dx = randn(g, t, rows, fout), torch.empty(rows, fin, device="cuda", dtype=t)
    dw, db = torch.empty(fout, fin, device="cuda", dtype=t), torch.empty(fout, device="cuda", dtype=t)
    lib, stream = dense._library(), torch.cuda.current_stream().cuda_stream
    for number in (2, 0):
        index = torch.tensor([number], dtype=torch.int32, device="cuda")
        layer = dense.ps_linear(dense._DTYPES[t], dense.ACTIVATIONS["gelu"], rows, fin, fout, 1, 3, None, index.data_ptr())
        for backward, operands in ((0, (x, w, b, None, y, z)), (1, (dy, x, w, z, dx, dw, db))):
            need = ctypes.c_uint64(0)
            assert lib.ps_linear_workspace_bytes(ctypes.byref(layer), backward, ctypes.byref(need)) == 0
            ws = torch.empty(max(need.value, 1), dtype=torch.uint8, device="cuda")
            args = [None if o is None else ctypes.byref(matrix(dense, o)) for o in operands]
            call = lib.ps_linear_backward if backward else lib.ps_linear_forward
            assert call(ctypes.byref(layer), *args, ws.data_ptr(), need.value, stream) == 0, lib.ps_dense_last_error()
            torch.cuda.synchronize()
        check_forward(y, x, w[number], b[number], None, "gelu", z)
        check_backward((dx, dw, db), dy, x, w[number], "gelu", z)


@pytest.mark.parametrize("dtype", ["bfloat16", "float32"])
def test_more_tiles_than_one_dimension_of_a_grid_holds(dense, dtype):  # noqa: F811
    """4097 groups of a row each and 262,208 columns: more blocks of 16 columns than a launch has room for, and 17.05 million tiles of 64 x 64,
    where 2^24 blocks of 256 threads make 2^32 threads."""
    import torch
    t, g = getattr(torch, dtype), gen(7)
    groups, narrow, wide = 4097, 16, 262208
    offsets = torch.arange(groups + 1, dtype=torch.int32, device="cuda")
    index = torch.zeros(groups, dtype=torch.int32, device="cuda")
    x, w = randn(g, t, groups, narrow), randn(g, t, wide, narrow, scale=0.25)
    y = dense.ps_grouped_linear_forward(x, offsets, w[None], weight_of_group=index)
    for c in range(0, wide, 16384):
        check_forward(y[:, c:c + 16384], x, w[c:c + 16384], None, None, "none")
    del y
    dy, v = randn(g, t, groups, narrow), randn(g, t, narrow, wide, scale=0.25)
    dx, _, _ = dense.ps_grouped_linear_backward(dy, torch.empty(groups, wide, device="cuda", dtype=t), offsets, v[None], weight_of_group=index, need_dw=False, need_db=False)
    for c in range(0, wide, 16384):
        check_backward((dx[:, c:c + 16384], None, None), dy, x[:, :1], v[:, c:c + 16384], "none", None)


@pytest.mark.parametrize("beside", [float("nan"), 1e38])
@pytest.mark.parametrize("rows,fin,fout", [(300, 100, 72), (1030, 136, 260), (1030, 135, 263)])
def test_what_lies_beside_an_operand_changes_nothing(dense, beside, rows, fin, fout):  # noqa: F811
    """fp32 operands that are views of wider rows: their products have the same bytes whatever the columns beside them hold."""
    import torch
    g = gen(rows + fin)
    values = [randn(g, torch.float32, rows, fin), randn(g, torch.float32, fout, fin), randn(g, torch.float32, rows, fout)]
    runs = []
    for fill in (0.0, beside):
        wide = [torch.full((v.shape[0], v.shape[1] + 300), fill, device="cuda") for v in values]
        x, w, dy = [b[:, 60:60 + v.shape[1]].copy_(v) for b, v in zip(wide, values)]
        runs.append((dense.ps_linear_forward(x, w), *dense.ps_linear_backward(dy, x, w)))
    check_forward(runs[1][0], values[0], values[1], None, None, "none")
    check_backward(runs[1][1:], values[2], values[0], values[1], "none", None)
    assert all(torch.equal(a, b) for a, b in zip(*runs))


# magnitudes of the two operands of a product; the third: every second row of the first is as large as makes ordinary products, 1 at most
EXTREMES = [(1.2e-37, 1e30, False), (1e30, 1.2e-37, False), (3e-37, 1e35, True), (1e-41, 1e37, False), (1e-42, 3e37, True), (1e-15, 1e-15, False), (1e-12, 3e-18, True)]


@pytest.mark.parametrize("rows,fin,fout", [(40, 64, 96), (200, 64, 96), (333, 200, 135), (700, 1025, 260)])
@pytest.mark.parametrize("a,b,mixed", EXTREMES)
def test_fp32_operands_of_extreme_sizes(dense, a, b, mixed, rows, fin, fout):  # noqa: F811
    """Products of ordinary size, of fp32 operands that the split into three bf16 parts does not hold in all their bits, or at all, and sums that
    are tiny: as exact as any others.  (Inputs and what is expected are made on the CPU, which keeps subnormal numbers.)"""
    import torch
    g = torch.Generator()
    g.manual_seed(rows + fin)
    def values(n, k, size, some=False):  # noqa: E306
        v = torch.randn(n, k, generator=g) * size
        if some:
            v[::2] = torch.randn(v[::2].shape, generator=g) * min(1.0, 1 / b)
        return v.cuda()
    x, w = values(rows, fin, a, mixed), values(fout, fin, b)
    y = dense.ps_linear_forward(x, w)
    check_forward(y.cpu(), x.cpu(), w.cpu(), None, None, "none")
    dy, v, u = values(rows, fout, a, mixed), values(fout, fin, b), values(rows, fin, b)
    dx, dw, _ = dense.ps_linear_backward(dy, u, v, need_db=False)
    check_backward((dx.cpu(), dw.cpu(), None), dy.cpu(), u.cpu(), v.cpu(), "none", None)


def test_a_handle_dropped_while_a_step_runs_on_another_stream(dense):  # noqa: F811
    """Its table and states are not given out again on the stream where they were made before that step is done."""
    import torch
    n = 3_000_017
    start, grad = torch.randn(n, device="cuda"), torch.randn(n, device="cuda")
    want, got = start.clone(), start.clone()
    dense.ps_adamw_step(dense.ps_adamw_create([want], [grad], state_bits=8), 1, 0.1)
    opt = dense.ps_adamw_create([got], [grad], state_bits=8)
    own = [opt.workspace, opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0]]
    places, sizes = {t.data_ptr() for t in own}, [t.numel() * t.element_size() for t in own]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        torch.cuda._sleep(200_000_000)  # a tenth of a second: a step that waits for its turn
        dense.ps_adamw_step(opt, 1, 0.1)
    del opt, own
    others = [torch.full((b,), 255, dtype=torch.uint8, device="cuda") for b in sizes]
    assert not places & {t.data_ptr() for t in others}
    torch.cuda.synchronize()
    assert torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
def test_more_groups_than_are_counted_beforehand(dense, dtype):  # noqa: F811
    """1300 groups, beyond the 1024 whose tiles the kernels count, a third of them empty and one of them large: forward and all gradients."""
    import torch
    t, g = getattr(torch, dtype), gen(9)
    sizes = [(0, 3, 5)[i % 3] if i != 700 else 2000 for i in range(1300)]
    edges = [0]
    for n in sizes:
        edges.append(edges[-1] + n)
    rows, fin, fout = edges[-1], 40, 24
    offsets = torch.tensor(edges, dtype=torch.int32, device="cuda")
    index = torch.tensor([i % 3 for i in range(len(sizes))], dtype=torch.int32, device="cuda")
    x, w, b, dy = randn(g, t, rows, fin), randn(g, t, 3, fout, fin, scale=fin ** -0.5), randn(g, t, 3, fout), randn(g, t, rows, fout)
    z = torch.empty(rows, fout, device="cuda", dtype=t)
    y = dense.ps_grouped_linear_forward(x, offsets, w, b, None, "silu", index, pre=z)
    dx, dw, db = dense.ps_grouped_linear_backward(dy, x, offsets, w, "silu", z, index)
    group = torch.repeat_interleave(torch.arange(len(sizes), device="cuda"), torch.tensor(sizes, device="cuda"))
    for k in range(3):
        r = (group % 3 == k).nonzero().squeeze(1)
        if len(r):
            check_forward(y[r], x[r], w[k], b[k], None, "silu", z[r])
            check_backward((dx[r], None, None), dy[r], x[r], w[k], "silu", z[r])
    for i in (0, 1, 2, 3, 699, 700, 701, 1023, 1024, 1025, 1297, 1298, 1299):
        s = slice(edges[i], edges[i + 1])
        if sizes[i]:
            check_backward((None, dw[i], db[i]), dy[s], x[s], w[i % 3], "silu", z[s])
    empty = torch.tensor(sizes, device="cuda") == 0
    assert bool((dw[empty] == 0).all()) and bool((db[empty] == 0).all()) and bool((dw[~empty] != 0).flatten(1).any(1).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_forward_on_both_sides_of_the_limits_for_few_rows(dense, dtype):  # noqa: F811
    """One group: rows times features, narrow results of deep contractions, rows that are no multiples of 16 bytes; groups: rows times columns, evenly
    spread or all in one group."""
    import torch
    t, g = getattr(torch, dtype), gen(11)
    for rows, fin, fout in ((24, 4096, 200), (25, 4096, 200), (64, 1536, 72), (64, 1544, 72), (2, 4096, 64), (2, 4104, 64), (2, 8200, 64), (2, 8200, 4096), (6, 4096, 16400),
                            (50, 1111, 96), (51, 1111, 96), (1, 4097, 300), (3, 4097, 300)):
        x, w, b, r = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, fout), randn(g, t, rows, fout)
        z = torch.empty(rows, fout, device="cuda", dtype=t)
        check_forward(dense.ps_linear_forward(x, w, b, r, "gelu", pre=z), x, w, b, r, "gelu", z)
    groups, fin, fout = 16, 72, 2056
    w, b = randn(g, t, groups, fout, fin, scale=fin ** -0.5), randn(g, t, groups, fout)
    for each in (4, 5, 15, 16, 40):
        for sizes in ([each] * groups, [0] * 7 + [each * groups] + [0] * 8):
            edges = [sum(sizes[:i]) for i in range(groups + 1)]
            x = randn(g, t, edges[-1], fin)
            y = dense.ps_grouped_linear_forward(x, torch.tensor(edges, dtype=torch.int32, device="cuda"), w, b, None, "relu")
            for i in range(groups):
                if sizes[i]:
                    s = slice(edges[i], edges[i + 1])
                    check_forward(y[s], x[s], w[i], b[i], None, "relu")
