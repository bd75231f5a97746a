"""Dense layers and AdamW on the GPU against their formulas in 64 bits.

Tolerances.  A result is rounded once, by at most half a step: half(t) = eps(t) / 2 of its magnitude, or, where it is
subnormal, half of the smallest subnormal number.  In front of that a sum of
K products and a bias, held in 32 bits, is off by at most (K + 2) steps of 2^-23 (matrix instructions may cut off instead of
rounding) of the sum S of the products' magnitudes; an activation's slope is below 1.13, and the activation itself is evaluated to
8 steps of 2^-23 of |z| + 1.  In a backward pass with an activation, dz is rounded to the operands' type first: half(t) of
the sum of the magnitudes |dz| |w|."""
import math

import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -23
TYPES = ["float32", "bfloat16", "float16"]


@pytest.fixture(scope="module")
def dense():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2406_05546_amd import dense as d
    d._library()
    return d


def half(t):
    import torch
    return torch.finfo(t).eps / 2


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def randn(g, dtype, *shape, scale=1.0):
    import torch
    return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)


def phi64(z):
    import torch
    return 0.5 * torch.special.erfc(-z * 0.5 ** 0.5)  # torch's ndtr has no bits left below -8


def act64(z, a):
    import torch
    return {"none": lambda: z, "relu": lambda: torch.where(z <= 0, torch.zeros_like(z), z), "gelu": lambda: z * phi64(z), "silu": lambda: z * torch.sigmoid(z)}[a]()


def slope64(z, a):
    import torch
    return {"none": lambda: torch.ones_like(z), "relu": lambda: (z > 0).to(z.dtype), "silu": lambda: torch.sigmoid(z) * (1 + z * torch.sigmoid(-z)),
            "gelu": lambda: phi64(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)}[a]()


def close(got, want, tol, what):
    import torch
    off = (got.double() - want).abs()
    info = torch.finfo(got.dtype)
    tol = tol + info.tiny * info.eps / 2
    bad = ~(off <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} values, worst {float((off / tol).nan_to_num(9e9).max()):.3g} times what it may be"


def check_forward(got, x, w, b, r, act, pre=None):
    x, w = x.double(), w.double()
    z = x @ w.t()
    size = x.abs() @ w.abs().t()
    if b is not None:
        z, size = z + b.double(), size + b.double().abs()
    ez = U * (x.shape[1] + 2) * size
    y = act64(z, act)
    ey = 1.13 * ez + (8 * U * (z.abs() + 1) if act in ("gelu", "silu") else 0)
    if r is not None:
        y = y + r.double()
        ey = ey + U * y.abs()
    close(got, y, ey + half(got.dtype) * (y.abs() + ey), f"y {tuple(got.shape)} {act}")
    if pre is not None:
        close(pre, z, ez + half(got.dtype) * (z.abs() + ez), "pre")


def check_backward(got, dy, x, w, act, z):
    t = dy.dtype
    dy, x, w = dy.double(), x.double(), w.double()
    if act != "none":
        s = slope64(z.double(), act)
        dz = dy * s
        each = dy.abs() * (16 * U * (1 + z.double().abs()) if act in ("gelu", "silu") else 0)  # the slope's evaluation
    else:
        dz, each = dy, 0 * dy
    rounded = each + (half(t) * dz.abs() if act != "none" else 0)
    if act != "none" and t.itemsize == 2 and str(t) == "torch.float16":
        rounded = rounded + 2.0 ** -25  # subnormal dz
    dx, dw, db = got
    if dx is not None:
        want, e = dz @ w, rounded @ w.abs() + U * (w.shape[0] + 2) * (dz.abs() @ w.abs())
        close(dx, want, e + half(t) * (want.abs() + e), "dx")
    if dw is not None:
        want, e = dz.t() @ x, rounded.t() @ x.abs() + U * (x.shape[0] + 2) * (dz.abs().t() @ x.abs())
        close(dw, want, e + half(t) * (want.abs() + e), "dw")
    if db is not None:
        want, e = dz.sum(0), each.sum(0) + U * (x.shape[0] + 2) * dz.abs().sum(0)
        close(db, want, e + half(t) * (want.abs() + e), "db")


# one row to more than a tile, features that fill tiles and stages and that do not, odd ones among them
SIZES = [(1, 1, 1), (1, 64, 64), (2, 7, 3), (5, 200, 33), (15, 128, 130), (16, 96, 64), (17, 72, 200), (33, 256, 48), (63, 65, 66), (64, 512, 128), (65, 129, 255),
         (100, 40, 264), (128, 64, 256), (130, 264, 136), (257, 320, 260), (300, 1000, 77), (512, 64, 512), (1025, 136, 72)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", SIZES)
def test_forward(dense, dtype, rows, fin, fout):
    import torch
    t = getattr(torch, dtype)
    g = gen(rows + fin + fout)
    x, w = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5)
    b, r = randn(g, t, fout), randn(g, t, rows, fout)
    for act, bias, residual, save in (("none", None, None, False), ("relu", b, None, True), ("gelu", b, r, True), ("silu", None, r, False)):
        pre = torch.empty(rows, fout, device="cuda", dtype=t) if save else None
        y = dense.ps_linear_forward(x, w, bias, residual, act, pre=pre)
        check_forward(y, x, w, bias, residual, act, pre)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", SIZES)
def test_backward(dense, dtype, rows, fin, fout):
    import torch
    t = getattr(torch, dtype)
    g = gen(rows + fin + fout)
    x, w, dy, z = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, rows, fout), randn(g, t, rows, fout, scale=2.0)
    for act in ("none", "relu", "gelu", "silu"):
        got = dense.ps_linear_backward(dy, x, w, act, pre=z if act != "none" else None)
        check_backward(got, dy, x, w, act, z)
    only = dense.ps_linear_backward(dy, x, w, "silu", pre=z, need_dx=False, need_db=False)
    assert only[0] is None and only[2] is None and torch.equal(only[1], got[1])
    only = dense.ps_linear_backward(dy, x, w, "silu", pre=z, need_dx=False, need_dw=False)
    assert torch.equal(only[2], got[2])


@pytest.mark.parametrize("dtype", TYPES)
def test_a_layer_as_large_as_the_largest_tiles(dense, dtype):
    import torch
    t = getattr(torch, dtype)
    g = gen(5)
    rows, fin, fout = 4096, 512, 4352
    x, w, b = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, fout)
    pre = torch.empty(rows, fout, device="cuda", dtype=t)
    y = dense.ps_linear_forward(x, w, b, None, "relu", pre=pre)
    check_forward(y, x, w, b, None, "relu", pre)
    dy = randn(g, t, rows, fout)
    check_backward(dense.ps_linear_backward(dy, x, w, "relu", pre=pre), dy, x, w, "relu", pre)
    x, dy = randn(g, t, 1024, 4096), randn(g, t, 1024, 4224)
    w = randn(g, t, 4224, 4096, scale=2.0 ** -6)
    check_backward(dense.ps_linear_backward(dy, x, w), dy, x, w, "none", None)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("first,extra", [(0, 8), (8, 16), (1, 3), (3, 5)])
def test_rows_apart_and_at_any_alignment(dense, dtype, first, extra):
    import torch
    t = getattr(torch, dtype)
    g = gen(first + extra)
    rows, fin, fout = 70, 96, 136
    def view(n, m):
        return randn(g, t, n, first + m + extra)[:, first:first + m]
    x, w, r, dy, z = view(rows, fin), view(fout, fin), view(rows, fout), view(rows, fout), view(rows, fout)
    b = randn(g, t, fout + 3)[3:]
    out = torch.full((rows, fout + 9), 7.0, device="cuda", dtype=t)
    pre = torch.full((rows, fout + 9), 7.0, device="cuda", dtype=t)
    y = dense.ps_linear_forward(x, w, b, r, "gelu", pre=pre[:, 5:-4], out=out[:, 5:-4])
    check_forward(y, x, w, b, r, "gelu", pre[:, 5:-4])
    for o in (out, pre):
        assert bool((o[:, :5] == 7).all()) and bool((o[:, -4:] == 7).all())
    dx, dw = torch.full((rows, fin + 3), 7.0, device="cuda", dtype=t), torch.full((fout, fin + 3), 7.0, device="cuda", dtype=t)
    got = dense.ps_linear_backward(dy, x, w, "gelu", pre=z, dx=dx[:, 1:-2], dw=dw[:, 1:-2])
    check_backward(got, dy, x, w, "gelu", z)
    for o in (dx, dw):
        assert bool((o[:, :1] == 7).all()) and bool((o[:, -2:] == 7).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_the_result_may_take_the_residuals_place(dense, dtype):
    import torch
    t = getattr(torch, dtype)
    for rows, fin, fout in ((3, 40, 24), (200, 64, 72), (64, 4096, 64)):
        g = gen(rows)
        x, w, r = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, rows, fout)
        want = dense.ps_linear_forward(x, w, None, r, "silu")
        got = dense.ps_linear_forward(x, w, None, r, "silu", out=r)
        assert got is r and torch.equal(got, want)


@pytest.mark.parametrize("dtype", TYPES)
def test_infinities_and_nan_stay_in_their_row_and_column(dense, dtype):
    import torch
    t = getattr(torch, dtype)
    for rows, fin, fout in ((3, 70, 33), (150, 72, 264)):
        g = gen(3)
        x, w = randn(g, t, rows, fin), randn(g, t, fout, fin)
        x[1, 5], x[2, 7], w[4, 0] = float("nan"), float("inf"), float("-inf")
        y = dense.ps_linear_forward(x, w, activation="relu").double()
        want = act64(x.double() @ w.double().t(), "relu")
        assert torch.equal(y.isnan(), want.isnan()) and torch.equal(y.isinf(), want.isinf()) and bool(y[1].isnan().all())
        fine = want.isfinite()
        assert float((y - want)[fine].abs().max()) <= 2 * half(t) * float(want[fine].abs().max()) + U * fin * fin
        dx, dw, db = dense.ps_linear_backward(y.to(t), x, w)
        assert bool(dx[1].isnan().all()) and bool(dw.isnan().all()) and bool(db.isnan().all())  # row 1 is NaN, and every column has it
        dy = randn(g, t, rows, fout)
        dy[0, 3] = float("inf")
        dx, dw, db = dense.ps_linear_backward(dy, x, randn(g, t, fout, fin))
        assert not bool(dx[0].isfinite().any()) and bool(dx[1:].isfinite().all())
        assert not bool(dw[3].isfinite().any()) and bool(db[3].isinf()) and bool(torch.cat([db[:3], db[4:]]).isfinite().all())


def test_activations_far_out(dense):
    import torch
    z = torch.tensor([-1e30, -200.0, -30.0, -9.0, -6.0, -1e-30, 0.0, 1e-30, 6.0, 30.0, 200.0, 1e30], device="cuda")[:, None]
    one = torch.ones(1, 1, device="cuda")
    for act in ("relu", "gelu", "silu"):
        y = dense.ps_linear_forward(z, one, activation=act).double()
        want = act64(z.double(), act)
        # relative, also where z is very negative and the result tiny (z is rounded before exp and erfc: 2^-24 z^2 in the exponent)
        close(y, want, want.abs() * (2e-6 + 2.0 ** -22 * z.double().square().clamp(max=200)) + 1e-37, act)
        dx = dense.ps_linear_backward(one.expand(12, 1).contiguous(), z, one, act, pre=z, need_dw=False)[0]
        close(dx, slope64(z.double(), act).nan_to_num(0.0), torch.full_like(z, 1e-5).double(), act + " slope")


@pytest.mark.parametrize("dtype", TYPES)
def test_gradients_against_differences(dense, dtype):
    """The loss sum(y * c) along random directions, y in 64 bits: the formula's gradients are the loss's, and the kernel's are
    checked against the formula's everywhere else."""
    import torch
    t = getattr(torch, dtype)
    rows, fin, fout = 9, 20, 12
    for act in ("gelu", "silu"):
        g = gen(7)
        x, w, b, c = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=0.3), randn(g, t, fout), randn(g, t, rows, fout)
        pre = torch.empty(rows, fout, device="cuda", dtype=t)
        dense.ps_linear_forward(x, w, b, None, act, pre=pre)
        grads = dense.ps_linear_backward(c, x, w, act, pre=pre)
        at = [x.double(), w.double(), b.double()]
        def loss(x, w, b):
            return float((act64(x @ w.t() + b, act) * c.double()).sum())
        for i, d in enumerate(grads):
            v = torch.randn(at[i].shape, device="cuda", dtype=torch.float64, generator=g)
            h = 1e-4
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            slope = (loss(*up) - loss(*down)) / (2 * h)
            # pre, dz and the gradient are rounded, each along every term of the sum: a few half steps of its magnitude
            tol = 8 * half(t) * float((d.double() * v).abs().sum()) + 40 * half(t) * float(c.double().abs().sum()) * (1 if i == 2 else 2) + 1e-5
            assert abs(slope - float((d.double() * v).sum())) <= tol


# ---- groups ---------------------------------------------------------------------------------------------------------

SPLITS = [[5], [0, 7, 0], [1, 1, 1, 1], [64, 0, 65, 130, 3], [300, 1, 0, 0, 200], [0, 0], [3] * 70 + [0] * 60 + [100]]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("fin,fout", [(64, 128), (33, 50)])
@pytest.mark.parametrize("split", SPLITS, ids=lambda s: f"{len(s)}groups{sum(s)}")
def test_groups(dense, dtype, fin, fout, split):
    import torch
    t = getattr(torch, dtype)
    g = gen(len(split) + fin)
    edges = [0]
    for n in split:
        edges.append(edges[-1] + n)
    rows, G, V = edges[-1], len(split), max(1, len(split) // 2)
    offsets = torch.tensor(edges, dtype=torch.int32, device="cuda")
    index = torch.tensor([(3 * i + 1) % V for i in range(G)], dtype=torch.int32, device="cuda")
    x, r, dy, z = randn(g, t, rows, fin), randn(g, t, rows, fout), randn(g, t, rows, fout), randn(g, t, rows, fout)
    for ids, mats in ((index, V), (None, G)):
        w, b = randn(g, t, mats, fout, fin, scale=fin ** -0.5), randn(g, t, mats, fout)
        pre = torch.empty_like(r)
        y = dense.ps_grouped_linear_forward(x, offsets, w, b, r, "silu", weight_of_group=ids, pre=pre)
        dx, dw, db = dense.ps_grouped_linear_backward(dy, x, offsets, w, "silu", pre=z, weight_of_group=ids)
        for i in range(G):
            s, k = slice(edges[i], edges[i + 1]), int(index[i]) if ids is not None else i
            if split[i]:
                check_forward(y[s], x[s], w[k], b[k], r[s], "silu", pre[s])
                check_backward((dx[s], dw[i], db[i]), dy[s], x[s], w[k], "silu", z[s])
            else:
                assert bool((dw[i] == 0).all()) and bool((db[i] == 0).all())


def test_rows_in_no_group_are_left_alone(dense):
    import torch
    t, g = torch.bfloat16, gen(1)
    rows, fin, fout = 200, 64, 96
    x, w, dy = randn(g, t, rows, fin), randn(g, t, 2, fout, fin), randn(g, t, rows, fout)
    offsets = torch.tensor([10, 50, 150], dtype=torch.int32, device="cuda")
    out, pre, dx = (torch.full((rows, n), 7.0, device="cuda", dtype=t) for n in (fout, fout, fin))
    dense.ps_grouped_linear_forward(x, offsets, w, activation="relu", pre=pre, out=out)
    z = pre.clone()
    _, dw, db = dense.ps_grouped_linear_backward(dy, x, offsets, w, "relu", pre=z, dx=dx)
    for o in (out, pre, dx):
        assert bool((o[:10] == 7).all()) and bool((o[150:] == 7).all()) and not bool((o[10:150] == 7).all(1).any())
    for i, s in enumerate((slice(10, 50), slice(50, 150))):
        check_forward(out[s], x[s], w[i], None, None, "relu", pre[s])
        check_backward((dx[s], dw[i], db[i]), dy[s], x[s], w[i], "relu", z[s])


def test_offsets_and_numbers_that_are_none(dense):
    """Offsets outside the rows are taken into them, a group that ends before it begins is empty, numbers of matrices go to
    the nearest: nothing outside the operands is read or written."""
    import torch
    t, g = torch.bfloat16, gen(2)
    rows, fin, fout = 100, 64, 64
    x, w = randn(g, t, rows, fin), randn(g, t, 2, fout, fin)
    offsets = torch.tensor([-5, 40, 30, 2 ** 31 - 1], dtype=torch.int32, device="cuda")  # groups 0..40, none, 30..100
    index = torch.tensor([-7, 0, 99], dtype=torch.int32, device="cuda")
    y = dense.ps_grouped_linear_forward(x, offsets, w, weight_of_group=index)
    check_forward(y[:30], x[:30], w[0], None, None, "none")
    check_forward(y[40:], x[40:], w[1], None, None, "none")
    dy = randn(g, t, rows, fout)
    dx, dw, db = dense.ps_grouped_linear_backward(dy, x, offsets, w, weight_of_group=index)
    check_backward((None, dw[0], db[0]), dy[:40], x[:40], w[0], "none", None)
    check_backward((dx[40:], None, None), dy[40:], x[40:], w[1], "none", None)
    check_backward((None, dw[2], db[2]), dy[30:], x[30:], w[1], "none", None)
    assert bool((dw[1] == 0).all()) and bool((db[1] == 0).all())


def test_gradients_into_rows_of_a_buffer(dense):
    """A group's gradients land in its row of the server's buffer, at whatever place in the row the layer has."""
    import torch
    t, g = torch.float32, gen(4)
    G, fin, fout, at, pitch = 5, 40, 24, 13, 1200
    offsets = torch.tensor([0, 9, 9, 30, 31, 50], dtype=torch.int32, device="cuda")
    rows = torch.full((G, pitch), 7.0, device="cuda")
    dw = rows[:, at:at + fout * fin].view(G, fout, fin)
    db = rows[:, at + fout * fin:at + fout * fin + fout]
    x, dy, w = randn(g, t, 50, fin), randn(g, t, 50, fout), randn(g, t, 1, fout, fin)
    index = torch.zeros(G, dtype=torch.int32, device="cuda")
    dense.ps_grouped_linear_backward(dy, x, offsets, w, weight_of_group=index, dw=dw, db=db)
    e = offsets.tolist()
    for i in range(G):
        check_backward((None, dw[i], db[i]), dy[e[i]:e[i + 1]], x[e[i]:e[i + 1]], w[0], "none", None)
    end = at + fout * fin + fout
    assert bool((rows[:, :at] == 7).all()) and bool((rows[:, end:] == 7).all())


# ---- streams, graphs, repeats ----------------------------------------------------------------------------------------

def test_the_same_bytes_every_time_and_on_another_stream(dense):
    import torch
    t, g = torch.bfloat16, gen(6)
    x, w, dy, z = randn(g, t, 3000, 128), randn(g, t, 136, 128), randn(g, t, 3000, 136), randn(g, t, 3000, 136)
    want = (dense.ps_linear_forward(x, w, None, z, "gelu"),) + dense.ps_linear_backward(dy, x, w, "gelu", pre=z)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for stream in (torch.cuda.current_stream(), side, side):
        with torch.cuda.stream(stream):
            got = (dense.ps_linear_forward(x, w, None, z, "gelu"),) + dense.ps_linear_backward(dy, x, w, "gelu", pre=z)
            same = [bool(torch.equal(a, b)) for a, b in zip(got, want)]
        assert all(same)
    torch.cuda.current_stream().wait_stream(side)


def test_captured_into_a_graph(dense):
    import torch
    t, g = torch.bfloat16, gen(8)
    offsets = torch.tensor([0, 3, 70, 70, 200], dtype=torch.int32, device="cuda")
    x, w, dy = randn(g, t, 200, 64), randn(g, t, 4, 72, 64), randn(g, t, 200, 72)
    z = torch.empty(200, 72, device="cuda", dtype=t)
    p = torch.zeros(4 * 72 * 64, device="cuda")
    grads = torch.zeros(1, 4 * 72 * 64, device="cuda", dtype=t)
    opt = dense.ps_adamw_create([p], [grads], state_bits=8)
    def step():
        y = dense.ps_grouped_linear_forward(x, offsets, w, None, None, "silu", pre=z)
        dx, dw, db = dense.ps_grouped_linear_backward(dy, x, offsets, w, "silu", pre=z)
        grads.copy_(dw.view(1, -1))
        dense.ps_adamw_step(opt, 3, 0.1)
        return y, dx, dw, db
    state = [p, opt.m[0], opt.v[0], opt.m_scale[0], opt.v_scale[0]]
    def zero():
        for s in state:
            s.zero_()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = step()
    for i in range(3):
        x.copy_(randn(g, t, 200, 64))
        offsets.copy_(torch.tensor([0, 3 + i, 70, 70 + i, 200], dtype=torch.int32))
        zero()
        want = step() + tuple(s.clone() for s in state)
        torch.cuda.synchronize()
        zero()
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(outs + tuple(state), want))


# ---- AdamW ---------------------------------------------------------------------------------------------------------

def adamw64(p, g, m, v, step, lr, b1, b2, eps, wd):
    m = b1 * m + (1 - b1) * g
    v = b2 * v + (1 - b2) * g * g
    p = p - lr * wd * p - lr / (1 - b1 ** step) * m / ((v / (1 - b2 ** step)).sqrt() + eps)
    return p, m, v


def encode(x, root):
    """The 8-bit state in 32-bit operations, one rounding each, as documented."""
    import torch
    n = x.numel()
    b = torch.zeros(-(-n // 256) * 256, device=x.device)
    b[:n] = x
    b = b.view(-1, 256)
    top = b.abs().amax(1).clamp(min=2.0 ** -100)
    q = (b * torch.div(torch.full_like(top, 448.0), top)[:, None]).to(torch.float8_e4m3fn).view(torch.uint8)
    if root:
        q = torch.where((b > 0) & (q == 0), torch.ones_like(q), q)
    return q.view(-1)[:n], top * (1.0 / 448.0)


COUNTS = [[1], [7], [256], [255, 257], [8, 2048, 2049, 3], [0, 5, 0], [100001], [16, 144, 4608, 32, 5120, 10]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("dtype,grad", [("float32", "float32"), ("bfloat16", "bfloat16"), ("float32", "bfloat16"), ("float16", "float16"), ("bfloat16", "float32")])
@pytest.mark.parametrize("rows", [1, 3])
@pytest.mark.parametrize("counts", COUNTS, ids=str)
def test_adamw(dense, bits, dtype, grad, rows, counts):
    import torch
    t, tg = getattr(torch, dtype), getattr(torch, grad)
    g = gen(sum(counts) + rows)
    lr, b1, b2, eps, scale = 0.01, 0.9, 0.99, 1e-8, 0.5
    decay = [0.1 * (i % 2) for i in range(len(counts))]
    params = [randn(g, t, n) for n in counts]
    grads = [randn(g, tg, rows, n, scale=0.1) for n in counts]
    copies = [torch.zeros(n, device="cuda", dtype=torch.bfloat16) if i % 2 else None for i, n in enumerate(counts)]
    opt = dense.ps_adamw_create(params, grads, state_bits=bits, weight_decay=decay, copies=copies)
    m, v = [torch.zeros(n, device="cuda", dtype=torch.float64) for n in counts], [torch.zeros(n, device="cuda", dtype=torch.float64) for n in counts]
    for step in (1, 2, 3):
        before = [p.double() for p in params]
        states = [tuple(s.double() for s in dense.ps_adamw_state(opt, i)) for i in range(len(counts))]
        codes = [(a.clone(), b.clone(), c.clone(), d.clone()) for a, b, c, d in zip(opt.m, opt.v, opt.m_scale, opt.v_scale)]
        for d in grads:
            d.copy_(randn(g, tg, *d.shape, scale=0.1))
        dense.ps_adamw_step(opt, step, lr, b1, b2, eps, grad_scale=scale)
        for i, n in enumerate(counts):
            if not n:
                continue
            rowsum = grads[i].double()
            gi, size = scale * rowsum.sum(0), scale * rowsum.abs().sum(0)
            m0, v0 = states[i]
            p, m1, v1 = adamw64(before[i], gi, m0, v0, step, lr, b1, b2, eps, decay[i])
            em = 2.0 ** -23 * ((rows + 2) * size + m0.abs() + m1.abs())
            # the update's size, of which every operation takes a few roundings, and what m's error makes of it
            root = (v1 / (1 - b2 ** step)).sqrt() + eps
            # relative error of the root: sums' errors against g itself where rows cancel
            ev = 2.0 ** -23 * (3 * v1 + (1 - b2) * (rows + 3) * size * size)
            er = (ev / (1 - b2 ** step)) / (2 * root.clamp(min=1e-30)) + 2.0 ** -22 * root
            update = lr / (1 - b1 ** step) * m1.abs() / root
            e = lr / (1 - b1 ** step) * em / root + update * (2.0 ** -21 + 2 * er / root) + 2.0 ** -22 * before[i].abs()
            close(params[i], p, e + half(t) * (p.abs() + e), "weights")
            if copies[i] is not None:
                close(copies[i], p, e + half(torch.bfloat16) * (p.abs() + e), "copy")
            if bits == 32:
                close(opt.m[i], m1, em + 1e-45, "m")
                close(opt.v[i], v1, ev + 1e-45, "v")
                continue
            total = grads[i][0].float()
            for k in range(1, rows):
                total = total + grads[i][k].float()
            total = total * scale
            def values(q, s):
                return q.view(torch.float8_e4m3fn).float() * s.repeat_interleave(256)[:n]
            old_m, old_root = values(codes[i][0], codes[i][2]), values(codes[i][1], codes[i][3])
            f32 = lambda c: float(torch.tensor(c, dtype=torch.float32))  # noqa: E731
            new_m = old_m * f32(b1) + total * f32(1 - b1)
            new_v = old_root * old_root * f32(b2) + total * total * f32(1 - b2)
            for got, got_scale, (want, want_scale) in ((opt.m[i], opt.m_scale[i], encode(new_m, False)), (opt.v[i], opt.v_scale[i], encode(new_v.sqrt(), True))):
                assert torch.equal(got, want) and torch.equal(got_scale, want_scale)
    dense.ps_adamw_destroy(opt)


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw_of_odd_addresses_and_rows_apart(dense, bits):
    """Tensors, states and gradient rows that begin anywhere give what aligned ones give, and nothing beside them is touched."""
    import torch
    g = gen(1)
    counts = [5, 300, 4099]
    for t in (torch.float32, torch.bfloat16):
        values = [randn(g, t, n) for n in counts]
        rows = [randn(g, t, 2, n) for n in counts]
        plain = dense.ps_adamw_create([p.clone() for p in values], rows, state_bits=bits, weight_decay=0.1)
        flat, wide = torch.full((6000,), 7.0, device="cuda", dtype=t), torch.full((2, 6001), 7.0, device="cuda", dtype=t)
        code = torch.zeros(6000, device="cuda", dtype=torch.uint8 if bits == 8 else torch.float32)
        at, parts, grads, ms, vs = 3, [], [], [], []
        code_v = code.clone()
        for p, r in zip(values, rows):
            n = p.numel()
            flat[at:at + n], wide[:, at:at + n] = p, r
            parts.append(flat[at:at + n])
            grads.append(wide[:, at:at + n])
            ms.append(code[at:at + n])
            vs.append(code_v[at:at + n])
            at += n + 5
        opt = dense.ps_adamw_create(parts, grads, state_bits=bits, weight_decay=0.1, m=ms, v=vs)
        for step in (1, 2):
            for o in (plain, opt):
                dense.ps_adamw_step(o, step, 0.01)
        for i in range(3):
            assert torch.equal(plain.params[i], opt.params[i]) and torch.equal(plain.m[i], opt.m[i]) and torch.equal(plain.v[i], opt.v[i])
        beside = torch.ones(6000, dtype=torch.bool, device="cuda")
        at = 3
        for n in counts:
            beside[at:at + n] = False
            at += n + 5
        assert bool((flat[beside] == 7).all()) and bool((code[beside] == 0).all()) and bool((code_v[beside] == 0).all())


def test_adamw_of_fewer_rows_than_there_are(dense):
    import torch
    g = gen(2)
    p, rows = randn(g, torch.float32, 1000), randn(g, torch.float32, 9, 1000)
    one, all_ = p.clone(), p.clone()
    dense.ps_adamw_step(dense.ps_adamw_create([one], [rows[:4].sum(0).clone()]), 1, 0.1)
    dense.ps_adamw_step(dense.ps_adamw_create([all_], [rows]), 1, 0.1, n_rows=4)
    assert float((one - all_).abs().max()) <= 1e-5
    opt = dense.ps_adamw_create([p], [rows])
    from paper_2406_05546_amd import binding as ps
    for n in (0, 10):
        with pytest.raises(ps.PsError) as e:
            dense.ps_adamw_step(opt, 1, 0.1, n_rows=n)
        assert e.value.status == ps.PS_EINVAL
    dense.ps_adamw_destroy(opt)
    with pytest.raises(ps.PsError):
        dense.ps_adamw_step(opt, 1, 0.1)


def test_adamw_values_that_are_not_finite(dense):
    import torch
    for bits in (32, 8):
        p, g = torch.ones(1024, device="cuda"), torch.full((1024,), 0.1, device="cuda")
        g[3], g[600] = float("nan"), float("inf")
        opt = dense.ps_adamw_create([p], [g], state_bits=bits)
        dense.ps_adamw_step(opt, 1, 0.1)
        fine = torch.ones(1024, dtype=torch.bool, device="cuda")
        fine[3] = fine[600] = False
        assert bool(p[fine].isfinite().all()) and bool(p[~fine].isnan().all())
        m, v = dense.ps_adamw_state(opt, 0)
        if bits == 32:
            assert bool(m[fine].isfinite().all()) and bool(m[3].isnan()) and bool(m[600].isinf()) and bool(v[600].isinf())
        else:  # their blocks as a whole
            for s in (m, v):
                bad = s.isnan().view(4, 256)
                assert bool(bad[0].all()) and bool(bad[2].all()) and not bool(bad[1].any()) and not bool(bad[3].any())


def test_adamw_states_that_are_tiny(dense):
    """Gradients whose states no scale can hold, and roots far below their block's largest: steps stay finite and bounded."""
    import torch
    g = torch.zeros(768, device="cuda")
    g[:256] = 1e-35
    g[256] = 1.0
    g[257:512] = 1e-7
    p = torch.zeros(768, device="cuda")
    opt = dense.ps_adamw_create([p], [g], state_bits=8)
    for step in range(1, 6):
        dense.ps_adamw_step(opt, step, 0.01)
    assert bool(p.isfinite().all()) and float(p.abs().max()) <= 5 * 0.01 * 1.001 and bool((p[512:] == 0).all())
    m, v = dense.ps_adamw_state(opt, 0)
    assert bool((v[256:512] > 0).all()) and bool((m[512:] == 0).all()) and bool((v[512:] == 0).all())
