"""Activations in 8 bits on the GPU: encoding and decoding to the bit against an encoder written here, and dense layers that keep their
pre-activations so, or read them and their inputs from there, against the same layers on the values that are held."""
import math

import pytest

from tests.test_gpu_dense import act64, check_backward, dense, gen, half, randn  # noqa: F401

pytestmark = pytest.mark.gpu
TYPES = ["float32", "bfloat16", "float16"]
INF = math.inf


def values_of_e4m3():
    """All values from 0 up, by their code."""
    import torch
    return torch.tensor([(m / 8 if e == 0 else 1 + m / 8) * 2.0 ** (max(e, 1) - 7) for e in range(16) for m in range(8)][:127], dtype=torch.float64)


def encode64(x):
    """Codes and scales (uint8) of a matrix on the CPU, value by value from the definition."""
    import torch
    rows, cols = x.shape
    blocks = -(-cols // 32)
    v = torch.zeros(rows, blocks * 32, dtype=torch.float64)
    v[:, :cols] = x.double()
    v = v.view(rows, blocks, 32)
    top = torch.where(v.isfinite(), v.abs(), 0.0).amax(2)
    scale = torch.full(top.shape, -126, dtype=torch.int64)
    for e in range(-126, 121):
        scale = torch.where((top > 448.0 * 2.0 ** (e - 1)) & (top <= 448.0 * 2.0 ** e) if e > -126 else top <= 448.0 * 2.0 ** e, e, scale)
    a = (v / torch.exp2(scale.double())[:, :, None]).abs()
    table = values_of_e4m3()
    finite = torch.where(a.isfinite(), a, 0.0)
    hi = torch.searchsorted(table, finite).clamp(0, 126)  # the first value not below
    lo = (hi - 1).clamp(min=0)
    up, down = table[hi] - finite, finite - table[lo]
    code = torch.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = torch.where((code == 0) & (a > 0), 1, code)
    beyond = table[code] * torch.exp2(scale.double())[:, :, None] > torch.finfo(x.dtype if x.dtype != torch.float64 else torch.float32).max
    code = torch.where(beyond, code - 1, code)
    code = torch.where(v.isfinite(), code, 127)
    code = code + 128 * (torch.signbit(v) & v.isfinite())
    return code.view(rows, blocks * 32)[:, :cols].to(torch.uint8), (scale + 127).to(torch.uint8)


def bits(c):
    """Codes and scales on the CPU; every NaN as one."""
    import torch
    code = c.codes.view(torch.uint8).cpu()
    return torch.where((code & 127) == 127, 127, code), c.scales.view(torch.uint8).cpu()


def check_encode(c, x):
    import torch
    code, scale = bits(c)
    want, want_scale = encode64(x.cpu())
    assert torch.equal(scale, want_scale), f"{int((scale != want_scale).sum())} scales"
    assert torch.equal(code, want), f"{int((code != want).sum())} codes"


def of_kind(kind, rows, cols, t, g):
    import torch
    x = torch.randn(rows, cols, device="cuda", generator=g)
    info = torch.finfo(t)
    if kind == "sizes":  # columns from subnormal to the largest
        x = x * torch.exp2(torch.linspace(math.log2(info.tiny) - 8, math.log2(info.max) - 3, cols, device="cuda"))
    elif kind == "zeros":
        x = torch.where(x > 0, x, torch.zeros_like(x))
        x[:, :40] = 0
    elif kind == "border":  # 448 and what is next to it, ties between codes
        x = torch.tensor([448, 449, 450, 447, 464, 1, 1.0625, 1.1875, 0.001, -0.0009765625, 0.00292969, -0.0, 896, 1.75, 1.7578125], device="cuda")[torch.randint(
            0, 15, (rows, cols), device="cuda", generator=g)] * torch.exp2(torch.randint(-6, 6, (rows, cols), device="cuda", generator=g).float())
    elif kind == "not finite":
        x[torch.rand(rows, cols, device="cuda", generator=g) < 0.05] = INF
        x[torch.rand(rows, cols, device="cuda", generator=g) < 0.05] = -INF
        x[torch.rand(rows, cols, device="cuda", generator=g) < 0.05] = math.nan
        x[0] = math.nan
    elif kind == "largest":
        x = torch.where(x > 0, info.max, -info.max) * (x.abs() > 0.5)
    return x.to(t)


SIZES = [(1, 1), (1, 8), (3, 31), (2, 32), (5, 33), (37, 1111), (64, 256), (130, 100), (257, 2048)]


@pytest.mark.parametrize("kind", ["plain", "sizes", "zeros", "border", "not finite", "largest"])
@pytest.mark.parametrize("dtype", TYPES)
def test_encode_and_decode(dense, dtype, kind):
    import torch
    t = getattr(torch, dtype)
    for rows, cols in SIZES:
        x = of_kind(kind, rows, cols, t, gen(rows + cols))
        c = dense.ps_checkpoint_encode(x)
        assert c.shape == (rows, cols) and c.codes.dtype == torch.float8_e4m3fn and c.scales.dtype == torch.float8_e8m0fnu
        check_encode(c, x)
        held = c.codes.double() * c.scales.double().repeat_interleave(32, 1)[:, :cols]
        for to in TYPES:
            y = dense.ps_checkpoint_decode(c, getattr(torch, to))
            want = held.to(getattr(torch, to))
            assert torch.equal(y.nan_to_num(7, 8, 9), want.nan_to_num(7, 8, 9)) and torch.equal(y.isnan(), want.isnan())
        # what is held: half a step, or the least code
        fine = x.double().isfinite()
        top = torch.where(fine, x.double().abs(), 0.0)
        top = torch.nn.functional.pad(top, (0, -cols % 32)).view(rows, -1, 32).amax(2).repeat_interleave(32, 1)[:, :cols]
        off = (held - x.double()).abs()
        assert bool((off[fine] <= (x.double().abs() / 16 + top * 2.0 ** -16 + 448 * 2.0 ** -135)[fine]).all())
        assert bool(((held == 0) == (x == 0))[fine].all()) and bool(held[~fine].isnan().all())


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_decode_with_an_activation(dense, act):
    import torch
    c = dense.ps_checkpoint_encode(torch.randn(70, 333, device="cuda", generator=gen(1)) * 3)
    z = c.codes.double() * c.scales.double().repeat_interleave(32, 1)[:, :333]
    for dtype in TYPES:
        t = getattr(torch, dtype)
        y, want = dense.ps_checkpoint_decode(c, t, act), act64(z, act)
        # as for a layer's activation: 8 steps of 2^-23 of |z| + 1, and the rounding
        tol = (8 * 2.0 ** -23 * (z.abs() + 1) if act != "relu" else 0) + half(t) * want.abs() + torch.finfo(t).tiny * half(t)
        assert bool(((y.double() - want).abs() <= tol).all())


@pytest.mark.parametrize("dtype", TYPES)
def test_the_largest_numbers_stay_finite(dense, dtype):
    import torch
    t = getattr(torch, dtype)
    top = torch.finfo(t).max
    x = (torch.tensor([1.0, -1.0, 0.999, 0.97, 0.96875, 0.968, 0.9375, 0.5, 1e-4, 0.0], device="cuda", dtype=torch.float64) * top).to(t).repeat(3, 7)
    c = dense.ps_checkpoint_encode(x)
    check_encode(c, x)
    y = dense.ps_checkpoint_decode(c, t)
    assert bool(y.isfinite().all()) and bool(((y.double() - x.double()).abs() <= x.double().abs() / 16 + top * 2.0 ** -16).all())
    # beside what is not finite, too
    x[:, ::9] = INF
    y = dense.ps_checkpoint_decode(dense.ps_checkpoint_encode(x), t)
    assert torch.equal(y.isfinite(), x.isfinite())


def test_rows_apart_and_at_any_place(dense):
    import torch
    for dtype in TYPES:
        t = getattr(torch, dtype)
        wide = randn(gen(2), t, 50, 301)
        wide[:, :3] = math.nan
        x = wide[:, 3:300]
        codes, scales = torch.full((50, 313), 77, device="cuda", dtype=torch.uint8), torch.full((50, 12), 99, device="cuda", dtype=torch.uint8)
        c = dense.ps_checkpoint_encode(x, dense.Checkpoint(codes[:, 5:302], scales[:, 1:11]))
        check_encode(c, x)
        assert bool((codes[:, :5] == 77).all()) and bool((codes[:, 302:] == 77).all()) and bool((scales[:, 0] == 99).all()) and bool((scales[:, 11] == 99).all())
        out = torch.full((50, 310), 5.0, device="cuda", dtype=t)
        y = dense.ps_checkpoint_decode(c, out=out[:, 1:298])
        assert torch.equal(y, dense.ps_checkpoint_decode(dense.ps_checkpoint_encode(x.contiguous()), t))
        assert bool((out[:, 0] == 5).all()) and bool((out[:, 298:] == 5).all())
    none = dense.ps_checkpoint_encode(torch.zeros(0, 40, device="cuda"))
    assert dense.ps_checkpoint_decode(none).shape == (0, 40)


def test_rows_beyond_32_bits(dense):
    import torch
    x = torch.zeros(70000, 32768, device="cuda", dtype=torch.bfloat16)
    x[69999, 32767], x[65537, 3], x[0, 0] = 3.0, -5.0, 7.0
    c = dense.ps_checkpoint_encode(x)
    assert int((c.codes.view(torch.uint8) & 127).count_nonzero()) == 3
    x.fill_(9.0)
    y = dense.ps_checkpoint_decode(c, out=x)
    assert (float(y[69999, 32767]), float(y[65537, 3]), float(y[0, 0])) == (3.0, -5.0, 7.0) and int(y.count_nonzero()) == 3


# one to few rows, features in no whole blocks, tiles of every size, contractions in parts
LAYERS = [(1, 64, 64), (3, 40, 33), (16, 96, 100), (65, 129, 255), (130, 264, 136), (256, 4096, 512), (300, 1000, 77), (512, 64, 512), (700, 1111, 1030), (2048, 512, 2048)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", LAYERS)
def test_forward_keeps_what_it_would_write(dense, dtype, rows, fin, fout):
    import torch
    t, g = getattr(torch, dtype), gen(rows + fin)
    x, w, b, r = randn(g, t, rows, fin), randn(g, t, fout, fin, scale=fin ** -0.5), randn(g, t, fout), randn(g, t, rows, fout)
    for act, bias, residual in (("gelu", b, None), ("relu", None, r), ("silu", b, r), ("none", None, None)):
        pre, kept = torch.empty(rows, fout, device="cuda", dtype=t), dense.ps_checkpoint_empty(rows, fout, "cuda:0")
        y = dense.ps_linear_forward(x, w, bias, residual, act, pre=pre)
        y8 = dense.ps_linear_forward(x, w, bias, residual, act, pre=kept)
        assert torch.equal(y, y8), act
        want = dense.ps_checkpoint_encode(pre)
        assert all(torch.equal(a, b) for a, b in zip(bits(kept), bits(want))), act


def test_layers_with_checkpoints_of_any_rows(dense):
    """Codes and scales that are parts of wider rows, at any place."""
    import torch
    for t in (torch.float32, torch.bfloat16):
        for rows, fin, fout in ((5, 40, 72), (300, 104, 264), (290, 33, 65)):
            g = gen(rows)
            x, w, dy = randn(g, t, rows, fin), randn(g, t, fout, fin), randn(g, t, rows, fout)

            def wide(cols):
                codes, scales = torch.full((rows, cols + 7), 77, device="cuda", dtype=torch.uint8), torch.full((rows, cols // 32 + 4), 99, device="cuda", dtype=torch.uint8)
                return codes, scales, dense.Checkpoint(codes[:, 3:cols + 3], scales[:, 1:(cols + 31) // 32 + 1])
            codes, scales, pre = wide(fout)
            dense.ps_linear_forward(x, w, activation="gelu", pre=pre)
            plain = dense.ps_checkpoint_empty(rows, fout, "cuda:0")
            dense.ps_linear_forward(x, w, activation="gelu", pre=plain)
            assert all(torch.equal(a, b) for a, b in zip(bits(pre), bits(plain)))
            assert bool((codes[:, :3] == 77).all()) and bool((codes[:, fout + 3:] == 77).all()) and bool((scales[:, 0] == 99).all()) and bool((scales[:, (fout + 31) // 32 + 1:] == 99).all())
            x8 = dense.ps_checkpoint_encode(x, wide(fin)[2])
            got, want = dense.ps_linear_backward(dy, x8, w, "gelu", pre=pre), dense.ps_linear_backward(dy, dense.ps_checkpoint_encode(x), w, "gelu", pre=plain)
            assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("cuts,fin,fout", [([0, 3, 3, 5, 9], 64, 100), ([2, 130, 131, 400, 420], 72, 264), ([10, 700, 1500], 256, 512)])
def test_forward_in_groups(dense, dtype, cuts, fin, fout):
    import torch
    t, g, n, rows = getattr(torch, dtype), gen(fin), len(cuts) - 1, cuts[-1] + 4
    offsets, index = torch.tensor(cuts, dtype=torch.int32).cuda(), torch.tensor([(2 * i + 1) % 3 for i in range(n)], dtype=torch.int32).cuda()
    x, w, b = randn(g, t, rows, fin), randn(g, t, 3, fout, fin, scale=fin ** -0.5), randn(g, t, 3, fout)
    pre, kept = torch.zeros(rows, fout, device="cuda", dtype=t), dense.ps_checkpoint_empty(rows, fout, "cuda:0")
    kept.codes.view(torch.uint8).fill_(55)
    kept.scales.view(torch.uint8).fill_(66)
    y = dense.ps_grouped_linear_forward(x, offsets, w, b, None, "gelu", index, pre=pre)
    y8 = dense.ps_grouped_linear_forward(x, offsets, w, b, None, "gelu", index, pre=kept)
    inside = slice(cuts[0], cuts[-1])
    assert torch.equal(y[inside], y8[inside])
    want = bits(dense.ps_checkpoint_encode(pre))
    for got, same, old in zip(bits(kept), want, (55, 66)):
        assert torch.equal(got[inside], same[inside])
        assert bool((got[:cuts[0]] == old).all()) and bool((got[cuts[-1]:] == old).all())


def test_forward_whose_sums_are_not_finite(dense):
    import torch
    x, w = randn(gen(3), torch.bfloat16, 300, 128), randn(gen(4), torch.bfloat16, 256, 128)
    x[7, 3], w[40, 9] = math.nan, INF
    pre, kept = torch.empty(300, 256, device="cuda", dtype=torch.bfloat16), dense.ps_checkpoint_empty(300, 256, "cuda:0")
    dense.ps_linear_forward(x, w, pre=pre)
    dense.ps_linear_forward(x, w, pre=kept)
    check_encode(kept, pre)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,fin,fout", LAYERS + [(0, 16, 24), (33, 2048, 4096)])
def test_backward(dense, dtype, rows, fin, fout):
    import torch
    t, g = getattr(torch, dtype), gen(rows + fin + fout)
    dy, w = randn(g, t, rows, fout), randn(g, t, fout, fin)
    x, z = randn(g, t, rows, fin), randn(g, t, rows, fout)
    x8, z8 = dense.ps_checkpoint_encode(x), dense.ps_checkpoint_encode(z)
    held_x, held_z = dense.ps_checkpoint_decode(x8, t), dense.ps_checkpoint_decode(z8, t)
    for act in ("gelu", "relu", "silu", "none"):
        got = dense.ps_linear_backward(dy, x8, w, act, pre=z8)
        check_backward(got, dy, held_x, w, act, held_z)
        # the same products of the same values, however the other operand is held
        only_pre, only_x = dense.ps_linear_backward(dy, x, w, act, pre=z8), dense.ps_linear_backward(dy, x8, w, act, pre=z)
        check_backward(only_pre, dy, x, w, act, held_z)
        check_backward(only_x, dy, held_x, w, act, z)
        plain = dense.ps_linear_backward(dy, held_x, w, act, pre=held_z)
        assert torch.equal(got[0], plain[0]) and torch.equal(got[2], plain[2])
        if fin % 8 == 0 and fout % 8 == 0:
            assert torch.equal(got[1], plain[1])
    dx, dw, db = dense.ps_linear_backward(dy, x8, w, "gelu", pre=z8, need_dx=False, need_db=False)
    assert dx is None and db is None and torch.equal(dw, dense.ps_linear_backward(dy, x8, w, "gelu", pre=z8)[1])
    dx, dw, db = dense.ps_linear_backward(dy, x8, w, "gelu", pre=z8, need_dw=False)
    assert dw is None and torch.equal(dx, dense.ps_linear_backward(dy, x, w, "gelu", pre=z8)[0])


@pytest.mark.parametrize("act", ["relu", "gelu", "silu"])
def test_backward_with_an_input_made_again(dense, act):
    import torch
    for dtype in TYPES:
        t, g = getattr(torch, dtype), gen(9)
        dy, w, before, z = randn(g, t, 200, 136), randn(g, t, 136, 72), randn(g, t, 200, 72), randn(g, t, 200, 136)
        b8, z8 = dense.ps_checkpoint_encode(before), dense.ps_checkpoint_encode(z)
        x = dense.ps_checkpoint_decode(b8, t, act)
        got = dense.ps_linear_backward(dy, b8, w, "gelu", pre=z8, x_activation=act)
        want = dense.ps_linear_backward(dy, x, w, "gelu", pre=z8)
        assert all(torch.equal(a, b) for a, b in zip(got, want))


@pytest.mark.parametrize("dtype", TYPES)
def test_backward_in_groups(dense, dtype):
    import torch
    t = getattr(torch, dtype)
    for cuts, fin, fout in (([0, 3, 3, 5, 9], 64, 100), ([2, 130, 131, 400, 420], 72, 264), ([1, 64, 128, 129, 1000], 33, 65)):
        g, n, rows = gen(fin), len(cuts) - 1, cuts[-1] + 4
        offsets, index = torch.tensor(cuts, dtype=torch.int32).cuda(), torch.tensor([(2 * i + 1) % 3 for i in range(n)], dtype=torch.int32).cuda()
        dy, w = randn(g, t, rows, fout), randn(g, t, 3, fout, fin)
        x8, z8 = dense.ps_checkpoint_encode(randn(g, t, rows, fin)), dense.ps_checkpoint_encode(randn(g, t, rows, fout))
        for c in (x8, z8):  # rows in no group: never in a sum
            c.codes.view(torch.uint8)[:cuts[0]] = 127
            c.codes.view(torch.uint8)[cuts[-1]:] = 127
        dx = torch.full((rows, fin), 3.0, device="cuda", dtype=t)
        _, dw, db = dense.ps_grouped_linear_backward(dy, x8, offsets, w, "silu", pre=z8, weight_of_group=index, dx=dx, x_activation="relu")
        x, z = dense.ps_checkpoint_decode(x8, t, "relu"), dense.ps_checkpoint_decode(z8, t)
        for k in range(n):
            s = slice(cuts[k], cuts[k + 1])
            check_backward((dx[s], dw[k], db[k]), dy[s], x[s], w[int(index[k])], "silu", z[s])
        assert bool((dx[:cuts[0]] == 3).all()) and bool((dx[cuts[-1]:] == 3).all())


def test_calls_in_a_graph_and_on_another_stream(dense):
    import torch
    g, t = gen(6), torch.bfloat16
    x, w, dy = randn(g, t, 300, 200), randn(g, t, 130, 200), randn(g, t, 300, 130)

    def step():
        x8, z8 = dense.ps_checkpoint_encode(x), dense.ps_checkpoint_empty(300, 130, "cuda:0")
        y = dense.ps_linear_forward(x, w, activation="gelu", pre=z8)
        few = dense.ps_checkpoint_empty(5, 130, "cuda:0")
        one = dense.ps_linear_forward(x[:5], w, activation="gelu", pre=few)
        return [y, one, *dense.ps_linear_backward(dy, x8, w, "gelu", pre=z8)] + [c.view(torch.uint8) for k in (x8, z8, few) for c in (k.codes, k.scales)]
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        there = step()
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip(there, step()))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = step()
        graphs.append((graph, out))
    for _ in range(3):
        x.normal_(generator=g)
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = step()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_calls_that_are_refused(dense):
    import torch
    from paper_2406_05546_amd.binding import PsError
    x, w, dy = torch.zeros(4, 64, device="cuda"), torch.zeros(40, 64, device="cuda"), torch.zeros(4, 40, device="cuda")
    x8, z8, C = dense.ps_checkpoint_encode(x), dense.ps_checkpoint_encode(dy), dense.Checkpoint
    bad = [lambda: dense.ps_checkpoint_encode(x[0]), lambda: dense.ps_checkpoint_encode(x.double()), lambda: dense.ps_checkpoint_encode(x.cpu()), lambda: dense.ps_checkpoint_encode(x.t()),
           lambda: dense.ps_checkpoint_encode(x, z8), lambda: dense.ps_checkpoint_encode(x, C(x8.codes, x8.scales[:, :1])), lambda: dense.ps_checkpoint_encode(x, C(x8.codes.float(), x8.scales)),
           lambda: dense.ps_checkpoint_encode(x, C(x8.codes, x8.scales.float())), lambda: dense.ps_checkpoint_encode(x, C(x8.codes.cpu(), x8.scales)),
           lambda: dense.ps_checkpoint_encode(x, C(x8.codes.view(torch.uint8)[:1].expand(4, 64), x8.scales)), lambda: dense.ps_checkpoint_encode(x, C(x8.codes, x8.scales.view(torch.uint8)[:1].expand(4, 2))),
           lambda: dense.ps_checkpoint_decode(x8, torch.float64), lambda: dense.ps_checkpoint_decode(x8, activation="tanh"), lambda: dense.ps_checkpoint_decode(x8, out=x[:3]),
           lambda: dense.ps_checkpoint_decode(C(x8.codes.cpu(), x8.scales.cpu())), lambda: dense.ps_linear_forward(x, w, pre=x8), lambda: dense.ps_linear_forward(x8, w),
           lambda: dense.ps_linear_backward(dy, x8, w, "gelu"), lambda: dense.ps_linear_backward(dy, x8, w, "gelu", pre=x8), lambda: dense.ps_linear_backward(dy, z8, w, "none"),
           lambda: dense.ps_linear_backward(dy, x, w, "gelu", pre=z8, x_activation="gelu"), lambda: dense.ps_linear_backward(dy, x8, w, "gelu", pre=z8, x_activation="tanh"),
           lambda: dense.ps_linear_backward(dy.bfloat16(), x8, w, "gelu", pre=z8)]
    for i, call in enumerate(bad):
        with pytest.raises(PsError):
            call()
            pytest.fail(f"call {i} was not refused")
