"""Log probabilities, entropies, alternatives and the gradient on the GPU, against their formulas in 64 bits.

Tolerances, with U = 2^-24.  t = (z - m) scale log2(e) has relative error 4 U (two products, a difference, the constant's rounding), 2^t by
the hardware is off by another 2^-23, so p is off by 2 U + 4 U |ln p| of itself.  A sum over n values in 32 bits is a chain of at most
n / 64 + 64 additions to a lane's sum and 10 between lanes, with a rescaling at each round: CHAIN = n / 64 + 128 steps of U.
So the sum s is off by dS = U (CHAIN + 2 + 4 sum p |ln(p s)|) of itself at most, L = log s by dS + 2 U |L| + U, and the sum of p t (all of one sign)
by U (CHAIN + 10 + 4 max...): every term p |t| by (6 + 8 |t|) U, weighted.  The entropy is the difference of L and that sum over s."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]
INF = float("inf")


@pytest.fixture(scope="module")
def tk():
    import torch
    assert torch.cuda.is_available(), "GPU tests need an MI355X"
    from paper_2406_05546_amd import tokens as t
    t._library()
    return t


def gen(seed):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def f32(x):
    import torch
    return torch.tensor(x, dtype=torch.float32).double().item()


def exact(z, scale):
    """m, L, entropy, log probabilities, and what L and the entropy may be off by."""
    import torch
    z = z.double()
    n = z.shape[1]
    m = z.amax(1, keepdim=True)
    x = (z - torch.where(m == -INF, 0.0, m)) * f32(scale)
    e = torch.exp(x)
    s = e.sum(1, keepdim=True)
    some = s > 0
    L = torch.log(s)
    p = torch.where(some, e / s, 0.0)
    x0 = torch.where(e > 0, x, 0.0)
    first, second = (p * x0.abs()).sum(1, keepdim=True), (p * x0 * x0).sum(1, keepdim=True)
    H = torch.where(some, L + first, 0.0)
    chain = n / 64 + 128
    off_s = U * (chain + 2 + 4 * first)
    off_L = torch.where(some, off_s + 2 * U * L.abs() + U, 0.0)
    off_H = torch.where(some, off_L + U * ((chain + 10) * first + 8 * second) + off_s * first + 4 * U * H, 0.0)
    # twice the lowest 32-bit number, -6.8e38, is no 32-bit number: its rounding is -inf
    logp = torch.where((z == -INF) | (x - L < -torch.finfo(torch.float32).max), -INF, x - L)
    return m, L, H, logp, off_L, off_H


def near(got, want, off, what):
    import torch
    got = got.double()
    same = torch.where(want.isinf(), got == want, (got - want).abs() <= off)
    assert bool(same.all()), f"{what}: {int((~same).sum())} of {same.numel()}, off by {float((got - want)[~same].abs().max()):.3g}"


def best_of(z, top):
    """Indices of the `top` largest, ties to the lowest, -1 behind what is not -inf."""
    import torch
    z = z.cpu().double()
    order = torch.sort(z, dim=1, descending=True, stable=True).indices[:, :top]
    order = torch.where(z.gather(1, order) == -INF, -1, order)
    return torch.nn.functional.pad(order, (0, top - order.shape[1]), value=-1)


def check_forward(tk, z, tok, scale, top):
    import torch
    got = tk.ps_logprob_forward(z, tok, scale, top)
    m, L, H, logp, off_L, off_H = exact(z, scale)
    vocab = z.shape[1]
    assert torch.equal(got.norm[:, :1].double(), m)
    near(got.norm[:, 1:2], L, off_L, "L")
    near(got.norm[:, 2:], H, off_H, "entropy")
    assert got.entropy.data_ptr() == got.norm.data_ptr() + 8
    if tok is not None:
        t = tok.long()
        there = (t >= 0) & (t < vocab)
        want = torch.where(there[:, None], logp.gather(1, t.clamp(0, vocab - 1)[:, None]), 0.0)
        x = torch.where(want.isinf(), 0.0, want + torch.where(L == -INF, 0.0, L))
        near(got.logp[:, None], want, off_L + U * (4 * x.abs() + 2 * want.abs()), "log probabilities")
    if top:
        want = best_of(z, top).cuda()
        assert got.top_tokens.dtype == torch.int32 and torch.equal(got.top_tokens.long(), want)
        value = torch.where(want < 0, -INF, logp.gather(1, want.clamp(min=0)))
        x = torch.where(value.isinf(), 0.0, value + torch.where(L == -INF, 0.0, L))
        near(got.top_logp, value, off_L + U * (4 * x.abs() + 2 * torch.where(value.isinf(), 0.0, value).abs()), "alternatives")
    else:
        assert got.top_logp is None and got.top_tokens is None
    return got


def logits_of(kind, rows, vocab, t, g):
    import torch
    z = torch.randn(rows, vocab, device="cuda", generator=g) * 3
    if kind == "ties":
        z = z.round()
    elif kind == "equal":
        z = torch.full_like(z, -2.5)
    elif kind == "zeros":
        z = torch.where(z > 0, 0.0, -0.0)  # both zeros are equal
    elif kind == "ascending":
        z = torch.arange(vocab, device="cuda").float().expand(rows, vocab) * (60.0 / vocab)
    elif kind == "descending":
        z = -torch.arange(vocab, device="cuda").float().expand(rows, vocab) * (60.0 / vocab)
    elif kind == "masked":
        z = z.masked_fill(torch.rand(vocab, device="cuda", generator=g) < 0.5, -INF)
        z[rows // 2] = -INF
    elif kind == "few":  # a handful of tokens is allowed, in some rows one or none
        keep = torch.rand(rows, vocab, device="cuda", generator=g) < 5.0 / vocab
        z = torch.where(keep, z, -INF)
    elif kind == "lowest":  # a mask of the type's lowest value
        z = torch.where(torch.rand(rows, vocab, device="cuda", generator=g) < 0.9, torch.finfo(t).min, z)
        z[0] = torch.finfo(t).min
    elif kind == "far":
        z = z * 300
    elif kind == "offset":
        z = z + 1000
    return z.contiguous().to(t)


KINDS = ["plain", "ties", "equal", "zeros", "ascending", "descending", "masked", "few", "lowest", "far", "offset"]
# a wavefront to a row, four, and sixteen; rounds of 1024 (fp32) and 2048 values
SIZES = [(1, 1), (1, 2), (3, 10), (9, 63), (5, 65), (64, 100), (2, 1023), (3, 1025), (7, 2048), (6, 2049), (5, 4099), (3, 8192), (4, 8193), (2, 50257)]


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
def test_forward(tk, dtype, kind):
    import torch
    t = getattr(torch, dtype)
    for i, (rows, vocab) in enumerate(SIZES):
        g = gen(rows + vocab)
        z = logits_of(kind, rows, vocab, t, g)
        tok = torch.randint(-1, vocab + 1, (rows,), device="cuda", generator=g)
        check_forward(tk, z, tok.to(torch.int32) if i % 2 else tok, (1.0, 0.7, 2.0)[i % 3], (0, 1, 5, 20, 32)[i % 5])
        check_forward(tk, z, tok, 1.0, 32)


@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_and_long_ones(tk, dtype):
    import torch
    t = getattr(torch, dtype)
    for rows, vocab, top in ((600, 9001, 5), (2050, 300, 3), (1, 131072, 20), (2, 300007, 32), (5000, 10, 0), (256, 60001, 7), (257, 60001, 7), (3, 1500000, 32)):
        g = gen(rows)
        z = (torch.randn(rows, vocab, device="cuda", generator=g) * 2).to(t)
        check_forward(tk, z, torch.randint(0, vocab, (rows,), device="cuda", generator=g), 1.0, top)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("dtype", TYPES)
def test_many_rows_of_a_few_rounds(tk, dtype, kind):
    """A wavefront for each; rows around eight rounds, and of fewer rows by one."""
    import torch
    t = getattr(torch, dtype)
    round_ = 4096 // t.itemsize
    for rows, vocab, top in ((2048, 8 * round_, 5), (2051, 8 * round_ - 3, 32), (2048, 8 * round_ + 1, 7), (2047, 3 * round_ + 5, 20), (3001, round_ + 1, 1), (2500, 2 * round_ + 9, 0)):
        g = gen(rows + vocab)
        z = logits_of(kind, rows, vocab, t, g)
        check_forward(tk, z, torch.randint(-1, vocab + 1, (rows,), device="cuda", generator=g), 0.8, top)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab", [(5, 2000), (3, 8192), (2, 50000), (300, 20000), (2, 131072)])
def test_large_values_that_few_lanes_have(tk, dtype, rows, vocab):
    """A row's vectors of 16 bytes go to 64, 256 or 1024 lanes in turn.  Where fewer lanes than there are alternatives have all that is large, the
    alternatives are not told by the lanes' largest values."""
    import torch
    t, g = getattr(torch, dtype), gen(vocab)
    vector = torch.arange(vocab, device="cuda") // (16 // t.itemsize)
    for period in (64, 256, 1024):
        z = torch.randn(rows, vocab, device="cuda", generator=g)
        z = torch.where(vector % period < 31, z + 50, z).to(t)
        check_forward(tk, z, None, 1.0, 32)
        check_forward(tk, torch.where(vector % period < 3, z + 50, 0).to(t), None, 1.0, 4)  # and many equal ones below


def test_rows_apart_and_at_any_place(tk):
    import torch
    for dtype in TYPES:
        t, g = getattr(torch, dtype), gen(1)
        wide = torch.randn(40, 3001, device="cuda", generator=g).to(t)
        wide[:, :1] = 99.0
        wide[:, 2500:] = float("nan")  # beside the rows: not looked at
        tok = torch.randint(0, 2499, (40, 3), device="cuda", generator=g)[:, 1]
        z = wide[:, 1:2500]
        got = check_forward(tk, z, tok, 1.0, 4)
        same = tk.ps_logprob_forward(z.contiguous(), tok.contiguous(), 1.0, 4)
        assert torch.equal(got.top_tokens, same.top_tokens)
        out = torch.full((40, 3001), 3.0, device="cuda", dtype=t)
        one, more = torch.randn(40, 2, device="cuda", generator=g)[:, 0], torch.ones(1, device="cuda").expand(40)
        d = tk.ps_logprob_backward(z, tok, got.norm, one, more, out=out[:, 1:2500])
        assert torch.equal(d, tk.ps_logprob_backward(z.contiguous(), tok, got.norm, one.contiguous(), more.contiguous()))
        assert bool((out[:, :1] == 3).all()) and bool((out[:, 2500:] == 3).all())


def test_without_tokens(tk):
    import torch
    z = torch.randn(20, 500, device="cuda", generator=gen(2))
    got = check_forward(tk, z, None, 1.0, 7)
    assert got.logp is None
    both = tk.ps_logprob_forward(z, torch.zeros(20, dtype=torch.int64, device="cuda"), 1.0, 7)
    assert torch.equal(got.norm, both.norm) and torch.equal(got.top_logp, both.top_logp)
    none = tk.ps_logprob_forward(z[:0], top=3)
    assert none.norm.shape == (0, 3) and none.top_tokens.shape == (0, 3)


@pytest.mark.parametrize("vocab", [10, 3000, 20000])
def test_rows_that_are_not_numbers(tk, vocab):
    import torch
    z = torch.randn(6, vocab, device="cuda", generator=gen(4))
    z[1, 7] = float("nan")
    z[3, 2] = INF
    z[4] = -INF
    z[4, 5] = float("nan")
    tok = torch.tensor([0, 1, 2, 3, 4, -1], device="cuda")
    got = tk.ps_logprob_forward(z, tok, 1.0, 3)
    for r in (1, 3, 4):
        assert bool(got.norm[r, 1:].isnan().all()) and bool(got.logp[r].isnan()) and bool(got.top_logp[r][got.top_tokens[r] >= 0].isnan().all())
    assert got.norm[3, 0] == INF and got.top_tokens[3, 0] == 2 and got.top_tokens[4].tolist() == [-1, -1, -1]
    fine = [0, 2, 5]
    alone = tk.ps_logprob_forward(z[fine], tok[fine], 1.0, 3)
    # Rows at other places in memory begin elsewhere in their first 16 bytes, and so are summed in another order: both are off by at most
    # what the forward pass may be, from the same numbers.
    _, L, H, logp, off_L, off_H = exact(z[fine], 1.0)
    assert torch.equal(alone.norm[:, 0], got.norm[fine, 0]) and torch.equal(alone.top_tokens, got.top_tokens[fine])
    for x in (alone.norm, got.norm[fine]):
        near(x[:, 1:2], L, off_L, "L")
        near(x[:, 2:], H, off_H, "entropy")
    for x in (alone.logp, got.logp[fine]):
        want = torch.where(tok[fine] < 0, 0.0, logp.gather(1, tok[fine].clamp(min=0)[:, None])[:, 0])
        near(x[:, None], want[:, None], off_L + U * (6 * want[:, None].abs() + 4 * L.abs()), "log probabilities")
    d = tk.ps_logprob_backward(z, tok, got.norm, torch.ones(6, device="cuda"), torch.ones(6, device="cuda"))
    for r in (1, 3, 4):
        assert bool(d[r].isnan().all())
    assert bool(d[fine].isfinite().all())


def check_backward(z, tok, norm, dlogp, dentropy, scale, got):
    """From the norm as it is: (m, L, H) of the forward pass, whose errors are its own."""
    import torch
    s, zd = f32(scale), z.double()
    m, L, H = (norm[:, i:i + 1].double() for i in range(3))
    empty = (m == -INF) & (L == -INF)
    logp = torch.where(empty, -INF, (zd - m) * s - L)
    p = torch.exp(logp)
    t = tok.long()
    there = (t >= 0) & (t < z.shape[1])
    gl = torch.where(there, dlogp.double(), 0.0)[:, None] if dlogp is not None else torch.zeros_like(m)
    gh = dentropy.double()[:, None] if dentropy is not None else torch.zeros_like(m)
    l0 = torch.where(p > 0, logp, 0.0)
    A, B = gl + gh * H, gh * l0
    want = -p * (A + B)
    # p: see above, with L log2(e) rounded twice more; A and B and their sum
    off_p = p * (2 * U + U * (4 * l0.abs() + 8 * L.abs()))
    off = off_p * (A + B).abs() + p * U * (4 * gl.abs() + 4 * (gh * H).abs() + 6 * B.abs() + gh.abs() * (4 * l0.abs() + 4 * L.abs()))
    # below 2^-126 the hardware's 2^t is 0
    off = off + torch.where(p < 2.0 ** -125, p, 0.0) * (A.abs() + (gh * logp.clamp(min=-1000)).abs())
    hit = torch.zeros_like(want).scatter_add_(1, t.clamp(0, z.shape[1] - 1)[:, None], gl)
    want, off = (want + hit) * s, (off + 2 * U * (hit.abs() + want.abs())) * s
    want, off = torch.where(empty, 0.0, want), torch.where(empty, 0.0, off)
    info = torch.finfo(got.dtype)
    tol = off + info.eps / 2 * (want.abs() + off) + info.tiny * info.eps / 2
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} values, worst {float(((got.double() - want).abs() / tol)[bad].max()):.3g}"


@pytest.mark.parametrize("kind", ["plain", "ties", "equal", "masked", "few", "lowest", "far", "offset"])
@pytest.mark.parametrize("dtype", TYPES)
def test_backward(tk, dtype, kind):
    import torch
    t = getattr(torch, dtype)
    for i, (rows, vocab) in enumerate(SIZES):
        g = gen(rows + vocab)
        z = logits_of(kind, rows, vocab, t, g)
        tok = torch.randint(-1, vocab + 1, (rows,), device="cuda", generator=g)
        scale = (1.0, 0.7, 2.0)[i % 3]
        norm = tk.ps_logprob_forward(z, tok, scale).norm
        dlogp, dentropy = torch.randn(rows, device="cuda", generator=g), torch.randn(rows, device="cuda", generator=g)
        for a, b in ((dlogp, dentropy), (dlogp, None), (None, dentropy)):
            check_backward(z, tok, norm, a, b, scale, tk.ps_logprob_backward(z, tok, norm, a, b, scale))
        both = tk.ps_logprob_backward(z, tok, norm, dlogp, dentropy, scale)
        assert not bool(tk.ps_logprob_backward(z, tok, norm, scale=scale).any())
        same = z.clone()
        assert tk.ps_logprob_backward(same, tok, norm, dlogp, dentropy, scale, out=same) is same and torch.equal(same, both)


def test_the_gradient_against_differences(tk):
    """Central differences of the forward pass in 32 bits: steps of 2^-5 have errors of third order, 2^-10 / 6 times a third derivative
    below 4, and those of the values, 1e-6, over 2^-4; together below 1e-3."""
    import torch
    g = gen(8)
    z = torch.randn(3, 12, device="cuda", generator=g)
    tok, dlogp, dentropy = torch.tensor([3, -1, 11], device="cuda"), torch.tensor([1.0, 2.0, -0.5], device="cuda"), torch.tensor([0.3, -1.0, 0.0], device="cuda")
    f = lambda x: (lambda r: (r.logp.double() * dlogp * (tok >= 0) + r.entropy.double() * dentropy).sum().item())(tk.ps_logprob_forward(x, tok, 1.5))  # noqa: E731
    grad = tk.ps_logprob_backward(z, tok, tk.ps_logprob_forward(z, tok, 1.5).norm, dlogp, dentropy, 1.5)
    h = 2.0 ** -5
    for r in range(3):
        for c in range(12):
            more, less = z.clone(), z.clone()
            more[r, c] += h
            less[r, c] -= h
            # scale^3 more for the third derivative
            assert abs((f(more) - f(less)) / (2 * h) - grad[r, c].item()) < 1e-3 * 1.5 ** 3 * 2


def test_rows_beyond_32_bits(tk):
    import torch
    rows, vocab = 9000, 250000  # 2.25e9 logits
    z = torch.zeros(rows, vocab, device="cuda", dtype=torch.bfloat16)
    z[:, 1234] = 12.0
    z[rows - 1, vocab - 1] = 13.0
    tok = torch.full((rows,), 1234, device="cuda")
    tok[rows - 1] = vocab - 1
    got = tk.ps_logprob_forward(z, tok, 1.0, 2)
    assert got.top_tokens[0].tolist() == [1234, 0] and got.top_tokens[rows - 1].tolist() == [vocab - 1, 1234]
    _, _, _, logp, off_L, _ = exact(z[-2:], 1.0)
    near(got.logp[-2:, None], logp.gather(1, tok[-2:, None]), off_L + 64 * U, "log probabilities")
    tk.ps_logprob_backward(z, tok, got.norm, torch.ones(rows, device="cuda"), out=z)
    want = 1 - torch.exp(got.logp[-1].double())
    assert abs(z[rows - 1, vocab - 1].double() - want) <= want * 2.0 ** -8 and float(z[rows - 2, vocab - 1]) < 0


def test_calls_in_a_graph_and_on_another_stream(tk):
    import torch
    g = gen(5)
    z, tok = torch.randn(70, 9001, device="cuda", generator=g).half(), torch.randint(0, 9001, (70,), device="cuda", generator=g)
    w = torch.full((1,), -1 / 70, device="cuda").expand(70)

    def both():
        r = tk.ps_logprob_forward(z, tok, 1.0, 8)
        return r.logp, r.norm, r.top_logp, r.top_tokens, tk.ps_logprob_backward(z, tok, r.norm, w, w)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        there = both()
    torch.cuda.current_stream().wait_stream(other)
    assert all(torch.equal(a, b) for a, b in zip(there, both()))
    graphs = []
    for _ in range(2):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = both()
        graphs.append((graph, out))
    for _ in range(3):
        z.copy_(torch.randn(70, 9001, device="cuda", generator=g))
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        want = both()
        for _, out in graphs:
            assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_calls_that_are_refused(tk):
    import torch
    from paper_2406_05546_amd.binding import PsError
    z, tok = torch.zeros(4, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    norm, one = torch.zeros(4, 3, device="cuda"), torch.zeros(4, device="cuda")
    bad = [lambda: tk.ps_logprob_forward(z[0], tok), lambda: tk.ps_logprob_forward(z.double(), tok), lambda: tk.ps_logprob_forward(z.t()[:4], tok),
           lambda: tk.ps_logprob_forward(z, tok[:3]), lambda: tk.ps_logprob_forward(z, tok.short()), lambda: tk.ps_logprob_forward(z, tok, top=33), lambda: tk.ps_logprob_forward(z, tok, top=-1),
           lambda: tk.ps_logprob_forward(z, tok, 0.0), lambda: tk.ps_logprob_forward(z, tok, float("nan")), lambda: tk.ps_logprob_forward(z[:1].expand(4, 8), tok),
           lambda: tk.ps_logprob_backward(z, None, norm, one), lambda: tk.ps_logprob_backward(z, tok, norm[:, :2], one), lambda: tk.ps_logprob_backward(z, tok, norm.double(), one),
           lambda: tk.ps_logprob_backward(z, tok, norm, one[:3]), lambda: tk.ps_logprob_backward(z, tok, norm, one.double()), lambda: tk.ps_logprob_backward(z, tok, norm, one, one[None]),
           lambda: tk.ps_logprob_backward(z, tok, norm, one, out=z.half()), lambda: tk.ps_logprob_backward(z, tok, norm, one, out=z[:3]),
           lambda: tk.ps_logprob_backward(z, tok, norm, one, out=z[:1].expand(4, 8)), lambda: tk.ps_logprob_backward(z, tok, norm.t().contiguous().t(), one)]
    for i, call in enumerate(bad):
        with pytest.raises(PsError):
            call()
            pytest.fail(f"call {i} was not refused")
