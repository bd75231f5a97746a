"""Rows of a table for given tokens and their gradient on the GPU, against their formulas in 64 bits.

Tolerances.  A result is rounded once, by at most half a step, eps(t) / 2 of its magnitude or half of the smallest subnormal
number; before that the product with the scale is rounded to 32 bits, 2^-24 of it, and a sum of n rows is off by at most n steps of
2^-24 of the sum of their magnitudes."""
import pytest

pytestmark = pytest.mark.gpu
U = 2.0 ** -24
TYPES = ["float32", "bfloat16", "float16"]


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


def f32(scale):
    import torch
    return torch.tensor(scale, dtype=torch.float32).double().item()


def close(got, want, before, what):
    """want in 64 bits, before: what it may be off by before it is rounded."""
    import torch
    info = torch.finfo(got.dtype)
    tol = before + info.eps / 2 * (want.abs() + before) + info.tiny * info.eps / 2
    bad = ~((got.double() - want).abs() <= tol)
    assert not bool(bad.any()), f"{what}: {int(bad.sum())} of {bad.numel()} values"


def owner_of(rows, offsets):
    """Group of each row, -1 for none."""
    import torch
    owner = torch.full((rows,), -1, dtype=torch.int64)
    if offsets is None:
        return torch.zeros(rows, dtype=torch.int64)
    for g, (lo, hi) in enumerate(zip(offsets, offsets[1:])):
        owner[max(0, lo):max(0, min(hi, rows))] = g
    return owner


def look64(tokens, table, scale, owner, index, before):
    """`before` where a row is in no group."""
    import torch
    out = before.double().clone()
    t, many, vocab = tokens.long(), table.dim() == 3, table.shape[-2]
    for r in range(len(t)):
        g = int(owner[r])
        if g < 0:
            continue
        m = (table[index[g]] if many else table)
        out[r] = m[int(t[r])].double() * f32(scale) if 0 <= int(t[r]) < vocab else 0.0
    return out


def gradient64(dy, tokens, vocab, scale, owner, groups):
    """Gradient and the sum of magnitudes and number of rows of each token, [groups, vocab, ...]."""
    import torch
    ok = (owner >= 0) & (tokens.long() >= 0) & (tokens.long() < vocab)
    at = (owner * vocab + tokens.long())[ok]
    total = torch.zeros(groups * vocab, dy.shape[1], dtype=torch.float64).index_add_(0, at, dy.double()[ok])
    size = torch.zeros(groups * vocab, dy.shape[1], dtype=torch.float64).index_add_(0, at, dy.double()[ok].abs())
    n = torch.zeros(groups * vocab, dtype=torch.float64).index_add_(0, at, torch.ones(int(ok.sum()), dtype=torch.float64))
    s = f32(scale)
    off = (n[:, None] + 2) * U * size * abs(s)
    return (total * s).view(groups, vocab, -1), off.view(groups, vocab, -1)


SIZES = [(1, 1, 1), (1, 7, 8), (2, 3, 5), (37, 100, 111), (64, 50, 64), (65, 1000, 513), (300, 17, 1024), (1000, 257, 72), (33, 5000, 2056)]


@pytest.mark.parametrize("bits", [32, 64])
@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,dim", SIZES)
def test_lookup(tk, dtype, rows, vocab, dim, bits):
    import torch
    t, g = getattr(torch, dtype), gen(rows + vocab + dim)
    table = torch.randn(vocab, dim, device="cuda", generator=g).to(t)
    tok = torch.randint(-2, vocab + 2, (rows,), device="cuda", generator=g).to(getattr(torch, f"int{bits}"))
    for scale in (1.0, -3.7):
        y = tk.ps_embedding_forward(tok, table, scale)
        assert y.shape == (rows, dim) and y.dtype == t
        want = look64(tok.cpu(), table.cpu(), scale, owner_of(rows, None), None, torch.zeros(rows, dim))
        close(y.cpu(), want, U * want.abs(), "rows")
        if scale == 1.0:
            assert torch.equal(y.cpu().double(), want)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("rows,vocab,dim,groups", [(1, 3, 4, 1), (50, 20, 33, 3), (129, 300, 256, 70), (513, 40, 520, 9)])
def test_lookup_in_groups(tk, dtype, rows, vocab, dim, groups):
    import torch
    t, g = getattr(torch, dtype), gen(rows + groups)
    cuts = sorted(torch.randint(0, rows + 1, (groups + 1,), generator=torch.Generator().manual_seed(rows)).tolist())
    index = torch.randint(0, 4, (groups,), generator=torch.Generator().manual_seed(7)).tolist()
    wide = torch.randn(4, vocab, dim + 3, device="cuda", generator=g).to(t)
    table = wide[:, :, 1:dim + 1]  # rows further apart than they are long, at odd places
    tok = torch.randint(-1, vocab + 1, (rows, 2), device="cuda", generator=g)[:, 1]
    out = torch.full((rows, dim + 1), 5.0, device="cuda", dtype=t)
    tk.ps_grouped_embedding_forward(tok, torch.tensor(cuts, dtype=torch.int32).cuda(), table, 0.5, torch.tensor(index, dtype=torch.int32).cuda(), out=out[:, :dim])
    want = look64(tok.cpu(), table.cpu(), 0.5, owner_of(rows, cuts), index, torch.full((rows, dim), 5.0))
    assert torch.equal(out[:, :dim].cpu().double(), want.to(t).double())
    assert bool((out[:, dim] == 5).all())


def test_lookup_where_padding_meets_values_that_are_not_finite(tk):
    import torch
    table = torch.full((3, 40), float("nan"), device="cuda")
    y = tk.ps_embedding_forward(torch.tensor([-1, 3, 1], device="cuda"), table, 2.0)
    assert bool((y[:2] == 0).all()) and bool(y[2].isnan().all())
    empty = tk.ps_embedding_forward(torch.zeros(0, dtype=torch.int64, device="cuda"), table)
    assert empty.shape == (0, 40)


KINDS = ["spread", "same", "two", "none", "ascending", "zipf"]


def some_tokens(kind, rows, vocab, g):
    import torch
    if kind == "same":
        return torch.full((rows,), vocab // 2, device="cuda")
    if kind == "none":
        return torch.full((rows,), -1, device="cuda")
    if kind == "two":
        return torch.where(torch.rand(rows, device="cuda", generator=g) < 0.3, 0, vocab - 1)
    if kind == "ascending":
        return torch.arange(rows, device="cuda") % vocab
    if kind == "zipf":
        return (torch.exp(torch.rand(rows, device="cuda", generator=g) * torch.log(torch.tensor(vocab + 1.0))) - 1).long().clamp(0, vocab - 1)
    return torch.randint(-1, vocab + 1, (rows,), device="cuda", generator=g)


# runs and chunks around 32 places, one block's sort and several, one to four digits
@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,vocab,dim", [(0, 5, 8), (1, 1, 1), (31, 4, 8), (32, 300, 33), (33, 2, 520), (64, 1, 7), (65, 70000, 3), (1000, 255, 24), (1000, 256, 24), (8192, 300, 5),
                                            (8193, 300, 5), (20000, 70000, 2), (30000, 11, 9), (3000, 1 << 22, 1), (16384, 3, 4)])
def test_gradient(tk, kind, rows, vocab, dim):
    import torch
    g = gen(rows + vocab + dim)
    tok = some_tokens(kind, rows, vocab, g)
    for dtype in TYPES:
        t = getattr(torch, dtype)
        dy = torch.randn(rows, dim, device="cuda", generator=g).to(t)
        got = tk.ps_embedding_backward(dy, tok.to(torch.int32) if dtype == "float32" else tok, vocab, 1.5)
        assert got.shape == (vocab, dim) and got.dtype == t
        want, off = gradient64(dy.cpu(), tok.cpu(), vocab, 1.5, owner_of(rows, None), 1)
        close(got.cpu(), want[0], off[0], f"{kind} {dtype}")
        assert torch.equal(got, tk.ps_embedding_backward(dy, tok, vocab, 1.5)), "the same bytes every time"


@pytest.mark.parametrize("rows,vocab,dim,groups", [(5, 3, 2, 1), (100, 6, 40, 3), (3000, 90, 17, 64), (9000, 4096, 4, 20)])
def test_gradient_in_groups(tk, rows, vocab, dim, groups):
    import torch
    g = gen(rows)
    cuts = sorted(torch.randint(0, rows + 1, (groups + 1,), generator=torch.Generator().manual_seed(rows)).tolist())
    offsets = torch.tensor(cuts, dtype=torch.int32).cuda()
    tok = some_tokens("zipf", rows, vocab, g)
    tok[::50] = -100
    wide = torch.randn(rows, dim + 5, device="cuda", generator=g)
    dy = wide[:, 2:dim + 2]
    total = vocab * dim
    queue = torch.full((groups, total + 11), 7.0, device="cuda")
    dtable = queue[:, 3:total + 3].unflatten(1, (vocab, dim))  # every worker's part of its row of a gradient buffer
    got = tk.ps_grouped_embedding_backward(dy, tok, offsets, vocab, -0.25, dtable=dtable)
    assert got is dtable and bool((queue[:, :3] == 7).all()) and bool((queue[:, total + 3:] == 7).all())
    want, off = gradient64(dy.cpu(), tok.cpu(), vocab, -0.25, owner_of(rows, cuts), groups)
    close(got.cpu(), want, off, "gradients")
    # a worker's gradient does not depend on the others
    for k in (0, groups // 2, groups - 1):
        alone = tk.ps_embedding_backward(dy[cuts[k]:cuts[k + 1]], tok[cuts[k]:cuts[k + 1]], vocab, -0.25)
        assert torch.equal(alone, got[k])


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("rows,vocab,dim", [(1, 1, 1), (16, 300, 7), (17, 2, 9), (64, 70000, 513), (255, 3, 1031), (300, 255, 64), (512, 256, 8), (512, 4097, 2049)])
def test_few_rows_and_many_give_the_same_bits(tk, kind, rows, vocab, dim):
    """The same rows with others of no token behind them, which take another way."""
    import torch
    g = gen(rows + dim)
    tok = some_tokens(kind, rows, vocab, g)
    more = torch.cat([tok, torch.full((600,), -1, device="cuda")])
    for dtype in TYPES:
        dy = torch.randn(rows + 600, dim, device="cuda", generator=g).to(getattr(torch, dtype))
        few, many = tk.ps_embedding_backward(dy[:rows], tok, vocab, 0.7), tk.ps_embedding_backward(dy, more, vocab, 0.7)
        assert torch.equal(few, many)
        want, off = gradient64(dy[:rows].cpu(), tok.cpu(), vocab, 0.7, owner_of(rows, None), 1)
        close(few.cpu(), want[0], off[0], f"{kind} {dtype}")


@pytest.mark.parametrize("vocab,dim,groups", [(1, 3, 70), (300, 40, 7), (1000, 520, 3), (5000, 4, 1)])
def test_few_rows_in_groups_and_many_give_the_same_bits(tk, vocab, dim, groups):
    """With groups without rows and rows before and behind all groups, in tokens and rows that are apart."""
    import torch
    g, rows = gen(vocab), 410
    cuts = sorted(torch.randint(5, rows - 9, (groups + 1,), generator=torch.Generator().manual_seed(groups)).tolist())
    if groups > 2:
        cuts[1] = cuts[2]
    offsets = torch.tensor(cuts, dtype=torch.int32).cuda()
    tok = some_tokens("zipf", rows + 200, vocab, g)[:, None].repeat(1, 3)[:, 1]
    dy = torch.randn(rows + 200, dim + 3, device="cuda", generator=g)[:, 1:dim + 1]
    few, many = tk.ps_grouped_embedding_backward(dy[:rows], tok[:rows], offsets, vocab), tk.ps_grouped_embedding_backward(dy, tok, offsets, vocab)
    assert torch.equal(few, many)
    want, off = gradient64(dy[:rows].cpu(), tok[:rows].cpu(), vocab, 1.0, owner_of(rows, cuts), groups)
    close(few.cpu(), want, off, "gradients")


def test_few_rows_in_a_graph(tk):
    import torch
    g = gen(6)
    tok, dy = torch.randint(0, 90, (200,), device="cuda", generator=g), torch.randn(200, 24, device="cuda", generator=g)
    tk.ps_embedding_backward(dy, tok, 90)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = tk.ps_embedding_backward(dy, tok, 90)
    for _ in range(3):
        tok.copy_(torch.randint(-1, 91, (200,), device="cuda", generator=g))
        dy.normal_(generator=g)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, tk.ps_embedding_backward(dy, tok, 90))


def test_keys_of_more_than_24_bits(tk):
    """Workers' tokens whose numbers, with the workers', pass what 32-bit floats hold."""
    import torch
    g, rows, vocab, groups = gen(2), 5000, 1 << 20, 20
    cuts = [rows * i // groups for i in range(groups + 1)]
    # neighbours, high and low, so that keys differ by one
    tok = torch.randint(0, 4, (rows,), device="cuda", generator=g) + torch.where(torch.rand(rows, device="cuda", generator=g) < 0.5, 0, vocab - 4)
    dy = torch.randn(rows, 1, device="cuda", generator=g)
    got = tk.ps_grouped_embedding_backward(dy, tok, torch.tensor(cuts, dtype=torch.int32).cuda(), vocab)
    want, off = gradient64(dy.cpu(), tok.cpu(), vocab, 1.0, owner_of(rows, cuts), groups)
    close(got.cpu(), want, off, "gradients")


@pytest.mark.parametrize("rows,vocab,dim,gap", [(40, 30, 5, 3), (40, 30, 1, 1), (100, 70, 300, 12), (20, 9, 40000, 5), (17000, 50, 24, 40)])
def test_gradient_in_rows_apart(tk, rows, vocab, dim, gap):
    """Lines shorter and longer than what a block clears, between others that stay as they are."""
    import torch
    for dtype in TYPES:
        t, g = getattr(torch, dtype), gen(rows + dim)
        dy, tok = torch.randn(rows, dim, device="cuda", generator=g).to(t), some_tokens("spread", rows, vocab, g)
        cuts = [0, rows // 3, rows]
        wide = torch.full((2, vocab + 1, dim + gap), 6.0, device="cuda", dtype=t)
        out = wide[:, :vocab, 1:dim + 1]
        tk.ps_grouped_embedding_backward(dy, tok, torch.tensor(cuts, dtype=torch.int32).cuda(), vocab, 0.5, dtable=out)
        want, off = gradient64(dy.cpu(), tok.cpu(), vocab, 0.5, owner_of(rows, cuts), 2)
        close(out.cpu(), want, off, "gradient")
        out.fill_(6.0)
        assert bool((wide == 6).all())


def test_many_groups_that_begin_at_a_row(tk):
    """Hundreds of empty groups between rows, and more groups than one look takes."""
    import torch
    g, rows, groups = gen(4), 150, 5000
    cuts = sorted(torch.randint(0, 10, (groups + 1,), generator=torch.Generator().manual_seed(1)).tolist())
    cuts[-700:] = sorted(torch.randint(10, rows, (700,), generator=torch.Generator().manual_seed(2)).tolist())
    offsets, index = torch.tensor(cuts, dtype=torch.int32).cuda(), (torch.arange(groups) % 7).to(torch.int32)
    table, tok = torch.randn(7, 20, 12, device="cuda", generator=g), torch.randint(0, 20, (rows,), device="cuda", generator=g)
    out = torch.zeros(rows, 12, device="cuda")
    tk.ps_grouped_embedding_forward(tok, offsets, table, 1.0, index.cuda(), out=out)
    owner = owner_of(rows, cuts)
    assert torch.equal(out.cpu().double(), look64(tok.cpu(), table.cpu(), 1.0, owner, index.tolist(), torch.zeros(rows, 12)))
    dy = torch.randn(rows, 3, device="cuda", generator=g)
    got = tk.ps_grouped_embedding_backward(dy, tok, offsets, 20)
    want, off = gradient64(dy.cpu(), tok.cpu(), 20, 1.0, owner, groups)
    close(got.cpu(), want, off, "gradients")


def test_offsets_of_any_contents_stay_inside(tk):
    import torch
    g = gen(3)
    table, tok = torch.randn(2, 10, 16, device="cuda", generator=g), torch.randint(0, 10, (40,), device="cuda", generator=g)
    dy = torch.randn(40, 16, device="cuda", generator=g)
    for cuts in ([0, 50, 20], [-5, 10, 1000], [30, 20, 10], [40, 40, 40], [2 ** 31 - 1, -2 ** 31, 7]):
        offsets = torch.tensor(cuts, dtype=torch.int32).cuda()
        out = torch.zeros(40, 16, device="cuda")
        tk.ps_grouped_embedding_forward(tok, offsets, table, 1.0, torch.tensor([99, -99], dtype=torch.int32).cuda(), out=out)
        for r in range(40):
            assert any(torch.equal(out[r], x) for x in (torch.zeros_like(out[r]), table[0, tok[r]], table[1, tok[r]]))
        assert bool(tk.ps_grouped_embedding_backward(dy, tok, offsets, 10).isfinite().all())
    one = torch.tensor([5, 30], dtype=torch.int32).cuda()  # rows in no group: no gradient
    got = tk.ps_grouped_embedding_backward(dy, tok, one, 10)
    want, off = gradient64(dy.cpu(), tok.cpu(), 10, 1.0, owner_of(40, [5, 30]), 1)
    close(got.cpu(), want, off, "gradient")


def test_the_gradient_against_differences(tk):
    """sum(dy * lookup(table)) is linear in the table: a change of one of its values changes it by the gradient, up to rounding.  The values
    are small whole numbers, so that nothing is rounded."""
    import torch
    g = gen(11)
    table = torch.randint(-4, 5, (6, 10), device="cuda", generator=g).float()
    tok = torch.randint(-1, 7, (50,), device="cuda", generator=g)
    dy = torch.randint(-4, 5, (50, 10), device="cuda", generator=g).float()
    grad = tk.ps_embedding_backward(dy, tok, 6, 2.0)
    f = lambda w: (dy.double() * tk.ps_embedding_forward(tok, w, 2.0).double()).sum().item()  # noqa: E731
    for v in range(6):
        for d in (0, 9):
            more = table.clone()
            more[v, d] += 1.0
            assert f(more) - f(table) == grad[v, d].item()


def test_values_that_are_not_finite_stay_with_their_token(tk):
    import torch
    dy = torch.ones(100, 24, device="cuda")
    tok = torch.arange(100, device="cuda") % 10
    dy[13] = float("nan")
    dy[14] = float("inf")
    got = tk.ps_embedding_backward(dy, tok, 12)
    assert bool(got[3].isnan().all()) and bool((got[4] == float("inf")).all())
    assert bool((got[[0, 1, 2, 5, 6, 7, 8, 9]] == 10).all()) and bool((got[10:] == 0).all())


def test_rows_beyond_32_bits(tk):
    """A table of more than 2^31 elements and of more than 4 GB, and a gradient buffer so."""
    import torch
    vocab, dim = 1100000, 2048
    table = torch.zeros(vocab, dim, device="cuda", dtype=torch.bfloat16)
    tok = torch.tensor([vocab - 1, 5, 1048576, vocab - 2], device="cuda")
    table[tok] = torch.arange(1, 5, device="cuda", dtype=torch.bfloat16)[:, None]
    y = tk.ps_embedding_forward(tok, table)
    assert torch.equal(y[:, 0].float().cpu(), torch.tensor([1., 2., 3., 4.])) and bool((y == y[:, :1]).all())
    table.fill_(9.0)
    got = tk.ps_embedding_backward(y, tok, vocab, dtable=table)
    assert torch.equal(got[tok], y)
    got[tok] = 0
    assert not bool(got.any())


def test_calls_in_a_graph_and_on_another_stream(tk):
    import torch
    g = gen(5)
    table = torch.randn(500, 96, device="cuda", generator=g)
    tok = torch.randint(0, 500, (9000,), device="cuda", generator=g)
    dy = torch.randn(9000, 96, device="cuda", generator=g)
    other = torch.cuda.Stream()
    other.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(other):
        y, d = tk.ps_embedding_forward(tok, table, 3.0), tk.ps_embedding_backward(dy, tok, 500, 3.0)
    torch.cuda.current_stream().wait_stream(other)
    assert torch.equal(y, tk.ps_embedding_forward(tok, table, 3.0)) and torch.equal(d, tk.ps_embedding_backward(dy, tok, 500, 3.0))
    graphs = []
    for _ in range(2):  # with workspaces of their own
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            out = tk.ps_embedding_forward(tok, table, 3.0), tk.ps_embedding_backward(dy, tok, 500, 3.0)
        graphs.append((graph, out))
    for _ in range(3):
        tok.copy_(torch.randint(-1, 501, (9000,), device="cuda", generator=g))
        dy.normal_(generator=g)
        for graph, out in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, out in graphs:
            assert torch.equal(out[0], tk.ps_embedding_forward(tok, table, 3.0)) and torch.equal(out[1], tk.ps_embedding_backward(dy, tok, 500, 3.0))


def test_calls_that_are_refused(tk):
    import torch
    from paper_2406_05546_amd.binding import PsError
    table, tok, dy = torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda"), torch.zeros(4, 8, device="cuda")
    offsets = torch.tensor([0, 4], dtype=torch.int32, device="cuda")
    bad = [lambda: tk.ps_embedding_forward(tok.float(), table), lambda: tk.ps_embedding_forward(tok.cpu(), table), lambda: tk.ps_embedding_forward(tok[None], table),
           lambda: tk.ps_embedding_forward(tok, table.double()), lambda: tk.ps_embedding_forward(tok, table.t()), lambda: tk.ps_embedding_forward(tok, table[None]),
           lambda: tk.ps_embedding_forward(tok, table, out=dy[:3]), lambda: tk.ps_embedding_forward(tok, table, out=dy.half()), lambda: tk.ps_embedding_forward(tok, table, float("nan")),
           lambda: tk.ps_grouped_embedding_forward(tok, offsets, table), lambda: tk.ps_grouped_embedding_forward(tok, offsets.long(), table[None]),
           lambda: tk.ps_grouped_embedding_forward(tok, offsets[:1], table[None]), lambda: tk.ps_grouped_embedding_forward(tok, offsets, table[None], table_of_group=offsets),
           lambda: tk.ps_embedding_backward(dy, tok[:3], 10), lambda: tk.ps_embedding_backward(dy[0], tok, 10), lambda: tk.ps_embedding_backward(dy, tok, 0),
           lambda: tk.ps_embedding_backward(dy, tok, (1 << 22) + 1), lambda: tk.ps_embedding_backward(dy, tok, 10, dtable=table[:9]), lambda: tk.ps_embedding_backward(dy, tok, 10, float("inf")),
           lambda: tk.ps_embedding_backward(dy[:, :1].expand(4, 8), tok, 10), lambda: tk.ps_embedding_backward(dy[:1].expand(4, 8), tok, 10)]
    for i, call in enumerate(bad):
        with pytest.raises(PsError):
            call()
            pytest.fail(f"call {i} was not refused")
