"""Calls of the operators on tokens at the ends of what they take: the largest and smallest scales, tokens beyond 32 bits, more rows than a launch has
blocks.  Tolerances as in test_gpu_logprob.py."""
import pytest

from tests.test_gpu_logprob import INF, U, check_backward, check_forward, f32, gen, tk  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("scale", [2e38, 1e30, 1e-30, 2e-38, 1e-42])
@pytest.mark.parametrize("rows,vocab", [(5, 40), (3, 5000), (2, 100001)])
def test_scales_at_the_ends(tk, rows, vocab, scale):
    import torch
    g = gen(vocab)
    # differences that a large scale leaves within reach, and for small ones values up to 1e38
    z = torch.randn(rows, vocab, device="cuda", generator=g) * max(min(3.0 / scale, 1e37), 1e-37)
    tok = torch.randint(-1, vocab + 1, (rows,), device="cuda", generator=g)
    if scale >= 1e-38:
        check_forward(tk, z, tok, scale, 3)
    norm = tk.ps_logprob_forward(z, tok, scale).norm
    d = tk.ps_logprob_backward(z, tok, norm, torch.full((rows,), 2.0 ** -8, device="cuda"), torch.full((rows,), -(2.0 ** -10), device="cuda"), scale)
    check_backward(z, tok, norm, torch.full((rows,), 2.0 ** -8, device="cuda"), torch.full((rows,), -(2.0 ** -10), device="cuda"), scale, d)


def test_a_gradient_beyond_the_numbers_is_infinite_where_it_is(tk):
    """scale times dlogp is no 32-bit number: infinite for the token, 0 for logits without probability."""
    import torch
    z = torch.full((3, 300), -1.0, device="cuda")
    z[:, 7] = 1.0
    tok = torch.tensor([9, 7, -1], device="cuda")
    norm = tk.ps_logprob_forward(z, tok, 2e38).norm
    four = torch.full((3,), 4.0, device="cuda")
    d = tk.ps_logprob_backward(z, tok, norm, four, None, 2e38)
    want = torch.zeros_like(d)
    want[0, 9], want[0, 7] = INF, -INF
    assert torch.equal(d, want)  # of the token with probability 1 it is 0
    # the entropy of a row of one token does not change
    assert not bool(tk.ps_logprob_backward(z, tok, norm, None, four, 2e38).any())


def test_tokens_beyond_32_bits_are_none(tk):
    import torch
    far = torch.tensor([2 ** 32 + 3, -2 ** 63, 2 ** 63 - 1, 2 ** 31 + 1, -2 ** 32, 3], device="cuda")
    z = torch.randn(6, 50, device="cuda", generator=gen(1))
    p = tk.ps_logprob_forward(z, far)
    assert bool((p.logp[:5] == 0).all()) and float(p.logp[5]) < 0
    d = tk.ps_logprob_backward(z, far, p.norm, torch.ones(6, device="cuda"))
    assert not bool(d[:5].any()) and bool(d[5].any())
    table, dy = torch.ones(50, 24, device="cuda"), torch.ones(6, 24, device="cuda")
    y = tk.ps_embedding_forward(far, table)
    assert not bool(y[:5].any()) and bool((y[5] == 1).all())
    want = torch.zeros(50, 24, device="cuda")
    want[3] = 1
    assert torch.equal(tk.ps_embedding_backward(dy, far, 50), want)
    for more in (600, 17000):  # by ranks, and sorted
        tok, many = torch.cat([far, far[:1].expand(more)]), torch.cat([dy, dy[:1].expand(more, 24)])
        assert torch.equal(tk.ps_embedding_backward(many, tok, 50), want)
    low = torch.tensor([-2 ** 31, 2 ** 31 - 1, 3], device="cuda", dtype=torch.int32)
    assert torch.equal(tk.ps_embedding_backward(dy[:3], low, 50), want)


def test_more_rows_than_blocks(tk):
    """A block has several of them in turn."""
    import torch
    g, rows = gen(3), 4300001
    z = torch.randn(rows, 5, device="cuda", generator=g)
    tok = torch.randint(-1, 5, (rows,), device="cuda", generator=g)
    p = check_forward(tk, z, tok, 1.0, 2)
    one = torch.ones(1, device="cuda").expand(rows)
    d = tk.ps_logprob_backward(z, tok, p.norm, one, one)
    for part in (slice(0, 1000), slice(rows - 1000, rows), slice(4194300, 4194310)):
        check_backward(z[part], tok[part], p.norm[part], one[part], one[part], 1.0, d[part])
    # every row's gradient adds up to 0: of five values, each off by a few U of 2 + ln 5 at most
    assert float(d.sum(1).abs().max()) <= 5 * 8 * U * 4
    table = torch.arange(5, device="cuda").float()[:, None] * torch.ones(3, device="cuda")
    y = tk.ps_embedding_forward(tok, table, 2.0)
    assert torch.equal(y[:, 1], tok.clamp(min=0).float() * 2)
    got = tk.ps_embedding_backward(torch.ones(rows, 3, device="cuda"), tok, 5)
    assert torch.equal(got[:, 2].long(), torch.bincount(tok + 1, minlength=6)[1:])  # whole numbers below 2^24


def test_calls_at_once_from_threads_on_streams(tk):
    """Each with its results and workspaces: gradients in one launch, by ranks and sorted, rows cut into parts, layers that keep 8 bits."""
    import threading
    import torch
    from paper_2406_05546_amd import dense
    g = gen(8)
    offsets = torch.tensor([0, 90, 30, 200], dtype=torch.int32).cuda()
    tok = torch.randint(-1, 300, (20000,), device="cuda", generator=g)
    dy, z = torch.randn(20000, 40, device="cuda", generator=g), torch.randn(3, 90001, device="cuda", generator=g)
    x, w = torch.randn(70, 96, device="cuda", generator=g).bfloat16(), torch.randn(200, 96, device="cuda", generator=g).bfloat16()

    def step():
        out = [tk.ps_grouped_embedding_backward(dy[:200], tok[:200], offsets, 300)] + [tk.ps_embedding_backward(dy[:n], tok[:n], 300) for n in (300, 9000, 20000)]
        p = tk.ps_logprob_forward(z, tok[:3], 1.0, 20)
        out += [p.logp, p.norm, p.top_logp, p.top_tokens, tk.ps_logprob_backward(z, tok[:3], p.norm, dy[:3, 0], dy[:3, 1])]
        for rows in (5, 70):
            pre = dense.ps_checkpoint_empty(rows, 200, "cuda:0")
            out.append(dense.ps_linear_forward(x[:rows], w, activation="gelu", pre=pre))
            out += [pre.codes.view(torch.uint8), pre.scales.view(torch.uint8)]
            out += dense.ps_linear_backward(out[-3], dense.ps_checkpoint_encode(x[:rows]), w, "gelu", pre=pre)
        return out
    want, bad = step(), []
    torch.cuda.synchronize()

    def run(k):
        stream = torch.cuda.Stream()
        with torch.cuda.stream(stream):
            for _ in range(10):
                if not all(torch.equal(a, b) for a, b in zip(step(), want)):
                    bad.append(k)
        stream.synchronize()
    threads = [threading.Thread(target=run, args=(k,)) for k in range(4)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not bad


def test_in_place_in_rows_of_any_place(tk):
    """The gradient over the logits where rows begin between multiples of 16 bytes, and nothing beside them."""
    import torch
    for t in (torch.float32, torch.bfloat16, torch.float16):
        for vocab, first in ((1, 1), (7, 3), (33, 5), (4097, 1), (20001, 7)):
            wide = torch.randn(9, vocab + 11, device="cuda", generator=gen(vocab)).to(t)
            z, before = wide[:, first:first + vocab], wide.clone()
            tok = torch.arange(9, device="cuda") % vocab
            p, a = tk.ps_logprob_forward(z, tok, 0.7), torch.randn(9, device="cuda", generator=gen(1))
            want = tk.ps_logprob_backward(z.contiguous(), tok, p.norm, a, a, 0.7)
            got = tk.ps_logprob_backward(z, tok, p.norm, a, a, 0.7, out=z)
            assert got is z and torch.equal(z, want)
            assert torch.equal(wide[:, :first], before[:, :first]) and torch.equal(wide[:, first + vocab:], before[:, first + vocab:])
