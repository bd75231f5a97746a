"""The embedding's gradient where rows are sorted: from 16385 rows on, by as many digits of 8 bits as groups times vocabulary have, and on either side of that
number.  Tolerances as in test_gpu_embedding.py; up to 16384 rows they are ranked, which has to give the same bits."""
import pytest

from tests.test_gpu_embedding import close, gen, gradient64, owner_of, some_tokens, tk  # noqa: F401

pytestmark = pytest.mark.gpu


# one digit to four; the result of an even number of passes lies elsewhere than that of an odd one
@pytest.mark.parametrize("kind", ["spread", "zipf", "same", "ascending"])
@pytest.mark.parametrize("rows,vocab,dim", [(16385, 255, 5), (16385, 256, 5), (17408, 257, 9), (20001, 50257, 3), (18000, 65535, 8), (17409, 65536, 4), (16400, 1 << 20, 1),
                                            (40000, 1000, 520)])
def test_digits(tk, kind, rows, vocab, dim):
    import torch
    g = gen(rows + vocab)
    tok = some_tokens(kind, rows, vocab, g)
    for dtype in ("float32", "bfloat16", "float16"):
        dy = torch.randn(rows, dim, device="cuda", generator=g).to(getattr(torch, dtype))
        got = tk.ps_embedding_backward(dy, tok.to(torch.int32) if dtype == "bfloat16" else tok, vocab, -0.75)
        want, off = gradient64(dy.cpu(), tok.cpu(), vocab, -0.75, owner_of(rows, None), 1)
        close(got.cpu(), want[0], off[0], f"{kind} {dtype}")


@pytest.mark.parametrize("rows,vocab,dim,groups", [(20000, 100, 8, 2), (17000, 300, 24, 65), (30000, 1 << 20, 1, 17), (16385, 1 << 22, 1, 4), (25000, 5, 12, 3000)])
def test_groups_with_rows_in_none(tk, rows, vocab, dim, groups):
    """Rows before and behind all groups, and groups without rows."""
    import torch
    g = gen(rows)
    cuts = sorted(torch.randint(100, rows - 200, (groups + 1,), generator=torch.Generator().manual_seed(vocab)).tolist())
    cuts[1] = cuts[0]
    tok = some_tokens("zipf", rows, vocab, g)
    tok[::37] = -1
    dy = torch.randn(rows, dim, device="cuda", generator=g)
    got = tk.ps_grouped_embedding_backward(dy, tok, torch.tensor(cuts, dtype=torch.int32).cuda(), vocab, 1.0)
    want, off = gradient64(dy.cpu(), tok.cpu(), vocab, 1.0, owner_of(rows, cuts), groups)
    close(got.cpu(), want, off, "gradients")
    # a worker alone, by ranks or in one launch
    for k in (1, groups // 2, groups - 1):
        if 0 < cuts[k + 1] - cuts[k] <= 16384:
            assert torch.equal(got[k], tk.ps_embedding_backward(dy[cuts[k]:cuts[k + 1]], tok[cuts[k]:cuts[k + 1]], vocab))


@pytest.mark.parametrize("kind", ["spread", "zipf", "same", "two", "none"])
@pytest.mark.parametrize("rows,vocab,dim", [(16384, 300, 24), (16383, 50257, 8), (16384, 3, 520), (9001, 70000, 3), (513, 40, 1024)])
def test_ranks_and_sort_give_the_same_bits(tk, kind, rows, vocab, dim):
    """The same rows with others of no token behind them, which are sorted."""
    import torch
    g, more = gen(rows + dim), 16385 - rows + 1000
    tok = torch.cat([some_tokens(kind, rows, vocab, g), torch.full((more,), -1, device="cuda")])
    for dtype in ("float32", "bfloat16"):
        dy = torch.randn(rows + more, dim, device="cuda", generator=g).to(getattr(torch, dtype))
        assert torch.equal(tk.ps_embedding_backward(dy[:rows], tok[:rows], vocab, 0.7), tk.ps_embedding_backward(dy, tok, vocab, 0.7))
