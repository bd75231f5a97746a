"""Embedding of rows in groups whose offsets do not ascend: what is one row's group has to be the same to the lookup, to the gradient of few rows
(one launch) and to that of many (sorted).  Rows with no token behind the others make many of few.

The gradient's tolerance is that of test_gpu_embedding.py: n steps of 2^-24 of the sum of magnitudes for n rows, and the product with the scale."""
import pytest

from tests.test_gpu_embedding import close, gen, gradient64, tk  # noqa: F401

pytestmark = pytest.mark.gpu


def by_lookup(tk, rows, cuts, dim):
    """Group of each row as the lookup has it, -1 for none: every group's table has its number."""
    import torch
    n = len(cuts) - 1
    table = torch.arange(1, n + 1, device="cuda", dtype=torch.float32)[:, None, None].expand(n, 1, dim).contiguous()
    out = torch.zeros(rows, dim, device="cuda")
    tk.ps_grouped_embedding_forward(torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.tensor(cuts, dtype=torch.int32).cuda(), table, out=out)
    assert bool((out == out[:, :1]).all())
    return out[:, 0].long().cpu() - 1


def last_that_begins(rows, cuts):
    """The last group that begins at a row or before, if it ends behind it."""
    import torch
    cuts, owner = [min(max(c, 0), rows) for c in cuts], torch.full((rows,), -1, dtype=torch.int64)
    for r in range(rows):
        g = max((g for g, c in enumerate(cuts[:-1]) if c <= r), default=-1)
        if g >= 0 and r < cuts[g + 1]:
            owner[r] = g
    return owner


def check_gradients(tk, rows, cuts, owner, vocab, dim, more):
    import torch
    g, n = gen(rows + dim), len(cuts) - 1
    offsets = torch.tensor(cuts, dtype=torch.int32).cuda()
    tok = torch.cat([torch.randint(-1, vocab, (rows,), device="cuda", generator=g), torch.full((more,), -1, device="cuda")])
    dy = torch.randn(rows + more, dim, device="cuda", generator=g)
    want, off = gradient64(dy[:rows].cpu(), tok[:rows].cpu(), vocab, 1.5, owner, n)
    got = tk.ps_grouped_embedding_backward(dy[:rows], tok[:rows], offsets, vocab, 1.5)
    close(got.cpu(), want, off, "gradients")
    if more:
        assert torch.equal(got, tk.ps_grouped_embedding_backward(dy, tok, offsets, vocab, 1.5))


CUTS = [[0, 30, 10, 40], [0, 10, 5, 20], [0, 40, 3, 25, 7, 33], [30, 20, 10], [0, 30, 5, 10], [5, 5, 40, 0, 12], [10, 40, 10, 40, 10], [0, 39, 38, 37, 40]]


@pytest.mark.parametrize("cuts", CUTS)
def test_a_row_is_in_one_group(tk, cuts):
    owner = last_that_begins(40, cuts)
    assert owner.tolist() == by_lookup(tk, 40, cuts, 16).tolist()
    check_gradients(tk, 40, cuts, owner, 3, 5, 600)


@pytest.mark.parametrize("rows,groups", [(410, 3), (512, 17), (130, 64), (200, 65), (512, 300), (500, 5000), (30000, 64), (30000, 65), (30000, 700)])
def test_any_offsets_mean_the_same_to_every_call(tk, rows, groups):
    import torch
    cuts = torch.randint(0, rows + 1, (groups + 1,), generator=torch.Generator().manual_seed(groups)).tolist()
    owner = by_lookup(tk, rows, cuts, 24)
    for dim in (8, 500):  # other numbers of rows to a block
        assert torch.equal(owner, by_lookup(tk, rows, cuts, dim))
    if groups <= 64 and rows <= 512:
        assert owner.tolist() == last_that_begins(rows, cuts).tolist()
    begin, end = torch.tensor(cuts)[owner], torch.tensor(cuts)[owner + 1]
    row = torch.arange(rows)
    assert bool(((owner < 0) | ((begin <= row) & (row < end))).all())
    check_gradients(tk, rows, cuts, owner, 3, 4, 600 if rows <= 512 else 0)


def test_ascending_offsets_beyond_one_look(tk):
    """More groups than are looked at together, rows before and behind them, every row in its own."""
    for rows, groups in ((512, 100), (300, 4200), (30000, 500)):
        import torch
        cuts = sorted(torch.randint(3, rows - 5, (groups + 1,), generator=torch.Generator().manual_seed(groups)).tolist())
        owner = torch.full((rows,), -1, dtype=torch.int64)
        for k in range(groups):
            owner[cuts[k]:cuts[k + 1]] = k
        assert torch.equal(owner, by_lookup(tk, rows, cuts, 24))
        check_gradients(tk, rows, cuts, owner, 3, 4, 600 if rows <= 512 else 0)
