"""Operators on tokens without a GPU: declared symbols, workspaces, and the calls that are refused before anything is launched."""
import ctypes
import os
import re

import pytest
import torch

from paper_2406_05546_amd import binding as ps
from paper_2406_05546_amd import dense, tokens

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOMEWHERE = 1 << 20  # an aligned address that no refused call looks at
HUGE = 1 << 40


def lib():
    return tokens._library()


def message():
    return dense._library().ps_dense_last_error().decode()


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "ps_tokens.h")).read()
    declared = re.findall(r"^PS_API\s+[\w\s\*]+?\b(\w+)\(", header, flags=re.M)
    assert sorted(declared) == sorted(tokens.EXPORTS)
    for name in declared:
        assert getattr(ps.load_library(), name) is not None
    assert int(re.search(r"PS_LOGPROB_MAX_TOP (\d+)", header).group(1)) == tokens.LOGPROB_MAX_TOP


def embedding(**kw):
    d = dict(dtype=dense.PS_BF16, n_groups=1, n_tables=1, rows=8, vocab=100, dim=16, offsets_dev=None, table_of_group_dev=None, scale=1.0)
    d.update(kw)
    return tokens.ps_embedding(**d)


def look(e, t=None, table=None, out=None):
    t = t or tokens.ps_tokens(SOMEWHERE, 1, 4)
    table = table or dense.ps_matrix(SOMEWHERE, 16, 1600)
    out = out or dense.ps_matrix(SOMEWHERE, 16, 0)
    return lib().ps_embedding_forward(ctypes.byref(e), ctypes.byref(t), ctypes.byref(table), ctypes.byref(out), None)


def gradient(e, t=None, dy=None, dtable=None, ws=SOMEWHERE, size=HUGE):
    t = t or tokens.ps_tokens(SOMEWHERE, 1, 4)
    dy = dy or dense.ps_matrix(SOMEWHERE, 16, 0)
    dtable = dtable or dense.ps_matrix(SOMEWHERE, 16, 1600)
    return lib().ps_embedding_backward(ctypes.byref(e), ctypes.byref(t), ctypes.byref(dy), ctypes.byref(dtable), ws, size, None)


BAD = [dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=(1 << 28) + 1), dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(dim=0), dict(dim=(1 << 22) + 1),
       dict(n_groups=0), dict(n_groups=2, n_tables=2), dict(n_groups=32769, n_tables=32769, offsets_dev=SOMEWHERE), dict(offsets_dev=SOMEWHERE + 2),
       dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=1e39)]


@pytest.mark.parametrize("bad", BAD)
def test_embeddings_that_are_refused(bad):
    e = embedding(**bad)
    n = ctypes.c_uint64(0)
    assert look(e) == ps.PS_EINVAL and "ps_embedding_forward" in message()
    assert gradient(e) == ps.PS_EINVAL and "ps_embedding_backward" in message()
    assert lib().ps_embedding_workspace_bytes(ctypes.byref(e), ctypes.byref(n)) == ps.PS_EINVAL and "ps_embedding_workspace_bytes" in message()


def test_more_sums_than_keys_are_refused():
    assert gradient(embedding(n_groups=512, n_tables=512, vocab=1 << 22, offsets_dev=SOMEWHERE)) == ps.PS_EINVAL


@pytest.mark.parametrize("bad", [dict(n_tables=0), dict(n_groups=3, n_tables=2, offsets_dev=SOMEWHERE), dict(offsets_dev=SOMEWHERE, table_of_group_dev=SOMEWHERE + 1)])
def test_tables_that_are_refused(bad):
    assert look(embedding(**bad)) == ps.PS_EINVAL


@pytest.mark.parametrize("t", [(None, 1, 4), (SOMEWHERE, 1, 2), (SOMEWHERE, 1, 0), (SOMEWHERE + 2, 1, 4), (SOMEWHERE + 4, 1, 8), (SOMEWHERE, -1, 4), (SOMEWHERE, (1 << 22) + 1, 4)])
def test_tokens_that_are_refused(t):
    given = tokens.ps_tokens(*t)
    assert look(embedding(), given) == ps.PS_EINVAL and gradient(embedding(), given) == ps.PS_EINVAL
    assert score(logprob(), given) == ps.PS_EINVAL and score_gradient(logprob(), given) == ps.PS_EINVAL


@pytest.mark.parametrize("m", [(None, 16, 1600), (SOMEWHERE + 1, 16, 1600), (SOMEWHERE, 15, 1600), (SOMEWHERE, (1 << 22) + 1, HUGE)])
def test_matrices_that_are_refused(m):
    m = dense.ps_matrix(*m)
    assert look(embedding(), table=m) == ps.PS_EINVAL and look(embedding(), out=m) == ps.PS_EINVAL
    assert gradient(embedding(), dy=m) == ps.PS_EINVAL and gradient(embedding(), dtable=m) == ps.PS_EINVAL
    overlap = dense.ps_matrix(SOMEWHERE, 16, 99 * 16 + 15)
    many = embedding(n_groups=2, n_tables=2, offsets_dev=SOMEWHERE)
    assert look(many, table=overlap) == ps.PS_EINVAL and gradient(many, dtable=overlap) == ps.PS_EINVAL
    assert score(logprob(vocab=16), logits=m) == ps.PS_EINVAL and score_gradient(logprob(vocab=16), logits=m) == ps.PS_EINVAL
    assert score_gradient(logprob(vocab=16), dlogits=m) == ps.PS_EINVAL


def test_workspace_of_a_gradient():
    def need(**kw):
        n = ctypes.c_uint64(0)
        assert lib().ps_embedding_workspace_bytes(ctypes.byref(embedding(**kw)), ctypes.byref(n)) == ps.PS_OK
        return n.value
    assert need(rows=0) == 0
    assert need(rows=512) == 0  # one launch
    assert need(n_groups=300, offsets_dev=SOMEWHERE, vocab=4194304, dim=1) > 0  # which would have too many threads
    # keys and order of 513 rows, twice, counts in two parts, two partial rows of 16 floats for every 16 rows, each to 256 bytes
    assert need(rows=513) == 4 * 2304 + 2304 + 2 * 33 * 16 * 4 + 128
    assert need(rows=100000) > 4 * 4 * 100000
    e = embedding(rows=600)
    assert gradient(e, size=need(rows=600) - 1) == ps.PS_ENOMEM
    assert gradient(e, ws=None) == ps.PS_EINVAL and gradient(e, ws=SOMEWHERE + 8) == ps.PS_EINVAL
    assert lib().ps_embedding_workspace_bytes(ctypes.byref(e), None) == ps.PS_EINVAL
    assert lib().ps_embedding_workspace_bytes(None, None) == ps.PS_EINVAL


def test_no_rows_need_nothing():
    e, none = embedding(rows=0), dense.ps_matrix(None, 16, 0)
    assert look(e, tokens.ps_tokens(None, 1, 4), out=none) == ps.PS_OK
    assert score(logprob(rows=0), tokens.ps_tokens(None, 1, 4), none, None, None) == ps.PS_OK
    assert score_gradient(logprob(rows=0), tokens.ps_tokens(None, 1, 4), none, none, None) == ps.PS_OK


def logprob(**kw):
    d = dict(dtype=dense.PS_BF16, top=0, rows=8, vocab=100, scale=1.0)
    d.update(kw)
    return tokens.ps_logprob(**d)


def score(l, t=None, logits=None, logp=SOMEWHERE, norm=SOMEWHERE, top_logp=SOMEWHERE, top_tokens=SOMEWHERE, ws=SOMEWHERE, size=HUGE):
    t = t or tokens.ps_tokens(SOMEWHERE, 1, 4)
    logits = logits or dense.ps_matrix(SOMEWHERE, 100, 0)
    return lib().ps_logprob_forward(ctypes.byref(l), ctypes.byref(t), ctypes.byref(logits), logp, norm, top_logp, top_tokens, ws, size, None)


def score_gradient(l, t=None, logits=None, dlogits=None, norm=SOMEWHERE, dlogp=(SOMEWHERE, 1), dentropy=(SOMEWHERE, 0)):
    t = t or tokens.ps_tokens(SOMEWHERE, 1, 4)
    logits, dlogits = logits or dense.ps_matrix(SOMEWHERE, 100, 0), dlogits or dense.ps_matrix(SOMEWHERE, 100, 0)
    return lib().ps_logprob_backward(ctypes.byref(l), ctypes.byref(t), ctypes.byref(logits), norm, ctypes.byref(tokens.ps_vector(*dlogp)),
                                     ctypes.byref(tokens.ps_vector(*dentropy)), ctypes.byref(dlogits), None)


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=(1 << 28) + 1), dict(vocab=0), dict(vocab=(1 << 22) + 1), dict(top=-1), dict(top=33),
                                 dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(scale=3e38)])
def test_log_probabilities_that_are_refused(bad):
    assert score(logprob(**bad)) == ps.PS_EINVAL and "ps_logprob_forward" in message()
    assert score_gradient(logprob(**bad)) == ps.PS_EINVAL and "ps_logprob_backward" in message()


def test_results_of_log_probabilities_that_are_refused():
    assert score(logprob(), norm=None) == ps.PS_EINVAL
    assert score(logprob(top=1), top_logp=None) == ps.PS_EINVAL and score(logprob(top=1), top_tokens=None) == ps.PS_EINVAL
    for name in ("logp", "norm", "top_logp", "top_tokens"):
        assert score(logprob(top=1), **{name: SOMEWHERE + 2}) == ps.PS_EINVAL
    assert score_gradient(logprob(), norm=None) == ps.PS_EINVAL and score_gradient(logprob(), norm=SOMEWHERE + 1) == ps.PS_EINVAL
    for bad in ((SOMEWHERE + 2, 1), (SOMEWHERE, -1), (SOMEWHERE, (1 << 22) + 1)):
        assert score_gradient(logprob(), dlogp=bad) == ps.PS_EINVAL and score_gradient(logprob(), dentropy=bad) == ps.PS_EINVAL
    assert lib().ps_logprob_forward(None, None, None, None, None, None, None, None, 0, None) == ps.PS_EINVAL


def test_workspace_of_log_probabilities():
    def need(**kw):
        n = ctypes.c_uint64(0)
        assert lib().ps_logprob_workspace_bytes(ctypes.byref(logprob(**kw)), ctypes.byref(n)) == ps.PS_OK
        return n.value
    assert need() == 0 and need(rows=0, vocab=1 << 20) == 0 and need(rows=1 << 14, vocab=1 << 20) == 0
    # a row that one block takes, and a longer one: parts of 8192 logits, three sums and the alternatives of each
    assert need(rows=1, vocab=1 << 16, top=5) == 0
    assert need(rows=1, vocab=1 << 18) == 512 and need(rows=1, vocab=1 << 18, top=5) == 512 + 32 * 5 * 8
    long = logprob(rows=1, vocab=1 << 18, top=5)
    logits = dense.ps_matrix(SOMEWHERE, 1 << 18, 0)
    assert score(long, logits=logits, size=512 + 32 * 5 * 8 - 1) == ps.PS_ENOMEM
    assert score(long, logits=logits, ws=None) == ps.PS_EINVAL and score(long, logits=logits, ws=SOMEWHERE + 8) == ps.PS_EINVAL
    assert lib().ps_logprob_workspace_bytes(ctypes.byref(long), None) == ps.PS_EINVAL
    assert lib().ps_logprob_workspace_bytes(ctypes.byref(logprob(top=33)), None) == ps.PS_EINVAL


def test_tensors_that_are_refused():
    x, t = torch.zeros(4, 8), torch.zeros(4, dtype=torch.int64)
    for call in (lambda: tokens.ps_embedding_forward(t, x), lambda: tokens.ps_embedding_backward(x, t, 10), lambda: tokens.ps_logprob_forward(x, t),
                 lambda: tokens.ps_logprob_backward(x, t, torch.zeros(4, 3), torch.zeros(4))):
        with pytest.raises(ps.PsError, match="not on a GPU"):
            call()
