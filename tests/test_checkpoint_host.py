"""Activations in 8 bits without a GPU: workspaces, and the calls that are refused before anything is launched."""
import ctypes

import pytest
import torch

from paper_2406_05546_amd import binding as ps
from paper_2406_05546_amd import dense
from tests.test_dense_host import SOMEWHERE, layer, matrices

HUGE = 1 << 40


def lib():
    return dense._library()


def need(l, backward, x8):
    n = ctypes.c_uint64(0)
    return lib().ps_linear_checkpoint_workspace_bytes(ctypes.byref(l), backward, x8, ctypes.byref(n)), n.value


def plain(l, backward):
    n = ctypes.c_uint64(0)
    assert lib().ps_linear_workspace_bytes(ctypes.byref(l), backward, ctypes.byref(n)) == ps.PS_OK
    return n.value


def test_workspace():
    l = layer(activation=2)
    # z of few rows in its own type first; z of many does not leave the kernel
    assert need(l, 0, 0) == (ps.PS_OK, plain(l, 0) + 512)
    many = layer(activation=2, rows=8192, in_features=2048, out_features=8192)
    assert need(many, 0, 0)[1] == plain(many, 0)
    # x [8][16] in bf16, as it is read
    assert need(l, 1, 0)[1] == plain(l, 1) and need(l, 1, 1)[1] == plain(l, 1) + 256
    odd = layer(activation=2, rows=7335, in_features=949, out_features=4658)  # copied to whole pieces anyway
    assert need(odd, 1, 1)[1] == plain(odd, 1)
    assert lib().ps_linear_checkpoint_workspace_bytes(ctypes.byref(l), 0, 0, None) == ps.PS_EINVAL
    assert need(layer(rows=-1), 1, 1)[0] == ps.PS_EINVAL


def code(call, dtype=1, rows=4, cols=40, x=(SOMEWHERE, 40, 0), c=(SOMEWHERE, SOMEWHERE, 40, 2), act=0):
    x, c = None if x is None else ctypes.byref(dense.ps_matrix(*x)), None if c is None else ctypes.byref(dense.ps_checkpoint(*c))
    if call == "encode":
        return lib().ps_checkpoint_encode(dtype, rows, cols, x, c, None)
    return lib().ps_checkpoint_decode(dtype, rows, cols, c, act, x, None)


BAD_CODES = [None, (None, SOMEWHERE, 40, 2), (SOMEWHERE, None, 40, 2), (SOMEWHERE, SOMEWHERE, 39, 2), (SOMEWHERE, SOMEWHERE, 40, 1), (SOMEWHERE, SOMEWHERE, (1 << 22) + 1, 2),
             (SOMEWHERE, SOMEWHERE, 40, (1 << 22) + 1)]


@pytest.mark.parametrize("call", ["encode", "decode"])
def test_codes_that_are_refused(call):
    for bad in (dict(dtype=3), dict(dtype=-1), dict(rows=-1), dict(rows=(1 << 28) + 1), dict(cols=0), dict(cols=(1 << 22) + 1), dict(x=None), dict(x=(None, 40, 0)), dict(x=(SOMEWHERE + 1, 40, 0)),
                dict(x=(SOMEWHERE, 39, 0)), dict(x=(SOMEWHERE, (1 << 22) + 1, 0))):
        assert code(call, **bad) == ps.PS_EINVAL, bad
        assert f"ps_checkpoint_{call}" in lib().ps_dense_last_error().decode()
    for c in BAD_CODES:
        assert code(call, c=c) == ps.PS_EINVAL, c
    assert code(call, rows=0, x=None, c=(None, None, 0, 0)) == ps.PS_OK
    for act in (-1, 4):
        assert code("decode", act=act) == ps.PS_EINVAL


def test_layers_with_codes_that_are_refused():
    l = layer(activation=2)
    m = {n: ctypes.byref(v) for n, v in matrices(["x", "w", "bias", "residual", "y", "pre", "dy", "dx", "dw", "db"], l).items()}

    def forward(pre, ws=SOMEWHERE, size=HUGE):
        return lib().ps_linear_forward_checkpoint(ctypes.byref(l), m["x"], m["w"], m["bias"], m["residual"], m["y"], None if pre is None else ctypes.byref(dense.ps_checkpoint(*pre)), ws, size, None)

    def backward(x8=None, pre8=None, act=0, ws=SOMEWHERE, size=HUGE):
        x, pre = None if x8 else m["x"], None if pre8 else m["pre"]
        x8, pre8 = (None if c is None else ctypes.byref(dense.ps_checkpoint(*c)) for c in (x8, pre8))
        return lib().ps_linear_backward_checkpoint(ctypes.byref(l), m["dy"], x, x8, act, m["w"], pre, pre8, m["dx"], m["dw"], m["db"], ws, size, None)
    good_x, good_pre = (SOMEWHERE, SOMEWHERE, 16, 1), (SOMEWHERE, SOMEWHERE, 24, 1)
    assert forward(None) == ps.PS_EINVAL
    for bad in ((None, SOMEWHERE, 24, 1), (SOMEWHERE, None, 24, 1), (SOMEWHERE, SOMEWHERE, 23, 1), (SOMEWHERE, SOMEWHERE, 24, 0)):
        assert forward(bad) == ps.PS_EINVAL and backward(good_x, bad) == ps.PS_EINVAL
    for bad in ((None, SOMEWHERE, 16, 1), (SOMEWHERE, None, 16, 1), (SOMEWHERE, SOMEWHERE, 15, 1), (SOMEWHERE, SOMEWHERE, 16, 0)):
        assert backward(bad, good_pre) == ps.PS_EINVAL
    for act in (-1, 4):
        assert backward(good_x, good_pre, act) == ps.PS_EINVAL
    assert forward(good_pre, size=need(l, 0, 0)[1] - 1) == ps.PS_ENOMEM and forward(good_pre, ws=None) == ps.PS_EINVAL
    assert backward(good_x, good_pre, size=need(l, 1, 1)[1] - 1) == ps.PS_ENOMEM and backward(good_x, good_pre, ws=None) == ps.PS_EINVAL
    assert lib().ps_linear_forward_checkpoint(None, *6 * [None], None, 0, None) == ps.PS_EINVAL


def test_tensors_that_are_refused():
    x = torch.zeros(4, 8)
    c = dense.ps_checkpoint_empty(4, 8, "cpu")
    for call in (lambda: dense.ps_checkpoint_encode(x), lambda: dense.ps_checkpoint_decode(c), lambda: dense.ps_linear_forward(x, torch.zeros(8, 8), pre=c),
                 lambda: dense.ps_linear_backward(x, c, torch.zeros(8, 8))):
        with pytest.raises(ps.PsError, match="GPU"):
            call()
