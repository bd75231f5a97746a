"""Dense layers and AdamW without a GPU: declared symbols, and the calls that are refused before anything is launched."""
import ctypes
import os
import re

import pytest

from paper_2406_05546_amd import binding as ps
from paper_2406_05546_amd import dense

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SOMEWHERE = 1 << 20  # an aligned address that no refused call looks at


def test_library_exports_every_declared_symbol():
    header = open(os.path.join(ROOT, "include", "ps_dense.h")).read()
    declared = re.findall(r"^PS_API\s+[\w\s\*]+?\b(\w+)\(", header, flags=re.M)
    assert sorted(declared) == sorted(dense.EXPORTS)
    for name in declared:
        assert getattr(ps.load_library(), name) is not None


def layer(**kw):
    d = dict(dtype=dense.PS_BF16, activation=0, rows=8, in_features=16, out_features=24, n_groups=1, n_weights=1, offsets_dev=None, weight_of_group_dev=None)
    d.update(kw)
    return dense.ps_linear(**d)


def need(l, backward=0):
    n = ctypes.c_uint64(0)
    return dense._library().ps_linear_workspace_bytes(ctypes.byref(l), backward, ctypes.byref(n)), n.value


def test_workspace_of_a_layer():
    assert need(layer()) == (ps.PS_OK, 0)
    # nothing to keep but the bias's partial sums without an activation, the rounded dz [8][24] with one
    plain, kept = need(layer(), 1)[1], need(layer(activation=1), 1)[1]
    assert plain > 0 and kept - plain == 512
    # a gradient of few tiles over many rows is cut up along the rows, in fp32
    assert need(layer(rows=1 << 16, in_features=64, out_features=64), 1)[1] >= 2 * 64 * 64 * 4
    assert dense._library().ps_dense_last_error() is not None


@pytest.mark.parametrize("bad", [dict(dtype=3), dict(dtype=-1), dict(activation=4), dict(activation=-1), dict(rows=-1), dict(rows=(1 << 28) + 1), dict(in_features=0),
                                 dict(out_features=0), dict(in_features=(1 << 22) + 1), dict(out_features=(1 << 22) + 1), dict(n_groups=0), dict(n_groups=2, n_weights=2),
                                 dict(n_groups=32769, n_weights=32769, offsets_dev=SOMEWHERE), dict(n_weights=0), dict(n_groups=3, n_weights=2, offsets_dev=SOMEWHERE),
                                 dict(offsets_dev=SOMEWHERE + 2), dict(offsets_dev=SOMEWHERE, weight_of_group_dev=SOMEWHERE + 1),
                                 dict(n_groups=32768, n_weights=1, offsets_dev=SOMEWHERE, weight_of_group_dev=SOMEWHERE, in_features=1 << 20, out_features=1 << 20)])
def test_layers_that_are_refused(bad):
    l = layer(**bad)
    assert need(l)[0] == ps.PS_EINVAL and b"ps_linear_workspace_bytes" in dense._library().ps_dense_last_error()
    m = dense.ps_matrix(SOMEWHERE, 24, 24 * 24)
    r = ctypes.byref(m)
    assert dense._library().ps_linear_forward(ctypes.byref(l), r, r, r, r, r, r, SOMEWHERE, 1 << 40, None) == ps.PS_EINVAL
    assert dense._library().ps_linear_backward(ctypes.byref(l), r, r, r, r, r, r, r, SOMEWHERE, 1 << 40, None) == ps.PS_EINVAL


NAMES_F, NAMES_B = ["x", "w", "bias", "residual", "y", "pre"], ["dy", "x", "w", "pre", "dx", "dw", "db"]


def matrices(names, l):
    fin, fout = l.in_features, l.out_features
    row = {"x": fin, "w": fin, "bias": fout, "residual": fout, "y": fout, "pre": fout, "dy": fout, "dx": fin, "dw": fin, "db": fout}
    return {n: dense.ps_matrix(SOMEWHERE, row[n], row[n] * (fout if n in ("w", "dw") else 1)) for n in names}


def forward(l, m, ws=SOMEWHERE, bytes_=1 << 40):
    return dense._library().ps_linear_forward(ctypes.byref(l), *[None if m[n] is None else ctypes.byref(m[n]) for n in NAMES_F], ws, bytes_, None)


def backward(l, m, ws=SOMEWHERE, bytes_=1 << 40):
    return dense._library().ps_linear_backward(ctypes.byref(l), *[None if m[n] is None else ctypes.byref(m[n]) for n in NAMES_B], ws, bytes_, None)


@pytest.mark.parametrize("name", NAMES_F)
def test_forward_operands_that_are_refused(name):
    l = layer()
    kinds = {"misaligned": dict(data_dev=SOMEWHERE + 1)}
    if name in ("x", "w", "y"):
        kinds["missing"] = dict(data_dev=None)
    if name != "bias":
        kinds["overlapping rows"] = dict(row=15)
        kinds["rows too far apart"] = dict(row=(1 << 22) + 8)
    for kind, change in kinds.items():
        m = matrices(NAMES_F, l)
        for k, v in change.items():
            setattr(m[name], k, v)
        assert forward(l, m) == ps.PS_EINVAL, kind
        assert name.encode() in dense._library().ps_dense_last_error()
        if kind == "missing":
            m[name] = None
            assert forward(l, m) == ps.PS_EINVAL


@pytest.mark.parametrize("name", NAMES_B)
def test_backward_operands_that_are_refused(name):
    l = layer(activation=2)
    kinds = {"misaligned": dict(data_dev=SOMEWHERE + 1)}
    if name in ("dy", "x", "w", "pre"):
        kinds["missing"] = dict(data_dev=None)
    if name != "db":
        kinds["overlapping rows"] = dict(row=15)
    for kind, change in kinds.items():
        m = matrices(NAMES_B, l)
        for k, v in change.items():
            setattr(m[name], k, v)
        assert backward(l, m) == ps.PS_EINVAL, kind
        assert name.encode() in dense._library().ps_dense_last_error()


def test_matrices_of_groups_that_overlap_are_refused():
    l = layer(n_groups=2, n_weights=2, offsets_dev=SOMEWHERE)
    m = matrices(NAMES_F, l)
    m["w"].matrix = 16 * 24 - 1
    assert forward(l, m) == ps.PS_EINVAL
    m = matrices(NAMES_B, l)
    m["dw"].matrix = 16 * 24 - 1
    assert backward(l, m) == ps.PS_EINVAL
    m = matrices(NAMES_B, l)
    m["db"].matrix = 23
    assert backward(l, m) == ps.PS_EINVAL


def test_workspaces_that_are_refused():
    l = layer(rows=4096, in_features=64, out_features=64, activation=1)
    m = matrices(NAMES_B, l)
    n = need(l, 1)[1]
    assert backward(l, m, SOMEWHERE, n - 1) == ps.PS_ENOMEM and backward(l, m, None, n) == ps.PS_EINVAL and backward(l, m, SOMEWHERE + 4, n) == ps.PS_EINVAL


def test_nothing_to_do_launches_nothing():
    l = layer(rows=0)
    m = matrices(NAMES_F, l)
    m["x"].data_dev = m["y"].data_dev = None  # tensors without elements have no address
    assert forward(l, m, None, 0) == ps.PS_OK
    m = matrices(NAMES_B, layer())
    m["dx"] = m["dw"] = m["db"] = None
    assert backward(layer(), m, None, 0) == ps.PS_OK


def adam(**kw):
    d = dict(param_dev=SOMEWHERE, grad_dev=SOMEWHERE, copy_dev=None, m_dev=SOMEWHERE, v_dev=SOMEWHERE, m_scale_dev=SOMEWHERE, v_scale_dev=SOMEWHERE, numel=100,
             grad_row=100, grad_rows=1, param_dtype=0, grad_dtype=0, copy_dtype=0, state_bits=8, weight_decay=0.0)
    d.update(kw)
    return (dense.ps_adamw_tensor * 1)(dense.ps_adamw_tensor(**d))


@pytest.mark.parametrize("bad", [dict(numel=-1), dict(param_dtype=3), dict(grad_dtype=-1), dict(copy_dev=SOMEWHERE, copy_dtype=7), dict(state_bits=16), dict(grad_rows=0),
                                 dict(grad_rows=2, grad_row=99), dict(weight_decay=-1.0), dict(weight_decay=float("nan")), dict(param_dev=None), dict(grad_dev=None),
                                 dict(m_dev=None), dict(v_dev=None), dict(m_scale_dev=None), dict(v_scale_dev=None), dict(param_dev=SOMEWHERE + 2),
                                 dict(grad_dev=SOMEWHERE + 1, grad_dtype=1), dict(state_bits=32, m_dev=SOMEWHERE + 1), dict(v_scale_dev=SOMEWHERE + 1),
                                 dict(copy_dev=SOMEWHERE + 1, copy_dtype=1), dict(numel=1 << 43)])
def test_tensors_of_a_step_that_are_refused(bad):
    n, h = ctypes.c_uint64(0), ctypes.c_void_p()
    lib = dense._library()
    assert lib.ps_adamw_workspace_bytes(adam(**bad), 1, ctypes.byref(n)) == ps.PS_EINVAL
    assert lib.ps_adamw_create(ctypes.byref(h), adam(**bad), 1, SOMEWHERE, 1 << 40, None) == ps.PS_EINVAL and not h.value
    assert lib.ps_dense_last_error() != b""


def test_tables_and_steps_that_are_refused():
    n, h = ctypes.c_uint64(0), ctypes.c_void_p()
    lib = dense._library()
    assert lib.ps_adamw_workspace_bytes(adam(), 1, ctypes.byref(n)) == ps.PS_OK and n.value >= 96
    assert lib.ps_adamw_workspace_bytes(None, 1, ctypes.byref(n)) == ps.PS_EINVAL and lib.ps_adamw_workspace_bytes(adam(), -1, ctypes.byref(n)) == ps.PS_EINVAL
    assert lib.ps_adamw_create(ctypes.byref(h), adam(), 1, None, 1 << 20, None) == ps.PS_EINVAL
    assert lib.ps_adamw_create(ctypes.byref(h), adam(), 1, SOMEWHERE + 8, 1 << 20, None) == ps.PS_EINVAL
    assert lib.ps_adamw_create(ctypes.byref(h), adam(), 1, SOMEWHERE, 16, None) == ps.PS_ENOMEM
    assert lib.ps_adamw_create(None, adam(), 1, SOMEWHERE, 1 << 20, None) == ps.PS_EINVAL and lib.ps_adamw_destroy(None) == ps.PS_EINVAL
    # an empty table needs no GPU, and its steps launch nothing
    assert lib.ps_adamw_create(ctypes.byref(h), None, 0, None, 0, None) == ps.PS_OK and h.value
    good = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, grad_scale=1.0, step=1, n_rows=1)
    assert lib.ps_adamw_step(h, ctypes.byref(dense.ps_adamw_options(**good)), None) == ps.PS_OK
    for bad in (dict(lr=-1.0), dict(lr=float("nan")), dict(lr=float("inf")), dict(beta1=1.0), dict(beta1=-0.1), dict(beta2=1.0), dict(beta2=float("nan")), dict(eps=0.0),
                dict(eps=1e-60), dict(grad_scale=float("inf")), dict(step=0), dict(n_rows=0)):
        assert lib.ps_adamw_step(h, ctypes.byref(dense.ps_adamw_options(**{**good, **bad})), None) == ps.PS_EINVAL, bad
    assert lib.ps_adamw_step(None, ctypes.byref(dense.ps_adamw_options(**good)), None) == ps.PS_EINVAL and lib.ps_adamw_step(h, None, None) == ps.PS_EINVAL
    assert lib.ps_adamw_destroy(h) == ps.PS_OK


def test_binding_refuses_tensors_that_are_not_on_a_gpu_or_do_not_fit():
    import torch
    x, w = torch.zeros(4, 8), torch.zeros(6, 8)
    for call in (lambda: dense.ps_linear_forward(x, w), lambda: dense.ps_linear_forward(x, torch.zeros(6, 7)), lambda: dense.ps_linear_forward(x.double(), w.double()),
                 lambda: dense.ps_linear_forward(x, w, activation="tanh"), lambda: dense.ps_linear_forward(x[0], w), lambda: dense.ps_linear_backward(x, x, w),
                 lambda: dense.ps_grouped_linear_forward(x, torch.zeros(1, dtype=torch.int32), w[None]), lambda: dense.ps_grouped_linear_forward(x, torch.zeros(3), w[None]),
                 lambda: dense.ps_grouped_linear_forward(x, torch.zeros(3, dtype=torch.int32), w), lambda: dense.ps_adamw_create([x], [x]), lambda: dense.ps_adamw_create([], []),
                 lambda: dense.ps_adamw_create([x], [x], state_bits=4)):
        with pytest.raises(ps.PsError) as e:
            call()
        assert e.value.status == ps.PS_EINVAL and str(e.value)
