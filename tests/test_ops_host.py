"""Host-side checks of the operators around the layer (no GPU needed): symbols
and structure layout of include/unif_moe_ops.h, workspace sizes, and the
arguments that are rejected before any HIP call."""
import ctypes
import math
import os
import re
import subprocess

import pytest
import torch

from paper_2608_10392_amd import _lib, ops
from synth import get_config, layer_config

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
HEADER = os.path.join(ROOT, "include", "unif_moe_ops.h")


@pytest.fixture(scope="module")
def L():
    return ops.lib()


def test_declared_symbols_are_exported(L):
    names = set(re.findall(r"^int32_t\s+(unif_moe_\w+)\s*\(", open(HEADER).read(), re.M))
    assert names == set(ops.EXPORTS)
    out = subprocess.run(["nm", "-D", "--defined-only", _lib.LIB_PATH], capture_output=True, text=True).stdout
    for n in names:
        assert re.search(rf"\bT {n}$", out, re.M), n


def test_structures_match_the_header(tmp_path):
    structs = dict(unif_moe_residual=ops.Residual, unif_moe_residual_grads=ops.ResidualGrads,
                   unif_moe_balance=ops.Balance)
    lines = [f' printf("{c} %zu\\n", sizeof({c}));' for c in structs]
    lines += [f' printf("{c}.{f} %zu\\n", offsetof({c}, {f}));' for c, p in structs.items() for f, _ in p._fields_]
    src = tmp_path / "layout.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "unif_moe_ops.h"\nint main(void) {\n'
                   + "\n".join(lines) + "\n return 0; }\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-I", os.path.dirname(HEADER), str(src), "-o", str(exe)], check=True)
    got = dict(l.split() for l in subprocess.run([str(exe)], capture_output=True, text=True).stdout.splitlines())
    for c, p in structs.items():
        assert int(got[c]) == ctypes.sizeof(p)
        for f, _ in p._fields_:
            assert int(got[f"{c}.{f}"]) == getattr(p, f).offset, f


# Addresses that no call touches: 1 GiB apart.
A = {k: (i + 1) << 30 for i, k in enumerate(
    "x f valid y h dy dh dx df ws out_gamma out_beta in_gamma in_beta gate "
    "d_out_gamma d_out_beta d_in_gamma d_in_beta d_gate".split())}


def residual(**kw):
    f = dict(n_tokens=100, d_model=64, dtype=1, stream_dtype=1, out_norm=1, in_norm=2, tokens_per_gate=0,
             out_eps=1e-6, in_eps=1e-6, residual_scale=1.0, **{k: A[k] for k in ops.PARAMS})
    f.update(kw)
    return ops.Residual(**f)


def forward(L, r, **kw):
    a = {k: A[k] for k in ("x", "f", "valid", "y", "h")}
    a.update(kw)
    return L.unif_moe_residual_forward(ctypes.byref(r), a["x"], a["f"], a["valid"], a["y"], a["h"], None)


def backward(L, r, dh_dtype=0, nbytes=1 << 29, grads=None, **kw):
    a = dict(A)
    a.update(kw)
    g = ops.ResidualGrads(**(dict({k: A["d_" + k] for k in ops.PARAMS}, **(grads or {}))))
    return L.unif_moe_residual_backward(ctypes.byref(r), a["y"], a["f"], a["valid"], a["dy"], a["dh"], dh_dtype,
                                        a["dx"], a["df"], ctypes.byref(g), a["ws"], nbytes, None)


BAD_RESIDUALS = [
    dict(n_tokens=-1), dict(d_model=0), dict(dtype=2), dict(stream_dtype=5), dict(dtype=0, stream_dtype=1),
    dict(out_norm=3), dict(in_norm=-1), dict(tokens_per_gate=-1), dict(out_eps=0.0), dict(in_eps=1e-39), dict(in_eps=math.nan),
    dict(out_eps=math.inf), dict(residual_scale=math.nan), dict(residual_scale=math.inf), dict(out_gamma=None),
    dict(in_gamma=None), dict(out_norm=0), dict(in_norm=0), dict(gate=A["gate"] + 2),
]


@pytest.mark.parametrize("bad", BAD_RESIDUALS)
def test_bad_descriptions_are_rejected(L, bad):
    n = ctypes.c_size_t(0)
    r = residual(**bad)
    assert L.unif_moe_residual_backward_workspace_size(ctypes.byref(r), ctypes.byref(n)) == _lib.EINVAL
    assert forward(L, r) == _lib.EINVAL
    assert backward(L, r) == _lib.EINVAL


def test_rows_out_of_range_are_unsupported(L):
    assert forward(L, residual(d_model=ops.RESIDUAL_MIN_D - 1)) == _lib.EUNSUPPORTED
    assert backward(L, residual(d_model=ops.RESIDUAL_MIN_D - 1)) == _lib.EUNSUPPORTED
    assert forward(L, residual(d_model=ops.RESIDUAL_MAX_D + 1)) == _lib.EUNSUPPORTED
    assert backward(L, residual(d_model=ops.RESIDUAL_MAX_D + 1)) == _lib.EUNSUPPORTED
    assert ops.residual_backward_workspace_size(residual(d_model=ops.RESIDUAL_MAX_D)) > 0


NONE_OUT = dict(out_norm=0, out_gamma=None, out_beta=None)
NONE_IN = dict(in_norm=0, in_gamma=None, in_beta=None)


def test_forward_rejects_bad_calls(L):
    row = 100 * 64 * 2
    for kw in (dict(x=None, f=None), dict(y=None, h=None), dict(f=None), dict(x=A["x"] + 1), dict(f=A["f"] + 1),
               dict(y=A["y"] + 1), dict(h=A["h"] + 1),
               dict(y=A["f"]), dict(h=A["x"]), dict(h=A["y"]), dict(y=A["x"] + 2), dict(y=A["x"] + row - 2),
               dict(h=A["gate"]), dict(y=A["valid"] & ~3), dict(h=A["in_gamma"] - row + 2)):
        assert forward(L, residual(), **kw) == _lib.EINVAL, kw
    assert forward(L, residual(**NONE_IN)) == _lib.EINVAL                      # h without N_in
    assert forward(L, residual(**NONE_OUT), f=None) == _lib.EINVAL             # a gate on no branch
    assert L.unif_moe_residual_forward(None, 1, 1, None, 1, 1, None) == _lib.EINVAL


def test_backward_rejects_bad_calls(L):
    for kw in (dict(dy=None, dh=None), dict(y=None), dict(f=None), dict(dh=None), dict(dx=A["y"]), dict(df=A["f"]),
               dict(df=A["dx"]), dict(dx=A["dy"] + 2), dict(df=A["dy"]), dict(dx=A["d_gate"]), dict(ws=A["dh"]),
               dict(dh=A["dh"] + 2), dict(dx=A["dx"] + 1), dict(grads=dict(gate=A["d_out_beta"])),
               dict(grads=dict(in_beta=A["d_in_beta"] + 1)), dict(dh_dtype=3)):
        assert backward(L, residual(), **kw) == _lib.EINVAL, kw
    # gradients of parameters that are not there
    assert backward(L, residual(gate=None)) == _lib.EINVAL
    assert backward(L, residual(in_beta=None)) == _lib.EINVAL
    # gradients of N_in without dh
    assert backward(L, residual(), y=None, dh=None) == _lib.EINVAL
    # fp32 layers have fp32 gradients
    f32 = residual(dtype=0, stream_dtype=0)
    assert backward(L, f32, dh_dtype=1) == _lib.EINVAL
    size = ops.residual_backward_workspace_size(residual())
    assert backward(L, residual(), nbytes=size - 1) == _lib.EWORKSPACE
    assert backward(L, residual(), ws=None) == _lib.EWORKSPACE


def test_no_tokens_need_no_launch(L):
    r = residual(n_tokens=0)
    assert forward(L, r) == 0
    assert backward(L, r, grads={k: None for k in ops.PARAMS}) == 0


CFG = layer_config(get_config("vit_s16", n_tokens=100, d_model=64, n_experts=4, n_blocks=8, max_shared=8))
B = {k: (i + 1) << 30 for i, k in enumerate(
    "alpha n_shared shared_mask n_res expert_ids weights valid X W loss counts dX_in dX dW_in dW ws".split())}
RECORD = ("alpha", "n_shared", "shared_mask", "n_res", "expert_ids", "weights")


def balance(L, cfg=CFG, bal=None, nbytes=1 << 29, **kw):
    a = dict(B)
    a.update(kw)
    c = _lib.make_config(cfg)
    b = bal or ops.Balance(tokens_per_group=0, unit=0, weight=1.0)
    rec = _lib.Routing(**{k: a[k] for k in RECORD})
    return L.unif_moe_balance_loss(ctypes.byref(c), ctypes.byref(b), ctypes.byref(rec), a["valid"], a["X"], a["W"],
                                   a["loss"], a["counts"], a["dX_in"], a["dX"], a["dW_in"], a["dW"], a["ws"], nbytes,
                                   None)


def test_balance_rejects_bad_calls(L):
    n = ctypes.c_size_t(0)
    for bad in (dict(tokens_per_group=-1, unit=0, weight=1.0), dict(tokens_per_group=0, unit=2, weight=1.0),
                dict(tokens_per_group=0, unit=0, weight=math.nan), dict(tokens_per_group=0, unit=1, weight=math.inf)):
        b, c = ops.Balance(**bad), _lib.make_config(CFG)
        assert balance(L, bal=b) == _lib.EINVAL
        assert L.unif_moe_balance_loss_workspace_size(ctypes.byref(c), ctypes.byref(b), ctypes.byref(n)) == _lib.EINVAL
    for kw in (dict(loss=None), dict(X=None), dict(W=None), dict(weights=None), dict(n_shared=None),
               dict(dX=None), dict(dW=None), dict(loss=B["loss"] + 2), dict(counts=B["counts"] + 4),
               dict(dX=B["dX_in"] + 4), dict(dX=B["X"]), dict(dW=B["W"]), dict(dW=B["dX"]), dict(loss=B["counts"]),
               dict(ws=B["weights"]), dict(dX=B["dW_in"]), dict(X=B["X"] + 1), dict(dW_in=B["dW_in"] + 1)):
        assert balance(L, **kw) == _lib.EINVAL, kw
    assert balance(L, cfg=dict(CFG, n_experts=0)) == _lib.EINVAL
    assert balance(L, cfg=dict(CFG, n_experts=65)) == _lib.EUNSUPPORTED
    narrow = dict(CFG, dtype="f32", d_model=ops.BALANCE_MIN_D - 1)
    assert balance(L, cfg=narrow) == balance(L, cfg=narrow, dX=None, dX_in=None) == _lib.EUNSUPPORTED
    size = ops.balance_loss_workspace_size(CFG, {})
    assert balance(L, nbytes=size - 1) == _lib.EWORKSPACE
    assert balance(L, ws=None) == _lib.EWORKSPACE


def test_binding_checks_tensors():
    """What only the binding sees: device, type, size and layout."""
    desc = dict(n_tokens=4, d_model=8, dtype="f32", in_norm="rms")
    with pytest.raises(_lib.UnifMoeError) as e:
        ops.make_residual(dict(desc, in_gamma=torch.ones(8)))
    assert e.value.status == _lib.EINVAL and "not on a GPU" in str(e.value)
    r = residual(n_tokens=4, d_model=8)
    r.device = None
    with pytest.raises(_lib.UnifMoeError, match="x is not on a GPU"):
        ops.residual_forward(r, torch.zeros(4, 8), None, None, None, None)
    with pytest.raises(KeyError):
        ops.make_residual(dict(desc, in_norm="batch"))
    for make, bad in ((ops.make_residual, dict(desc, gamma=None)), (ops.make_balance, dict(lam=0.1))):
        with pytest.raises(_lib.UnifMoeError, match="unknown keys"):
            make(bad)
