"""What DeviceLayer takes as its inputs (no GPU needed): every layout of the
right type and size gives the same values, anything else is refused before the
library is called."""
import numpy as np
import pytest
import torch

from paper_2608_10392_amd import _lib
from paper_2608_10392_amd.layer import DeviceLayer, to_device

N, D, K, B, M = 6, 32, 2, 2, 16
CFG = dict(n_tokens=N, d_model=D, n_experts=K, n_blocks=B, block_width=M, mass_threshold=0.7)
rng = np.random.default_rng(0)


def words(*shape):
    return rng.integers(0, 1 << 15, shape, dtype=np.uint16)


def bits(t):
    return t.view(torch.int16).numpy().view(np.uint16)


def transposed(t):
    """The same values, stored column by column."""
    return t.transpose(-1, -2).contiguous().transpose(-1, -2)


@pytest.mark.parametrize("layout", [lambda t: t, transposed, lambda t: torch.cat([t, t], -1)[..., :t.shape[-1]],
                                    lambda t: torch.stack([t, t])[1]])
def test_tensors_of_any_layout(layout):
    x = rng.standard_normal((4, 3)).astype(np.float32)
    got = to_device(layout(torch.from_numpy(x)), "f32", "cpu")
    assert got.is_contiguous() and np.array_equal(got.numpy(), x)
    w = words(4, 6)
    for t in (torch.from_numpy(w.view(np.int16)), torch.from_numpy(w), torch.from_numpy(w.view(np.int16)).view(torch.bfloat16)):
        got = to_device(layout(t.view(torch.int16)).view(t.dtype), "bf16", "cpu")
        assert got.dtype == torch.bfloat16 and got.is_contiguous() and np.array_equal(bits(got), w)


def test_arrays_of_any_layout():
    x, w = rng.standard_normal((3, 4)).astype(np.float32), words(3, 4)
    assert np.array_equal(to_device(x.T, "f32", "cpu").numpy(), x.T) and to_device(x.T, "f32", "cpu").is_contiguous()
    assert np.array_equal(bits(to_device(w.T, "bf16", "cpu")), w.T)
    assert np.array_equal(bits(to_device(w.view(np.int16)[::2], "bf16", "cpu")), w[::2])
    for kind in (np.uint8, "V2"):
        assert np.array_equal(bits(to_device(w.view(kind), "bf16", "cpu")), w)
    assert to_device(None, "f32", "cpu") is None


@pytest.mark.parametrize("dtype, a", [
    ("f32", torch.zeros(4, 3, dtype=torch.bfloat16)), ("f32", torch.zeros(4, 3, dtype=torch.float64)),
    ("f32", np.zeros((4, 3))), ("f32", np.zeros((4, 3), np.uint16)), ("bf16", torch.zeros(4, 3)),
    ("bf16", torch.zeros(4, 3, dtype=torch.float16)), ("bf16", np.zeros((4, 3), np.float32)),
    ("bf16", np.zeros((4, 3), np.float16)),
])
def test_other_types_are_refused(dtype, a):
    with pytest.raises(_lib.UnifMoeError, match="array is torch") as e:
        to_device(a, dtype, "cpu")
    assert e.value.status == _lib.EINVAL


def layer(dtype="bf16", **kw):
    make = words if dtype == "bf16" else lambda *s: rng.standard_normal(s).astype(np.float32)
    a = dict(X=make(N, D), valid=None, W_router=np.zeros((K + 1, D), np.float32), prototypes=np.zeros((B, D), np.float32),
             W_up=make(K + 1, B * M, D), W_down=make(K + 1, D, B * M))
    a.update(kw)
    return DeviceLayer(dict(CFG, dtype=dtype), **a, device="cpu"), a


def test_layer_takes_arrays_and_tensors():
    for dtype in ("bf16", "f32"):
        _, a = layer(dtype)
        t = {k: transposed(torch.from_numpy(a[k])) for k in ("X", "W_up", "W_down")}
        got, _ = layer(dtype, **t)
        for k in t:
            v = getattr(got, k)
            assert v.is_contiguous() and np.array_equal(bits(v) if dtype == "bf16" else v.numpy(), a[k])
    # rows past the layer's are not read, and another shape of as many elements is the same data
    got, _ = layer(X=words(N + 3, D), W_up=words((K + 1) * B * M, D))
    assert got.X.shape[0] == N + 3


@pytest.mark.parametrize("bad", [
    dict(X=words(N - 1, D)), dict(X=words(N, D - 1)), dict(X=words(2 * N, 2 * D)), dict(X=torch.zeros(N, D)),
    dict(W_up=words(K, B * M, D)), dict(W_up=words(K + 1, B * M, 2 * D)), dict(W_down=words(K + 1, D, B * M - 1)),
    dict(W_down=np.zeros((K + 1, D, B * M), np.float32)), dict(X=words(N * D - 1)), dict(X=words(N * D + 1)),
])
def test_layer_refuses(bad):
    with pytest.raises(_lib.UnifMoeError, match=f"{list(bad)[0]} is"):
        layer(**bad)


def test_gradient_and_block_input_are_checked(monkeypatch):
    """dY and a block's X: refused before the library is called."""
    dev, _ = layer("f32")
    for fn in ("layer_backward", "block_forward", "layer_backward_workspace_size", "block_forward_workspace_size"):
        monkeypatch.setattr(_lib, fn, lambda *a, **k: pytest.fail("called"))
    blk = dict(norm="none", residual=True, ln_eps=1e-6)
    for bad in (torch.zeros(N, D, dtype=torch.bfloat16), torch.zeros(N - 1, D), np.zeros((N, D)), torch.zeros(N, D + 1)):
        with pytest.raises(_lib.UnifMoeError, match="dY is"):
            dev.backward(bad)
        with pytest.raises(_lib.UnifMoeError, match="X is"):
            dev.block_forward(blk, X=bad)
    # a transposed gradient reaches the library in the layer's order
    dY, seen = torch.randn(N, D), {}
    monkeypatch.setattr(_lib, "layer_backward_workspace_size", lambda c: 1)
    monkeypatch.setattr(_lib, "layer_backward", lambda *a, **k: seen.update(dY=a[7]))
    dev.backward(transposed(dY))
    assert seen["dY"].is_contiguous() and torch.equal(seen["dY"], dY)
