"""A training step of a block built from the operators: N_in, the layer, the
join, and back with the balance and the diversity loss (DeviceBlock, MI355X
only), against the same step in 64 bits: the oracle's layer between norms
written out here.

fp32 layers: the layer's gradients agree with the oracle within 1e-4 of their
largest value (the tolerance of its own backward), so the step's do: the norms
around it have gains near 1, and their errors are far below. bf16 layers: the
layer's own bound 1e-2, and N_in(x) and df are rounded to bf16 on the way, each
2^-9 of values that the sums average: 2e-2. Tokens near a routing decision on
either side are marked padded.
"""
import numpy as np
import pytest
import torch

import oracle.unif_moe_oracle as O
from paper_2608_10392_amd import _lib, ops
from paper_2608_10392_amd.layer import DeviceBlock, DeviceLayer
from synth import generate, get_config, layer_config
from tests import parity

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
EPS = 1e-6


def norm(u, gamma, beta):
    c = u - u.mean(1, keepdim=True)
    return c / torch.sqrt((c * c).mean(1, keepdim=True) + EPS) * gamma + beta


@pytest.mark.parametrize("dtype, stream", [("f32", "f32"), ("bf16", "bf16"), ("bf16", "f32")])
def test_training_step(dtype, stream):
    print(f"\n[gpu] block step {dtype}, stream {stream}", flush=True)
    over = dict(n_tokens=320, d_model=128, n_experts=5, n_blocks=4, block_width=64, max_shared=4)
    base = dict(f32="tiny_f32", bf16="vit_s16")[dtype]
    g = generate(get_config(base, **over))
    cfg, n, d, K = g["cfg"], 320, 128, 5
    rng = np.random.default_rng(3)
    f64 = lambda a: torch.from_numpy(np.ascontiguousarray(a)).double()
    t = torch.float32 if stream == "f32" else torch.bfloat16
    layer_t = torch.float32 if dtype == "f32" else torch.bfloat16
    x = f64(rng.standard_normal((n, d)) * 2 + 0.3).to(t)
    dy = f64(rng.standard_normal((n, d))).to(t)
    p = dict(in_gamma=1 + 0.2 * rng.standard_normal(d), in_beta=0.1 * rng.standard_normal(d),
             out_gamma=1 + 0.2 * rng.standard_normal(d), out_beta=0.1 * rng.standard_normal(d),
             gate=0.5 + 0.3 * rng.standard_normal((5, d)))
    p = {k: f64(v).float() for k, v in p.items()}
    bal, div = dict(tokens_per_group=64, weight=0.5), 0.25

    # 64-bit side: h as the layer sees it (rounded to its type)
    leaf = {k: v.double().requires_grad_() for k, v in p.items()}
    xr = x.double().requires_grad_()
    h64 = norm(xr, leaf["in_gamma"], leaf["in_beta"])
    h = h64.detach().to(layer_t)
    hb = h.numpy() if dtype == "f32" else h.view(torch.int16).numpy().view(np.uint16)
    rec = O.route(cfg, hb, None, g["W_router"], g["prototypes"])
    margin, _ = O.margins(cfg, rec)
    # h may round either way where the fp32 norm is a little off: a routing
    # margin well above that keeps the decisions
    valid = (margin >= 50 * parity.MARGIN).astype(np.uint8)
    valid[100:128] = 0
    rec = O.route(cfg, hb, valid, g["W_router"], g["prototypes"])
    real = torch.from_numpy(valid).bool()[:, None]
    Y, _ = O.forward(cfg, hb, valid, g["W_router"], g["prototypes"], g["W_up"], g["W_down"], rec=rec)
    f = torch.from_numpy(np.asarray(Y, np.float64)).requires_grad_()
    gate = leaf["gate"][torch.arange(n) // 64]
    y = 0.75 * xr + gate * norm(f, leaf["out_gamma"], leaf["out_beta"])
    (torch.where(real, y, 0.0) * dy.double()).sum().backward()
    df = f.grad.to(layer_t).double().numpy()
    lg = O.backward(cfg, hb, valid, g["W_router"], g["prototypes"], g["W_up"], g["W_down"], df)
    hin = torch.from_numpy(O._as_f32(hb, dtype).astype(np.float64)).requires_grad_()
    W = f64(g["W_router"]).requires_grad_()
    l = hin @ W[1:].T
    s = torch.softmax(l, dim=1) * real
    ids, k = torch.from_numpy(rec["expert_ids"].astype(np.int64)), torch.from_numpy(rec["n_res"].astype(np.int64))
    chosen = torch.zeros(n, K + 1, dtype=torch.float64).scatter_(
        1, ids.clamp(min=0), (torch.arange(K)[None] < k[:, None]).double())[:, 1:] * real
    loads = chosen.view(5, 64, K).sum(1)
    loss = K / 5 * (loads / loads.sum(1, keepdim=True) * s.view(5, 64, K).sum(1)
                    / real.view(5, 64, 1).sum(1)).sum()
    gram = W @ W.T - torch.eye(K + 1, dtype=torch.float64)
    (bal["weight"] * loss + div * gram.norm()).backward()
    dh = torch.from_numpy(lg["dX"]) + hin.grad
    h64.backward(torch.where(real, dh, 0.0))
    want = dict(dx=xr.grad * real, dW_up=lg["dW_up"], dW_down=lg["dW_down"], dW_router=lg["dW_router"] + W.grad.numpy(),
                **{k: v.grad for k, v in leaf.items()})

    # device side
    dev = DeviceLayer(layer_config(cfg), hb, valid, g["W_router"], g["prototypes"], g["W_up"], g["W_down"], device=DEV)
    block = DeviceBlock(dev, dict(in_norm="layer", out_norm="layer", in_eps=EPS, out_eps=EPS, residual_scale=0.75,
                                  tokens_per_gate=64, **{k: v.to(DEV) for k, v in p.items()}), stream)
    xd = x.to(DEV)
    yd = block.forward(xd)
    got = block.backward(xd, dy.to(DEV), bal, div)
    torch.cuda.synchronize()
    grec = dev.routing_numpy()
    assert np.array_equal(grec["n_res"][valid == 1], rec["n_res"][valid == 1])
    assert got["counts"][:, 1:].cpu().tolist() == loads.long().tolist()
    tol = 1e-4 if dtype == "f32" else 2e-2
    assert abs(float(got["balance"]) - float(loss.detach())) <= tol * float(loss.detach())
    assert abs(float(got["diversity"]) - float(gram.detach().norm())) <= 1e-5 * float(gram.detach().norm())
    want["y"], got["y"] = torch.where(real, y.detach(), 0.0), yd
    for key, w in want.items():
        w = torch.as_tensor(w)
        err = float((got[key].double().cpu() - w).abs().max()) / float(w.abs().max())
        print(f"[gpu] {key}: {err:.1e} x max", flush=True)
        assert err <= tol, f"{key}: {err:.2e} of the largest value"
    assert bool((got["dx"][torch.from_numpy(valid == 0).to(DEV)] == 0).all())


def step_inputs():
    """A small fp32 block, its input and an output gradient."""
    g = generate(get_config("tiny_f32", n_tokens=320, d_model=128, n_experts=5, n_blocks=4, block_width=64, max_shared=4))
    rng = np.random.default_rng(4)
    rand = lambda *s: torch.from_numpy(rng.standard_normal(s).astype(np.float32)).to(DEV)
    dev = DeviceLayer(layer_config(g["cfg"]), g["X"], None, g["W_router"], g["prototypes"], g["W_up"], g["W_down"],
                      device=DEV)
    block = DeviceBlock(dev, dict(in_norm="rms", out_norm="layer", in_eps=EPS, out_eps=EPS, in_gamma=1 + 0.1 * rand(128),
                                  out_gamma=1 + 0.1 * rand(128), out_beta=0.1 * rand(128)))
    return block, rand(320, 128), rand(320, 128)


def step(block, x, dy, stream=None):
    y = block.forward(x, stream=stream)
    return dict(block.backward(x, dy, dict(tokens_per_group=64, weight=0.5), 0.25, stream=stream), y=y)


def agree(got, want):
    # the layer's own sums may come in another order: a few fp32 steps of the largest value
    for key, w in want.items():
        err = float((got[key].double() - w.double()).abs().max())
        assert err <= 1e-5 * float(w.double().abs().max()), f"{key}: {err:.2e}"


@pytest.mark.parametrize("raw", [False, True])
def test_step_on_another_stream(raw, monkeypatch):
    """What a step allocates on another stream belongs to that stream."""
    print(f"\n[gpu] block step on another stream, raw handle {raw}", flush=True)
    block, x, dy = step_inputs()
    want = step(block, x, dy)
    torch.cuda.synchronize()
    side, seen = torch.cuda.Stream(), []
    alloc = _lib.alloc_workspace
    monkeypatch.setattr(_lib, "alloc_workspace",
                        lambda *a: (seen.append(torch.cuda.current_stream().cuda_stream), alloc(*a))[1])
    got = step(block, x, dy, side.cuda_stream if raw else side)
    side.synchronize()
    assert seen and set(seen) == {side.cuda_stream}
    assert torch.cuda.current_stream().cuda_stream != side.cuda_stream
    agree(got, want)


def test_step_captured():
    """A captured step's replays, with eager steps between them."""
    print("\n[gpu] block step captured", flush=True)
    block, x, dy = step_inputs()
    want = {k: v.clone() for k, v in step(block, x, dy).items()}
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = step(block, x, dy)
    for _ in range(3):
        for v in got.values():
            v.fill_(-1)
        graph.replay()
        torch.cuda.synchronize()
        agree(got, want)
        agree(step(block, x, dy), want)
        torch.cuda.synchronize()
