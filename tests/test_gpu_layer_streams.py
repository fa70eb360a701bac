"""Layer and block calls on a given stream (MI355X only): the stream they run on,
by object or raw handle, 0 (the null stream) among them, and what they allocate
there, with the results of the same calls on the current stream."""
import pytest
import torch

from paper_2608_10392_amd import _lib
from paper_2608_10392_amd.layer import DeviceLayer
from synth import block_inputs, generate, get_config, layer_config, upstream_grad
from tests.test_gpu_block_step import DEV, agree, step, step_inputs

pytestmark = pytest.mark.gpu


def record_allocations(monkeypatch):
    seen, alloc = [], _lib.alloc_workspace
    monkeypatch.setattr(_lib, "alloc_workspace",
                        lambda *a: (seen.append(torch.cuda.current_stream().cuda_stream), alloc(*a))[1])
    return seen


def streams():
    side = torch.cuda.Stream()
    return dict(side=side, handle=side.cuda_stream, null=0, default=torch.cuda.default_stream()), side


@pytest.mark.parametrize("name", ["side", "handle", "null", "default"])
def test_block_step(name, monkeypatch):
    print(f"\n[gpu] block step on a given stream: {name}", flush=True)
    block, x, dy = step_inputs()
    want = step(block, x, dy)
    torch.cuda.synchronize()
    given, side = streams()
    other = torch.cuda.Stream()
    seen = record_allocations(monkeypatch)
    with torch.cuda.stream(other):   # neither the given one nor the null stream
        got = step(block, x, dy, given[name])
        assert torch.cuda.current_stream() == other
    torch.cuda.synchronize()
    assert seen and set(seen) == {side.cuda_stream if name in ("side", "handle") else 0}
    agree(got, want)


@pytest.mark.parametrize("name", ["side", "handle", "null", "default"])
def test_layer_calls(name, monkeypatch):
    print(f"\n[gpu] layer calls on a given stream: {name}", flush=True)
    g = generate(get_config("tiny_f32", n_tokens=320, d_model=128, n_experts=5, n_blocks=4, block_width=64, max_shared=4))
    (blk, Xb), dY = block_inputs(g, "pre"), upstream_grad(g)
    make = lambda: DeviceLayer(layer_config(g["cfg"]), g["X"], g["valid"], g["W_router"], g["prototypes"], g["W_up"],
                               g["W_down"], device=DEV)

    def calls(dev, s):
        out = dict(block=dev.block_forward(blk, Xb, s).clone())
        out["Y"] = dev.forward(s).clone()
        out.update(dev.backward(dY, s), routed=dev.route(stream=s)["weights"].clone())
        return out, dev.stats(s)

    want, stats = calls(make(), None)
    torch.cuda.synchronize()
    given, side = streams()
    seen = record_allocations(monkeypatch)
    dev = make()
    torch.cuda.synchronize()
    # with the given stream current too, since the clones between the calls run there
    stream = side if name in ("side", "handle") else torch.cuda.default_stream()
    with torch.cuda.stream(stream):
        got, n = calls(dev, given[name])
    torch.cuda.synchronize()
    assert len(seen) == 5 and set(seen) == {stream.cuda_stream}
    assert n == stats
    agree(got, want)
    # with another stream current
    dev, other = make(), torch.cuda.Stream()
    torch.cuda.synchronize()
    seen.clear()
    with torch.cuda.stream(other):
        grads = dev.backward(dY, given[name])
    torch.cuda.synchronize()
    assert seen == [stream.cuda_stream]
    agree(grads, {k: want[k] for k in grads})
