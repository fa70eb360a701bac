"""Padded tokens beside router weights that are not finite (MI355X only): their
rows of dX are the incoming ones, or zero, whatever the router holds."""
import pytest
import torch

from tests.test_gpu_balance import Case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype, n, d, K", [("f32", 450, 100, 5), ("bf16", 450, 96, 17), ("bf16", 30001, 768, 16),
                                            ("bf16", 30001, 1024, 64), ("f32", 30001, 200, 33)])
@pytest.mark.parametrize("padding", ["some", "all"])
def test_router_weights_that_are_not_finite(dtype, n, d, K, padding):
    print(f"\n[gpu] balance {n} x {d} {dtype} K={K}, NaN in the router, {padding} tokens padded", flush=True)
    c = Case(n, d, K, dtype=dtype, per=300, padded=(lambda t: t % 3 == 1) if padding == "some" else (lambda t: t >= 0))
    rows = c.valid == 0
    c.X[rows] = float("nan")
    finite = c.run()
    c.W[1] = float("nan")
    c.W[K, ::2] = float("inf")
    got = c.run()
    # the router's rows reach dX alone
    for k in ("loss", "counts", "dW"):
        assert torch.equal(got[k], finite[k])
    assert torch.equal(got["dX"][rows], c.dX_in[rows])
    assert bool(torch.isnan(got["dX"][~rows]).all())
    # dX alone, in place, and written
    alone = c.run(dW_in=None, dW=None, X=None)
    assert torch.equal(alone["dX"][rows], c.dX_in[rows])
    o = dict(c.outputs(), dX=c.dX_in.clone())
    c.run(o, dX_in=o["dX"])
    assert torch.equal(o["dX"][rows], c.dX_in[rows])
    assert bool((c.run(dX_in=None)["dX"][rows] == 0).all())
    assert bool((c.run(dX_in=None, dW_in=None, dW=None, X=None)["dX"][rows] == 0).all())
