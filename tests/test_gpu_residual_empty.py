"""Parameters that only padded tokens meet (MI355X only): a gate pooled from an
empty sequence is 0 / 0. Whatever they hold, padded rows are zero in every
output and reach no gradient. Bounds as in test_gpu_residual.py."""
import pytest
import torch

from paper_2608_10392_amd import ops
from tests.test_gpu_residual import DEV, TYPES, U, Case, check

pytestmark = pytest.mark.gpu

NAN, INF = float("nan"), float("inf")


def empty_sequences(c):
    """NaN and infinities in the gate rows of sequences without a real token;
    returns which those are and the gate with finite rows in their place."""
    groups = c.params["gate"].shape[0]
    real = torch.zeros(groups, device=DEV).index_add_(0, torch.arange(c.n, device=DEV) // c.per, c.valid.float())
    empty = real == 0
    clean = c.params["gate"].clone()
    c.params["gate"][empty] = NAN
    c.params["gate"][empty, ::3] = INF
    return empty, clean


@pytest.mark.parametrize("n, d, per, types", [
    (450, 96, 50, TYPES[0]), (450, 768, 50, TYPES[1]), (450, 1000, 50, TYPES[2]), (450, 1500, 50, TYPES[4]),
    (450, 64, 1, TYPES[0]), (5000, 768, 197, TYPES[0]), (20011, 64, 7, TYPES[3]), (20011, 768, 5, TYPES[0]),
    (5000, 2500, 30, TYPES[0]), (5000, 2500, 600, TYPES[2])])
@pytest.mark.parametrize("out", ["none", "layer", "rms"])
def test_gates_of_empty_sequences(n, d, per, types, out):
    print(f"\n[gpu] residual {n} x {d} {types} out {out}, every third of the sequences of {per} tokens empty", flush=True)
    c = Case(n, d, types, out=out, gate=True, per=per, padded=lambda t: ((t // per) % 3 == 1) | (t % 11 == 4))
    empty, clean = empty_sequences(c)
    assert bool(empty.any()) and not bool(empty.all())
    rows = c.valid == 0
    (y, h), got = c.forward(), c.backward()
    c.params["gate"] = clean
    (wy, ty), (wh, th) = c.forward64()
    check("y", y, wy, ty)
    check("h", h, wh, th)
    want = c.backward64()
    for k, v in got.items():
        check(k, v, *want[k])
    for v in (y, h, got["dx"], got["df"]):
        assert bool((v[rows] == 0).all())
    assert bool((got["gate"][empty] == 0).all())


@pytest.mark.parametrize("n, d", [(5, 48), (300, 768), (3000, 96), (300, 1024), (70, 3000)])
@pytest.mark.parametrize("per", [0, 40, 100000])
def test_no_real_token(n, d, per):
    """Every parameter NaN and no real token: every gradient is zero."""
    print(f"\n[gpu] residual {n} x {d}, a gate per {per} tokens, all padded", flush=True)
    c = Case(n, d, gate=True, per=per, padded=lambda t: t >= 0)
    for k, v in c.params.items():
        v.fill_(NAN if k != "out_beta" else INF)
    for v in (*c.forward(), *c.backward().values()):
        assert bool((v == 0).all())


@pytest.mark.parametrize("per", [0, 7])
def test_one_real_token(per):
    """A single real token: its row and the gradients are those of a call on it
    alone; a NaN column of a parameter stays out of the padded rows."""
    print(f"\n[gpu] residual, one real token, a gate per {per} tokens", flush=True)
    for n, d in ((900, 96), (900, 768), (500, 1500)):
        c = Case(n, d, gate=True, per=per, padded=lambda t: t != 41)
        if per:
            c.params["gate"][torch.arange(c.params["gate"].shape[0], device=DEV) != 41 // per] = NAN
        got = c.backward()
        one = Case(1, d, gate=True)
        for k in ("x", "f", "dy", "dh"):
            setattr(one, k, getattr(c, k)[41:42].contiguous())
        one.params = {k: (v[41 // per:41 // per + 1] if per and k == "gate" else v) for k, v in c.params.items()}
        one.res = ops.make_residual(dict(n_tokens=1, d_model=d, dtype="bf16", stream_dtype="bf16", out_norm="layer",
                                         in_norm="rms", out_eps=c.res.out_eps, in_eps=c.res.in_eps,
                                         residual_scale=c.scale, **one.params))
        want = one.backward()
        for k in ("dx", "df"):
            assert torch.equal(got[k][41:42], want[k]) and bool((got[k][c.valid == 0] == 0).all())
        for k in ("in_gamma", "in_beta", "out_gamma", "out_beta"):
            assert torch.equal(got[k], want[k])
        # gamma A + beta D, A and D the same in both: one rounding in fp64's sum for a single gate row, for one of
        # several u |beta D| for the product and u |sum| for the rest, so that they differ by at most u |beta D| +
        # 2 u |sum| to first order (D from d out_beta = gate D, whose roundings are of second order here)
        sums, row = want["gate"].view(-1).double(), one.params["gate"].view(-1).double()
        limit = U * ((c.params["out_beta"] * want["out_beta"] / row).abs() + 2 * sums.abs()) * (1 + 2.0 ** -20)
        assert bool(((got["gate"][41 // per if per else 0] - sums).abs() <= limit).all())
        c.params["in_gamma"][5] = c.params["out_gamma"][9] = NAN
        got = c.backward()
        assert bool((got["dx"][c.valid == 0] == 0).all()) and bool((got["df"][c.valid == 0] == 0).all())
        assert bool(torch.isnan(got["dx"][41]).all()) and bool(torch.isnan(got["df"][41]).all())
