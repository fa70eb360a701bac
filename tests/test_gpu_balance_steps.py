"""The balance loss where a workgroup of the gradients takes several steps of 16
tokens and a group many pieces (MI355X only), against the 64-bit definition
with the bounds of test_gpu_balance.py: dW adds at most 16 tokens a step one
after the other, steps as asserted here, far below the N / 32 + 64 of its bound;
a wave's fp32 sums of affinities stay those of at most 64 tokens."""
import pytest
import torch

from tests.test_gpu_balance import U, Case, check

pytestmark = pytest.mark.gpu


def steps(n, d, K):
    """16-token steps per workgroup: the token ranges are as many as run at once
    (12 or 8 waves per compute unit, four strips of 64 columns per workgroup)."""
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    strips = -(-d // 64)
    slabs = -(-strips // 4)
    ranges = max(1, cus * ((12 if K <= 16 else 8) // -(-strips // slabs)) // slabs)
    return -(-(-(-n // 16)) // ranges)


def sizes(c):
    s = steps(c.n, c.d, c.K)
    assert s > 1, "one step per workgroup: nothing here for this device"
    return s


@pytest.mark.parametrize("K", [1, 16, 17, 33, 64])
@pytest.mark.parametrize("dtype, n, d", [("bf16", 50011, 768), ("f32", 40001, 1003)])
@pytest.mark.parametrize("unit, per, padded", [("tokens", 0, False), ("blocks", 0, True), ("blocks", 197, False),
                                               ("tokens", 197, True)])
def test_many_steps(dtype, n, d, K, unit, per, padded):
    c = Case(n, d, K, dtype=dtype, unit=unit, per=per, padded=(lambda t: t % 37 > 20) if padded else None)
    if padded:
        c.X[c.valid == 0] = float("nan")
    got = check(c, f"{n} x {d} {dtype} K={K} {unit} groups of {per}, padded {padded}, {sizes(c)} steps")
    if padded:
        assert torch.equal(got["dX"][c.valid == 0], c.dX_in[c.valid == 0])
    # each gradient alone, both in place, and written rather than added
    assert torch.equal(c.run(dW_in=None, dW=None, X=None)["dX"], got["dX"])
    assert torch.equal(c.run(dX_in=None, dX=None, W=None)["dW"], got["dW"])
    o = dict(c.outputs(), dX=c.dX_in.clone(), dW=c.dW_in.clone())
    c.run(o, dX_in=o["dX"], dW_in=o["dW"])
    assert all(torch.equal(o[k], got[k]) for k in o)
    c.dX_in = c.dW_in = None
    check(c, "the same, written")


@pytest.mark.parametrize("K", [1, 8, 33, 64])
@pytest.mark.parametrize("unit", ["tokens", "blocks"])
@pytest.mark.parametrize("n, per", [(50011, 0), (50011, 20000), (9000, 1025)])
def test_many_pieces(n, per, unit, K):
    """Groups of more than 1,024 tokens, in up to 98 pieces of 512: with 33 and
    64 experts more than 16 pieces a stretch."""
    for padded in (None, lambda t: (t % 37 > 20) | (t // 700 % 5 == 0)):
        c = Case(n, 64, K, dtype="bf16", unit=unit, per=per, padded=padded)
        if padded:
            c.X[c.valid == 0] = float("nan")
        got = check(c, f"{n} x 64 K={K} {unit} groups of {per}, padded {padded is not None}")
        o = c.run(counts=got["counts"].clone().fill_(7), dX_in=None, dX=None, dW_in=None, dW=None, X=None, W=None)
        assert torch.equal(o["loss"], got["loss"])


def test_all_padded_groups_of_many_pieces():
    """Long groups without a valid token count as 0, the others as if alone."""
    c = Case(12000, 96, 9, dtype="bf16", per=3000, padded=lambda t: t // 3000 % 2 == 1)
    c.X[c.valid == 0] = float("nan")
    got = check(c, "12000 x 96, every other group of 3000 empty")
    assert bool((got["counts"][1::2] == 0).all())


def test_foreign_ids_are_not_counted():
    """A token whose ids are all outside 1..K takes exactly its own loads away,
    and its affinities reach neither the loss nor a gradient."""
    print("\n[gpu] balance: foreign ids, counted", flush=True)
    for per in (0, 30):
        c = Case(120, 64, 6, per=per, dtype="f32")
        want, ids, k = c.run(), c.rec["expert_ids"][7].clone(), int(c.rec["n_res"][7])
        c.rec["expert_ids"][7] = torch.tensor([0, -5, 7, 1 << 30, -(1 << 31), 99], dtype=torch.int32, device=ids.device)
        c.rec["n_res"][7], c.rec["weights"][7] = 6, 0.3
        got = c.run()
        loads = want["counts"].clone()
        loads[0].index_add_(0, ids[:k].long(), torch.full((k,), -1, dtype=torch.int64, device=ids.device))
        assert torch.equal(got["counts"], loads)
        assert torch.equal(got["dX"][7], c.dX_in[7])
        # the definition with that token's affinities and choices at zero; it stays a valid token of its group
        c.rec["expert_ids"][7], c.rec["n_res"][7], c.rec["weights"][7] = ids, 0, 0.0
        w = c.want()
        assert torch.equal(got["counts"], w["counts"])
        for name in ("loss", "dX", "dW"):
            assert bool(((got[name].double() - w[name][0]).abs() <= w[name][1] + 2 * U * (w[name][0].abs() + w[name][1])
                         + 2.0 ** -126).all()), name
