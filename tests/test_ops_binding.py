"""The operators around the layer at their host side (no GPU needed):
descriptions whose integers do not fit the library's, and outputs over arrays
that a call is given but does not read."""
import ctypes

import pytest

from paper_2608_10392_amd import _lib, ops

DESC = dict(n_tokens=6, d_model=8, dtype="f32", in_norm="none")


@pytest.mark.parametrize("key", ["n_tokens", "d_model", "tokens_per_gate"])
@pytest.mark.parametrize("value", [1 << 31, (1 << 32) + 3, -(1 << 31) - 1, 1 << 70])
def test_integers_past_32_bits(key, value):
    """A gate row per 2^32 + 3 tokens is one row: cut to 32 bits it would be one
    per 3 tokens, and the second read past the gate's end."""
    with pytest.raises(_lib.UnifMoeError, match=f"{key} {value} is past 32 bits") as e:
        ops.make_residual(dict(DESC, **{key: value}))
    assert e.value.status == _lib.EINVAL
    if key == "tokens_per_gate":
        with pytest.raises(_lib.UnifMoeError, match="tokens_per_group .* is past 32 bits"):
            ops.make_balance(dict(tokens_per_group=value))


def test_the_largest_integers_pass():
    top = (1 << 31) - 1
    r = ops.make_residual(dict(DESC, n_tokens=top, tokens_per_gate=top))
    assert (r.n_tokens, r.tokens_per_gate) == (top, top)
    assert ops.make_balance(dict(tokens_per_group=top)).tokens_per_group == top
    assert ops.make_balance({}).tokens_per_group == 0


@pytest.mark.parametrize("output", ["loss", "counts", "dX", "dW", "ws"])
@pytest.mark.parametrize("array", ["alpha", "n_shared", "shared_mask", "n_res", "expert_ids", "weights"])
def test_outputs_over_the_record_are_rejected(output, array):
    """All six arrays of the record are inputs, also the two that the loss does
    not read."""
    names = "alpha n_shared shared_mask n_res expert_ids weights valid X W loss counts dX_in dX dW_in dW ws".split()
    at = {k: (i + 1) << 40 for i, k in enumerate(names)}
    at[output] = at[array] + 64   # inside the array's 100 elements
    cfg = _lib.make_config(dict(n_tokens=100, d_model=64, n_experts=4, n_blocks=8, block_width=64, dtype="bf16",
                                mass_threshold=0.6))
    rec = _lib.Routing(**{k: at[k] for k in names[:6]})
    bal = ops.make_balance({})
    status = ops.lib().unif_moe_balance_loss(
        ctypes.byref(cfg), ctypes.byref(bal), ctypes.byref(rec), at["valid"], at["X"], at["W"], at["loss"], at["counts"],
        at["dX_in"], at["dX"], at["dW_in"], at["dW"], at["ws"], 1 << 36, None)
    assert status == _lib.EINVAL
