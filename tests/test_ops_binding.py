"""The binding of the operators around the layer (no GPU needed): descriptions
whose integers do not fit the library's."""
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
