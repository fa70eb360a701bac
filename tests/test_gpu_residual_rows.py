"""Padded tokens between real ones inside a team's rows, up to more than 64 rows a
team, in every team width (MI355X only), and N_in alone. Bounds as in
test_gpu_residual.py: at most 80 rows a team here and at most 64 teams in a
workgroup, one after the other: below the 192 roundings of a parameter's sum."""
import pytest
import torch

from tests.test_gpu_residual import TYPES, Case, Norm, check

pytestmark = pytest.mark.gpu

CUS = 256


def rows(n, d, forward):
    """Tokens per team of a launch: a team's lanes hold 3 x 4 columns each up to 64
    lanes, a workgroup the rows past 1,024 columns; 64 (16 in wide rows) waves per
    compute unit in the forward's launch, 8 in the backward's."""
    if d > 1024:
        waves = -(-d // 512)
        most = CUS * max(1, (16 if forward else 8) // waves)
    else:
        lanes = next(l for l in (8, 16, 32, 64) if l == 64 or l * 12 >= d)
        block = 256 if forward else 512
        most = CUS * max(1, (64 if forward else 8) // (block // 64)) * (block // lanes)
    return -(-n // most)


def poison(c):
    pad = c.valid == 0
    for t in (c.x, c.f, c.dy, c.dh):
        t[pad] = float("nan")
        t[pad, ::2] = float("inf")
    return pad


PADDINGS = dict(alternating=lambda t: t % 2 == 1, runs=lambda t: t % 71 > 50, most=lambda t: t % 9 != 4)


@pytest.mark.parametrize("padding", list(PADDINGS))
@pytest.mark.parametrize("n, d, least, per, types", [
    (60_000, 33, 3, 37, TYPES[1]), (1_100_000, 20, 64, 5000, TYPES[0]), (40_000, 130, 4, 0, TYPES[0]), (30_000, 384, 7, 5, TYPES[2]),
    (20_000, 512, 9, 197, TYPES[3]), (20_000, 1000, 9, 333, TYPES[0]), (140_000, 400, 64, 777, TYPES[4]),
    (20_000, 2500, 78, 150, TYPES[0]), (20_000, 1100, 39, 0, TYPES[4]), (5_000, 8000, 19, 7, TYPES[1])])
def test_padded_rows_between_real_ones_backward(n, d, least, per, types, padding):
    assert least < rows(n, d, False) <= 80
    print(f"\n[gpu] residual {n} x {d} {types} backward, {rows(n, d, False)} rows a team, {padding} padded", flush=True)
    c = Case(n, d, types, gate=True, per=per, padded=PADDINGS[padding])
    pad = poison(c)
    got, want = c.backward(), c.backward64()
    for k, v in got.items():
        check(k, v, *want[k])
    assert bool((got["dx"][pad] == 0).all()) and bool((got["df"][pad] == 0).all())


@pytest.mark.parametrize("padding", list(PADDINGS))
@pytest.mark.parametrize("n, d, least, per, types", [
    (300_000, 33, 2, 37, TYPES[1]), (200_000, 130, 3, 0, TYPES[0]), (100_000, 384, 3, 5, TYPES[2]), (60_000, 512, 3, 197, TYPES[3]),
    (60_000, 1000, 3, 333, TYPES[0]), (60_000, 2500, 78, 150, TYPES[0]), (50_000, 1100, 38, 0, TYPES[4]), (30_000, 8000, 117, 7, TYPES[1])])
def test_padded_rows_between_real_ones_forward(n, d, least, per, types, padding):
    assert least < rows(n, d, True)
    print(f"\n[gpu] residual {n} x {d} {types} forward, {rows(n, d, True)} rows a team, {padding} padded", flush=True)
    c = Case(n, d, types, gate=True, per=per, padded=PADDINGS[padding])
    pad = poison(c)
    (y, h), want = c.forward(), c.forward64()
    check("y", y, *want[0])
    check("h", h, *want[1])
    assert bool((y[pad] == 0).all()) and bool((h[pad] == 0).all())
    # over x itself, as a step that keeps one stream does
    x = c.x.clone()
    y2, h2 = c.forward(x=x, y=x)
    assert torch.equal(y, y2) and torch.equal(h, h2)


@pytest.mark.parametrize("inn", ["layer", "rms"])
@pytest.mark.parametrize("n, d, types", [(70, 192, TYPES[0]), (1000, 768, TYPES[2]), (333, 1000, TYPES[4]), (90, 2500, TYPES[3]),
                                         (30_000, 64, TYPES[1])])
def test_norm_in_front_alone(n, d, types, inn):
    """No branch and no y: h = N_in(s x), what a block's first call forms."""
    print(f"\n[gpu] residual N_in alone {n} x {d} {types} {inn}", flush=True)
    for beta in (True, False):
        c = Case(n, d, types, out="none", inn=inn, beta=beta, padded=lambda t: t % 5 == 2)
        pad = poison(c)
        _, h = c.forward(f=None, y=None)
        real = (c.valid != 0)[:, None]
        v = c.scale * torch.where(real, c.x.double(), 0.0)
        want = Norm(inn, v, c._p("in_gamma", 1.0), c._p("in_beta", 0.0), 2 * 2.0 ** -24 * v.abs())
        check("h", h, want.out * real, want.tol_out * real)
        assert bool((h[pad] == 0).all())
        y, both = c.forward(f=None)
        assert torch.equal(both, h)
        check("y", y, v, 2 * 2.0 ** -24 * v.abs())
