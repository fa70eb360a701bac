"""The residual join (unif_moe_residual_forward / _backward) against its
definition in 64 bits (MI355X only).

Bounds, per element, with u = 2^-24 (half an fp32 step) and sums of absolute
values that the 64-bit side forms next to each result. A row sum is at most 16
terms in a lane, six butterfly steps and eight waves: 30 roundings; statistics
add a division, a square root and products. C = 64 u times the terms' absolute
values covers each row quantity to first order. A parameter's sum over the
tokens adds at most 128 terms one after the other in these tests before the
teams' and workgroups' (32 more): P = 192 u. Outputs in bf16 add half a step,
2^-9 of the value (2^-8 eps / 2), and the smallest normal's step.
"""
import itertools

import pytest
import torch

from paper_2608_10392_amd import _lib, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
C, P = 64 * U, 192 * U
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "f32": torch.float32}
TYPES = [("bf16", "bf16", "f32"), ("bf16", "bf16", "bf16"), ("bf16", "f32", "f32"), ("bf16", "f32", "bf16"),
         ("f32", "f32", "f32")]
EPS = 1e-5


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


class Norm:
    """hat = normalised rows, r their scale, with bounds of the fp32 errors of
    hat given that of the input rows (tol)."""

    def __init__(self, kind, u, gamma, beta, tol):
        self.kind, self.gamma = kind, gamma
        if kind == "none":
            self.hat, self.r, self.out, self.tol_hat, self.tol_out = u, None, u, tol, tol
            return
        m = lambda v: v.mean(1, keepdim=True)
        c = u - m(u) if kind == "layer" else u
        self.r = 1 / torch.sqrt(m(c * c) + EPS)
        self.hat = c * self.r
        tol_c = tol + (m(tol) + C * (u.abs() + m(u.abs())) if kind == "layer" else 0)
        rel_r = C + self.r ** 2 * m(c.abs() * tol_c)
        self.tol_hat = tol_c * self.r + self.hat.abs() * rel_r
        self.rel_r = rel_r
        g = gamma.abs()
        self.out = self.hat * gamma + beta
        self.tol_out = self.tol_hat * g + 4 * U * ((self.hat * gamma).abs() + beta.abs())

    def grad(self, a, tol):
        """Gradient of the input rows from that of hat, and its bound."""
        if self.kind == "none":
            return a, tol
        m = lambda v: v.mean(1, keepdim=True)
        q = m(a * self.hat)
        s = m(a) if self.kind == "layer" else 0 * q
        g = self.r * (a - s - self.hat * q)
        tq = m(tol * self.hat.abs() + a.abs() * self.tol_hat) + C * m((a * self.hat).abs())
        ts = m(tol) + C * m(a.abs()) if self.kind == "layer" else 0 * q
        t = self.r * (tol + ts + self.hat.abs() * tq + self.tol_hat * q.abs())
        t = t + (self.rel_r + 8 * U) * self.r * (a.abs() + s.abs() + (self.hat * q).abs())
        return g, t


class Case:
    """Inputs of one join on the device."""

    def __init__(self, n, d, types=("bf16", "bf16", "f32"), out="layer", inn="rms", gate=None, per=0, beta=True,
                 scale=0.75, padded=None, seed=0):
        self.n, self.d, self.types, self.per, self.scale = n, d, types, per, scale
        self.out, self.inn = out, inn
        gen = torch.Generator(device=DEV)
        gen.manual_seed(1000 * n + d + seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)
        layer, stream, dh = (T[t] for t in types)
        self.x = ((0.5 + 2 * torch.rand(n, 1, generator=gen, device=DEV)) * rnd(n, d) + 0.5 * rnd(d)).to(stream)
        self.f, self.dy, self.dh = (0.6 * rnd(n, d)).to(layer), rnd(n, d).to(stream), rnd(n, d).to(dh)
        self.params = {}
        for side, kind in (("out", out), ("in", inn)):
            if kind != "none":
                self.params[side + "_gamma"] = 1 + 0.3 * rnd(d)
                if beta:
                    self.params[side + "_beta"] = 0.2 * rnd(d)
        if gate:
            self.params["gate"] = 0.4 + 0.5 * rnd(ops.gate_rows(n, per), d)
        self.valid = None
        if padded is not None:
            self.valid = padded(torch.arange(n, device=DEV)).logical_not().to(torch.uint8)
        self.res = ops.make_residual(dict(
            n_tokens=n, d_model=d, dtype=types[0], stream_dtype=types[1], out_norm=out, in_norm=inn, out_eps=EPS,
            in_eps=EPS, residual_scale=scale, tokens_per_gate=per, **self.params))

    # 64-bit side ----------------------------------------------------------
    def _p(self, k, other):
        return self.params[k].double() if k in self.params else torch.full((1, self.d), other, dtype=torch.float64, device=DEV)

    def _gate(self):
        if "gate" not in self.params:
            return torch.ones(1, 1, dtype=torch.float64, device=DEV)
        g = self.params["gate"].double()
        return g[torch.arange(self.n, device=DEV) // self.per] if self.per else g

    def _real(self):
        return torch.ones(self.n, 1, dtype=torch.bool, device=DEV) if self.valid is None else self.valid.bool()[:, None]

    def forward64(self):
        real, zero = self._real(), torch.zeros((), dtype=torch.float64, device=DEV)
        x, f = (torch.where(real, v.double(), zero) for v in (self.x, self.f))
        b = Norm(self.out, f, self._p("out_gamma", 1.0), self._p("out_beta", 0.0), torch.zeros_like(f))
        g = self._gate()
        v = self.scale * x + g * b.out
        tol = g.abs() * b.tol_out + 4 * U * ((self.scale * x).abs() + (g * b.out).abs())
        h = Norm(self.inn, v, self._p("in_gamma", 1.0), self._p("in_beta", 0.0), tol)
        return [(w * real, t * real) for w, t in ((v, tol), (h.out, h.tol_out))]

    def backward64(self, dy=True, dh=True):
        real, zero = self._real(), torch.zeros((), dtype=torch.float64, device=DEV)
        y, f, gy, gh = (torch.where(real, v.double(), zero) for v in (self.x, self.f, self.dy, self.dh))
        if not dy:
            gy = 0 * gy
        o, t = {}, {}
        D, tD = gy, torch.zeros_like(gy)
        if dh:
            nin = Norm(self.inn, y, self._p("in_gamma", 1.0), self._p("in_beta", 0.0), torch.zeros_like(y))
            o["in_beta"], t["in_beta"] = gh.sum(0), P * gh.abs().sum(0)
            o["in_gamma"] = (gh * nin.hat).sum(0)
            t["in_gamma"] = (gh.abs() * nin.tol_hat + P * (gh * nin.hat).abs()).sum(0)
            a = gh * nin.gamma
            w, tw = nin.grad(a, U * a.abs())
            D, tD = D + w, tw + 2 * U * (D.abs() + w.abs())
        o["dx"], t["dx"] = self.scale * D, abs(self.scale) * (tD + U * D.abs())
        nout = Norm(self.out, f, self._p("out_gamma", 1.0), self._p("out_beta", 0.0), torch.zeros_like(f))
        g = self._gate()
        per = D * nout.out
        tper = tD * nout.out.abs() + D.abs() * nout.tol_out + P * per.abs()
        if "gate" in self.params:
            rows = self.params["gate"].shape[0]
            at = torch.arange(self.n, device=DEV) // (self.per or self.n)
            add = lambda v: torch.zeros(rows, self.d, dtype=torch.float64, device=DEV).index_add_(0, at, v * real)
            o["gate"], t["gate"] = add(per), add(tper)
        dn, tdn = D * g, tD * g.abs() + U * (D * g).abs()
        o["out_beta"], t["out_beta"] = dn.sum(0), (tdn + P * dn.abs()).sum(0)
        o["out_gamma"] = (dn * nout.hat).sum(0)
        t["out_gamma"] = (tdn * nout.hat.abs() + dn.abs() * nout.tol_hat + P * (dn * nout.hat).abs()).sum(0)
        b = dn * nout.gamma if self.out != "none" else dn
        o["df"], t["df"] = nout.grad(b, tdn * (nout.gamma.abs() if self.out != "none" else 1) + U * b.abs())
        return {k: (v * real if k in ("dx", "df") else v, t[k]) for k, v in o.items()}

    # device side ----------------------------------------------------------
    def forward(self, **kw):
        a = dict(x=self.x, f=self.f, y=torch.full_like(self.x, 7.0), h=torch.full_like(self.f, 7.0))
        a.update(kw)
        ops.residual_forward(self.res, a["x"], a["f"], self.valid, a["y"], a["h"])
        return a["y"], a["h"]

    def outputs(self):
        o = dict(dx=torch.full_like(self.x, 7.0), df=torch.full_like(self.f, 7.0))
        return dict(o, **{k: torch.full_like(v, 7.0) for k, v in self.params.items()})

    def backward(self, o=None, ws=None, **kw):
        o = self.outputs() if o is None else o
        a = dict(y=self.x, f=self.f, dy=self.dy, dh=self.dh, dx=o.get("dx"), df=o.get("df"))
        a.update(kw)
        ws = _lib.alloc_workspace(ops.residual_backward_workspace_size(self.res), DEV) if ws is None else ws
        ops.residual_backward(self.res, a["y"], a["f"], self.valid, a["dy"], a["dh"], a["dx"], a["df"],
                              {k: v for k, v in o.items() if k in ops.PARAMS}, ws)
        return o


def check(name, got, want, tol):
    tiny = 2.0 ** -126
    limit = tol + half_step(got.dtype) * (want.abs() + tol) + tiny
    over = (got.double() - want).abs() - limit
    assert torch.isfinite(got).all(), name
    assert float(over.max()) <= 0, f"{name}: {float((got.double() - want).abs().max()):.3e} off, over by {float(over.max()):.3e}"


def check_both(c, label):
    print(f"\n[gpu] residual {label}", flush=True)
    y, h = c.forward(**({} if c.inn != "none" else dict(h=None)))
    (wy, ty), (wh, th) = c.forward64()
    check("y", y, wy, ty)
    if c.inn != "none":
        check("h", h, wh, th)
    dh = c.inn != "none"
    got = c.backward(**({} if dh else dict(y=None, dh=None)))
    want = c.backward64(dh=dh)
    for k, v in got.items():
        check(k, v, *want[k])


WIDTHS = [4, 5, 6, 7, 8, 63, 64, 65, 128, 200, 256, 257, 384, 512, 513, 768, 1000, 1024, 1025, 1536, 2048, 4096, 5120, 8191,
          8192]


@pytest.mark.parametrize("d", WIDTHS)
def test_widths(d):
    types = TYPES[WIDTHS.index(d) % 5]
    check_both(Case(37, d, types, gate=True), f"37 x {d} {types}")


@pytest.mark.parametrize("n", [1, 2, 3, 31, 64, 65, 197, 1001, 4099])
def test_token_counts(n):
    check_both(Case(n, 96, gate=True, per=5), f"{n} x 96, a gate per 5 tokens")


@pytest.mark.parametrize("types", TYPES)
@pytest.mark.parametrize("out, inn", list(itertools.product(("none", "layer", "rms"), repeat=2)))
def test_norms_and_types(types, out, inn):
    for gate, beta in ((None, True), (True, False)):
        check_both(Case(45, 320, types, out, inn, gate, beta=beta), f"45 x 320 {types} {out} {inn} gate {gate} beta {beta}")


@pytest.mark.parametrize("d", [64, 200, 768, 1000, 2500])
@pytest.mark.parametrize("n, per", [(1000, 1), (1000, 3), (1000, 64), (1000, 999), (1000, 1000), (1000, 5000),
                                    (5000, 197), (20011, 2500)])
def test_gates_per_group(n, per, d):
    check_both(Case(n, d, gate=True, per=per, out="rms"), f"{n} x {d}, a gate per {per} tokens")


PADDINGS = dict(every_third=lambda t: t % 3 == 1, all=lambda t: t >= 0, all_but_last=lambda t: t < t.numel() - 1,
                tail=lambda t: t % 50 > 20, whole_groups=lambda t: (t // 50) % 2 == 0)


@pytest.mark.parametrize("padding", list(PADDINGS))
@pytest.mark.parametrize("d", [96, 768, 1500])
def test_padded_tokens(padding, d):
    """Padded rows hold NaN and infinities in every input; their outputs are
    zero and they reach no gradient."""
    c = Case(450, d, gate=True, per=50, padded=PADDINGS[padding])
    rows = c.valid == 0
    for t in (c.x, c.f, c.dy, c.dh):
        t[rows] = float("nan")
        t[rows, ::2] = float("inf")
    check_both(c, f"450 x {d} padded {padding}")
    for t in (*c.forward(), *[v for k, v in c.backward().items() if k in ("dx", "df")]):
        assert bool((t[rows] == 0).all())


def test_absent_inputs_and_outputs():
    print("\n[gpu] residual: absent tensors", flush=True)
    c = Case(70, 192, ("bf16", "f32", "f32"), gate=True)
    y, h = c.forward()
    only_y, _ = c.forward(h=None)
    _, only_h = c.forward(y=None)
    assert torch.equal(y, only_y) and torch.equal(h, only_h)
    # no residual: as with x = 0
    (y0, h0), (yz, hz) = c.forward(x=None), c.forward(x=torch.zeros_like(c.x))
    assert torch.equal(y0, yz) and torch.equal(h0, hz)
    full = c.backward()
    for keep in (("dx",), ("df",), ("gate", "in_beta"), ("out_gamma",), ()):
        o = c.backward({k: v for k, v in c.outputs().items() if k in keep})
        assert all(torch.equal(o[k], full[k]) for k in keep)
    assert torch.equal(c.backward(dy=None)["dx"], c.backward(dy=torch.zeros_like(c.dy))["dx"])
    # no branch: N_in alone
    b = Case(70, 192, out="none", gate=None)
    (y, h), (wy, _) = b.forward(f=None), b.forward64()
    check("y", y, b.scale * b.x.double(), 2 * U * b.x.double().abs())
    o = b.outputs()
    o.pop("df")
    o = b.backward(o, f=None)
    want = b.backward64()
    for k in o:
        check(k, o[k], *want[k])
    # no N_in: y's gradient alone
    n = Case(70, 192, inn="none", gate=True)
    o = n.backward(y=None, dh=None)
    for k, v in o.items():
        check(k, v, *n.backward64(dh=False)[k])


def test_in_place():
    """y over x and dx over dy."""
    print("\n[gpu] residual: in place", flush=True)
    for d in (130, 768, 3000):
        c = Case(333, d, gate=True)
        (y, h), o = c.forward(), c.backward()
        x, dy = c.x.clone(), c.dy.clone()
        y2, h2 = c.forward(x=x, y=x)
        assert torch.equal(y, y2) and torch.equal(h, h2)
        o2 = c.backward(dict(c.outputs(), dx=dy), dy=dy)
        assert all(torch.equal(o[k], o2[k]) for k in o)


@pytest.mark.parametrize("types", [TYPES[0], TYPES[3], TYPES[4]])
@pytest.mark.parametrize("d", [65, 200, 768, 1030])
def test_alignment_and_neighbours(types, d):
    """Tensors that start one element into their storage, with a band behind
    every output that stays as it was."""
    print(f"\n[gpu] residual: unaligned {d} {types}", flush=True)
    c = Case(50, d, types, gate=True, per=7)
    (y, h), o = c.forward(), c.backward()

    def shifted(t, fill=None):
        flat = torch.full((t.numel() + 65,), 3.0, dtype=t.dtype, device=DEV)
        view = flat[1:1 + t.numel()].view(t.shape)
        if fill is None:
            view.copy_(t)
        return flat, view

    for k in ("x", "f", "dy", "dh"):
        setattr(c, k, shifted(getattr(c, k))[1])
    fy, y2 = shifted(y, True)
    fh, h2 = shifted(h, True)
    c.forward(y=y2, h=h2)
    bands, o2 = {}, {}
    for k, v in o.items():
        bands[k], o2[k] = shifted(v, True)
    c.backward(o2)
    assert torch.equal(y, y2) and torch.equal(h, h2)
    assert all(torch.equal(o[k], o2[k]) for k in o)
    for flat in (fy, fh, *bands.values()):
        assert float(flat[0]) == 3.0 and bool((flat[-64:] == 3.0).all())


def test_workspace_bounds_and_repeats():
    """Any contents of the workspace, a band behind it, the same bits again."""
    print("\n[gpu] residual: workspace", flush=True)
    for n, d, per in ((3000, 64, 7), (700, 768, 0), (700, 768, 30), (90, 6000, 20)):
        c = Case(n, d, gate=True, per=per)
        size = ops.residual_backward_workspace_size(c.res)
        first = c.backward()
        for fill in (0, 255):
            ws = torch.full((size + 256,), fill, dtype=torch.uint8, device=DEV)
            ws[size:] = 77
            o = c.backward(ws=ws[:size])
            assert all(torch.equal(o[k], first[k]) for k in o)
            assert bool((ws[size:] == 77).all())


def test_large_rows_of_equal_values():
    """Rows without variance, zero rows and rows with a large offset."""
    print("\n[gpu] residual: flat rows", flush=True)
    for inn in ("layer", "rms"):
        c = Case(16, 700, ("f32", "f32", "f32"), out="layer", inn=inn, gate=True, scale=1.0)
        c.x[0], c.f[0] = 0.0, 0.0
        c.x[1], c.f[1] = 3.5, -2.25
        c.f[2:4] += 1000.0
        check_both(c, f"flat rows {inn}")


def test_streams_and_graphs():
    """On another stream, and captured: every replay equals the eager call on
    the inputs it was replayed with."""
    print("\n[gpu] residual: streams and graphs", flush=True)
    c = Case(600, 768, gate=True, per=197)
    (y, h), o = c.forward(), c.backward()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    ws = [_lib.alloc_workspace(ops.residual_backward_workspace_size(c.res), DEV) for _ in range(2)]
    with torch.cuda.stream(side):
        y2, h2 = c.forward()
        o2 = c.backward(ws=ws[0])
    o3 = c.backward(ws=ws[1])
    torch.cuda.synchronize()
    assert torch.equal(y, y2) and torch.equal(h, h2)
    assert all(torch.equal(o[k], o2[k]) and torch.equal(o[k], o3[k]) for k in o)
    y4, h4, o4 = torch.empty_like(y), torch.empty_like(h), c.outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.forward(y=y4, h=h4)
        c.backward(o4, ws[0])
    for i in range(3):
        c.x.mul_(0.5 + i)
        c.dh.add_(0.25)
        (y, h), o = c.forward(), c.backward(ws=ws[1])
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(y, y4) and torch.equal(h, h4)
        assert all(torch.equal(o[k], o4[k]) for k in o)


def test_no_tokens():
    print("\n[gpu] residual: no tokens", flush=True)
    c = Case(0, 96, gate=True)
    c.forward()
    o = c.backward()
    torch.cuda.synchronize()
    assert all(bool((o[k] == 0).all()) for k in c.params)


def test_gradient_against_differences():
    """The gradients against central differences of the 64-bit forward."""
    print("\n[gpu] residual: differences", flush=True)
    c = Case(6, 24, ("f32", "f32", "f32"), gate=True, per=4)
    # the backward reads the forward's y
    dy, dh, x0 = c.dy.double(), c.dh.double(), c.x.clone()
    c.backward_y = c.forward64()[0][0].float()
    got = c.backward(y=c.backward_y)

    def loss():
        (y, _), (h, _) = c.forward64()
        return float((y * dy).sum() + (h * dh).sum())

    for name, t in dict(dx=c.x, df=c.f, **c.params).items():
        flat, g = t.view(-1), got[name].reshape(-1)
        for i in range(0, flat.numel(), max(1, flat.numel() // 9)):
            keep = float(flat[i])
            step = 2.0 ** -9
            flat[i] = keep + step
            hi, up = float(flat[i]), loss()
            flat[i] = keep - step
            lo, down = float(flat[i]), loss()
            flat[i] = keep
            # third differences are of the order of the values here: step^2 = 4e-6
            assert abs((up - down) / (hi - lo) - float(g[i])) <= 1e-3 * (1 + abs(float(g[i]))), (name, i)


@pytest.mark.parametrize("bad, what", [
    (dict(x=lambda t: t.t().contiguous().t()), "x is not a contiguous"), (dict(f=lambda t: t.float()), "f is torch.float32"),
    (dict(y=lambda t: t[:-1]), "y is not a contiguous tensor of"), (dict(h=lambda t: t.cpu()), "h is not on a GPU"),
])
def test_binding_refuses(bad, what):
    c = Case(20, 32)
    a = dict(x=c.x, f=c.f, y=torch.empty_like(c.x), h=torch.empty_like(c.f))
    a.update({k: fn(a[k]) for k, fn in bad.items()})
    with pytest.raises(_lib.UnifMoeError, match=what) as e:
        ops.residual_forward(c.res, a["x"], a["f"], None, a["y"], a["h"])
    assert e.value.status == _lib.EINVAL


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 bytes: the last rows are those of a call of
    their own."""
    n, d, tail = 700_001, 1600, 33
    print(f"\n[gpu] residual: {n} x {d}", flush=True)
    gen = torch.Generator(device=DEV)
    gen.manual_seed(5)
    rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)
    x, f = rnd(n, d), rnd(n, d).to(torch.bfloat16)
    p = dict(in_gamma=1 + 0.2 * rnd(d), out_gamma=1 + 0.2 * rnd(d), gate=rnd(1, d))
    desc = dict(d_model=d, dtype="bf16", stream_dtype="f32", in_norm="rms", out_norm="layer", **p)
    got, want = [], []
    for rows, out in ((slice(0, n), got), (slice(n - tail, n), want)):
        xs, fs = x[rows], f[rows]
        res = ops.make_residual(dict(desc, n_tokens=len(xs)))
        y, h = torch.empty_like(xs), torch.empty_like(fs)
        ops.residual_forward(res, xs, fs, None, y, h)
        out += [y[-tail:].clone(), h[-tail:].clone()]
        ws = _lib.alloc_workspace(ops.residual_backward_workspace_size(res), DEV)
        ops.residual_backward(res, xs, fs, None, xs, fs, y, h, None, ws)
        out += [y[-tail:].clone(), h[-tail:].clone()]
        del y, h
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    torch.cuda.empty_cache()


def test_absent_stream_in_mixed_types():
    """No x and no y beside an fp32 stream, a workspace at an odd address, and
    both gradients from one tensor."""
    print("\n[gpu] residual: absent stream", flush=True)
    for d in (4, 7, 129, 2049):
        c = Case(1, d, ("bf16", "f32", "f32"), gate=True)
        _, want = c.forward(x=torch.zeros_like(c.x))
        _, h = c.forward(x=None, y=None)
        assert torch.equal(h, want)
        c = Case(40, d, ("f32", "f32", "f32"), gate=True, per=7)
        c.dh = c.dy
        size = ops.residual_backward_workspace_size(c.res)
        first, ws = c.backward(), torch.empty(size + 3, dtype=torch.uint8, device=DEV)
        o = c.backward(ws=ws[3:])
        assert all(torch.equal(o[k], first[k]) for k in o)
        for k, v in o.items():
            check(k, v, *c.backward64()[k])
