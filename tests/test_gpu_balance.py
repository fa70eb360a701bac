"""The balance loss (unif_moe_balance_loss) against its definition in 64 bits
(MI355X only).

Bounds with u = 2^-24 and sums of absolute values formed next to each result:
dl_tj = p_tj (a_j - sum_m p_tm a_m) sums K <= 64 terms and rounds a_j once: 80 u
of its terms' absolute values. dX adds K terms to it (another 80 u of their
absolute values), dW adds at most N / 32 + 64 terms one after the other. The
loss sums affinities of at most 256 tokens in fp32, the rest in fp64, and is
rounded once: 300 u of it. Loads are whole numbers and equal.
"""
import pytest
import torch

import paper_2608_10392_amd as unif
from paper_2608_10392_amd import _lib, ops

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
DEV = "cuda:0"
T = {"bf16": torch.bfloat16, "f32": torch.float32}


class Case:
    def __init__(self, n, d, K, B=8, dtype="f32", per=0, unit="tokens", padded=None, add=True, weight=0.5, seed=0):
        self.n, self.d, self.K, self.B, self.per, self.unit, self.weight = n, d, K, B, per, unit, weight
        gen = torch.Generator(device=DEV)
        gen.manual_seed(10 * n + d + K + seed)
        rnd = lambda *s: torch.randn(*s, generator=gen, device=DEV)
        self.cfg = dict(n_tokens=n, d_model=d, n_experts=K, n_blocks=B, block_width=64, dtype=dtype,
                        mass_threshold=0.7)
        self.bal = dict(tokens_per_group=per, unit=unit, weight=weight)
        self.valid = None
        real = torch.ones(n, dtype=torch.bool, device=DEV)
        if padded is not None:
            real = padded(torch.arange(n, device=DEV)).logical_not()
            self.valid = real.to(torch.uint8)
        self.real = real
        p, order = torch.sort(torch.softmax(1.5 * rnd(n, K), dim=1), dim=1, descending=True, stable=True)
        k = torch.randint(1, K + 1, (n,), generator=gen, device=DEV)
        b = torch.randint(1, max(B, 2), (n,), generator=gen, device=DEV)
        self.rec = dict(alpha=torch.rand(n, generator=gen, device=DEV), n_shared=torch.where(real, b, 0).int(),
                        shared_mask=torch.zeros(n, dtype=torch.int64, device=DEV), n_res=torch.where(real, k, 0).int(),
                        expert_ids=torch.where(real[:, None], order + 1, -1).int().contiguous(),
                        weights=torch.where(real[:, None], p, 0.0).contiguous())
        self.X, self.W = rnd(n, d).to(T[dtype]), rnd(K + 1, d) / d ** 0.5
        self.dX_in = 1e-3 * rnd(n, d) if add else None
        self.dW_in = 1e-3 * rnd(K + 1, d) if add else None

    def outputs(self):
        f = dict(dtype=torch.float32, device=DEV)
        return dict(loss=torch.full((1,), 7.0, **f), dX=torch.full((self.n, self.d), 7.0, **f),
                    dW=torch.full((self.K + 1, self.d), 7.0, **f),
                    counts=torch.full((ops.gate_rows(self.n, self.per), self.K + 1), 7, dtype=torch.int64, device=DEV))

    def run(self, o=None, ws=None, **kw):
        o = self.outputs() if o is None else o
        a = dict(X=self.X, W=self.W, dX_in=self.dX_in, dW_in=self.dW_in, **{k: o.get(k) for k in ("counts", "dX", "dW")})
        a.update(kw)
        ws = unif.alloc_workspace(unif.balance_loss_workspace_size(self.cfg, self.bal), DEV) if ws is None else ws
        unif.balance_loss(self.cfg, self.bal, self.rec, self.valid, a["X"], a["W"], o["loss"], a["counts"],
                          a["dX_in"], a["dX"], a["dW_in"], a["dW"], ws)
        return o

    def want(self):
        n, K, B = self.n, self.K, self.B
        R = self.per or max(n, 1)
        G = ops.gate_rows(n, self.per)
        ids, f64 = self.rec["expert_ids"], dict(dtype=torch.float64, device=DEV)
        real = self.real
        p, chosen = torch.zeros(n, K + 1, **f64), torch.zeros(n, K + 1, **f64)
        at = torch.where(real[:, None], ids, 0).long()
        p.scatter_(1, at, self.rec["weights"].double())
        chosen.scatter_(1, at, (torch.arange(K, device=DEV)[None] < self.rec["n_res"][:, None]).double())
        p, chosen = p[:, 1:] * real[:, None], chosen[:, 1:] * real[:, None]
        b = self.rec["n_shared"].double()
        unit = torch.ones_like(b) if self.unit == "tokens" else B - b
        shared = (real.double() if self.unit == "tokens" else b * real)[:, None]
        group = torch.arange(n, device=DEV) // R
        per = lambda v: torch.zeros(G, v.shape[1], **f64).index_add_(0, group, v)
        load, tokens, mass = per(chosen * unit[:, None]), per(real.double()[:, None]), per(p)
        share = load / load.sum(1, keepdim=True).clamp(min=1)
        loss = K * (share * mass / tokens.clamp(min=1)).sum() / max(G, 1)
        a = (self.weight * K / max(G, 1) * share / tokens.clamp(min=1))[group]
        q = (p * a).sum(1, keepdim=True)
        dl = p * (a - q)
        tdl = 80 * U * p * (a + q)
        W, X = self.W[1:].double().abs(), torch.where(real[:, None], self.X.double(), 0.0)
        dX, dW = dl @ self.W[1:].double(), torch.zeros(K + 1, self.d, **f64)
        tdX, tdW = tdl @ W + 80 * U * (dl.abs() @ W), torch.zeros_like(dW)
        dW[1:] = dl.T @ X
        tdW[1:] = tdl.T @ X.abs() + (n / 32 + 64) * U * (dl.abs().T @ X.abs())
        if self.dX_in is not None:
            dX, dW = dX + self.dX_in, dW + self.dW_in
        return dict(loss=(loss[None], 300 * U * loss[None]), counts=torch.cat([per(shared), load], 1).long(),
                    dX=(dX, tdX), dW=(dW, tdW))


def check(c, label):
    print(f"\n[gpu] balance {label}", flush=True)
    got, want = c.run(), c.want()
    assert torch.equal(got["counts"], want["counts"])
    for k in ("loss", "dX", "dW"):
        w, t = want[k]
        assert torch.isfinite(got[k]).all(), k
        over = (got[k].double() - w).abs() - t - 2 * U * (w.abs() + t) - 2.0 ** -126
        assert w.numel() == 0 or float(over.max()) <= 0, f"{k}: over by {float(over.max()):.3e} of {float(w.abs().max()):.3e}"
    return got


@pytest.mark.parametrize("K", [1, 2, 3, 6, 8, 15, 16, 17, 31, 32, 33, 47, 48, 49, 63, 64])
def test_expert_counts(K):
    for dtype, d in (("f32", 100), ("bf16", 160)):
        for unit in ("tokens", "blocks"):
            check(Case(333, d, K, dtype=dtype, unit=unit, per=0 if K % 2 else 50), f"333 x {d} K={K} {dtype} {unit}")


@pytest.mark.parametrize("dtype, d", [("f32", 8), ("f32", 9), ("f32", 63), ("f32", 127), ("f32", 128), ("f32", 130), ("f32", 1025),
                                      ("f32", 2500), ("bf16", 32), ("bf16", 96), ("bf16", 384), ("bf16", 768),
                                      ("bf16", 1024), ("bf16", 1056), ("bf16", 4096)])
def test_widths(dtype, d):
    check(Case(150, d, 7, dtype=dtype), f"150 x {d} {dtype}")
    check(Case(150, d, 40, dtype=dtype, add=False), f"150 x {d} {dtype} K=40 written")


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 255, 256, 257, 1000, 4099, 20011])
def test_token_counts(n):
    for per in (0, 1, 2, 63, 64, 65, 197, 256, 300, 5000):
        if n < 20011 or per in (0, 197, 5000):
            check(Case(n, 64, 6, dtype="bf16", per=per), f"{n} x 64 groups of {per}")


PADDINGS = dict(every_third=lambda t: t % 3 == 1, all=lambda t: t >= 0, all_but_last=lambda t: t < t.numel() - 1,
                tail=lambda t: t % 50 > 20, whole_groups=lambda t: (t // 50) % 2 == 0)


@pytest.mark.parametrize("padding", list(PADDINGS))
@pytest.mark.parametrize("per", [0, 50, 130])
def test_padded_tokens(padding, per):
    """Padded tokens' rows of X hold NaN; they reach nothing, and their rows of
    dX are the incoming ones."""
    c = Case(450, 96, 9, dtype="bf16", per=per, padded=PADDINGS[padding])
    rows = c.valid == 0
    c.X[rows] = float("nan")
    got = check(c, f"450 x 96 padded {padding} groups of {per}")
    assert torch.equal(got["dX"][rows], c.dX_in[rows])
    c.dX_in = c.dW_in = None
    assert bool((c.run()["dX"][rows] == 0).all())


def test_no_load():
    """Groups whose tokens share every block have no load in blocks."""
    c = Case(200, 64, 5, B=4, unit="blocks", per=50)
    c.rec["n_shared"][50:120] = 4
    got = check(c, "groups without load")
    assert bool((got["dX"][50:100] == c.dX_in[50:100]).all())
    c.rec["n_shared"][:] = 4
    assert float(c.run()["loss"]) == 0.0


def test_uniform_and_collapsed():
    """The loss is 1 for even loads and affinities and K for all on one expert."""
    print("\n[gpu] balance: extremes", flush=True)
    K = 8
    c = Case(64 * K, 64, K, add=False, weight=1.0)
    c.rec["weights"][:] = 1.0 / K
    c.rec["n_res"][:] = 1
    c.rec["expert_ids"][:] = 1 + (torch.arange(64 * K, device=DEV)[:, None] + torch.arange(K, device=DEV)[None]) % K
    got = c.run()
    assert abs(float(got["loss"]) - 1.0) <= 300 * U
    assert float(got["dX"].abs().max()) <= 80 * U / 64
    c.rec["weights"][:] = 0.0
    c.rec["weights"][:, 0] = 1.0
    c.rec["expert_ids"][:] = 1 + torch.arange(K, device=DEV)
    assert abs(float(c.run()["loss"]) - K) <= 300 * U * K


def test_absent_outputs_and_in_place():
    print("\n[gpu] balance: absent and in place", flush=True)
    for dtype, d in (("bf16", 352), ("f32", 101)):
        c = Case(777, d, 11, dtype=dtype, per=100)
        full = c.run()
        o = c.run(counts=None, dX_in=None, dX=None, dW_in=None, dW=None, X=None, W=None)
        assert torch.equal(o["loss"], full["loss"])
        assert torch.equal(c.run(dW_in=None, dW=None, X=None)["dX"], full["dX"])
        assert torch.equal(c.run(dX_in=None, dX=None, W=None)["dW"], full["dW"])
        o = dict(c.outputs(), dX=c.dX_in.clone(), dW=c.dW_in.clone())
        c.run(o, dX_in=o["dX"], dW_in=o["dW"])
        assert all(torch.equal(o[k], full[k]) for k in o)
        assert torch.equal(full["dW"][0], c.dW_in[0])


@pytest.mark.parametrize("dtype, d", [("bf16", 96), ("f32", 131)])
def test_alignment_and_neighbours(dtype, d):
    """Tensors one element into their storage, bands behind the outputs."""
    print(f"\n[gpu] balance: unaligned {dtype}", flush=True)
    c = Case(100, d, 6, dtype=dtype, per=30)
    full = c.run()

    def shifted(t):
        flat = torch.full((t.numel() + 65,), 3, dtype=t.dtype, device=DEV)
        view = flat[1:1 + t.numel()].view(t.shape)
        view.copy_(t)
        return flat, view

    for k in ("X", "W", "dX_in", "dW_in"):
        setattr(c, k, shifted(getattr(c, k))[1])
    c.rec = {k: shifted(v)[1] for k, v in c.rec.items()}
    bands, o = {}, {}
    for k, v in c.outputs().items():
        bands[k], o[k] = shifted(v)
    c.run(o)
    assert all(torch.equal(o[k], full[k]) for k in o)
    for flat in bands.values():
        assert float(flat[0]) == 3 and bool((flat[-64:] == 3).all())


def test_workspace_streams_and_graphs():
    print("\n[gpu] balance: workspace, streams, graphs", flush=True)
    c = Case(3000, 256, 16, dtype="bf16", per=197)
    first = c.run()
    size = unif.balance_loss_workspace_size(c.cfg, c.bal)
    for fill in (0, 255):
        ws = torch.full((size + 256,), fill, dtype=torch.uint8, device=DEV)
        ws[size:] = 77
        o = c.run(ws=ws[:size])
        assert all(torch.equal(o[k], first[k]) for k in o)
        assert bool((ws[size:] == 77).all())
    side, ws2 = torch.cuda.Stream(), unif.alloc_workspace(size, DEV)
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        o2 = c.run(ws=ws2)
    o1 = c.run(ws=ws[:size])
    torch.cuda.synchronize()
    assert all(torch.equal(o1[k], first[k]) and torch.equal(o2[k], first[k]) for k in first)
    o = c.outputs()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.run(o, ws2)
    for i in range(3):
        c.X.mul_(0.5)
        c.rec["n_res"].clamp_(max=9 - 3 * i)
        eager = c.run(ws=ws[:size])
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(eager[k], o[k]) for k in o)


def test_no_tokens():
    print("\n[gpu] balance: no tokens", flush=True)
    for per in (0, 10):
        c = Case(0, 64, 5, per=per)
        o = c.run()
        torch.cuda.synchronize()
        assert float(o["loss"]) == 0.0 and torch.equal(o["dW"], c.dW_in) and bool((o["counts"] == 0).all())


def test_foreign_ids_are_ignored():
    """Expert ids outside 1..K are neither read nor counted."""
    print("\n[gpu] balance: foreign ids", flush=True)
    c = Case(120, 64, 6)
    want = c.run()
    c.rec["expert_ids"][7], c.rec["n_res"][7] = torch.tensor([0, -5, 7, 1 << 30, -(1 << 31), 99], dtype=torch.int32, device=DEV), 6
    c.rec["weights"][7] = 0.3
    got = c.run()
    assert torch.isfinite(got["dX"]).all() and torch.equal(got["dX"][7], c.dX_in[7])
    assert int(got["counts"][0, 1:].sum()) < int(want["counts"][0, 1:].sum()) + 1


def test_counts_match_the_statistics():
    """The loads of a routed batch are unif_moe_stats' tokens per expert."""
    print("\n[gpu] balance: against statistics", flush=True)
    from paper_2608_10392_amd.layer import DeviceLayer
    from synth import generate, get_config, layer_config
    g = generate(get_config("bert_base_padded", n_tokens=1024, d_model=256, n_experts=8, n_blocks=16, block_width=64))
    dev = DeviceLayer(layer_config(g["cfg"]), g["X"], g["valid"], g["W_router"], g["prototypes"])
    dev.route()
    stats = dev.stats()
    loss, counts = dev.balance_loss(dict(tokens_per_group=128))
    assert counts.sum(0).tolist() == stats["expert_tokens"][:9]
    _, blocks = dev.balance_loss(dict(unit="blocks"))
    assert int(blocks.sum()) == stats["activated_blocks"]
    assert 1.0 <= float(loss) <= 8.0


def test_binding_refuses():
    c = Case(20, 32, 4)
    for kw, what in ((dict(X=c.X.double()), "X is torch.float64"), (dict(W=c.W[1:]), "W_router is not a contiguous"),
                     (dict(dX_in=c.dX_in.t().contiguous().t()), "dX_in is not a contiguous")):
        with pytest.raises(_lib.UnifMoeError, match=what):
            c.run(**kw)


def test_offsets_past_32_bits():
    """Tensors of more than 2^32 bytes: the last group's rows of dX are those of
    a call of its own, with the weight of its share of the mean."""
    per, groups, d, K = 1024, 1280, 1024, 4
    n = per * groups
    print(f"\n[gpu] balance: {n} x {d}", flush=True)
    c = Case(n, d, K, dtype="bf16", per=per, weight=640.0, add=False)
    o = c.run()
    last = Case(per, d, K, dtype="bf16", weight=0.5, add=False)
    last.rec, last.X, last.W = {k: v[-per:].contiguous() for k, v in c.rec.items()}, c.X[-per:], c.W
    want = last.run()
    assert torch.equal(o["counts"][-1:], want["counts"])
    # the slopes' quotients may round differently: two fp32 steps of a sum of K terms' absolute values
    err = (o["dX"][-per:] - want["dX"]).abs().max()
    assert float(err) <= 8 * K * U * float(want["dX"].abs().max())
    del c, o
    torch.cuda.empty_cache()
