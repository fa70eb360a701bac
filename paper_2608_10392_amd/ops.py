"""ctypes binding of the operators around the layer (include/unif_moe_ops.h).

Argument marshalling only, as in _lib.py. Tensors are torch device tensors;
their type, size, layout and device are checked here (what the library cannot
see from a pointer), everything else by the library. A call runs on the device
of its tensors and, where no stream is given, on that device's current stream.
"""
import ctypes

from . import _lib
from ._lib import EINVAL, UnifMoeError, alloc_workspace  # noqa: F401

ROW_NORMS = {"none": 0, "layer": 1, "rms": 2}
BALANCE_UNITS = {"tokens": 0, "blocks": 1}
RESIDUAL_MIN_D, RESIDUAL_MAX_D = 4, 8192
BALANCE_MIN_D = 8
PARAMS = ("out_gamma", "out_beta", "in_gamma", "in_beta", "gate")


class Residual(ctypes.Structure):
    """unif_moe_residual; make_residual notes the parameter tensors it points to
    (and so keeps them) and their device."""
    params, device = {}, None
    _fields_ = [("n_tokens", ctypes.c_int32), ("d_model", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("stream_dtype", ctypes.c_int32), ("out_norm", ctypes.c_int32), ("in_norm", ctypes.c_int32),
                ("tokens_per_gate", ctypes.c_int32), ("out_eps", ctypes.c_float), ("in_eps", ctypes.c_float),
                ("residual_scale", ctypes.c_float)] + [(k, ctypes.c_void_p) for k in PARAMS]


class ResidualGrads(ctypes.Structure):
    _fields_ = [(k, ctypes.c_void_p) for k in PARAMS]


class Balance(ctypes.Structure):
    _fields_ = [("tokens_per_group", ctypes.c_int32), ("unit", ctypes.c_int32), ("weight", ctypes.c_float)]


RESIDUAL_KEYS = frozenset(k for k, _ in Residual._fields_)
BALANCE_KEYS = frozenset(k for k, _ in Balance._fields_)
EXPORTS = ("unif_moe_residual_forward", "unif_moe_residual_backward_workspace_size", "unif_moe_residual_backward",
           "unif_moe_balance_loss_workspace_size", "unif_moe_balance_loss")
_LIB = None


def lib():
    """The loaded HIP library with these operators' signatures."""
    global _LIB
    if _LIB is None:
        L = _lib.lib()
        vp, sz, i32 = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int32
        resp, szp = ctypes.POINTER(Residual), ctypes.POINTER(sz)
        cfgp, balp = ctypes.POINTER(_lib.Config), ctypes.POINTER(Balance)
        L.unif_moe_residual_forward.argtypes = [resp, vp, vp, vp, vp, vp, vp]
        L.unif_moe_residual_backward_workspace_size.argtypes = [resp, szp]
        L.unif_moe_residual_backward.argtypes = [resp, vp, vp, vp, vp, vp, i32, vp, vp,
                                                 ctypes.POINTER(ResidualGrads), vp, sz, vp]
        L.unif_moe_balance_loss_workspace_size.argtypes = [cfgp, balp, szp]
        L.unif_moe_balance_loss.argtypes = [cfgp, balp, ctypes.POINTER(_lib.Routing), vp, vp, vp, vp, vp, vp, vp, vp,
                                            vp, vp, sz, vp]
        for name in EXPORTS:
            getattr(L, name).restype = i32
        _LIB = L
    return _LIB


def _refuse(where, what):
    e = UnifMoeError(EINVAL, where)
    e.args = (f"{e.args[0]}: {what}",)
    raise e


def _known(where, desc, keys):
    if not keys.issuperset(desc):
        _refuse(where, f"unknown keys {sorted(set(desc) - keys)}")


def _int32(where, desc, key, other=None):
    """An integer of the description; ctypes would cut it to 32 bits."""
    v = int(desc[key] if other is None else desc.get(key, other))
    if not -1 << 31 <= v < 1 << 31:
        _refuse(where, f"{key} {v} is past 32 bits")
    return v


class _Tensors:
    """Checks a call's tensors (all on one GPU) and yields their pointers."""
    __slots__ = ("where", "device")

    def __init__(self, where, device=None):
        self.where, self.device = where, device   # device: index of the tensors' GPU

    def __call__(self, name, t, dtype, numel):
        if t is None:
            return None
        device = t.get_device()
        if t.dtype is dtype and t.numel() == numel and device == self.device and t.is_contiguous():
            return t.data_ptr()
        if device < 0 or not t.is_cuda:
            _refuse(self.where, f"{name} is not on a GPU")
        if t.dtype != dtype:
            _refuse(self.where, f"{name} is {t.dtype}, not {dtype}")
        if t.numel() != numel or not t.is_contiguous():
            _refuse(self.where, f"{name} is not a contiguous tensor of {numel} elements")
        if self.device is not None and device != self.device:
            _refuse(self.where, f"{name} is on GPU {device}, other tensors on GPU {self.device}")
        self.device = device
        return t.data_ptr()

    def workspace(self, t):
        if t is None:
            return None, 0
        return self("workspace", t, t.dtype, t.numel()), t.nbytes

    def call(self, fn, args, stream):
        """fn(*args, stream) with the tensors' device current."""
        import torch
        if self.device is None or self.device == torch.cuda.current_device():
            status = fn(*args, _stream(stream, self.device))
        else:
            with torch.cuda.device(self.device):
                status = fn(*args, _stream(stream, self.device))
        if status != _lib.OK:
            _lib._check(status, self.where)


def _stream(stream, device):
    if stream is None and device is not None:
        import torch
        return torch._C._cuda_getCurrentRawStream(device)
    return _lib._stream(stream)


def _torch_dtype(code):
    import torch
    return torch.bfloat16 if code == _lib.DTYPES["bf16"] else torch.float32


def gate_rows(n_tokens, tokens_per_gate):
    """Rows of a gate: one, or one per tokens_per_gate consecutive tokens."""
    return -(-n_tokens // tokens_per_gate) if tokens_per_gate else 1


def make_residual(desc):
    """Residual structure from a dict: n_tokens, d_model, dtype and
    stream_dtype ("bf16", "f32"; stream_dtype defaults to dtype), out_norm and
    in_norm ("none", "layer", "rms"), out_eps, in_eps, residual_scale (1),
    tokens_per_gate (0), and fp32 device tensors (or None) out_gamma, out_beta,
    in_gamma, in_beta [d] and gate [rows, d]. Calls with the same description
    can share the structure."""
    import torch
    _known("make_residual", desc, RESIDUAL_KEYS)
    n, d = (_int32("make_residual", desc, k) for k in ("n_tokens", "d_model"))
    per = _int32("make_residual", desc, "tokens_per_gate", 0)
    r = Residual(n_tokens=n, d_model=d, dtype=_lib.DTYPES[desc["dtype"]],
                 stream_dtype=_lib.DTYPES[desc.get("stream_dtype", desc["dtype"])],
                 out_norm=ROW_NORMS[desc.get("out_norm", "none")], in_norm=ROW_NORMS[desc.get("in_norm", "none")],
                 tokens_per_gate=per, out_eps=float(desc.get("out_eps", 1e-6)), in_eps=float(desc.get("in_eps", 1e-6)),
                 residual_scale=float(desc.get("residual_scale", 1.0)))
    at = _Tensors("make_residual")
    r.params = {k: desc.get(k) for k in PARAMS}
    for k, t in r.params.items():
        rows = gate_rows(n, per) if k == "gate" and per >= 0 and n >= 0 else 1
        setattr(r, k, at(k, t, torch.float32, rows * d))
    r.device = at.device
    return r


def _residual(res, where):
    r = make_residual(res) if isinstance(res, dict) else res
    return r, _Tensors(where, r.device)


def residual_forward(res, x, f, valid, y, h, stream=None):
    """y = residual_scale x + gate N_out(f) and h = N_in(y) of every token
    (unif_moe_residual_forward); x or f, and y or h, may be None, y may be x."""
    import torch
    r, at = _residual(res, "unif_moe_residual_forward")
    n, s, l = r.n_tokens * r.d_model, _torch_dtype(r.stream_dtype), _torch_dtype(r.dtype)
    args = (ctypes.byref(r), at("x", x, s, n), at("f", f, l, n), at("valid", valid, torch.uint8, r.n_tokens),
            at("y", y, s, n), at("h", h, l, n))
    at.call(lib().unif_moe_residual_forward, args, stream)


def residual_backward_workspace_size(res):
    r, at = _residual(res, "unif_moe_residual_backward_workspace_size")
    size = ctypes.c_size_t(0)
    _lib._check(lib().unif_moe_residual_backward_workspace_size(ctypes.byref(r), ctypes.byref(size)), at.where)
    return size.value


def residual_backward(res, y, f, valid, dy, dh, dx, df, grads, workspace, stream=None):
    """Gradients of the join (unif_moe_residual_backward): dx and df (or
    None), and into ``grads`` (dict by parameter name, or None) those of the
    parameters. dh is fp32 or of the layer's type; dx may be dy."""
    import torch
    r, at = _residual(res, "unif_moe_residual_backward")
    n, s, l = r.n_tokens * r.d_model, _torch_dtype(r.stream_dtype), _torch_dtype(r.dtype)
    h = torch.float32 if dh is None or dh.dtype == torch.float32 else l
    g = ResidualGrads()
    for k, t in (grads or {}).items():
        if k not in PARAMS:
            _refuse(at.where, f"no parameter {k!r}")
        setattr(g, k, at("gradient of " + k, t, torch.float32,
                         r.d_model * (gate_rows(r.n_tokens, r.tokens_per_gate) if k == "gate" else 1)))
    args = (ctypes.byref(r), at("y", y, s, n), at("f", f, l, n), at("valid", valid, torch.uint8, r.n_tokens),
            at("dy", dy, s, n), at("dh", dh, h, n), _lib.DTYPES["f32" if h == torch.float32 else "bf16"],
            at("dx", dx, s, n), at("df", df, l, n), ctypes.byref(g), *at.workspace(workspace))
    at.call(lib().unif_moe_residual_backward, args, stream)


def make_balance(bal):
    """Balance structure from a dict: tokens_per_group (0: one group), unit
    ("tokens", "blocks"), weight (1)."""
    _known("make_balance", bal, BALANCE_KEYS)
    return Balance(tokens_per_group=_int32("make_balance", bal, "tokens_per_group", 0),
                   unit=BALANCE_UNITS[bal.get("unit", "tokens")], weight=float(bal.get("weight", 1.0)))


def balance_loss_workspace_size(cfg, bal):
    c, b = _lib.make_config(cfg), make_balance(bal)
    size = ctypes.c_size_t(0)
    _lib._check(lib().unif_moe_balance_loss_workspace_size(ctypes.byref(c), ctypes.byref(b), ctypes.byref(size)),
                "unif_moe_balance_loss_workspace_size")
    return size.value


def balance_loss(cfg, bal, routing, valid, X, W_router, loss, counts, dX_in, dX, dW_router_in, dW_router, workspace,
                 stream=None):
    """Balance loss over a routing record into ``loss`` [1], the loads into
    ``counts`` [groups, K+1] int64, and weight times the loss's gradient, added
    to dX_in and dW_router_in (or None), into dX and dW_router
    (unif_moe_balance_loss). counts, dX and dW_router may be None, dX may be
    dX_in and dW_router may be dW_router_in."""
    import torch
    c, b = _lib.make_config(cfg), make_balance(bal)
    at = _Tensors("unif_moe_balance_loss")
    N, K, d = c.n_tokens, c.n_experts, c.d_model
    f32, i32 = torch.float32, torch.int32
    kinds = dict(alpha=(f32, N), n_shared=(i32, N), shared_mask=(torch.int64, N), n_res=(i32, N),
                 expert_ids=(i32, N * K), weights=(f32, N * K))
    rec = _lib.Routing(**{k: at("record's " + k, routing[k], *kind) for k, kind in kinds.items()})
    groups = gate_rows(N, b.tokens_per_group)
    args = (ctypes.byref(c), ctypes.byref(b), ctypes.byref(rec), at("valid", valid, torch.uint8, N),
            at("X", X, _torch_dtype(c.dtype), N * d), at("W_router", W_router, f32, (K + 1) * d),
            at("loss", loss, f32, 1), at("counts", counts, torch.int64, groups * (K + 1)),
            at("dX_in", dX_in, f32, N * d), at("dX", dX, f32, N * d),
            at("dW_router_in", dW_router_in, f32, (K + 1) * d), at("dW_router", dW_router, f32, (K + 1) * d),
            *at.workspace(workspace))
    at.call(lib().unif_moe_balance_loss, args, stream)
