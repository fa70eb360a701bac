"""Device-resident UniF-MoE layer: moves one layer's inputs to the GPU once
and calls the HIP library on them (torch supplies memory and streams)."""
import contextlib
import functools
import inspect
import math

import numpy as np

from . import _lib, ops


def to_device(a, dtype_name, device, name="array", shape=None):
    """numpy array or torch tensor -> contiguous torch device tensor of the
    format: bf16 data arrives as 16-bit words (or as a bfloat16 tensor), f32
    data as float32. Other types are refused, and with ``shape`` what does not
    hold it: other sizes, unless only the first dimension is larger. A device
    tensor that is laid out so already is used as it is, without a copy."""
    import torch
    if a is None:
        return None
    if not torch.is_tensor(a):
        a = np.ascontiguousarray(a)
        if dtype_name == "bf16" and (a.dtype.kind not in "fc" or a.dtype.name == "bfloat16"):
            a = a.view(np.int16)   # the words, however they are typed
        a = torch.from_numpy(a)
    if dtype_name == "bf16" and a.dtype in (torch.int16, torch.uint16):
        a = a.view(torch.bfloat16)
    want = torch.bfloat16 if dtype_name == "bf16" else torch.float32
    if a.dtype != want:
        ops._refuse("to_device", f"{name} is {a.dtype}, not {want}")
    if shape is not None and a.numel() != math.prod(shape):
        if a.dim() != len(shape) or a.shape[1:] != shape[1:] or a.shape[0] < shape[0]:
            ops._refuse("to_device", f"{name} is {tuple(a.shape)}, not {tuple(shape)}")
    return a.to(device).contiguous()


def _on_stream(method):
    """Runs ``method`` with its ``stream`` argument (a torch stream, another
    object's ``cuda_stream``, a raw handle, or None: the layer's device's current
    one) current, and so its device: what it allocates belongs to that stream, so
    memory it frees on return is not handed out before the stream's work on it is
    done."""
    args_of = inspect.signature(method).parameters
    at = list(args_of).index("stream") - 1   # among the arguments behind self
    by_position = args_of["stream"].kind is inspect.Parameter.POSITIONAL_OR_KEYWORD

    @functools.wraps(method)
    def run(self, *args, **kwargs):
        import torch
        given = by_position and len(args) > at
        stream = args[at] if given else kwargs.get("stream")
        device = getattr(self, "layer", self).Y.get_device()
        if not isinstance(stream, torch.cuda.Stream):
            stream = getattr(stream, "cuda_stream", stream)
        if isinstance(stream, int):
            # 0 is the null stream's handle, which ExternalStream takes for none at all
            stream = torch.cuda.ExternalStream(stream, device=device) if stream else torch.cuda.default_stream(device)
        if given:
            args = (*args[:at], stream, *args[at + 1:])
        else:
            kwargs["stream"] = stream
        here = device >= 0 and device == torch.cuda.current_device()
        if stream is None:
            apart = None if here or device < 0 else torch.cuda.device(device)
        else:   # to enter a stream takes 6 us of the host's time, to see that it is current 1
            apart = None if here and ops._stream(None, device) == stream.cuda_stream else torch.cuda.stream(stream)
        with apart or contextlib.nullcontext():
            return method(self, *args, **kwargs)
    return run


class DeviceLayer:
    """Inputs of one layer on the device, plus output, record and workspace.

    ``cfg`` is a layer description dict (dtype "bf16" or "f32"); arrays are
    numpy: X and the expert weights as bf16 bits (uint16) or float32 (or
    tensors, see to_device), the router and prototypes as float32, ``valid`` as
    uint8 or None. The calls share the output, the record and the workspaces:
    those on different streams, and replays of graphs that hold such calls, are
    ordered by the caller, who keeps the layer until their work is done.
    """

    def __init__(self, cfg, X, valid, W_router, prototypes, W_up=None, W_down=None,
                 device="cuda:0"):
        import torch
        self.cfg = dict(cfg)
        self.device = device
        dt = cfg["dtype"]
        N, d, K = cfg["n_tokens"], cfg["d_model"], cfg["n_experts"]
        H = cfg["n_blocks"] * cfg["block_width"]
        self.X = to_device(X, dt, device, "X", (N, d))
        self.valid = None if valid is None else torch.from_numpy(np.ascontiguousarray(valid, np.uint8)).to(device)
        self.W_router = to_device(np.asarray(W_router, np.float32), "f32", device)
        self.prototypes = to_device(np.asarray(prototypes, np.float32), "f32", device)
        self.W_up = to_device(W_up, dt, device, "W_up", (K + 1, H, d))
        self.W_down = to_device(W_down, dt, device, "W_down", (K + 1, d, H))
        self.Y = torch.empty((N, d), dtype=torch.bfloat16 if dt == "bf16" else torch.float32,
                             device=device)
        self.routing = _lib.alloc_routing(N, K, device)
        self.ws_forward = None
        self.ws_route = None
        self.ws_stats = None

    @_on_stream
    def forward(self, stream=None, routing=True):
        if self.ws_forward is None:
            self.ws_forward = _lib.alloc_workspace(_lib.layer_forward_workspace_size(self.cfg), self.device)
        _lib.layer_forward(self.cfg, self.X, self.valid, self.W_router, self.prototypes,
                           self.W_up, self.W_down, self.Y, self.ws_forward,
                           routing=self.routing if routing else None, stream=stream)
        return self.Y

    @_on_stream
    def block_forward(self, blk, X=None, stream=None, routing=True):
        """The transformer block around the layer (``blk`` as
        synth.block_inputs returns it: numpy parameters, moved to the device
        on each call). ``X`` replaces the layer input (the residual stream)."""
        c = self.cfg
        Xd = self.X if X is None else to_device(X, c["dtype"], self.device, "X", (c["n_tokens"], c["d_model"]))
        b = dict(norm=blk["norm"], residual=blk["residual"], ln_eps=blk["ln_eps"])
        for k in ("ln_gamma", "ln_beta", "b_up", "b_down"):
            b[k] = None if blk.get(k) is None else to_device(np.asarray(blk[k], np.float32), "f32",
                                                              self.device)
        ws = _lib.alloc_workspace(_lib.block_forward_workspace_size(self.cfg, b), self.device)
        _lib.block_forward(self.cfg, b, Xd, self.valid, self.W_router, self.prototypes,
                           self.W_up, self.W_down, self.Y, ws,
                           routing=self.routing if routing else None, stream=stream)
        return self.Y

    @_on_stream
    def backward(self, dY, stream=None):
        """Gradients of sum(dY * Y) (dY in the layer's format, see to_device): dict of
        fp32 device tensors dX, dW_up, dW_down, dW_router."""
        import torch
        c = self.cfg
        N, d, K = c["n_tokens"], c["d_model"], c["n_experts"]
        H = c["n_blocks"] * c["block_width"]
        dYd = to_device(dY, c["dtype"], self.device, "dY", (N, d))
        f = dict(dtype=torch.float32, device=self.device)
        g = dict(dX=torch.empty((N, d), **f), dW_up=torch.empty((K + 1, H, d), **f),
                 dW_down=torch.empty((K + 1, d, H), **f), dW_router=torch.empty((K + 1, d), **f))
        ws = _lib.alloc_workspace(_lib.layer_backward_workspace_size(c), self.device)
        _lib.layer_backward(c, self.X, self.valid, self.W_router, self.prototypes, self.W_up,
                            self.W_down, dYd, g["dX"], g["dW_up"], g["dW_down"], g["dW_router"], ws,
                            stream=stream)
        return g

    @_on_stream
    def diversity_loss(self, weight, dW_router, *, stream=None):
        """L_div of the router as a device scalar; weight times its gradient is
        added to ``dW_router``."""
        import torch
        loss = torch.empty(1, dtype=torch.float32, device=self.device)
        ws = _lib.alloc_workspace(_lib.diversity_loss_workspace_size(self.cfg), self.device)
        _lib.diversity_loss(self.cfg, self.W_router, weight, loss, dW_router, ws, stream=stream)
        return loss

    @_on_stream
    def balance_loss(self, bal, dX=None, dW_router=None, *, stream=None):
        """Balance loss and per-expert loads (device tensors) over the layer's
        routing record, which forward and route leave there for the layer's X (not
        a forward without the record, and not block_forward, whose layer sees
        another input); weight times the loss's gradient is added to ``dX`` and
        ``dW_router`` where given."""
        import torch
        c = self.cfg
        rows = ops.gate_rows(c["n_tokens"], bal.get("tokens_per_group", 0))
        loss = torch.empty(1, dtype=torch.float32, device=self.device)
        counts = torch.empty((rows, c["n_experts"] + 1), dtype=torch.int64, device=self.device)
        ws = _lib.alloc_workspace(ops.balance_loss_workspace_size(c, bal), self.device)
        ops.balance_loss(c, bal, self.routing, self.valid, self.X, self.W_router, loss, counts, dX, dX, dW_router,
                         dW_router, ws, stream=stream)
        return loss, counts

    @_on_stream
    def route(self, out=None, stream=None):
        if self.ws_route is None:
            self.ws_route = _lib.alloc_workspace(_lib.route_workspace_size(self.cfg), self.device)
        out = self.routing if out is None else out
        _lib.route(self.cfg, self.X, self.valid, self.W_router, self.prototypes, out,
                   self.ws_route, stream=stream)
        return out

    @_on_stream
    def stats(self, stream=None):
        if self.ws_stats is None:
            self.ws_stats = _lib.alloc_workspace(_lib.stats_workspace_size(self.cfg), self.device)
        return _lib.stats(self.cfg, self.routing, self.valid, self.ws_stats, stream=stream)

    def routing_numpy(self):
        r = {k: v.cpu().numpy() for k, v in self.routing.items()}
        r["shared_mask"] = r["shared_mask"].view(np.uint64)
        return r

    def output_numpy(self):
        import torch
        if self.cfg["dtype"] == "bf16":
            return self.Y.view(torch.int16).cpu().numpy().view(np.uint16)
        return self.Y.cpu().numpy()


class DeviceBlock:
    """A block around the layer in training: y = residual_scale x + gate
    N_out(F(N_in(x))), with F the layer, and the gradients of a loss of y with
    the balance loss and the diversity loss added.

    ``params`` is the join's description (ops.make_residual) without sizes and
    types; its in_norm ("layer" or "rms": the layer's input is always N_in's)
    belongs to N_in in front of the layer, the rest to the join behind it.
    ``stream_dtype`` is the residual stream's type. A forward leaves the layer's
    input and output in ``layer`` (X, Y and the record), where the backward of
    the last forward finds them. Each direction is two calls of the join's
    operators, N_in alone and the join without a next norm: 10 bytes an element
    in bf16 forward and 18 backward, where one call with the next block's N_in
    moves 8 and 14. In bf16 dx is rounded once by each of the two.
    """

    def __init__(self, layer, params, stream_dtype=None):
        self.layer, self.params = layer, dict(params)
        c = layer.cfg
        size = dict(n_tokens=c["n_tokens"], d_model=c["d_model"], dtype=c["dtype"],
                    stream_dtype=stream_dtype or c["dtype"])
        before = {k: v for k, v in params.items() if k in ("in_norm", "in_eps", "in_gamma", "in_beta")}
        behind = {k: v for k, v in params.items() if k not in before}
        self.before = ops.make_residual(dict(size, **before))
        self.behind = ops.make_residual(dict(size, **behind))

    @_on_stream
    def forward(self, x, *, stream=None):
        import torch
        L = self.layer
        L.X = torch.empty((L.cfg["n_tokens"], L.cfg["d_model"]), dtype=L.Y.dtype, device=L.device)
        ops.residual_forward(self.before, x, None, L.valid, None, L.X, stream=stream)
        f = L.forward(stream=stream)
        y = torch.empty_like(x)
        ops.residual_forward(self.behind, x, f, L.valid, y, None, stream=stream)
        return y

    @_on_stream
    def backward(self, x, dy, balance=None, diversity=0.0, *, stream=None):
        """Gradients of the last forward: dx, the layer's (dW_up, dW_down,
        dW_router) and the parameters', and the losses."""
        import torch
        L = self.layer
        like = {k: torch.empty_like(v) for k, v in self.params.items() if k in ops.PARAMS and v is not None}
        df, dx = torch.empty_like(L.Y), torch.empty_like(dy)
        ws = [_lib.alloc_workspace(ops.residual_backward_workspace_size(r), L.device)
              for r in (self.behind, self.before)]
        ops.residual_backward(self.behind, None, L.Y, L.valid, dy, None, dx, df,
                              {k: v for k, v in like.items() if not k.startswith("in_")}, ws[0], stream=stream)
        g = L.backward(df, stream=stream)
        if balance is not None:
            g["balance"], g["counts"] = L.balance_loss(balance, g["dX"], g["dW_router"], stream=stream)
        if diversity:
            g["diversity"] = L.diversity_loss(diversity, g["dW_router"], stream=stream)
        ops.residual_backward(self.before, x, None, L.valid, dx, g.pop("dX"), dx, None,
                              {k: v for k, v in like.items() if k.startswith("in_")}, ws[1], stream=stream)
        return dict(g, dx=dx, **like)
