"""Device-side plumbing around the bindings: uploads numpy inputs as torch tensors, owns the
output/scratch buffers of one layer, of a sequence of layers or of a training step and hands raw
results back.  No arithmetic of the layers happens here."""
import numpy as np
import torch

from . import adamw, astl, gswa, lnorm, relpos, synth

_PARAMS = ("w_qkv", "b_qkv", "w_proj", "b_proj", "table")


def to_device(a, dtype, device="cuda:0"):
    """numpy fp32 values -> device tensor of storage type 'f32' or 'bf16' (RNE on the host)."""
    if dtype == "f32":
        return torch.from_numpy(np.ascontiguousarray(a, dtype=np.float32)).to(device)
    bits = synth.to_bf16_bits(a).reshape(np.shape(a))
    return torch.from_numpy(bits.view(np.int16)).to(device).view(torch.bfloat16)


def to_host(t):
    return t.detach().float().cpu().numpy()


class DeviceLayer:
    """Buffers of one GSWA layer call on the GPU (inputs, outputs, saved state, scratch)."""

    def __init__(self, B, H, W, C, heads, groups, window, shift, dtype, flags=0, device="cuda:0",
                 dqk=0):
        self.desc = gswa.make_desc(B, H, W, C, heads, groups, window, shift, dtype, flags, dqk)
        self.dtype, self.device = dtype, device
        self.shape = (B, H, W, C)
        tdt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.saved_bytes, self.fwd_ws_bytes, self.bwd_ws_bytes = gswa.gswa_query_bytes(self.desc)
        self.y = torch.empty(self.shape, dtype=tdt, device=device)
        self.dx = torch.empty(self.shape, dtype=tdt, device=device)
        self.saved = torch.empty(self.saved_bytes, dtype=torch.uint8, device=device)
        ws_bytes = max(self.fwd_ws_bytes + self.saved_bytes, self.bwd_ws_bytes)
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        shp = synth.param_shapes(C, heads, groups, window, dqk)
        self.grads = {k: torch.empty(shp[k], dtype=torch.float32, device=device) for k in _PARAMS}
        self.params = None
        self.x = self.dy = None

    def set_params(self, p):
        self.params = {k: to_device(p[k], self.dtype, self.device) for k in _PARAMS}

    def set_inputs(self, x, dy=None):
        self.x = to_device(x, self.dtype, self.device)
        self.dy = None if dy is None else to_device(dy, self.dtype, self.device)

    def forward(self, keep=True, stream=None):
        p = self.params
        gswa.gswa_forward(self.desc, self.x, p["w_qkv"], p["b_qkv"], p["w_proj"], p["b_proj"],
                          p["table"], self.y, self.saved if keep else None, self.ws, stream)

    def backward(self, stream=None):
        p, g = self.params, self.grads
        gswa.gswa_backward(self.desc, self.x, self.dy, p["w_qkv"], p["b_qkv"], p["w_proj"],
                           p["b_proj"], p["table"], self.saved, self.dx, g["w_qkv"], g["b_qkv"],
                           g["w_proj"], g["b_proj"], g["table"], self.ws, stream)

    def results(self):
        out = {"y": to_host(self.y), "dx": to_host(self.dx)}
        out.update({"d" + k: to_host(v) for k, v in self.grads.items()})
        return out


class DeviceBlock:
    """Buffers of one whole-layer call (LayerNorms, attention, MLP, skips) on the GPU."""

    def __init__(self, B, H, W, C, heads, groups, window, shift, dtype, hidden, eps=1e-5, flags=0,
                 device="cuda:0", dqk=0):
        self.desc = astl.make_desc(B, H, W, C, heads, groups, window, shift, dtype, hidden, eps, flags, dqk)
        self.dtype, self.device = dtype, device
        self.shape = (B, H, W, C)
        tdt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.saved_bytes, self.fwd_ws_bytes, self.bwd_ws_bytes = astl.astl_query_bytes(self.desc)
        self.y = torch.empty(self.shape, dtype=tdt, device=device)
        self.dx = torch.empty(self.shape, dtype=tdt, device=device)
        self.saved = torch.empty(self.saved_bytes, dtype=torch.uint8, device=device)
        ws_bytes = max(self.fwd_ws_bytes + self.saved_bytes, self.bwd_ws_bytes)
        self.ws = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
        shp = synth.astl_param_shapes(C, heads, groups, window, hidden, dqk)
        self.grads = {k: torch.empty(s, dtype=torch.float32, device=device) for k, s in shp.items()}
        self.params = None
        self.x = self.dy = None

    @staticmethod
    def _fields(d):
        """synth's names -> the field names of the C structs (the bias table is `table` there)."""
        return {("bias_table" if k == "table" else k): v for k, v in d.items()}

    def set_params(self, p):
        self.params = {k: to_device(v, self.dtype, self.device) for k, v in p.items()}

    def set_inputs(self, x, dy=None):
        self.x = to_device(x, self.dtype, self.device)
        self.dy = None if dy is None else to_device(dy, self.dtype, self.device)

    def forward(self, keep=True, stream=None):
        astl.astl_forward(self.desc, self.x, self._fields(self.params), self.y,
                          self.saved if keep else None, self.ws, stream)

    def backward(self, stream=None):
        astl.astl_backward(self.desc, self.x, self.dy, self._fields(self.params), self.saved, self.dx,
                           self._fields(self.grads), self.ws, stream)

    def results(self):
        out = {"y": to_host(self.y), "dx": to_host(self.dx)}
        out.update({"d" + k: to_host(v) for k, v in self.grads.items()})
        return out


class DeviceStack:
    """Buffers of a sequence of whole layers (alternating shift) behind the stack entry points."""

    def __init__(self, B, H, W, C, heads, groups, window, shift, dtype, hidden, n_layers, checkpoint_every=0,
                 eps=1e-5, flags=0, device="cuda:0", dqk=0, band_windows=0, inference_only=False):
        """band_windows > 0: inference runs band by band (forward(keep=False)), with that many window rows
        per band.  inference_only: no buffers for the backward pass."""
        self.band_windows = band_windows
        self.desc = astl.make_stack_desc(B, H, W, C, heads, groups, window, shift, dtype, hidden, n_layers,
                                         checkpoint_every, eps, flags, dqk)
        self.dtype, self.device, self.n_layers = dtype, device, n_layers
        self.shape = (B, H, W, C)
        tdt = torch.float32 if dtype == "f32" else torch.bfloat16
        self.saved_bytes, self.fwd_ws_bytes, self.bwd_ws_bytes = astl.astl_stack_query_bytes(self.desc)
        self.y = torch.empty(self.shape, dtype=tdt, device=device)
        if band_windows:
            self.fwd_ws_bytes = astl.astl_stack_tiled_query_bytes(self.desc, band_windows)
        if inference_only:
            self.saved_bytes = self.bwd_ws_bytes = 0
            self.dx = self.saved = None
            self.grads = []
        else:
            self.dx = torch.empty(self.shape, dtype=tdt, device=device)
            self.saved = torch.empty(self.saved_bytes, dtype=torch.uint8, device=device)
            shp = synth.astl_param_shapes(C, heads, groups, window, hidden, dqk)
            self.grads = [{k: torch.empty(s, dtype=torch.float32, device=device) for k, s in shp.items()}
                          for _ in range(n_layers)]
        self.ws = torch.empty(max(self.fwd_ws_bytes, self.bwd_ws_bytes), dtype=torch.uint8, device=device)
        self.params = None
        self.x = self.dy = None

    def set_params(self, per_layer):
        self.params = [{k: to_device(v, self.dtype, self.device) for k, v in p.items()} for p in per_layer]

    def set_inputs(self, x, dy=None):
        self.x = to_device(x, self.dtype, self.device)
        self.dy = None if dy is None else to_device(dy, self.dtype, self.device)

    def forward(self, keep=True, stream=None):
        if self.band_windows and not keep:
            astl.astl_stack_forward_tiled(self.desc, self.x, [DeviceBlock._fields(p) for p in self.params], self.y,
                                          self.band_windows, self.ws, stream)
            return
        astl.astl_stack_forward(self.desc, self.x, [DeviceBlock._fields(p) for p in self.params], self.y,
                                self.saved if keep else None, self.ws, stream)

    def forward_tiled(self, band_windows, stream=None):
        """Inference band by band; the scratch is allocated here, at the size the library asks for."""
        need = astl.astl_stack_tiled_query_bytes(self.desc, band_windows)
        ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        astl.astl_stack_forward_tiled(self.desc, self.x, [DeviceBlock._fields(p) for p in self.params], self.y,
                                      band_windows, ws, stream)
        return need

    def backward(self, stream=None):
        astl.astl_stack_backward(self.desc, self.x, self.dy, [DeviceBlock._fields(p) for p in self.params],
                                 self.saved, self.dx, [DeviceBlock._fields(g) for g in self.grads], self.ws, stream)

    def results(self):
        out = {"y": to_host(self.y), "dx": to_host(self.dx)}
        for l, g in enumerate(self.grads):
            out.update({f"{l}.d{k}": to_host(v) for k, v in g.items()})
        return out


class DeviceTrainer:
    """One training step of a sequence of whole layers with a LayerNorm at its end: ``forward`` leaves z = LN(stack(x)), ``backward`` takes
    the loss's gradient ``dz`` to every parameter's, ``update`` is one AdamW step, clipped by the norm of all gradients.  bf16 parameters
    have an fp32 copy.

    ``edges``: the bias tables of the layers come from learned tables of buckets of offsets (see include/relpos.h); None: every row of
    a table is learned.  A step allocates nothing and reads nothing back, so it can be captured into a graph; ``set_params`` and ``set_inputs``
    wait for the steps under way and put new values where the old ones were, so a captured step goes on with them.

    ``skip_nonfinite``: an update whose gradients' norm is infinite or NaN changes nothing, the count of steps included; without it such a
    gradient stays in parameters and states for good.  ``lr_scale``, a value on the device, multiplies the learning rate: a schedule for steps that
    are captured, whose ``lr`` is that of their capture."""

    DECAYED = ("w_qkv", "w_proj", "w_fc1", "w_fc2")

    def __init__(self, B, H, W, C, heads, groups, window, shift, dtype, hidden, n_layers, checkpoint_every=0, eps=1e-5, flags=0,
                 device="cuda:0", dqk=0, edges=None, lr=2e-4, betas=(0.9, 0.999), adam_eps=1e-8, weight_decay=0.01, max_norm=1.0,
                 state_bits=32, seed=0, skip_nonfinite=False):
        if flags & gswa.GSWA_ACCUM_WGRAD:
            raise ValueError("a step's gradients are its own: GSWA_ACCUM_WGRAD is not taken")
        self.stack = DeviceStack(B, H, W, C, heads, groups, window, shift, dtype, hidden, n_layers, checkpoint_every, eps, flags,
                                 device, dqk)
        self.lr, self.weight_decay, self.max_norm = lr, weight_decay, max_norm
        self.norm_desc = lnorm.make_desc(B * H * W, C, dtype, eps)
        self.bias_desc = None if edges is None else relpos.make_desc(heads, edges, dtype, relpos.RELPOS_BIDIRECTIONAL, window=window)
        self.adam_desc = adamw.make_desc(*betas, adam_eps, state_bits, adamw.ADAMW_SKIP_NONFINITE if skip_nonfinite else 0, seed)
        new = lambda *shape, dtype=self.stack.y.dtype: torch.empty(shape, dtype=dtype, device=device)  # noqa: E731
        self.z, self.stack.dy = new(B, H, W, C), new(B, H, W, C)
        self._x, self._dz, self.dz = new(B, H, W, C), new(B, H, W, C), None
        self.grads = {"norm_w": new(C, dtype=torch.float32), "norm_b": new(C, dtype=torch.float32)}
        for l, g in enumerate(self.stack.grads):
            self.grads.update({f"{l}.{k}": v for k, v in g.items() if edges is None or k != "table"})
            if edges is not None:
                self.grads[f"{l}.buckets"] = new(self.bias_desc.buckets, heads, dtype=torch.float32)
        self.norm_ws = new(lnorm.lnorm_query_bytes(self.norm_desc), dtype=torch.uint8)
        self.bias_ws = None if edges is None else new(relpos.relpos_query_bytes(self.bias_desc) + 256, dtype=torch.uint8)
        self.step = torch.zeros(1, dtype=torch.int64, device=device)
        self.grad_norm = torch.zeros((), device=device)
        self.lr_scale = torch.ones((), device=device)
        self.params = self.masters = self.states = self.plan = self.plan_buffer = None

    def set_params(self, per_layer, norm_w, norm_b):
        """per_layer: numpy parameters of each layer as synth.astl_params names them, with ``buckets`` in the place of ``table`` where
        the tables come from buckets.  States and the count of steps start at zero."""
        s = self.stack
        named = {"norm_w": norm_w, "norm_b": norm_b}
        for l, p in enumerate(per_layer):
            named.update({f"{l}.{k}": v for k, v in p.items()})
        if set(named) != set(self.grads):
            raise ValueError(f"parameters missing: {sorted(set(self.grads) - set(named))}, unknown: {sorted(set(named) - set(self.grads))}")
        for k, v in named.items():
            if np.asarray(v).size != self.grads[k].numel():
                raise ValueError(f"{k} has {np.asarray(v).size} values, {self.grads[k].numel()} are needed")
        if self.params is None:
            self._allocate(named, len(per_layer))
        self._settle()
        tensors = []
        for k, v in named.items():
            p, states = self.params[k], self.states[k]
            p.copy_(to_device(v, s.dtype, "cpu").reshape(p.shape))
            tensors.append(dict(states, p=p, g=self.grads[k], weight_decay=self.weight_decay if k.split(".")[-1] in self.DECAYED else 0.0))
            if self.masters:
                tensors[-1]["master"] = self.masters[k]
                self.masters[k].copy_(to_device(v, "f32", "cpu").reshape(p.shape))
            for state in states.values():
                state.zero_()
        self.step.zero_()
        if self.plan_buffer is None:
            self.plan_buffer = torch.empty(adamw.adamw_query_bytes(self.adam_desc, tensors), dtype=torch.uint8, device=s.device)
        self.plan = adamw.adamw_plan(self.adam_desc, tensors, self.plan_buffer)
        self._settle()

    def _allocate(self, named, layers):
        """What a step reads and writes of parameters and states."""
        s, eight = self.stack, self.adam_desc.state_bits == 8
        new = lambda shape, dtype: torch.empty(shape, dtype=dtype, device=s.device)  # noqa: E731
        self.params = {k: new(np.shape(v), s.y.dtype) for k, v in named.items()}
        self.masters = {k: new(np.shape(v), torch.float32) for k, v in named.items()} if s.dtype == "bf16" else {}
        s.params = [{k.split(".")[-1]: v for k, v in self.params.items() if k.startswith(f"{l}.") and not k.endswith(".buckets")}
                    for l in range(layers)]
        if self.bias_desc is not None:
            for p, g in zip(s.params, s.grads):
                p["table"] = new(g["table"].shape, s.y.dtype)
        self.states = {}
        for k, p in self.params.items():
            n = p.numel()
            self.states[k] = {m: new(n, torch.uint8 if eight else torch.float32) for m in ("m", "v")}
            if eight:
                self.states[k].update({m: new(-(-n // adamw.BLOCK), torch.uint8) for m in ("m_exp", "v_exp")})

    def _settle(self):
        """Values change when no step is under way, on whatever stream, and are there for the next one."""
        if self.step.is_cuda:
            torch.cuda.synchronize(self.step.device)

    def set_inputs(self, x, dz=None):
        """Without dz there is nothing for ``backward`` to start from."""
        s, shape = self.stack, self.z.shape
        for a in (x, dz):
            if a is not None and np.asarray(a).size != self.z.numel():
                raise ValueError(f"{np.asarray(a).size} values, {tuple(shape)} are needed")
        self._settle()
        s.x, self.dz = self._x, None if dz is None else self._dz
        for t, a in ((s.x, x), (self.dz, dz)):
            if a is not None:
                t.copy_(to_device(a, s.dtype, "cpu").reshape(shape))
        self._settle()

    def forward(self, stream=None):
        s = self.stack
        if self.bias_desc is not None:
            for l, p in enumerate(s.params):
                relpos.relpos_forward(self.bias_desc, self.params[f"{l}.buckets"], p["table"], stream)
        s.forward(True, stream)
        lnorm.lnorm_forward(self.norm_desc, s.y, None, self.params["norm_w"], self.params["norm_b"], self.z, None, stream)

    def backward(self, stream=None):
        s, g = self.stack, self.grads
        lnorm.lnorm_backward(self.norm_desc, s.y, self.dz, self.params["norm_w"], None, s.dy, g["norm_w"], g["norm_b"], self.norm_ws, stream)
        s.backward(stream)
        if self.bias_desc is not None:
            for l, p in enumerate(s.grads):
                relpos.relpos_backward(self.bias_desc, p["table"], g[f"{l}.buckets"], self.bias_ws, stream)

    def update(self, stream=None):
        adamw.adamw_norm(self.plan, self.grad_norm, stream)
        adamw.adamw_step(self.plan, self.step, self.lr, self.lr_scale, self.grad_norm, self.max_norm, stream)
