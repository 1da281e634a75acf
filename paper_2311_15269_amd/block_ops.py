"""Thin ctypes binding of include/tessel_block_ops.h: the operators that the blocks of a schedule run -- causal attention over
packed sequences, the norms around a block with gate and residual scale, activation checkpoints in 8 bits and their use in
the backward pass.

Tensors are torch's, on the GPU; every call runs on torch's current stream and allocates its outputs and workspace there
(a tensor that another stream wrote is the caller's to wait for, as with torch's own operators).  There is no CPU fallback.
Nothing here records torch's automatic differentiation: forward and backward are two calls.
"""
import ctypes as C
import math

from . import binding

EXPORTS = (
    "tessel_block_last_hip_error", "tessel_packing_create", "tessel_packing_destroy", "tessel_packing_table_bytes", "tessel_packing_bind",
    "tessel_attention_forward", "tessel_attention_backward_workspace_bytes", "tessel_attention_backward",
    "tessel_residual_norm_forward", "tessel_residual_norm_backward_workspace_bytes", "tessel_residual_norm_backward",
    "tessel_checkpoint_store", "tessel_checkpoint_restore", "tessel_gated_forward", "tessel_gated_backward",
    "tessel_weight_gradient_workspace_bytes", "tessel_weight_gradient",
)

E_INVALID_ARG = -1
E_UNSUPPORTED = -9
GROUP = 64
ACT = {"silu": 0, "gelu": 1}
GATE_NONE, GATE_CHANNEL, GATE_TOKEN = 0, 1, 2


class Heads(C.Structure):
    _fields_ = [("data", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("stride", C.c_int64)]


class Attention(C.Structure):
    _fields_ = [("type", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32), ("scale", C.c_float),
                ("q", Heads), ("k", Heads), ("v", Heads), ("o", Heads), ("lse", C.c_void_p), ("d_o", Heads),
                ("dq", Heads), ("dk", Heads), ("dv", Heads)]


class ResidualNorm(C.Structure):
    _fields_ = [("type", C.c_int32), ("gate_kind", C.c_int32), ("tokens", C.c_int64), ("channels", C.c_int32), ("scale", C.c_float),
                ("eps", C.c_float), ("x", Rows), ("y", Rows), ("gate", Rows), ("pre", C.c_void_p), ("post", C.c_void_p),
                ("stats", C.c_void_p), ("r", Rows), ("h", Rows), ("dr", Rows), ("dh", Rows), ("dx", Rows), ("dy", Rows),
                ("dgate", Rows), ("dpre", C.c_void_p), ("dpost", C.c_void_p), ("dgate_channel", C.c_void_p), ("accumulate", C.c_int32)]


class CheckpointDesc(C.Structure):
    _fields_ = [("values", C.c_void_p), ("exponents", C.c_void_p), ("value_stride", C.c_int64), ("exponent_stride", C.c_int64),
                ("tokens", C.c_int64), ("channels", C.c_int32), ("type", C.c_int32)]


class WeightGrad(C.Structure):
    _fields_ = [("x", CheckpointDesc), ("dy", Rows), ("outputs", C.c_int32), ("accumulate", C.c_int32), ("dw", C.c_void_p),
                ("dw_stride", C.c_int64)]


_lib = None


def _library():
    global _lib
    if _lib is None:
        lib = binding.load_library()
        ptr, size = C.c_void_p, C.POINTER(C.c_size_t)
        lib.tessel_packing_create.argtypes = [ptr, C.c_int32, C.c_int64, C.POINTER(C.c_void_p)]
        lib.tessel_packing_destroy.argtypes = [ptr]
        lib.tessel_packing_destroy.restype = None
        lib.tessel_packing_table_bytes.argtypes = [ptr, size]
        lib.tessel_packing_bind.argtypes = [ptr, ptr, C.c_size_t, ptr]
        lib.tessel_attention_forward.argtypes = [ptr, C.POINTER(Attention), ptr]
        lib.tessel_attention_backward_workspace_bytes.argtypes = [ptr, C.POINTER(Attention), size]
        lib.tessel_attention_backward.argtypes = [ptr, C.POINTER(Attention), ptr, C.c_size_t, ptr]
        lib.tessel_residual_norm_forward.argtypes = [C.POINTER(ResidualNorm), ptr]
        lib.tessel_residual_norm_backward_workspace_bytes.argtypes = [C.POINTER(ResidualNorm), size]
        lib.tessel_residual_norm_backward.argtypes = [C.POINTER(ResidualNorm), ptr, C.c_size_t, ptr]
        for f in (lib.tessel_checkpoint_store, lib.tessel_checkpoint_restore):
            f.argtypes = [C.POINTER(CheckpointDesc), C.POINTER(Rows), ptr]
        lib.tessel_gated_forward.argtypes = [C.c_int] + [C.POINTER(Rows)] * 3 + [C.POINTER(CheckpointDesc)] * 2 + [ptr]
        lib.tessel_gated_backward.argtypes = [C.c_int, C.POINTER(Rows)] + [C.POINTER(CheckpointDesc)] * 2 + [C.POINTER(Rows)] * 3 + [ptr]
        lib.tessel_weight_gradient_workspace_bytes.argtypes = [C.POINTER(WeightGrad), size]
        lib.tessel_weight_gradient.argtypes = [C.POINTER(WeightGrad), ptr, C.c_size_t, ptr]
        _lib = lib
    return _lib


def _stream(t):
    import torch
    return torch.cuda.current_stream(t.device).cuda_stream


def _refuse(text):
    raise binding.TesselError(E_INVALID_ARG, text)


def _type(t):
    import torch
    code = {torch.bfloat16: 0, torch.float16: 1, torch.float32: 2}.get(t.dtype)
    if code is None:
        raise binding.TesselError(E_UNSUPPORTED, "no operator for tensors of type %s" % t.dtype)
    return code


def _same(like, shape, *tensors):
    """all on the GPU of `like`, of its type and of this shape"""
    for t in tensors:
        if not t.is_cuda or t.device != like.device or t.dtype != like.dtype or tuple(t.shape) != tuple(shape):
            _refuse("expected a %s tensor of shape %s on %s, got %s %s on %s" % (like.dtype, tuple(shape), like.device, t.dtype, tuple(t.shape), t.device))


def _heads(t):
    """a [tokens, heads, dim] tensor; one whose last dimension is not contiguous, or whose strides or start are not multiples of
    16 bytes, is refused"""
    if t.shape[2] > 1 and t.stride(2) != 1:
        _refuse("the last dimension has to be contiguous")
    return Heads(t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1] * t.shape[2], t.stride(1) if t.shape[1] > 1 else t.shape[2])


def _rows(t):
    if t.dim() != 2 or (t.shape[1] > 1 and t.stride(1) != 1):
        _refuse("expected [tokens, channels] with contiguous channels, got strides %s" % (t.stride(),))
    return Rows(t.data_ptr(), t.stride(0) if t.shape[0] > 1 else t.shape[1])


def _vector(t, channels, like):
    import torch
    if t.dtype != torch.float32 or tuple(t.shape) != (channels,) or (channels > 1 and t.stride(0) != 1) or t.device != like.device:
        _refuse("expected %d contiguous 32-bit numbers on %s, got %s %s" % (channels, like.device, t.dtype, tuple(t.shape)))
    return t.data_ptr()


def _workspace(n, like):
    import torch
    return torch.empty(max(16, n), dtype=torch.uint8, device=like.device)


class Packing:
    """tessel_packing_*: sequences of these lengths one behind the other in total_tokens tokens (default: their sum), and attention over
    them.  Holds the device table of their tiles; made once, it serves any layer, stream and head layout."""

    def __init__(self, lengths, total_tokens=None, device=None):
        import torch
        lib = _library()
        self.lengths = [int(n) for n in lengths]
        self.tokens = sum(self.lengths) if total_tokens is None else int(total_tokens)
        array = (C.c_int32 * max(1, len(self.lengths)))(*self.lengths)
        h = C.c_void_p()
        binding._check(lib.tessel_packing_create(array, len(self.lengths), self.tokens, C.byref(h)))
        self._h = h
        n = C.c_size_t()
        binding._check(lib.tessel_packing_table_bytes(h, C.byref(n)))
        self._table = torch.empty(n.value, dtype=torch.uint8, device="cuda" if device is None else device)
        self._made_on = _stream(self._table)
        binding._check(lib.tessel_packing_bind(h, self._table.data_ptr(), n.value, self._made_on))

    def close(self):
        if getattr(self, "_h", None) and _lib is not None:
            _lib.tessel_packing_destroy(self._h)
        self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:       # interpreter shutdown
            pass

    def _describe(self, q, k, v, scale):
        import torch
        if q.dim() != 3 or k.dim() != 3 or q.device != self._table.device:
            _refuse("expected [tokens, heads, dim] on %s" % self._table.device)
        heads, dim = q.shape[1], q.shape[2]
        _same(q, (self.tokens, heads, dim), q)
        _same(q, (self.tokens, k.shape[1], dim), k, v)
        scale = 1 / math.sqrt(max(1, dim)) if scale is None else scale
        if _stream(q) != self._made_on:                     # (the table must not be given away while that stream still reads it)
            self._table.record_stream(torch.cuda.current_stream(q.device))
        return Attention(type=_type(q), heads=heads, kv_heads=k.shape[1], dim=dim, scale=scale, q=_heads(q), k=_heads(k), v=_heads(v))

    def attention(self, q, k, v, scale=None):
        """tessel_attention_forward: q [tokens, heads, dim], k and v [tokens, kv_heads, dim] -> (o like q, lse [heads, tokens])"""
        import torch
        a = self._describe(q, k, v, scale)
        o = torch.empty(q.shape, dtype=q.dtype, device=q.device)
        lse = torch.empty(q.shape[1], self.tokens, dtype=torch.float32, device=q.device)
        a.o, a.lse = _heads(o), lse.data_ptr()
        binding._check(_library().tessel_attention_forward(self._h, C.byref(a), _stream(q)))
        return o, lse

    def attention_backward(self, d_o, q, k, v, o, lse, scale=None):
        """tessel_attention_backward: (dq, dk, dv) from the gradient of o and what the forward call took and gave"""
        import torch
        lib = _library()
        a = self._describe(q, k, v, scale)
        _same(q, q.shape, d_o, o)
        if lse.dtype != torch.float32 or tuple(lse.shape) != (q.shape[1], self.tokens) or not lse.is_contiguous() or lse.device != q.device:
            _refuse("lse is not what the forward call gave")
        dq, dk, dv = (torch.empty(t.shape, dtype=t.dtype, device=t.device) for t in (q, k, v))
        a.o, a.lse, a.d_o, a.dq, a.dk, a.dv = _heads(o), lse.data_ptr(), _heads(d_o), _heads(dq), _heads(dk), _heads(dv)
        n = C.c_size_t()
        binding._check(lib.tessel_attention_backward_workspace_bytes(self._h, C.byref(a), C.byref(n)))
        ws = _workspace(n.value, q)
        binding._check(lib.tessel_attention_backward(self._h, C.byref(a), ws.data_ptr(), ws.numel(), _stream(q)))
        return dq, dk, dv


def _describe_norm(x, y, pre, post, gate, scale, eps):
    if x.dim() != 2:
        _refuse("expected [tokens, channels]")
    _same(x, x.shape, x, y)
    n, c = x.shape
    a = ResidualNorm(type=_type(x), tokens=n, channels=c, scale=scale, eps=eps, x=_rows(x), y=_rows(y), pre=_vector(pre, c, x),
                     post=None if post is None else _vector(post, c, x))
    if gate is None:
        a.gate_kind = GATE_NONE
    elif gate.dim() == 1:
        a.gate_kind, a.gate = GATE_CHANNEL, Rows(_vector(gate, c, x), 0)
    else:
        _same(x, x.shape, gate)
        a.gate_kind, a.gate = GATE_TOKEN, _rows(gate)
    return a


def residual_norm(x, y, pre, post=None, gate=None, scale=1.0, eps=1e-6):
    """tessel_residual_norm_forward: (r, h, stats) with r = scale x + gate n(y, post), h = n(r, pre).  post None: y itself; gate:
    None, [channels] in 32 bits or [tokens, channels] like x."""
    import torch
    a = _describe_norm(x, y, pre, post, gate, scale, eps)
    r, h = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for _ in range(2))
    stats = torch.empty(2, x.shape[0], dtype=torch.float32, device=x.device)
    a.r, a.h, a.stats = _rows(r), _rows(h), stats.data_ptr()
    binding._check(_library().tessel_residual_norm_forward(C.byref(a), _stream(x)))
    return r, h, stats


def residual_norm_backward(dr, dh, x, y, stats, pre, post=None, gate=None, scale=1.0, into=None):
    """tessel_residual_norm_backward: (dx, dy, dpre, dpost, dgate), None for what the forward call did not have.  `into`: (dpre, dpost,
    dgate) of earlier micro-batches, to which the parameters' gradients are added (dgate: of a gate for the channels)."""
    import torch
    lib = _library()
    a = _describe_norm(x, y, pre, post, gate, scale, 0.0)
    _same(x, x.shape, dr, dh)
    if stats.dtype != torch.float32 or tuple(stats.shape) != (2, x.shape[0]) or not stats.is_contiguous() or stats.device != x.device:
        _refuse("stats is not what the forward call gave")
    dx, dy = (torch.empty(x.shape, dtype=x.dtype, device=x.device) for _ in range(2))
    a.stats, a.dr, a.dh, a.dx, a.dy = stats.data_ptr(), _rows(dr), _rows(dh), _rows(dx), _rows(dy)
    dpre, dpost, dgate = into if into is not None else (None, None, None)
    c = x.shape[1]
    if into is None:
        dpre = torch.empty(c, dtype=torch.float32, device=x.device)
        dpost = torch.empty_like(dpre) if post is not None else None
        dgate = torch.empty_like(dpre) if a.gate_kind == GATE_CHANNEL else None
    a.accumulate = 0 if into is None else 1
    a.dpre = _vector(dpre, c, x)
    if post is not None:
        a.dpost = _vector(dpost, c, x)
    if a.gate_kind == GATE_CHANNEL:
        a.dgate_channel = _vector(dgate, c, x)
    elif a.gate_kind == GATE_TOKEN:
        dgate = torch.empty(x.shape, dtype=x.dtype, device=x.device)
        a.dgate = _rows(dgate)
    n = C.c_size_t()
    binding._check(lib.tessel_residual_norm_backward_workspace_bytes(C.byref(a), C.byref(n)))
    ws = _workspace(n.value, x)
    binding._check(lib.tessel_residual_norm_backward(C.byref(a), ws.data_ptr(), ws.numel(), _stream(x)))
    return dx, dy, dpre, dpost, dgate


class Checkpoint:
    """An activation [tokens, channels] in 8 bits: `values` [tokens, channels up to the next multiple of 64] and `exponents`
    [tokens, groups of 64 channels], of a tensor of type `dtype`."""

    def __init__(self, tokens, channels, dtype, device):
        import torch
        groups = -(-channels // GROUP)
        self.tokens, self.channels, self.dtype, self.device = tokens, channels, dtype, torch.device(device)
        self.values = torch.empty(tokens, groups * GROUP, dtype=torch.int8, device=device)
        self.exponents = torch.empty(tokens, groups, dtype=torch.uint8, device=device)

    @property
    def nbytes(self):
        return self.values.numel() + self.exponents.numel()

    def _desc(self):
        import torch
        return CheckpointDesc(self.values.data_ptr(), self.exponents.data_ptr(), self.values.shape[1], self.exponents.shape[1], self.tokens,
                              self.channels, _type(torch.empty(0, dtype=self.dtype)))

    def _like(self, *tensors):
        for t in tensors:
            if not t.is_cuda or t.device != self.values.device or t.dtype != self.dtype or tuple(t.shape) != (self.tokens, self.channels):
                _refuse("expected %s [%d, %d] on %s, got %s %s" % (self.dtype, self.tokens, self.channels, self.values.device, t.dtype, tuple(t.shape)))


def _new_checkpoint(x):
    if x.dim() != 2 or not x.is_cuda:
        _refuse("expected [tokens, channels] on the GPU")
    _type(x)
    return Checkpoint(x.shape[0], x.shape[1], x.dtype, x.device)


def checkpoint(x):
    """tessel_checkpoint_store: x [tokens, channels] in 8 bits"""
    c = _new_checkpoint(x)
    binding._check(_library().tessel_checkpoint_store(C.byref(c._desc()), C.byref(_rows(x)), _stream(x)))
    return c


def restore(c):
    """tessel_checkpoint_restore: what a checkpoint stands for, in the type of what was stored"""
    import torch
    x = torch.empty(c.tokens, c.channels, dtype=c.dtype, device=c.values.device)
    binding._check(_library().tessel_checkpoint_restore(C.byref(c._desc()), C.byref(_rows(x)), _stream(x)))
    return x


def _act(act):
    if act not in ACT:
        _refuse("no activation %r: one of %s" % (act, ", ".join(ACT)))
    return ACT[act]


def gated(g, u, act="silu"):
    """tessel_gated_forward: (a, checkpoint of g, checkpoint of u) with a = act(g) u"""
    import torch
    kind = _act(act)
    kg, ku = _new_checkpoint(g), _new_checkpoint(u)
    kg._like(u)
    a = torch.empty(g.shape, dtype=g.dtype, device=g.device)
    binding._check(_library().tessel_gated_forward(kind, C.byref(_rows(g)), C.byref(_rows(u)), C.byref(_rows(a)), C.byref(kg._desc()),
                                                   C.byref(ku._desc()), _stream(g)))
    return a, kg, ku


def gated_backward(da, kg, ku, act="silu", with_output=False):
    """tessel_gated_backward: (dg, du), or (dg, du, a) with the checkpoints' own act(g) u"""
    import torch
    kind = _act(act)
    kg._like(da)
    dg, du = (torch.empty(da.shape, dtype=da.dtype, device=da.device) for _ in range(2))
    a = torch.empty(da.shape, dtype=da.dtype, device=da.device) if with_output else None
    binding._check(_library().tessel_gated_backward(kind, C.byref(_rows(da)), C.byref(kg._desc()), C.byref(ku._desc()), C.byref(_rows(dg)),
                                                    C.byref(_rows(du)), C.byref(_rows(a)) if with_output else None, _stream(da)))
    return (dg, du, a) if with_output else (dg, du)


def weight_gradient(dy, x, into=None):
    """tessel_weight_gradient: dy^T x [outputs, channels] in 32 bits, for dy [tokens, outputs] and a checkpoint x [tokens, channels]; added
    to `into` (and that returned) if it is given"""
    import torch
    lib = _library()
    if dy.dim() != 2 or not dy.is_cuda or dy.device != x.values.device or dy.dtype != x.dtype or dy.shape[0] != x.tokens:
        _refuse("dy %s %s does not go with a checkpoint of %s [%d, %d]" % (dy.dtype, tuple(dy.shape), x.dtype, x.tokens, x.channels))
    shape = (dy.shape[1], x.channels)
    if into is not None and (into.dtype != torch.float32 or tuple(into.shape) != shape or into.device != dy.device or (shape[1] > 1 and into.stride(1) != 1)):
        _refuse("the sum has to be 32-bit %s on %s" % (shape, dy.device))
    dw = torch.empty(shape, dtype=torch.float32, device=dy.device) if into is None else into
    a = WeightGrad(x=x._desc(), dy=_rows(dy), outputs=shape[0], accumulate=0 if into is None else 1, dw=dw.data_ptr(),
                   dw_stride=dw.stride(0) if shape[0] > 1 else shape[1])
    n = C.c_size_t()
    binding._check(lib.tessel_weight_gradient_workspace_bytes(C.byref(a), C.byref(n)))
    ws = _workspace(n.value, dy)
    binding._check(lib.tessel_weight_gradient(C.byref(a), ws.data_ptr(), ws.numel(), _stream(dy)))
    return dw
