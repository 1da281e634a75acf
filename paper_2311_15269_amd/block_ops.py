"""Thin ctypes binding of include/tessel_block_ops.h: the operators that the blocks of a schedule run -- causal attention over
packed sequences, the norms around a block with gate and residual scale, activation checkpoints in 8 bits and their use in
the backward pass.

Tensors are torch's, on the GPU; every call runs on torch's current stream and allocates its outputs and workspace there
(a tensor that another stream wrote is the caller's to wait for, as with torch's own operators).  There is no CPU fallback.
Nothing here records torch's automatic differentiation: forward and backward are two calls, and a tensor that requires a gradient is
refused while torch records (under torch.no_grad(), and in the passes of a torch.autograd.Function, it is taken as it is).
"""
import ctypes as C
import math

from . import binding

EXPORTS = (
    "tessel_block_last_hip_error", "tessel_packing_create", "tessel_packing_destroy", "tessel_packing_table_bytes", "tessel_packing_bind",
    "tessel_attention_forward_workspace_bytes", "tessel_attention_forward", "tessel_attention_backward_workspace_bytes", "tessel_attention_backward",
    "tessel_residual_norm_forward", "tessel_residual_norm_backward_workspace_bytes", "tessel_residual_norm_backward",
    "tessel_checkpoint_store", "tessel_checkpoint_restore", "tessel_gated_forward", "tessel_gated_backward",
    "tessel_weight_gradient_workspace_bytes", "tessel_weight_gradient",
)

E_INVALID_ARG = -1
E_TOOBIG = -4
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


def _flat(struct):
    """The same layout with the fields of the structures inside side by side: one call fills it, which is most of what a small call costs
    on the host."""
    fields = []
    for name, kind in struct._fields_:
        fields += [(name + "_" + n, k) for n, k in kind._fields_] if issubclass(kind, C.Structure) else [(name, kind)]
    flat = type("Flat" + struct.__name__, (C.Structure,), {"_fields_": fields})
    assert C.sizeof(flat) == C.sizeof(struct)
    return flat


_FlatAttention, _FlatNorm, _FlatWeight = _flat(Attention), _flat(ResidualNorm), _flat(WeightGrad)
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
        # (structures by address: the nested ones above and their flat twins alike)
        lib.tessel_attention_forward_workspace_bytes.argtypes = [ptr, ptr, size]
        lib.tessel_attention_forward.argtypes = [ptr, ptr, ptr, C.c_size_t, ptr]
        lib.tessel_attention_backward_workspace_bytes.argtypes = [ptr, ptr, size]
        lib.tessel_attention_backward.argtypes = [ptr, ptr, ptr, C.c_size_t, ptr]
        lib.tessel_residual_norm_forward.argtypes = [ptr, ptr]
        lib.tessel_residual_norm_backward_workspace_bytes.argtypes = [ptr, size]
        lib.tessel_residual_norm_backward.argtypes = [ptr, ptr, C.c_size_t, ptr]
        for f in (lib.tessel_checkpoint_store, lib.tessel_checkpoint_restore):
            f.argtypes = [ptr, ptr, ptr]
        lib.tessel_gated_forward.argtypes = [C.c_int] + [ptr] * 6
        lib.tessel_gated_backward.argtypes = [C.c_int] + [ptr] * 7
        lib.tessel_weight_gradient_workspace_bytes.argtypes = [ptr, size]
        lib.tessel_weight_gradient.argtypes = [ptr, ptr, C.c_size_t, ptr]
        _lib = lib
    return _lib


def _refuse(text):
    raise binding.TesselError(E_INVALID_ARG, text)


MOST = 0x7FFFFFFF       # that the structures' 32-bit fields hold: of more they take the low bits without a word


def _too_big(size):
    raise binding.TesselError(E_TOOBIG, "%d does not fit 32 bits" % size)


def _stream(t):
    """the current stream, which is one of the current GPU, so that a tensor of another one is refused"""
    import torch
    if t.is_cuda and t.get_device() != torch.cuda.current_device():
        _refuse("a tensor on %s, but the current GPU is number %d" % (t.device, torch.cuda.current_device()))
    raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
    return torch.cuda.current_stream(t.device).cuda_stream if raw is None else raw(t.get_device())


def _refuse_gradient(t):
    import torch
    if torch.is_grad_enabled():
        _refuse("a tensor of shape %s requires a gradient, which no operator here records: detach it or call under torch.no_grad()" % (tuple(t.shape),))


_TYPES = {}


def _type(t):
    import torch
    if not _TYPES:
        _TYPES.update({torch.bfloat16: 0, torch.float16: 1, torch.float32: 2})
    code = _TYPES.get(t.dtype)
    if code is None:
        raise binding.TesselError(E_UNSUPPORTED, "no operator for tensors of type %s" % t.dtype)
    return code


def _same(like, shape, *tensors):
    """all on the GPU of `like`, of its type and of this shape"""
    dtype, at = like.dtype, like.get_device()
    for t in tensors:
        if not t.is_cuda or t.dtype is not dtype or t.shape != shape or t.get_device() != at:
            _refuse("expected a %s tensor of shape %s on %s, got %s %s on %s" % (like.dtype, tuple(shape), like.device, t.dtype, tuple(t.shape), t.device))
        if t.requires_grad:
            _refuse_gradient(t)


def _heads(t):
    """a [tokens, heads, dim] tensor: start and strides.  One whose last dimension is not contiguous, or whose strides or start are not
    multiples of 16 bytes, is refused."""
    n, heads, dim = t.shape
    token, head, last = t.stride()
    if last != 1 and dim > 1:
        _refuse("the last dimension has to be contiguous")
    return t.data_ptr(), token if n > 1 else heads * dim, head if heads > 1 else dim


def _rows(t):
    """a [tokens, channels] tensor: start and stride"""
    stride = t.stride()
    if len(stride) != 2 or (stride[1] != 1 and t.shape[1] > 1):
        _refuse("expected [tokens, channels] with contiguous channels, got strides %s" % (stride,))
    return t.data_ptr(), stride[0] if t.shape[0] > 1 else t.shape[1]


def _vector(t, channels, like):
    if _type(t) != 2 or t.shape != (channels,) or not t.is_contiguous() or t.get_device() != like.get_device():
        _refuse("expected %d contiguous 32-bit numbers on %s, got %s %s" % (channels, like.device, t.dtype, tuple(t.shape)))
    if t.requires_grad:
        _refuse_gradient(t)
    return t.data_ptr()


def _like(t):
    """a contiguous tensor of the same shape, type and place (half the time of torch.empty with all of them)"""
    import torch
    return torch.empty_like(t, memory_format=torch.contiguous_format)


def _workspace(n, like):
    import torch
    return like.new_empty((max(16, n),), dtype=torch.uint8)


class Packing:
    """tessel_packing_*: sequences of these lengths one behind the other in total_tokens tokens (default: their sum), and attention over
    them.  Holds the device table of their tiles; made once, it serves any layer, stream and head layout."""

    def __init__(self, lengths, total_tokens=None, device=None):
        import torch
        lib = _library()
        self.lengths = [int(n) for n in lengths]
        self.tokens = sum(self.lengths) if total_tokens is None else int(total_tokens)
        if min(self.lengths, default=0) < 0:
            _refuse("a length of %d" % min(self.lengths))
        if max(self.lengths, default=0) > MOST:
            _too_big(max(self.lengths))
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

    def _describe(self, q, k, v, scale, stream):
        import torch
        if q.dim() != 3 or k.dim() != 3 or q.device != self._table.device:
            _refuse("expected [tokens, heads, dim] on %s" % self._table.device)
        heads, kv_heads, dim = q.shape[1], k.shape[1], q.shape[2]
        if heads > MOST or kv_heads > MOST or dim > MOST:
            _too_big(max(heads, kv_heads, dim))
        _same(q, (self.tokens, heads, dim), q)
        _same(q, (self.tokens, kv_heads, dim), k, v)
        if stream != self._made_on:                         # (the table must not be given away while that stream still reads it)
            self._table.record_stream(torch.cuda.current_stream(q.device))
        return (_type(q), heads, kv_heads, dim, 1 / math.sqrt(max(1, dim)) if scale is None else scale, *_heads(q), *_heads(k), *_heads(v))

    def attention(self, q, k, v, scale=None):
        """tessel_attention_forward: q [tokens, heads, dim], k and v [tokens, kv_heads, dim] -> (o like q, lse [heads, tokens])"""
        import torch
        lib, stream = _library(), _stream(q)
        described = self._describe(q, k, v, scale, stream)
        o = _like(q)
        lse = q.new_empty((q.shape[1], self.tokens), dtype=torch.float32)
        a = _FlatAttention(*described, *_heads(o), lse.data_ptr())
        n = C.c_size_t()
        binding._check(lib.tessel_attention_forward_workspace_bytes(self._h, C.byref(a), C.byref(n)))
        ws = _workspace(n.value, q) if n.value else None
        binding._check(lib.tessel_attention_forward(self._h, C.byref(a), None if ws is None else ws.data_ptr(), n.value, stream))
        return o, lse

    def attention_backward(self, d_o, q, k, v, o, lse, scale=None):
        """tessel_attention_backward: (dq, dk, dv) from the gradient of o and what the forward call took and gave"""
        import torch
        lib, stream = _library(), _stream(q)
        described = self._describe(q, k, v, scale, stream)
        _same(q, q.shape, d_o, o)
        if lse.dtype is not torch.float32 or lse.shape != (q.shape[1], self.tokens) or not lse.is_contiguous() or lse.get_device() != q.get_device():
            _refuse("lse is not what the forward call gave")
        dq, dk, dv = _like(q), _like(k), _like(v)
        a = _FlatAttention(*described, *_heads(o), lse.data_ptr(), *_heads(d_o), *_heads(dq), *_heads(dk), *_heads(dv))
        n = C.c_size_t()
        binding._check(lib.tessel_attention_backward_workspace_bytes(self._h, C.byref(a), C.byref(n)))
        ws = _workspace(n.value, q)
        binding._check(lib.tessel_attention_backward(self._h, C.byref(a), ws.data_ptr(), ws.numel(), stream))
        return dq, dk, dv


def _describe_norm(x, y, pre, post, gate, scale, eps):
    if x.dim() != 2:
        _refuse("expected [tokens, channels]")
    n, c = x.shape
    if c > MOST:
        _too_big(c)
    _same(x, x.shape, x, y)
    if gate is None:
        kind, at = GATE_NONE, (None, 0)
    elif gate.dim() == 1:
        kind, at = GATE_CHANNEL, (_vector(gate, c, x), 0)
    else:
        _same(x, x.shape, gate)
        kind, at = GATE_TOKEN, _rows(gate)
    return (_type(x), kind, n, c, scale, eps, *_rows(x), *_rows(y), *at, _vector(pre, c, x), None if post is None else _vector(post, c, x))


def residual_norm(x, y, pre, post=None, gate=None, scale=1.0, eps=1e-6):
    """tessel_residual_norm_forward: (r, h, stats) with r = scale x + gate n(y, post), h = n(r, pre).  post None: y itself; gate:
    None, [channels] in 32 bits or [tokens, channels] like x."""
    import torch
    described = _describe_norm(x, y, pre, post, gate, scale, eps)
    n, c = described[2], described[3]
    r, h, stats = _like(x), _like(x), x.new_empty((2, n), dtype=torch.float32)
    a = _FlatNorm(*described, stats.data_ptr(), r.data_ptr(), c, h.data_ptr(), c)
    binding._check(_library().tessel_residual_norm_forward(C.byref(a), _stream(x)))
    return r, h, stats


def residual_norm_backward(dr, dh, x, y, stats, pre, post=None, gate=None, scale=1.0, into=None):
    """tessel_residual_norm_backward: (dx, dy, dpre, dpost, dgate), None for what the forward call did not have.  `into`: (dpre, dpost,
    dgate) of earlier micro-batches, to which the parameters' gradients are added (dgate: of a gate for the channels)."""
    import torch
    lib = _library()
    described = _describe_norm(x, y, pre, post, gate, scale, 0.0)
    kind, shape, c = described[1], x.shape, described[3]
    _same(x, shape, dr, dh)
    if stats.dtype is not torch.float32 or stats.shape != (2, shape[0]) or not stats.is_contiguous() or stats.get_device() != x.get_device():
        _refuse("stats is not what the forward call gave")
    dx, dy = _like(x), _like(x)
    if into is None:
        new = x.new_empty((3, c), dtype=torch.float32)
        dpre, dpost, dgate = new.unbind(0)
        first = new.data_ptr()
        to = [first, first + 4 * c, first + 8 * c]
    else:
        dpre, dpost, dgate = into
        to = [_vector(dpre, c, x), None if post is None else _vector(dpost, c, x), _vector(dgate, c, x) if kind == GATE_CHANNEL else None]
    if post is None:
        dpost = to[1] = None
    at = (None, 0)
    if kind != GATE_CHANNEL:
        dgate = to[2] = None
    if kind == GATE_TOKEN:
        dgate = _like(x)
        at = (dgate.data_ptr(), c)
    a = _FlatNorm(*described, stats.data_ptr(), None, 0, None, 0, *_rows(dr), *_rows(dh), dx.data_ptr(), c, dy.data_ptr(), c, *at, *to,
                  0 if into is None else 1)
    n = C.c_size_t()
    binding._check(lib.tessel_residual_norm_backward_workspace_bytes(C.byref(a), C.byref(n)))
    ws = _workspace(n.value, x)
    binding._check(lib.tessel_residual_norm_backward(C.byref(a), ws.data_ptr(), ws.numel(), _stream(x)))
    return dx, dy, dpre, dpost, dgate


class Checkpoint:
    """An activation [tokens, channels] in 8 bits: `values` [tokens, channels up to the next multiple of 64] and `exponents`
    [tokens, groups of 64 channels], of a tensor of type `dtype`."""

    def __init__(self, like):
        """room for a tensor like this one"""
        import torch
        tokens, channels = like.shape
        if channels > MOST:
            _too_big(channels)
        groups = -(-channels // GROUP)
        self.tokens, self.channels, self.dtype, self.device = tokens, channels, like.dtype, like.device
        # (one tensor for both: half the time of two)
        self._room = like.new_empty((tokens * groups * (GROUP + 1),), dtype=torch.uint8)
        self._groups, self._at = groups, like.get_device()
        first = self._room.data_ptr()
        self._words = (first, first + tokens * groups * GROUP, groups * GROUP, groups, tokens, channels, _type(like))
        self._desc = CheckpointDesc(*self._words)

    @property
    def values(self):
        import torch
        return self._room[:self.tokens * self._groups * GROUP].view(torch.int8).view(self.tokens, self._groups * GROUP)

    @property
    def exponents(self):
        return self._room[self.tokens * self._groups * GROUP:].view(self.tokens, self._groups)

    @property
    def nbytes(self):
        return self._room.numel()

    def _like(self, t):
        if not t.is_cuda or t.dtype is not self.dtype or t.shape != (self.tokens, self.channels) or t.get_device() != self._at:
            _refuse("expected %s [%d, %d] on %s, got %s %s" % (self.dtype, self.tokens, self.channels, self.device, t.dtype, tuple(t.shape)))
        if t.requires_grad:
            _refuse_gradient(t)


def _new_checkpoint(x):
    if x.dim() != 2 or not x.is_cuda:
        _refuse("expected [tokens, channels] on the GPU")
    if x.requires_grad:
        _refuse_gradient(x)
    return Checkpoint(x)


def checkpoint(x):
    """tessel_checkpoint_store: x [tokens, channels] in 8 bits"""
    c = _new_checkpoint(x)
    rows = Rows(*_rows(x))
    binding._check(_library().tessel_checkpoint_store(C.byref(c._desc), C.byref(rows), _stream(x)))
    return c


def restore(c):
    """tessel_checkpoint_restore: what a checkpoint stands for, in the type of what was stored"""
    x = c._room.new_empty((c.tokens, c.channels), dtype=c.dtype)
    rows = Rows(x.data_ptr(), c.channels)
    binding._check(_library().tessel_checkpoint_restore(C.byref(c._desc), C.byref(rows), _stream(x)))
    return x


def _act(act):
    if act not in ACT:
        _refuse("no activation %r: one of %s" % (act, ", ".join(ACT)))
    return ACT[act]


def gated(g, u, act="silu"):
    """tessel_gated_forward: (a, checkpoint of g, checkpoint of u) with a = act(g) u"""
    kind = _act(act)
    kg = _new_checkpoint(g)
    kg._like(u)
    ku = _new_checkpoint(u)
    a = _like(g)
    rows = Rows(*_rows(g)), Rows(*_rows(u)), Rows(a.data_ptr(), kg.channels)
    binding._check(_library().tessel_gated_forward(kind, C.byref(rows[0]), C.byref(rows[1]), C.byref(rows[2]), C.byref(kg._desc),
                                                   C.byref(ku._desc), _stream(g)))
    return a, kg, ku


def gated_backward(da, kg, ku, act="silu", with_output=False):
    """tessel_gated_backward: (dg, du), or (dg, du, a) with the checkpoints' own act(g) u"""
    kind = _act(act)
    kg._like(da)
    if ku._at != kg._at:
        _refuse("checkpoints on %s and %s" % (kg.device, ku.device))
    outs = [_like(da) for _ in range(3 if with_output else 2)]
    rows = [Rows(t.data_ptr(), kg.channels) for t in outs]
    d = Rows(*_rows(da))
    binding._check(_library().tessel_gated_backward(kind, C.byref(d), C.byref(kg._desc), C.byref(ku._desc), C.byref(rows[0]), C.byref(rows[1]),
                                                    C.byref(rows[2]) if with_output else None, _stream(da)))
    return tuple(outs)


def weight_gradient(dy, x, into=None):
    """tessel_weight_gradient: dy^T x [outputs, channels] in 32 bits, for dy [tokens, outputs] and a checkpoint x [tokens, channels]; added
    to `into` (and that returned) if it is given"""
    import torch
    lib = _library()
    if dy.dim() != 2 or not dy.is_cuda or dy.get_device() != x._at or dy.dtype is not x.dtype or dy.shape[0] != x.tokens:
        _refuse("dy %s %s does not go with a checkpoint of %s [%d, %d]" % (dy.dtype, tuple(dy.shape), x.dtype, x.tokens, x.channels))
    if dy.requires_grad:
        _refuse_gradient(dy)
    shape = (dy.shape[1], x.channels)
    if shape[0] > MOST:
        _too_big(shape[0])
    if into is None:
        dw = dy.new_empty(shape, dtype=torch.float32)
    else:
        dw = into
        if dw.dtype is not torch.float32 or dw.shape != shape or dw.get_device() != dy.get_device() or (shape[1] > 1 and dw.stride(1) != 1):
            _refuse("the sum has to be 32-bit %s on %s" % (shape, dy.device))
        if dw.requires_grad:
            _refuse_gradient(dw)
    a = _FlatWeight(*x._words, *_rows(dy), shape[0], 0 if into is None else 1, dw.data_ptr(), dw.stride(0) if shape[0] > 1 else shape[1])
    n = C.c_size_t()
    binding._check(lib.tessel_weight_gradient_workspace_bytes(C.byref(a), C.byref(n)))
    need = n.value
    ws = _workspace(need, dy) if need else None
    binding._check(lib.tessel_weight_gradient(C.byref(a), ws.data_ptr() if need else None, need, _stream(dy)))
    return dw
