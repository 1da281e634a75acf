"""Thin ctypes binding of include/tessel_block_ops.h: the operators that the blocks of a schedule run -- causal attention over
packed sequences, the norms around a block with gate and residual scale, activation checkpoints in 8 bits and their use in
the backward pass -- and what lies between the tokens and the attention: the embedding of a shard of the vocabulary, the norms of
queries and keys with the rotation by position, dropout whose mask is never stored.

Tensors are torch's, on the GPU; every call runs on torch's current stream and allocates its outputs and workspace there
(a tensor that another stream wrote is the caller's to wait for, as with torch's own operators).  There is no CPU fallback.
Nothing here records torch's automatic differentiation: forward and backward are two calls, and a tensor that requires a gradient is
refused while torch records (under torch.no_grad(), and in the passes of a torch.autograd.Function, it is taken as it is).
"""
import ctypes as C
import math
import operator
import struct

from . import binding

EXPORTS = (
    "tessel_block_last_hip_error", "tessel_packing_create", "tessel_packing_destroy", "tessel_packing_table_bytes", "tessel_packing_bind",
    "tessel_attention_forward_workspace_bytes", "tessel_attention_forward", "tessel_attention_backward_workspace_bytes", "tessel_attention_backward",
    "tessel_residual_norm_forward", "tessel_residual_norm_backward_workspace_bytes", "tessel_residual_norm_backward",
    "tessel_checkpoint_store", "tessel_checkpoint_restore", "tessel_gated_forward", "tessel_gated_backward",
    "tessel_weight_gradient_workspace_bytes", "tessel_weight_gradient",
    "tessel_dropout_apply", "tessel_embedding_forward", "tessel_embedding_backward_workspace_bytes", "tessel_embedding_backward",
    "tessel_rotation_forward", "tessel_rotation_backward_workspace_bytes", "tessel_rotation_backward",
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


class Drop(C.Structure):
    _fields_ = [("seed", C.c_uint64), ("number", C.c_uint64), ("step", C.c_void_p), ("rate", C.c_float)]


class DropoutRows(C.Structure):
    _fields_ = [("type", C.c_int32), ("channels", C.c_int32), ("tokens", C.c_int64), ("x", Rows), ("y", Rows), ("drop", Drop)]


class Embedding(C.Structure):
    _fields_ = [("type", C.c_int32), ("index_type", C.c_int32), ("token", C.c_void_p), ("tokens", C.c_int64), ("first", C.c_int64),
                ("rows", C.c_int32), ("channels", C.c_int32), ("scale", C.c_float), ("table", Rows), ("out", Rows), ("d_out", Rows),
                ("dtable", C.c_void_p), ("dtable_stride", C.c_int64), ("accumulate", C.c_int32), ("drop", Drop)]


class Rotation(C.Structure):
    _fields_ = [("type", C.c_int32), ("index_type", C.c_int32), ("heads", C.c_int32), ("kv_heads", C.c_int32), ("dim", C.c_int32),
                ("turning", C.c_int32), ("neighbours", C.c_int32), ("eps", C.c_float), ("tokens", C.c_int64), ("position", C.c_void_p),
                ("frequency", C.c_void_p), ("wq", C.c_void_p), ("wk", C.c_void_p), ("q", Heads), ("k", Heads), ("q_out", Heads),
                ("k_out", Heads), ("dq_out", Heads), ("dk_out", Heads), ("dq", Heads), ("dk", Heads), ("dwq", C.c_void_p),
                ("dwk", C.c_void_p), ("accumulate", C.c_int32)]


def _flat(nested):
    """The same layout with the fields of the structures inside side by side: one call fills it, which is most of what a small call costs
    on the host."""
    fields = []
    for name, kind in nested._fields_:
        fields += [(name + "_" + n, k) for n, k in kind._fields_] if issubclass(kind, C.Structure) else [(name, kind)]
    flat = type("Flat" + nested.__name__, (C.Structure,), {"_fields_": fields})
    assert C.sizeof(flat) == C.sizeof(nested)
    return flat


def _packed(nested):
    """The same layout as bytes from the values of all fields, a third of the time that filling a structure takes (missing pointers: 0)"""
    codes = {C.c_int32: "i", C.c_int64: "q", C.c_uint64: "Q", C.c_float: "f", C.c_void_p: "P"}
    whole = struct.Struct("@" + "".join(codes[kind] for _, kind in _flat(nested)._fields_) + "0q")
    assert whole.size == C.sizeof(nested)
    return whole.pack


_FlatAttention, _FlatNorm, _FlatWeight = _flat(Attention), _flat(ResidualNorm), _flat(WeightGrad)
_pack_dropout, _pack_embedding, _pack_rotation = _packed(DropoutRows), _packed(Embedding), _packed(Rotation)
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
        for f in (lib.tessel_dropout_apply, lib.tessel_embedding_forward, lib.tessel_rotation_forward):
            f.argtypes = [ptr, ptr]
        for f in (lib.tessel_embedding_backward_workspace_bytes, lib.tessel_rotation_backward_workspace_bytes):
            f.argtypes = [ptr, size]
        for f in (lib.tessel_embedding_backward, lib.tessel_rotation_backward):
            f.argtypes = [ptr, ptr, C.c_size_t, ptr]
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
    """a [tokens, heads, dim] tensor: start and strides.  One whose last dimension is not contiguous is refused (by the attention in the library also one whose strides or
    start are not multiples of 16 bytes)."""
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
        self._positions = None
        binding._check(lib.tessel_packing_bind(h, self._table.data_ptr(), n.value, self._made_on))

    @property
    def positions(self):
        """each token's place in its sequence, as rotate() takes it: int32 [tokens], made at the first use, which so is not for a stream that is being
        captured; noughts for tokens of no sequence.  To be read on the stream that is current now, also when the packing is gone by then."""
        import torch
        stream = torch.cuda.current_stream(self._table.device)
        if self._positions is None:
            places = torch.zeros(self.tokens, dtype=torch.int32)
            begin = 0
            for n in self.lengths:
                places[begin:begin + n] = torch.arange(n, dtype=torch.int32)
                begin += n
            self._positions, self._placed_on = places.to(self._table.device), stream
        elif stream != self._placed_on:                     # (as with the table: not given away while that stream still reads it)
            self._positions.record_stream(stream)
        return self._positions

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


class Dropout:
    """A dropout: which values it keeps follows from `seed`, `number` (which dropout of the program this is: a layer's, of a micro-batch) and where
    they stand, so the backward pass, and a block that computes its activations again, draw the same ones.  `step`: an int64 tensor of one
    number on the GPU, added to `number` when a kernel runs (a captured graph that counts it up draws anew in every replay).  An object
    stays what it was made as."""

    def __init__(self, rate, seed, number=0, step=None):
        import torch
        if not 0 <= rate < 1:
            _refuse("a dropout rate of %r: from 0 to below 1" % (rate,))
        seed, number = operator.index(seed), operator.index(number)
        for n in (seed, number):
            if not 0 <= n < 1 << 64:
                _refuse("%r is no number of 64 bits" % (n,))
        if step is not None and (step.dtype is not torch.int64 or step.numel() != 1 or not step.is_cuda):
            _refuse("step has to be one int64 number on the GPU")
        self._step = step
        self._words = (seed, number, 0 if step is None else step.data_ptr(), float(rate))

    rate = property(lambda self: self._words[3])
    seed = property(lambda self: self._words[0])
    number = property(lambda self: self._words[1])
    step = property(lambda self: self._step)

    def _at(self, like):
        if self._step is not None and self._step.get_device() != like.get_device():
            _refuse("step on %s, the tensors on %s" % (self._step.device, like.device))
        return self._words


_NO_DROP = (0, 0, 0, 0.0)


def _on_gpu(t, dims):
    if t.dim() != len(dims) or not t.is_cuda:
        _refuse("expected [%s] on the GPU, got %s on %s" % (", ".join(dims), tuple(t.shape), t.device))
    if max(t.shape) > MOST:
        _too_big(max(t.shape))
    if t.requires_grad:
        _refuse_gradient(t)


def _index(t, n, like):
    """type and address of a whole number for each token"""
    import torch
    kind = 1 if t.dtype is torch.int64 else 0 if t.dtype is torch.int32 else None
    if kind is None:
        raise binding.TesselError(E_UNSUPPORTED, "tokens and positions are int32 or int64, not %s" % t.dtype)
    if t.shape != (n,) or t.get_device() != like.get_device() or (n > 1 and t.stride(0) != 1):
        _refuse("expected %d contiguous whole numbers on %s, got %s on %s" % (n, like.device, tuple(t.shape), t.device))
    return kind, t.data_ptr()


def dropout(x, drop):
    """tessel_dropout_apply: x [tokens, channels] with what `drop` (a Dropout) drops as zeros and the rest by 1 / (1 - rate); the same call on the
    gradient of what it gave is the backward pass"""
    _on_gpu(x, ("tokens", "channels"))
    y = _like(x)
    n, c = x.shape
    binding._check(_library().tessel_dropout_apply(_pack_dropout(_type(x), c, n, *_rows(x), y.data_ptr(), c, *drop._at(x)), _stream(x)))
    return y


def _number(n):
    """a number that 32 bits hold"""
    if not -3.4e38 < n < 3.4e38:
        _refuse("%r is no number of 32 bits" % (n,))
    return n


def _whole_first(first):
    first = operator.index(first)
    if not 0 <= first <= 1 << 62:
        _refuse("the first row of a shard has to be 0 to 2^62, not %r" % (first,))
    return first


def embed(tokens, table, scale=1.0, first=0, drop=None):
    """tessel_embedding_forward: scale times the rows of table [rows, channels] that tokens (int32 or int64) ask for, after `drop` (a Dropout) if
    there is one -> [tokens, channels].  The table holds the rows from `first` on of a vocabulary; tokens of other rows, and negative ones, get zeros."""
    _on_gpu(table, ("rows", "channels"))
    rows, c = table.shape
    if tokens.dim() != 1 or tokens.shape[0] > MOST:
        _refuse("expected at most 2^31 - 1 tokens in one dimension, got %s" % (tuple(tokens.shape),))
    n = tokens.shape[0]
    kind, at = _index(tokens, n, table)
    out = table.new_empty((n, c))
    a = _pack_embedding(_type(table), kind, at, n, _whole_first(first), rows, c, _number(scale), *_rows(table), out.data_ptr(), c, 0, 0, 0, 0, 0,
                        *(_NO_DROP if drop is None else drop._at(table)))
    binding._check(_library().tessel_embedding_forward(a, _stream(table)))
    return out


def embed_backward(d_out, tokens, rows, scale=1.0, first=0, drop=None, into=None):
    """tessel_embedding_backward: the gradient [rows, channels] of the table in 32 bits from that of what embed() gave; added to `into` (and that
    returned) if it is given, of which rows that no token asked for are neither read nor written.  The same bits each time; the rows of one shard are not
    added up in the order of another that holds them."""
    import torch
    lib = _library()
    _on_gpu(d_out, ("tokens", "channels"))
    n, c = d_out.shape
    rows = operator.index(rows)
    if not 0 < rows <= MOST:
        _refuse("a table of %r rows" % (rows,))
    kind, at = _index(tokens, n, d_out)
    if into is None:
        dtable = d_out.new_empty((rows, c), dtype=torch.float32)
    else:
        dtable = into
        if dtable.dtype is not torch.float32 or dtable.shape != (rows, c) or dtable.get_device() != d_out.get_device() or (c > 1 and dtable.stride(1) != 1):
            _refuse("the sum has to be 32-bit %s on %s" % ((rows, c), d_out.device))
        if dtable.requires_grad:
            _refuse_gradient(dtable)
    a = _pack_embedding(_type(d_out), kind, at, n, _whole_first(first), rows, c, _number(scale), 0, 0, 0, 0, *_rows(d_out), dtable.data_ptr(),
                        dtable.stride(0) if rows > 1 else c, 0 if into is None else 1, *(_NO_DROP if drop is None else drop._at(d_out)))
    size = C.c_size_t()
    binding._check(lib.tessel_embedding_backward_workspace_bytes(a, C.byref(size)))
    ws = _workspace(size.value, d_out) if size.value else None
    binding._check(lib.tessel_embedding_backward(a, 0 if ws is None else ws.data_ptr(), size.value, _stream(d_out)))
    return dtable


def frequencies(turning, base=10000.0, device=None):
    """base^(-2 i / turning) for the pairs i of `turning` channels, in 64 bits: what rotate() takes"""
    import torch
    if turning < 0 or turning % 2:
        _refuse("%r channels are no pairs" % (turning,))
    return torch.exp(torch.arange(0, turning, 2, dtype=torch.float64, device="cuda" if device is None else device) * (-math.log(base) / max(1, turning)))


def _describe_rotation(q, k, positions, frequency, wq, wk, eps, neighbours):
    import torch
    at, shape = q.get_device(), q.shape
    if len(shape) != 3 or k.dim() != 3 or at < 0:
        _refuse("expected [tokens, heads, dim] on the GPU, got %s and %s on %s" % (tuple(shape), tuple(k.shape), q.device))
    n, heads, dim = shape
    kv_heads, pairs = k.shape[1], frequency.numel()
    if max(n, heads, kv_heads, dim) > MOST:
        _too_big(max(n, heads, kv_heads, dim))
    if q.requires_grad:
        _refuse_gradient(q)
    _same(q, (n, kv_heads, dim), k)
    if frequency.dtype is not torch.float64 or frequency.dim() != 1 or not frequency.is_contiguous() or frequency.get_device() != at:
        _refuse("frequencies are contiguous 64-bit numbers on %s" % q.device)
    if frequency.requires_grad:
        _refuse_gradient(frequency)
    if 2 * pairs > dim:
        _refuse("%d pairs of %d channels" % (pairs, dim))
    kind, where = _index(positions, n, q)
    if wq is None and wk is None:
        weights = (0, 0)
    elif wq is None or wk is None:
        _refuse("weights for both, queries and keys, or for neither")
    else:
        weights = (_vector(wq, dim, q), _vector(wk, dim, q))
    return (_type(q), kind, heads, kv_heads, dim, 2 * pairs, 1 if neighbours else 0, _number(eps), n, where, frequency.data_ptr(), *weights, *_heads(q), *_heads(k))


def rotate(q, k, positions, frequency, wq=None, wk=None, eps=1e-6, neighbours=False):
    """tessel_rotation_forward: q [tokens, heads, dim] and k [tokens, kv_heads, dim] -> both, each head normed with wq or wk [dim] (None: as it is) and its
    first 2 len(frequency) channels turned pair by pair by the angles positions x frequency: channels i and i + len(frequency), or with `neighbours`
    2 i and 2 i + 1.  positions: int32 or int64 [tokens] (Packing.positions: those of its sequences); frequency: 64-bit numbers (see frequencies)."""
    described = _describe_rotation(q, k, positions, frequency, wq, wk, eps, neighbours)
    qo, ko = _like(q), _like(k)
    a = _pack_rotation(*described, *_heads(qo), *_heads(ko), 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0, 0)
    binding._check(_library().tessel_rotation_forward(a, _stream(q)))
    return qo, ko


def rotate_backward(dq_out, dk_out, q, k, positions, frequency, wq=None, wk=None, eps=1e-6, neighbours=False, into=None, out=None):
    """tessel_rotation_backward: (dq, dk, dwq, dwk) from the gradients of what rotate() gave and from what it took; dwq and dwk are None without norms, and
    added to `into` = (dwq, dwk) if it is given.  `out` = (dq, dk): tensors to write the gradients to, of any strides (parts of the gradient of a
    joint projection)."""
    import torch
    lib = _library()
    described = _describe_rotation(q, k, positions, frequency, wq, wk, eps, neighbours)
    _same(q, q.shape, dq_out)
    _same(q, k.shape, dk_out)
    dim = q.shape[2]
    if out is None:
        dq, dk = _like(q), _like(k)
    else:
        dq, dk = out
        _same(q, q.shape, dq)
        _same(q, k.shape, dk)
    dwq = dwk = None
    to = (0, 0)
    if wq is not None and into is None:
        new = q.new_empty((2, dim), dtype=torch.float32)
        dwq, dwk = new.unbind(0)
        to = (new.data_ptr(), new.data_ptr() + 4 * dim)
    elif wq is not None:
        dwq, dwk = into
        to = (_vector(dwq, dim, q), _vector(dwk, dim, q))
    a = _pack_rotation(*described, 0, 0, 0, 0, 0, 0, *_heads(dq_out), *_heads(dk_out), *_heads(dq), *_heads(dk), *to, 0 if into is None else 1)
    size = C.c_size_t()
    binding._check(lib.tessel_rotation_backward_workspace_bytes(a, C.byref(size)))
    ws = _workspace(size.value, q) if size.value else None
    binding._check(lib.tessel_rotation_backward(a, None if ws is None else ws.data_ptr(), size.value, _stream(q)))
    return dq, dk, dwq, dwk
