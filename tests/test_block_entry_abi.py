"""What the library refuses of the operators between the tokens and the attention before it touches a GPU, and what the binding refuses before that.  No GPU, no
compute calls."""
import ctypes as C

import pytest
import torch

from paper_2311_15269_amd import binding, block_ops as B
from tests.test_block_ops_abi import AT, INVALID, OK, TOOBIG, UNSUPPORTED, WORKSPACE

NAN, INF = float("nan"), float("inf")


def drop(**change):
    d = B.Drop(seed=1, number=2, step=None, rate=0.5)
    for name, value in change.items():
        setattr(d, name, value)
    return d


def change_of(a, change):
    for name, value in change.items():
        setattr(a, name, value)
    return a


@pytest.mark.parametrize("change, code", [
    ({"tokens": 0}, OK), ({"tokens": 0, "x": B.Rows(None, 0), "y": B.Rows(None, 0)}, OK),
    ({"tokens": -1}, INVALID), ({"channels": 0}, INVALID), ({"type": 3}, UNSUPPORTED), ({"x": B.Rows(None, 64)}, INVALID), ({"x": B.Rows(AT + 1, 64)}, INVALID),
    ({"x": B.Rows(AT, -1)}, INVALID), ({"y": B.Rows(AT, 63)}, INVALID), ({"y": B.Rows(None, 64)}, INVALID), ({"tokens": 1 << 31}, TOOBIG),
    ({"tokens": (1 << 31) - 1, "channels": 17}, TOOBIG), ({"tokens": 1 << 24, "channels": (1 << 31) - 1}, TOOBIG),
    ({"tokens": 1, "channels": (1 << 30) + 1}, TOOBIG),
    ({"drop": drop(rate=1.0)}, INVALID), ({"drop": drop(rate=-0.5)}, INVALID), ({"drop": drop(rate=NAN)}, INVALID), ({"drop": drop(rate=INF)}, INVALID),
    ({"drop": drop(step=AT + 4)}, INVALID), ({"tokens": 0, "drop": drop(step=AT)}, OK),
])
def test_dropout_refuses(change, code):
    a = change_of(B.DropoutRows(type=0, channels=64, tokens=5, x=B.Rows(AT, 64), y=B.Rows(AT, 64), drop=drop()), change)
    assert B._library().tessel_dropout_apply(C.byref(a), None) == code


def embedding(**change):
    return change_of(B.Embedding(type=0, index_type=1, token=AT, tokens=5, first=0, rows=10, channels=64, scale=1.0, table=B.Rows(AT, 64), out=B.Rows(AT, 64),
                                 d_out=B.Rows(AT, 64), dtable=AT, dtable_stride=64, accumulate=0, drop=drop(rate=0.0)), change)


@pytest.mark.parametrize("change, code", [
    ({"tokens": -1}, INVALID), ({"rows": 0}, INVALID), ({"channels": 0}, INVALID), ({"tokens": 1 << 31}, TOOBIG), ({"rows": (1 << 24) + 1}, TOOBIG), ({"channels": (1 << 24) + 1}, TOOBIG),
    ({"tokens": (1 << 31) - 1, "channels": 17}, TOOBIG), ({"type": 3}, UNSUPPORTED), ({"index_type": 2}, UNSUPPORTED), ({"first": -1}, INVALID), ({"first": (1 << 62) + 1}, INVALID),
    ({"scale": NAN}, INVALID), ({"scale": INF}, INVALID), ({"token": None}, INVALID), ({"token": AT + 4}, INVALID), ({"drop": drop(rate=1.0)}, INVALID),
])
def test_embedding_refuses(change, code):
    lib, a = B._library(), embedding(**change)
    assert lib.tessel_embedding_forward(C.byref(a), None) == code
    assert lib.tessel_embedding_backward(C.byref(a), AT, 1 << 50, None) == code


@pytest.mark.parametrize("rate", [0.0, 0.5])
@pytest.mark.parametrize("tokens, channels, code", [
    # 2^32 - 256 chunks of eight channels, in rows that leave none, and nearly half, of their lanes over
    ((1 << 31) - 128, 16, INVALID), ((1 << 31) - 127, 16, TOOBIG), (1431655680, 17, INVALID), (1431655681, 17, TOOBIG), (1200000000, 24, INVALID), (80000000, 257, INVALID), (130150516, 257, INVALID),
    (130150517, 257, TOOBIG), ((1 << 26) - 4, 512, INVALID), (1 << 26, 512, TOOBIG), (66076416, 513, INVALID), (66076417, 513, TOOBIG), ((1 << 31) - 128, 9, INVALID),
])
def test_rows_of_as_many_chunks_as_a_launch_has_threads(tokens, channels, rate, code):
    """(INVALID: a table and rows that are not there, looked for behind the sizes.)"""
    none = B.Rows(None, 0)
    for kind in range(3):
        a = B.DropoutRows(type=kind, channels=channels, tokens=tokens, x=none, y=none, drop=drop(rate=rate))
        assert B._library().tessel_dropout_apply(C.byref(a), None) == code
        a = embedding(type=kind, channels=channels, tokens=tokens, table=none, out=none, drop=drop(rate=rate))
        assert B._library().tessel_embedding_forward(C.byref(a), None) == code


def test_embedding_passes_refuse_their_own():
    lib, n = B._library(), C.c_size_t()
    for change, code in (({"tokens": 0}, OK), ({"tokens": 0, "token": None, "out": B.Rows(None, 0)}, OK), ({"table": B.Rows(None, 64)}, INVALID), ({"table": B.Rows(AT + 1, 64)}, INVALID),
                         ({"out": B.Rows(AT, 63)}, INVALID), ({"out": B.Rows(None, 64)}, INVALID)):
        assert lib.tessel_embedding_forward(C.byref(embedding(**change)), None) == code, change
    for change in ({"d_out": B.Rows(None, 64)}, {"d_out": B.Rows(AT, -64)}, {"dtable": None}, {"dtable": AT + 2}, {"dtable_stride": 63}):
        assert lib.tessel_embedding_backward(C.byref(embedding(**change)), AT, 1 << 50, None) == INVALID, change
    for change, code in (({}, OK), ({"rows": 1 << 24}, OK), ({"tokens": 0}, OK), ({"rows": 0}, INVALID), ({"tokens": 1 << 31}, TOOBIG)):
        assert lib.tessel_embedding_backward_workspace_bytes(C.byref(embedding(**change)), C.byref(n)) == code
    assert lib.tessel_embedding_backward_workspace_bytes(C.byref(embedding()), None) == INVALID
    a = embedding(tokens=5000)
    assert lib.tessel_embedding_backward_workspace_bytes(C.byref(a), C.byref(n)) == OK
    if n.value:
        for at, size in ((None, n.value), (AT + 8, n.value), (AT, n.value - 1)):
            assert lib.tessel_embedding_backward(C.byref(a), at, size, None) == WORKSPACE
    assert lib.tessel_embedding_forward(None, None) == lib.tessel_embedding_backward(None, None, 0, None) == INVALID


def rotation(**change):
    def heads(n):
        return B.Heads(AT, n * 64, 64)
    return change_of(B.Rotation(type=0, index_type=1, heads=4, kv_heads=2, dim=64, turning=64, neighbours=0, eps=1e-6, tokens=5, position=AT, frequency=AT, wq=AT, wk=AT,
                                q=heads(4), k=heads(2), q_out=heads(4), k_out=heads(2), dq_out=heads(4), dk_out=heads(2), dq=heads(4), dk=heads(2), dwq=AT, dwk=AT,
                                accumulate=0), change)


@pytest.mark.parametrize("change, code", [
    ({"tokens": -1}, INVALID), ({"heads": 0}, INVALID), ({"kv_heads": 0}, INVALID), ({"dim": 0}, INVALID), ({"dim": 63}, INVALID), ({"turning": 66}, INVALID), ({"turning": 3}, INVALID),
    ({"turning": -2}, INVALID), ({"dim": 258}, TOOBIG), ({"tokens": 1 << 31}, TOOBIG), ({"tokens": (1 << 26) + 64, "heads": 64}, TOOBIG), ({"heads": (1 << 24) + 1}, TOOBIG), ({"kv_heads": (1 << 31) - 1}, TOOBIG),
    ({"type": 3}, UNSUPPORTED), ({"index_type": 5}, UNSUPPORTED), ({"eps": -1.0}, INVALID), ({"eps": NAN}, INVALID), ({"eps": INF}, INVALID), ({"wq": None}, INVALID), ({"wk": None}, INVALID),
    ({"wq": AT + 2}, INVALID), ({"frequency": None}, INVALID), ({"frequency": AT + 4}, INVALID), ({"position": None}, INVALID), ({"position": AT + 4}, INVALID),
    ({"q": B.Heads(None, 256, 64)}, INVALID), ({"q": B.Heads(AT + 1, 256, 64)}, INVALID), ({"k": B.Heads(AT, -2, 64)}, INVALID), ({"k": B.Heads(AT, 1 << 41, 64)}, INVALID),
])
def test_rotation_refuses(change, code):
    lib, a = B._library(), rotation(**change)
    assert lib.tessel_rotation_forward(C.byref(a), None) == code
    assert lib.tessel_rotation_backward(C.byref(a), AT, 1 << 50, None) == code


def test_rotation_of_many_tokens():
    """a wave for all heads of a token where there are many: 2^26 waves are the threads of a launch"""
    n = C.c_size_t()
    for tokens, heads, code in (((1 << 26) - 4, 64, OK), (1 << 26, 64, TOOBIG), ((1 << 31) - 1, 1, OK), (1 << 20, 1 << 20, OK), (1, 1 << 24, OK)):
        a = rotation(tokens=tokens, heads=heads, kv_heads=heads, dim=128 if heads > 1 else 2, turning=0)
        assert B._library().tessel_rotation_backward_workspace_bytes(C.byref(a), C.byref(n)) == code, (tokens, heads)


def test_rotation_passes_refuse_their_own():
    lib, n = B._library(), C.c_size_t()
    assert lib.tessel_rotation_forward(C.byref(rotation(tokens=0)), None) == OK
    assert lib.tessel_rotation_forward(C.byref(rotation(tokens=0, q=B.Heads(None, 0, 0), position=None)), None) == OK
    # results that lie on themselves: tokens or heads on each other, tokens inside a token's heads
    for bad in (B.Heads(None, 256, 64), B.Heads(AT, 0, 64), B.Heads(AT, 256, 0), B.Heads(AT, 255, 64), B.Heads(AT, 256, 63), B.Heads(AT, 64, 64), B.Heads(AT, 64, 319), B.Heads(AT, 63, 320)):
        assert lib.tessel_rotation_forward(C.byref(rotation(q_out=bad)), None) == INVALID
        assert lib.tessel_rotation_backward(C.byref(rotation(dq=bad)), AT, 1 << 50, None) == INVALID
    for change in ({"dwq": None}, {"dwk": AT + 1}, {"dq_out": B.Heads(None, 256, 64)}, {"dk": B.Heads(AT, 64, 64)}):
        assert lib.tessel_rotation_backward(C.byref(rotation(**change)), AT, 1 << 50, None) == INVALID, change
    a = rotation()
    assert lib.tessel_rotation_backward_workspace_bytes(C.byref(a), C.byref(n)) == OK and n.value > 0
    for at, size in ((None, n.value), (AT + 8, n.value), (AT, n.value - 1)):
        assert lib.tessel_rotation_backward(C.byref(a), at, size, None) == WORKSPACE
    assert lib.tessel_rotation_backward_workspace_bytes(C.byref(rotation(wq=None, wk=None)), C.byref(n)) == OK and n.value == 0
    assert lib.tessel_rotation_backward_workspace_bytes(C.byref(a), None) == lib.tessel_rotation_forward(None, None) == lib.tessel_rotation_backward(None, None, 0, None) == INVALID


def test_sizes_that_do_not_fit_32_bits_are_refused():
    """2^32 + 5 channels, heads or tokens are not 5"""
    class There(torch.Tensor):
        is_cuda = True
    wide = torch.zeros(1, 1, dtype=torch.bfloat16).expand(1, (1 << 32) + 5).as_subclass(There)
    token = torch.zeros(1, dtype=torch.int64)
    for call in (lambda: B.dropout(wide, B.Dropout(0.5, 1)), lambda: B.embed(token, wide), lambda: B.embed_backward(wide, token, 5),
                 lambda: B.embed(token.expand((1 << 32) + 5), wide[:, :8].as_subclass(There)), lambda: B.rotate(wide.view(1, -1, 1), wide.view(1, -1, 1), token, torch.zeros(0))):
        with pytest.raises(binding.TesselError) as error:
            call()
        assert error.value.code in (TOOBIG, INVALID)
    with pytest.raises(binding.TesselError):
        B.embed_backward(torch.zeros(1, 8).as_subclass(There), token, (1 << 32) + 5)


def test_numbers_that_are_none_of_64_bits_are_refused():
    for args in ((0.5, 1 << 64), (0.5, -1), (0.5, 1, 1 << 64), (1.0, 1), (-0.1, 1), (NAN, 1)):
        with pytest.raises(binding.TesselError) as error:
            B.Dropout(*args)
        assert error.value.code == INVALID
    for first in (-1, (1 << 62) + 1):
        with pytest.raises(binding.TesselError):
            B._whole_first(first)
    for call in (lambda: B.Dropout(0.5, 1.5), lambda: B.Dropout(0.5, 1, 2.5), lambda: B._whole_first(1.5)):
        with pytest.raises(TypeError):
            call()
    for n in (1e39, -1e39, NAN, INF):
        with pytest.raises(binding.TesselError):
            B._number(n)
    for turning in (-2, 5):
        with pytest.raises(binding.TesselError):
            B.frequencies(turning, device="cpu")


def test_a_dropout_stays_what_it_is():
    drop = B.Dropout(0.25, 7, 8)
    assert (drop.rate, drop.seed, drop.number, drop.step) == (0.25, 7, 8, None)
    with pytest.raises(AttributeError):
        drop.number = 9
