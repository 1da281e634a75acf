"""A launch holds 2^32 - 1 threads: calls of more are TOOBIG before they reach the GPU.  No GPU."""
import ctypes as C

import pytest

from paper_2311_15269_amd import block_ops as B
from tests.test_block_ops_abi import AT, INVALID, OK, TOOBIG, WORKSPACE, attention, kept, packing


@pytest.mark.parametrize("sequences, heads, kv_heads, code", [
    # one token each: a tile a sequence; the passes over queries take workgroups of 256 for each head, that over keys of 512 for each of keys
    (1 << 10, (1 << 14) - 1, 1, WORKSPACE), (1 << 10, 1 << 14, 1, TOOBIG), (1 << 10, (1 << 13) - 1, (1 << 13) - 1, WORKSPACE),
    (1 << 10, 1 << 13, 1 << 13, TOOBIG), (1 << 20, 8, 8, TOOBIG), (1 << 20, 8, 4, WORKSPACE), (1 << 20, 16, 1, TOOBIG), (1 << 22, 1 << 8, 1, TOOBIG),
])
def test_attention_of_more_workgroups_than_a_launch_holds(sequences, heads, kv_heads, code):
    lib = B._library()
    rc, h = packing([1] * sequences)
    assert rc == OK
    a = attention(heads=heads, kv_heads=kv_heads)
    n = C.c_size_t()
    for name in ("q", "o", "d_o", "dq"):
        setattr(a, name, B.Heads(AT, heads * 64, 64))
    for name in ("k", "v", "dk", "dv"):
        setattr(a, name, B.Heads(AT, kv_heads * 64, 64))
    assert lib.tessel_attention_backward(h, C.byref(a), AT, 1 << 50, None) == code                  # (WORKSPACE: valid, but not bound)
    assert lib.tessel_attention_backward_workspace_bytes(h, C.byref(a), C.byref(n)) == (TOOBIG if code == TOOBIG else OK)
    lib.tessel_packing_destroy(h)


def test_a_forward_pass_has_limits_of_its_own():
    """2^23 workgroups of the kernel over keys are too many, of the forward pass not"""
    lib = B._library()
    rc, h = packing([1] * (1 << 10))
    a = attention(heads=1 << 13, kv_heads=1 << 13)
    for name in ("q", "k", "v", "o"):
        setattr(a, name, B.Heads(AT, 64 << 13, 64))
    assert lib.tessel_attention_forward(h, C.byref(a), AT, 1 << 50, None) == WORKSPACE
    lib.tessel_packing_destroy(h)


@pytest.mark.parametrize("outputs, channels, code", [
    (1, (1 << 31) - 1, TOOBIG), (8, (1 << 31) - 1, TOOBIG), (1, (1 << 30) - 128, INVALID), (1 << 24, 1 << 20, TOOBIG), ((1 << 31) - 1, 64, TOOBIG),
])
def test_weight_gradients_of_more_tiles_than_a_launch_holds(outputs, channels, code):
    """tiles of 128 x 128 (256 x 256) by 512 threads; counted without leaving 32 bits"""
    lib = B._library()
    stride = -(-channels // 64) * 64
    a = B.WeightGrad(x=kept(tokens=0, channels=channels, value_stride=0, exponent_stride=0), dy=B.Rows(None, 0), outputs=outputs, dw=None, dw_stride=stride)
    assert lib.tessel_weight_gradient(C.byref(a), None, 0, None) == code
