"""Refusal of strides whose extents 64 bits do not hold: without it the checks for overlaps would compare wrapped numbers (no device needed)."""
import ctypes

import pytest

from tests.test_cache_host import L, append, attention, cache  # noqa: F401

TOKENS = 2 ** 24 + 1  # times a stride of 2^39 elements of two bytes: 2^64


@pytest.mark.parametrize("field", ["q_token_stride", "k_token_stride", "v_token_stride", "q_out_token_stride"])
@pytest.mark.parametrize("stride", [2 ** 33, 2 ** 38, 2 ** 39, 2 ** 40 - 1])
def test_append(L, field, stride):
    a = append(tokens=TOKENS, **{field: stride})
    assert L.dq8_cache_append(0, ctypes.byref(cache()), ctypes.byref(a), None) == 3 and b"stride" in L.dq8_last_error()


@pytest.mark.parametrize("field", ["q_token_stride", "out_token_stride"])
@pytest.mark.parametrize("stride", [2 ** 33, 2 ** 38, 2 ** 39, 2 ** 40 - 1])
def test_attention(L, field, stride):
    a = attention(tokens=TOKENS, batch=TOKENS, **{field: stride})
    assert L.dq8_cache_attention(0, ctypes.byref(cache()), ctypes.byref(a), None, 0, None) == 3 and b"stride" in L.dq8_last_error()
    assert L.dq8_cache_attention_workspace_bytes(ctypes.byref(cache()), ctypes.byref(a)) == 0


def test_many_heads(L):
    """65535 heads are all that a call takes: strides up to the limit of any stride fit."""
    a = append(heads=65535, tokens=1, q_head_stride=2 ** 40)
    assert L.dq8_cache_append(0, ctypes.byref(cache()), ctypes.byref(a), None) == 3 and b"stride" in L.dq8_last_error()
    a = append(heads=0, q_weight=None, tokens=1, k_head_stride=2 ** 40)
    assert L.dq8_cache_append(0, ctypes.byref(cache()), ctypes.byref(a), None) == 3 and b"stride" in L.dq8_last_error()
