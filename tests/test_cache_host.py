"""The calls for a paged cache of keys and values, as far as they need no device: exports and refusals."""
import ctypes
import os
import re

import numpy as np
import pytest

from paper_1511_04561_amd import build as dq8_build
from paper_1511_04561_amd import dq8

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def L():
    dq8_build.build(force=False)
    lib = ctypes.CDLL(dq8_build.LIB)
    lib.dq8_last_error.restype = ctypes.c_char_p
    lib.dq8_cache_append.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p]
    lib.dq8_cache_attention.argtypes = [ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_size_t, ctypes.c_void_p]
    lib.dq8_cache_attention_workspace_bytes.argtypes = [ctypes.c_void_p, ctypes.c_void_p]
    lib.dq8_cache_attention_workspace_bytes.restype = ctypes.c_size_t
    return lib


BUFFERS = [np.zeros(1 << 16, np.float64) for _ in range(12)]


def at(i, offset=0):
    """An address in host memory: never followed, every call here ends before it touches a device."""
    return (BUFFERS[i].ctypes.data + 63) // 64 * 64 + offset


def cache(**other):
    c = dq8._Cache(at(0), at(1), 2, 2, 16, 64)
    for name, value in other.items():
        setattr(c, name, value)
    return c


def append(**other):
    a = dq8._Append(type=1, tokens=3, heads=4, q=at(2), k=at(3), v=at(4), q_out=at(5), slots=at(6), positions=at(7), rotation=at(8), n_positions=9, half=32,
                    q_weight=at(9), k_weight=at(10), eps=1e-6)
    a.q_token_stride = a.q_out_token_stride = 256
    a.k_token_stride = a.v_token_stride = 128
    a.q_head_stride = a.k_head_stride = a.v_head_stride = a.q_out_head_stride = 64
    for name, value in other.items():
        setattr(a, name, value)
    return a


def attention(**other):
    a = dq8._Attention(type=1, tokens=3, heads=4, q=at(2), out=at(5), batch=3, max_pages=1, pages=at(6), lens=at(7), softmax_scale=0.125)
    a.q_token_stride = a.out_token_stride = 256
    a.q_head_stride = a.out_head_stride = 64
    for name, value in other.items():
        setattr(a, name, value)
    return a


def test_every_declared_call_is_exported(L):
    header = open(os.path.join(ROOT, "include", "dq8_cache.h")).read()
    header = re.sub(r"/\*.*?\*/", "", header, flags=re.S)
    names = sorted(set(re.findall(r"\b(dq8_[a-z0-9_]+)\s*\(", header)))
    assert names == ["dq8_cache_append", "dq8_cache_attention", "dq8_cache_attention_workspace_bytes"]
    assert all(hasattr(L, n) for n in names)


def test_the_structs_are_those_of_the_header(tmp_path):
    """Sizes and offsets of the Python structures against the compiler's."""
    import subprocess
    pairs = [("dq8_cache", dq8._Cache), ("dq8_append", dq8._Append), ("dq8_attention", dq8._Attention)]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "dq8_cache.h"', "int main(void) {"]
    for name, s in pairs:
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f, _ in s._fields_]
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    got = [int(v) for v in subprocess.check_output([str(exe)]).split()]
    want = []
    for _, s in pairs:
        want += [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    assert got == want


CACHE_REFUSALS = [(2, -1, {}), (2, 4, {}), (1, 0, {"codes": None}), (1, 0, {"scales": None}), (3, 0, {"codes": at(0, 8)}), (3, 0, {"scales": at(1, 4)}),
                  (3, 0, {"dim": 0}), (3, 0, {"dim": 24}), (3, 0, {"dim": 272}), (3, 0, {"dim": -16}), (3, 0, {"page_size": 8}), (3, 0, {"page_size": 48}),
                  (3, 0, {"page_size": 2048}), (3, 0, {"page_size": 0}), (3, 0, {"kv_heads": 0}), (3, 0, {"kv_heads": 70000}), (3, 0, {"pages": 0}),
                  (3, 0, {"pages": 1 << 27}), (3, 0, {"pages": 1 << 63}), (3, 0, {"kv_heads": 8192, "page_size": 1024, "dim": 256, "pages": 1})]


@pytest.mark.parametrize("status,kind,change", CACHE_REFUSALS)
def test_refused_caches(L, status, kind, change):
    c, a, t = cache(**change), append(), attention()
    assert L.dq8_cache_append(kind, ctypes.byref(c), ctypes.byref(a), None) == status and L.dq8_last_error()
    assert L.dq8_cache_attention(kind, ctypes.byref(c), ctypes.byref(t), None, 0, None) == status
    if kind == 0:
        assert L.dq8_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(t)) == 0


@pytest.mark.parametrize("status,change", [
    (3, {"type": 3}), (3, {"type": -1}), (3, {"heads": -1}), (3, {"heads": 70000}), (1, {"k": None}), (1, {"v": None}), (1, {"slots": None}), (1, {"q": None}),
    (1, {"q_out": None}), (1, {"positions": None}), (3, {"tokens": 1 << 31}), (3, {"tokens": 1 << 28}), (3, {"heads": 0}), (3, {"half": 0}), (3, {"half": 33}),
    (3, {"half": -1}), (3, {"n_positions": 0}), (3, {"n_positions": 1 << 40}), (3, {"eps": float("nan")}), (3, {"eps": -1.0}), (3, {"eps": float("inf")}),
    (3, {"k_token_stride": 1 << 50}), (3, {"k": at(3, 1)}), (3, {"q": at(2, 1)}), (3, {"rotation": at(8, 2)}), (3, {"k_weight": at(10, 1)}),
    (3, {"slots": at(6, 4)}), (3, {"positions": at(7, 4)}), (3, {"q_out": at(0)}), (3, {"q_out": at(1)}), (3, {"k": at(0)}), (3, {"v": at(1, 2)}),
    (3, {"q_out": at(2, 2)}), (3, {"q_out": at(3)}), (3, {"rotation": at(5)}), (3, {"slots": at(5)}), (3, {"slots": at(0)}), (3, {"q_weight": at(5)})])
def test_refused_appends(L, status, change):
    c, a = cache(), append(**change)
    assert L.dq8_cache_append(0, ctypes.byref(c), ctypes.byref(a), None) == status and L.dq8_last_error()


@pytest.mark.parametrize("status,change", [
    (3, {"type": 0}), (3, {"type": 3}), (3, {"heads": 0}), (3, {"heads": 3}), (3, {"heads": 70000}), (1, {"q": None}), (1, {"out": None}), (1, {"pages": None}),
    (1, {"lens": None}), (3, {"tokens": 4}), (3, {"batch": 0}), (3, {"tokens": 1 << 31}), (3, {"batch": 1 << 31, "tokens": 1 << 31}),
    (3, {"max_pages": 0}), (3, {"max_pages": 1 << 27}), (3, {"window": -1}), (3, {"softmax_scale": float("nan")}),
    (3, {"softmax_scale": float("-inf")}), (3, {"q_token_stride": 1 << 41}), (3, {"q": at(2, 1)}), (3, {"pages": at(6, 2)}), (3, {"lens": at(7, 1)}),
    (3, {"out": at(2)}), (3, {"out": at(0)}), (3, {"out": at(1)}), (3, {"out": at(6)}), (3, {"out": at(7)}), (3, {"starts": at(5)}), (3, {"starts": at(8, 2)})])
def test_refused_attentions(L, status, change):
    c, a = cache(), attention(**change)
    assert L.dq8_cache_attention(0, ctypes.byref(c), ctypes.byref(a), None, 0, None) == status and L.dq8_last_error()


def test_refused_workspaces_and_structs(L):
    c, a = cache(), attention()
    assert L.dq8_cache_attention(0, ctypes.byref(c), ctypes.byref(a), at(8, 8), 64, None) == 3
    for i in (0, 1, 2, 5, 6, 7):
        assert L.dq8_cache_attention(0, ctypes.byref(c), ctypes.byref(a), at(i), 64, None) == 3
    assert L.dq8_cache_attention(0, None, ctypes.byref(a), None, 0, None) == 1
    assert L.dq8_cache_attention(0, ctypes.byref(c), None, None, 0, None) == 1
    assert L.dq8_cache_append(0, None, ctypes.byref(append()), None) == 1
    assert L.dq8_cache_append(0, ctypes.byref(c), None, None) == 1


def test_calls_without_tokens_launch_nothing(L):
    c = cache()
    assert L.dq8_cache_append(0, ctypes.byref(c), ctypes.byref(append(tokens=0, k=None, v=None, slots=None, q=None)), None) == 0
    assert L.dq8_cache_attention(0, ctypes.byref(c), ctypes.byref(attention(tokens=0, q=None, out=None)), None, 0, None) == 0
    assert L.dq8_cache_attention(0, ctypes.byref(c), ctypes.byref(attention(tokens=0, batch=0, pages=None)), None, 0, None) == 0
    assert L.dq8_cache_attention(0, ctypes.byref(c), ctypes.byref(attention(batch=0, starts=at(8))), None, 0, None) == 0
    assert L.dq8_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(attention(tokens=0))) == 0
