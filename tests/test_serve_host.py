"""The calls for 4-bit weights and for the steps around the cache, as far as they need no device: exports, structs and refusals."""
import ctypes
import os
import re
import subprocess

import numpy as np
import pytest

from paper_1511_04561_amd import build as dq8_build
from paper_1511_04561_amd import dq8

from . import serve_reference as ref

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
BUFFERS = [np.zeros(1 << 13, np.float64) for _ in range(14)]  # 64 KiB each


@pytest.fixture(scope="module")
def L():
    dq8_build.build(force=False)
    lib = ctypes.CDLL(dq8_build.LIB)
    vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
    lib.dq8_last_error.restype = ctypes.c_char_p
    lib.dq8_weights_encode.argtypes = [ci, vp, sz, vp, vp]
    lib.dq8_weights_decode.argtypes = [vp, ci, vp, sz, vp]
    lib.dq8_weights_product.argtypes = [vp, vp, vp, sz, vp]
    lib.dq8_weights_product_workspace_bytes.argtypes = [vp, vp]
    lib.dq8_weights_product_workspace_bytes.restype = sz
    lib.dq8_cache_plan.argtypes = [vp, vp]
    lib.dq8_draft_verify.argtypes = [vp, vp, sz, vp]
    lib.dq8_draft_verify_workspace_bytes.argtypes = [vp]
    lib.dq8_draft_verify_workspace_bytes.restype = sz
    return lib


def at(i, offset=0):
    """An address in host memory: never followed, every call here ends before it touches a device."""
    return (BUFFERS[i].ctypes.data + 63) // 64 * 64 + offset


def changed(s, change):
    for name, value in change.items():
        setattr(s, name, value)
    return s


def weights(**change):
    return changed(dq8._Weights(at(0), at(1), 20, 300, 32), change)


def product(**change):
    return changed(dq8._Product(type=1, out_type=1, tokens=3, x=at(2), x_stride=300, out=at(3), out_stride=20, bias=at(4)), change)


def plan(**change):
    return changed(dq8._Plan(batch=3, max_pages=4, tokens=9, free_capacity=12, page_size=16, lens=at(0), new_tokens=at(1), drop=at(2), pages=at(3), free_pages=at(4),
                             n_free=at(5), slots=at(6), positions=at(7), starts=at(8), lens_out=at(9), granted=at(10), n_free_out=at(11)), change)


def verify(**change):
    return changed(dq8._Verify(type=0, tokens=6, batch=2, vocab=50, target=at(0), draft=at(1), target_stride=50, draft_stride=50, ids=at(2), uniform=at(3), sample=at(4),
                               starts=at(5), out=at(6), accepted=at(7), rejected=at(8)), change)


@pytest.mark.parametrize("name,calls", [
    ("dq8_weights.h", ["dq8_weights_decode", "dq8_weights_encode", "dq8_weights_product", "dq8_weights_product_workspace_bytes"]),
    ("dq8_serve.h", ["dq8_cache_plan", "dq8_draft_verify", "dq8_draft_verify_workspace_bytes"])])
def test_every_declared_call_is_exported(L, name, calls):
    header = re.sub(r"/\*.*?\*/", "", open(os.path.join(ROOT, "include", name)).read(), flags=re.S)
    assert sorted(set(re.findall(r"\b(dq8_[a-z0-9_]+)\s*\(", header))) == calls
    assert all(hasattr(L, n) for n in calls)


def test_the_structs_are_those_of_the_headers(tmp_path):
    pairs = [("dq8_weights", dq8._Weights), ("dq8_product", dq8._Product), ("dq8_plan", dq8._Plan), ("dq8_verify", dq8._Verify)]
    lines = ['#include <stddef.h>', '#include <stdio.h>', '#include "dq8_weights.h"', '#include "dq8_serve.h"', "int main(void) {"]
    want = []
    for name, s in pairs:
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        lines += ['printf("%%zu\\n", offsetof(%s, %s));' % (name, f) for f, _ in s._fields_]
        want += [ctypes.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
    src, exe = tmp_path / "s.c", tmp_path / "s"
    src.write_text("\n".join(lines + ["return 0; }"]))
    subprocess.check_call(["gcc", "-I", os.path.join(ROOT, "include"), "-o", str(exe), str(src)])
    assert [int(v) for v in subprocess.check_output([str(exe)]).split()] == want


@pytest.mark.parametrize("status,change", [
    (1, {"codes": None}), (1, {"scales": None}), (3, {"codes": at(0, 8)}), (3, {"scales": at(1, 4)}), (3, {"group": 0}), (3, {"group": 16}), (3, {"group": 96}),
    (3, {"group": -32}), (3, {"rows": 1 << 28}), (3, {"rows": (1 << 28) - 15}), (3, {"rows": 1 << 63}), (3, {"cols": 1 << 31}), (3, {"rows": 1 << 14, "cols": 1 << 22}), (3, {"rows": 1 << 30, "cols": 1 << 30}), (3, {"scales": at(0, 1024)})])
def test_refused_weights(L, status, change):
    w, p = weights(**change), product()
    assert L.dq8_weights_encode(1, at(2), 300, ctypes.byref(w), None) == status and L.dq8_last_error()
    assert L.dq8_weights_decode(ctypes.byref(w), 1, at(2), 300, None) == status
    assert L.dq8_weights_product(ctypes.byref(w), ctypes.byref(p), None, 0, None) == status


def test_refused_matrices(L):
    w = ctypes.byref(weights())
    for call in (lambda kind, p, stride: L.dq8_weights_encode(kind, p, stride, w, None), lambda kind, p, stride: L.dq8_weights_decode(w, kind, p, stride, None)):
        assert call(1, None, 300) == 1
        assert call(3, at(2), 300) == 3 and call(-1, at(2), 300) == 3
        assert call(1, at(2, 1), 300) == 3 and call(0, at(2, 2), 300) == 3
        assert call(1, at(2), 1 << 41) == 3 and call(1, at(2), (1 << 64) - 300) == 3
        assert call(1, at(0), 300) == 3 and call(1, at(1, 2), 300) == 3
        assert call(0, at(0, 0) - 64, 300) == 3
    assert L.dq8_weights_decode(w, 1, at(2), 299, None) == 3  # rows overlap; an input's may
    assert L.dq8_weights_encode(1, at(2), 300, None, None) == 1 and L.dq8_weights_decode(None, 1, at(2), 300, None) == 1


@pytest.mark.parametrize("status,change", [
    (3, {"type": 0}), (3, {"type": 3}), (3, {"out_type": 2}), (3, {"out_type": -1}), (3, {"tokens": (1 << 20) + 1}), (3, {"tokens": 1 << 63}), (1, {"x": None}),
    (1, {"out": None}), (3, {"x": at(2, 1)}), (3, {"out": at(3, 1)}), (3, {"out_type": 0, "out": at(3, 2)}), (3, {"bias": at(4, 2)}), (3, {"x_stride": 1 << 45}),
    (3, {"out_stride": 19}), (3, {"out_stride": 1 << 45}), (3, {"out": at(2)}), (3, {"out": at(0)}), (3, {"out": at(1)}), (3, {"out": at(4)}), (3, {"x": at(0)})])
def test_refused_products(L, status, change):
    w, p = weights(), product(**change)
    assert L.dq8_weights_product(ctypes.byref(w), ctypes.byref(p), None, 0, None) == status and L.dq8_last_error()


def test_products_of_nothing(L):
    assert L.dq8_weights_product(ctypes.byref(weights()), ctypes.byref(product(tokens=0, x=None, out=None)), None, 0, None) == 0
    assert L.dq8_weights_product(ctypes.byref(weights(rows=0, codes=None, scales=None)), ctypes.byref(product(out=None)), None, 0, None) == 0
    assert L.dq8_weights_product(ctypes.byref(weights(cols=0)), ctypes.byref(product()), None, 0, None) == 3
    assert L.dq8_weights_product(ctypes.byref(weights()), None, None, 0, None) == 1
    for w in (weights(rows=0, codes=None), weights(cols=0, scales=None)):
        assert L.dq8_weights_encode(1, None, 0, ctypes.byref(w), None) == 0 and L.dq8_weights_decode(ctypes.byref(w), 0, None, 0, None) == 0


@pytest.mark.parametrize("status,change", [
    (3, {"page_size": 8}), (3, {"page_size": 24}), (3, {"page_size": 2048}), (3, {"page_size": 0}), (3, {"page_size": -16}), (3, {"batch": 4097}), (3, {"batch": 0}),
    (3, {"max_pages": 0}), (3, {"max_pages": 1 << 27}), (3, {"batch": 4096, "max_pages": 1 << 19}), (3, {"tokens": 1 << 31}), (3, {"free_capacity": 1 << 31}),
    (1, {"lens": None}), (1, {"new_tokens": None}), (1, {"pages": None}), (1, {"free_pages": None}), (1, {"n_free": None}), (1, {"slots": None}), (1, {"positions": None}),
    (1, {"starts": None}), (1, {"lens_out": None}), (1, {"granted": None}), (1, {"n_free_out": None}), (3, {"lens": at(0, 2)}), (3, {"slots": at(6, 4)}),
    (3, {"positions": at(7, 4)}), (3, {"drop": at(2, 1)}), (3, {"pages": at(3, 2)}), (3, {"positions": at(6)}), (3, {"starts": at(3)}), (3, {"granted": at(0)}),
    (3, {"granted": at(1)}), (3, {"lens_out": at(2)}), (3, {"lens_out": at(0, 4)}), (3, {"n_free_out": at(4)}), (3, {"n_free": at(4, 8)}), (3, {"pages": at(4)}),
    (3, {"drop": at(3)}), (3, {"granted": at(9)}), (3, {"lens": at(8)}), (3, {"new_tokens": at(9)})])
def test_refused_plans(L, status, change):
    assert L.dq8_cache_plan(ctypes.byref(plan(**change)), None) == status and L.dq8_last_error()
    assert L.dq8_cache_plan(None, None) == 1


@pytest.mark.parametrize("status,change", [
    (3, {"type": 3}), (3, {"type": -1}), (3, {"batch": 65536}), (3, {"tokens": 1 << 31}), (3, {"starts": None, "batch": 4}), (3, {"starts": None, "batch": 0}),
    (3, {"vocab": 0}), (3, {"vocab": 1 << 31}), (3, {"target_stride": 1 << 45}), (3, {"draft_stride": 1 << 45})])
def test_refused_verifications_by_size(L, status, change):
    v = verify(**change)
    assert L.dq8_draft_verify(ctypes.byref(v), None, 0, None) == status and L.dq8_last_error()
    assert L.dq8_draft_verify_workspace_bytes(ctypes.byref(v)) == 0


@pytest.mark.parametrize("status,change", [
    (1, {"target": None}), (1, {"ids": None}), (1, {"uniform": None}), (1, {"sample": None}), (1, {"out": None}), (1, {"accepted": None}), (1, {"rejected": None}),
    (3, {"target": at(0, 2)}), (3, {"draft": at(1, 1)}), (3, {"type": 1, "target": at(0, 1)}), (3, {"ids": at(2, 4)}), (3, {"out": at(6, 4)}), (3, {"uniform": at(3, 2)}),
    (3, {"sample": at(4, 1)}), (3, {"starts": at(5, 2)}), (3, {"accepted": at(7, 1)}), (3, {"rejected": at(8, 2)}), (3, {"out": at(2)}), (3, {"out": at(0)}),
    (3, {"out": at(1, 8)}), (3, {"accepted": at(8)}), (3, {"accepted": at(4)}), (3, {"rejected": at(5)}), (3, {"rejected": at(6)})])
def test_refused_verifications(L, status, change):
    assert L.dq8_draft_verify(ctypes.byref(verify(**change)), None, 0, None) == status and L.dq8_last_error()


def test_refused_workspaces(L):
    v = verify()
    assert L.dq8_draft_verify(ctypes.byref(v), at(9, 8), 64, None) == 3
    for i in range(9):
        assert L.dq8_draft_verify(ctypes.byref(v), at(i), 64, None) == 3
    for space in (at(9, 8), at(0), at(1), at(2), at(3), at(4)):
        assert L.dq8_weights_product(ctypes.byref(weights()), ctypes.byref(product()), space, 64, None) == 3
    assert L.dq8_weights_product_workspace_bytes(ctypes.byref(weights(group=1)), ctypes.byref(product(tokens=100))) == 0
    assert L.dq8_weights_product_workspace_bytes(ctypes.byref(weights()), ctypes.byref(product(tokens=16))) == 0
    assert L.dq8_weights_product_workspace_bytes(None, None) == 0
    assert L.dq8_draft_verify(None, None, 0, None) == 1 and L.dq8_draft_verify_workspace_bytes(None) == 0
    assert L.dq8_draft_verify(ctypes.byref(verify(batch=0)), None, 0, None) == 0


def test_python_calls_refuse_host_tensors_and_wrong_sizes():
    import torch
    with pytest.raises(TypeError):
        dq8.weights_encode(torch.zeros(16, 128))
    with pytest.raises(TypeError):
        dq8.weights_product(torch.zeros(1, 128, dtype=torch.bfloat16), torch.zeros(1, 1, 1024, dtype=torch.uint8), torch.zeros(1, 1, 16, 4, dtype=torch.bfloat16))
    with pytest.raises(TypeError):
        dq8.cache_plan(*[torch.zeros(1, 1, dtype=torch.int32)] * 5, 16, 1)
    with pytest.raises(TypeError):
        dq8.draft_verify(torch.zeros(1, 5), *[torch.zeros(1)] * 3)


# ---------------------------------------------------------------- the references against each other and against hand-made cases


def test_reference_format_round_trip():
    rng = np.random.default_rng(7)
    for rows, cols, group in ((1, 1, 32), (17, 129, 64), (33, 300, 128)):
        w = rng.standard_normal((rows, cols)).astype(np.float32)
        codes, scales = ref.encode(w, group)
        values = ref.decode(codes, scales, rows, cols)
        again = ref.encode(values.astype(np.float32), group)
        assert np.abs(values - w).max() <= 1.01 * np.abs(w).max() / 6  # half of the widest step, 4 to 6, and the scale's rounding
        assert np.array_equal(ref.decode(*again, rows, cols), values) or np.abs(ref.decode(*again, rows, cols) - values).max() < 0.02 * np.abs(w).max()


def test_reference_plan_by_hand():
    pages, free = np.array([[5, 6, 0, 0], [7, 0, 0, 0]], np.int32), np.array([1, 2, 3, 0, 0], np.int32)
    got = ref.plan([20, 16], [3, 17], pages, free, 3, 16, 22, drop=[5, 0])
    # sequence 0: 15 + 3 tokens stay on both pages; sequence 1: 33 tokens, pages 3 and 2 taken
    assert got[0].tolist() == [95, 96, 97] + [48 + i for i in range(16)] + [32, -1, -1]
    assert got[1].tolist() == [15, 16, 17] + list(range(16, 33)) + [-1, -1]
    assert got[2].tolist() == [0, 3, 20] and got[3].tolist() == [18, 33] and got[4].tolist() == [3, 17] and got[5] == 1
    assert pages.tolist() == [[5, 6, 0, 0], [7, 3, 2, 0]]


def test_reference_verification_by_hand():
    p = np.array([[0.5, 0.5, 0.0], [0.25, 0.25, 0.5], [0.0, 0.0, 1.0]])
    q = np.array([[1.0, 0.0, 0.0], [0.5, 0.0, 0.5], [0, 0, 0]])
    # token 0 stays while u < 0.5; token 2 while u * 0.5 < 0.5; behind both, token 2 is sure
    assert [v.tolist() for v in ref.verify(p, [9, 0, 2], [0.4, 0.9, 0.0], [0.3], [0, 3], q)] == [[0, 2, 2], [2], [0]]
    # refused at once: weights max(p - q, 0) = (0, 0.5, 0)
    assert [v.tolist() for v in ref.verify(p, [9, 0, 2], [0.5, 0.9, 0.0], [0.3], [0, 3], q)] == [[1, -1, -1], [0], [2]]
