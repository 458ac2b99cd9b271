"""Python binding of the dq8 C ABI (include/dq8.h): argument marshalling only.

Every function takes torch CUDA tensors (device memory) and enqueues the library's
HIP kernels on torch's current stream.  Nothing is computed here and there is no
fallback: if libdq8.so is missing or a call fails, an exception is raised.

A call with ordinary arguments is marshalled by the extension _binding.so (csrc/dq8_binding.cpp); it returns None for
any other, which then takes the code here: the same library call, and the place where wrong arguments are reported.
Scratch memory is handed in by the extension only, and not while the stream is captured: without it (tensors on another device
than the current one, error statistics without `stats` and `means`, captured calls) long arrays with one scale, sets of tensors and
the statistics of one block take a launch or two more.
"""
import ctypes
import os

import torch

DYNAMIC_TREE, LINEAR, STATIC_TREE, MANTISSA = 0, 1, 2, 3
SCALES_GIVEN = 1
MAX_K = 32

_HERE = os.path.dirname(os.path.abspath(__file__))
# DQ8_LIBRARY names another build of the same library (e.g. one compiled with -DDQ8_TUNABLE for experiments).
LIB_PATH = os.environ.get("DQ8_LIBRARY") or os.path.join(_HERE, "libdq8.so")
_lib = None


class _Unbound:
    """Stands for the extension until the library is loaded: every call takes the code here, which loads it."""

    def __getattr__(self, name):
        return lambda *args: None


_native = _Unbound()


class Dq8Error(RuntimeError):
    pass


class _Cache(ctypes.Structure):  # dq8_cache of include/dq8_cache.h
    _fields_ = [("codes", ctypes.c_void_p), ("scales", ctypes.c_void_p), ("pages", ctypes.c_size_t),
                ("kv_heads", ctypes.c_int), ("page_size", ctypes.c_int), ("dim", ctypes.c_int)]


class _Append(ctypes.Structure):  # dq8_append
    _fields_ = ([("type", ctypes.c_int), ("tokens", ctypes.c_size_t), ("heads", ctypes.c_int)]
                + [(f, ctypes.c_void_p) for f in ("q", "k", "v", "q_out")]
                + [("%s_%s_stride" % (f, w), ctypes.c_size_t) for f in ("q", "k", "v", "q_out") for w in ("token", "head")]
                + [(f, ctypes.c_void_p) for f in ("slots", "positions", "rotation")]
                + [("n_positions", ctypes.c_size_t), ("half", ctypes.c_int), ("interleaved", ctypes.c_int),
                   ("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("eps", ctypes.c_double)])


class _Attention(ctypes.Structure):  # dq8_attention
    _fields_ = ([("type", ctypes.c_int), ("tokens", ctypes.c_size_t), ("heads", ctypes.c_int), ("q", ctypes.c_void_p), ("out", ctypes.c_void_p)]
                + [("%s_%s_stride" % (f, w), ctypes.c_size_t) for f in ("q", "out") for w in ("token", "head")]
                + [("batch", ctypes.c_size_t), ("max_pages", ctypes.c_size_t)]
                + [(f, ctypes.c_void_p) for f in ("pages", "lens", "starts")]
                + [("max_new", ctypes.c_size_t), ("window", ctypes.c_int), ("softmax_scale", ctypes.c_float)])


def lib():
    """The loaded shared library (loaded on first use)."""
    global _lib, _native
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise Dq8Error("%s not found: build it with `python -m paper_1511_04561_amd.build` "
                           "(there is no fallback path)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, sz, ci = ctypes.c_void_p, ctypes.c_size_t, ctypes.c_int
        L.dq8_codebook.argtypes = [ci, vp]
        L.dq8_init.argtypes = []
        L.dq8_absmax.argtypes = [vp, sz, sz, vp, vp]
        L.dq8_encode.argtypes = [ci, vp, sz, sz, vp, vp, ctypes.c_uint, vp]
        L.dq8_decode.argtypes = [ci, vp, vp, sz, sz, vp, vp]
        L.dq8_decode_accumulate_avg.argtypes = [ci, ctypes.POINTER(vp), ctypes.POINTER(vp), ci, sz, sz, vp, vp]
        L.dq8_decode_accumulate_avg_local.argtypes = [ci, ctypes.POINTER(vp), ctypes.POINTER(vp), ci, vp, sz, sz, vp, vp]
        L.dq8_decode_avg_encode.argtypes = [ci, ctypes.POINTER(vp), ctypes.POINTER(vp), ci, vp, sz, sz, vp, vp, vp]
        L.dq8_error_stats.argtypes = [ci, vp, sz, sz, vp, ctypes.c_uint, vp, vp, vp]
        L.dq8_absmax_segments.argtypes = [vp, sz, vp, sz, vp, vp]
        L.dq8_encode_segments.argtypes = [ci, vp, sz, vp, sz, vp, vp, ctypes.c_uint, vp]
        L.dq8_decode_segments.argtypes = [ci, vp, vp, sz, vp, sz, vp, vp]
        L.dq8_decode_accumulate_avg_segments.argtypes = [ci, ctypes.POINTER(vp), ctypes.POINTER(vp), ci, vp, sz, vp, sz, vp, vp]
        for f in (L.dq8_codebook, L.dq8_init, L.dq8_absmax, L.dq8_encode, L.dq8_decode, L.dq8_decode_accumulate_avg,
                  L.dq8_decode_accumulate_avg_local, L.dq8_decode_avg_encode, L.dq8_absmax_segments, L.dq8_encode_segments,
                  L.dq8_decode_segments, L.dq8_decode_accumulate_avg_segments):
            f.restype = ci
        L.dq8_cache_append.argtypes = [ci, ctypes.POINTER(_Cache), ctypes.POINTER(_Append), vp]
        L.dq8_cache_append.restype = ci
        L.dq8_cache_attention.argtypes = [ci, ctypes.POINTER(_Cache), ctypes.POINTER(_Attention), vp, sz, vp]
        L.dq8_cache_attention.restype = ci
        L.dq8_cache_attention_workspace_bytes.argtypes = [ctypes.POINTER(_Cache), ctypes.POINTER(_Attention)]
        L.dq8_cache_attention_workspace_bytes.restype = sz
        dbl = ctypes.c_double
        L.dq8_model_speedup.argtypes = [ci, dbl, dbl, dbl, ci, dbl, dbl, ctypes.POINTER(dbl)]
        L.dq8_model_penalty.argtypes = [ctypes.POINTER(dbl), ctypes.POINTER(dbl), sz, ctypes.POINTER(dbl)]
        L.dq8_model_speedup.restype = ci
        L.dq8_model_penalty.restype = ci
        L.dq8_last_error.restype = ctypes.c_char_p
        try:
            from . import _binding
        except ImportError as e:
            raise Dq8Error("%s/_binding.so cannot be loaded (%s): build it with `python -m paper_1511_04561_amd.build`" % (_HERE, e)) from e
        _binding.bind(Dq8Error, {name: ctypes.cast(getattr(L, name), vp).value for name in _BOUND})
        _native = _binding
        _lib = L
    return _lib


_BOUND = ("dq8_absmax", "dq8_encode_ws", "dq8_workspace_bytes", "dq8_decode", "dq8_absmax_segments", "dq8_encode_segments_ws",
          "dq8_workspace_bytes_segments", "dq8_decode_segments",
          "dq8_decode_accumulate_avg", "dq8_decode_accumulate_avg_local", "dq8_decode_accumulate_avg_segments",
          "dq8_decode_avg_encode", "dq8_error_stats_ws", "dq8_workspace_bytes_stats", "dq8_cache_append", "dq8_cache_attention",
          "dq8_cache_attention_workspace_bytes", "dq8_last_error")


def _check(rc, what):
    if rc != 0:
        raise Dq8Error("%s failed (status %d): %s" % (what, rc, lib().dq8_last_error().decode()))


def n_blocks(n, block):
    if n == 0:
        return 0
    b = n if (block == 0 or block > n) else block
    return (n + b - 1) // b


def _dev(t, dtype, what):
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % what)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % what)
    return t


def _device_and_stream_calls(c):
    """The current device and the raw handle of a device's current stream, as calls: those of torch's C module `c` (private names,
    seen in torch 2.10) where it has both, else the public ones."""
    if hasattr(c, "_cuda_getDevice") and hasattr(c, "_cuda_getCurrentRawStream"):
        return c._cuda_getDevice, c._cuda_getCurrentRawStream
    return torch.cuda.current_device, lambda index: torch.cuda.current_stream(index).cuda_stream


_current_device, _raw_stream = _device_and_stream_calls(torch._C)


def _enqueue(fn, index, *args):
    """Calls the library function `fn` with `args` and torch's current stream on device `index`, which is made current for the
    call if it is not.

    The stream is asked for as the raw handle: torch.cuda.current_stream() builds a Stream object first (2.9 us; the handle
    0.07)."""
    if index == _current_device():
        rc = fn(*args, _raw_stream(index))
    else:
        with torch.cuda.device(index):
            rc = fn(*args, _raw_stream(index))
    if rc != 0:
        _check(rc, fn.__name__)


def codebook(kind):
    """The 256 table values of a data type as a CPU float32 tensor."""
    cb = torch.empty(256, dtype=torch.float32)
    _check(lib().dq8_codebook(int(kind), cb.data_ptr()), "dq8_codebook")
    return cb


def init():
    _check(lib().dq8_init(), "dq8_init")


def absmax(x, block=0, scales=None):
    done = _native.absmax(x, block, scales)
    if done is not None:
        return done
    x = _dev(x, torch.float32, "x")
    n = x.numel()
    if scales is None:
        scales = torch.empty(n_blocks(n, block), dtype=torch.float32, device=x.device)
    _dev(scales, torch.float32, "scales")
    if scales.numel() < n_blocks(n, block):
        raise ValueError("scales too small")
    _enqueue(lib().dq8_absmax, x.get_device(), x.data_ptr(), n, int(block), scales.data_ptr())
    return scales


def encode(kind, x, block=0, scales=None, codes=None, scales_given=False):
    """Returns (codes, scales).  With scales_given the passed scales are used as they are."""
    done = _native.encode(kind, x, block, scales, codes, scales_given)
    if done is not None:
        return done
    x = _dev(x, torch.float32, "x")
    n = x.numel()
    if scales is None:
        if scales_given:
            raise ValueError("scales_given needs scales")
        scales = torch.empty(n_blocks(n, block), dtype=torch.float32, device=x.device)
    if codes is None:
        codes = torch.empty(n, dtype=torch.uint8, device=x.device)
    _dev(scales, torch.float32, "scales")
    _dev(codes, torch.uint8, "codes")
    if scales.numel() < n_blocks(n, block) or codes.numel() < n:
        raise ValueError("output buffers too small")
    _enqueue(lib().dq8_encode, x.get_device(), int(kind), x.data_ptr(), n, int(block), scales.data_ptr(), codes.data_ptr(),
             SCALES_GIVEN if scales_given else 0)
    return codes, scales


def decode(kind, codes, scales, block=0, out=None):
    done = _native.decode(kind, codes, scales, block, out)
    if done is not None:
        return done
    codes = _dev(codes, torch.uint8, "codes")
    scales = _dev(scales, torch.float32, "scales")
    n = codes.numel()
    if scales.numel() < n_blocks(n, block):
        raise ValueError("scales too small")
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=codes.device)
    _dev(out, torch.float32, "out")
    if out.numel() < n:
        raise ValueError("out too small")
    _enqueue(lib().dq8_decode, codes.get_device(), int(kind), codes.data_ptr(), scales.data_ptr(), n, int(block), out.data_ptr())
    return out


MAX_SEGMENTS = 4095


def _bounds(bounds, n):
    """bounds: int64 device tensor of n_seg + 1 ascending element offsets from 0 to n (read by the kernels only)."""
    b = _dev(bounds, torch.int64, "bounds")
    if b.numel() < 2:
        raise ValueError("bounds needs at least two entries")
    return b, b.numel() - 1


def absmax_segments(x, bounds, scales=None):
    done = _native.absmax_segments(x, bounds, scales)
    if done is not None:
        return done
    x = _dev(x, torch.float32, "x")
    b, n_seg = _bounds(bounds, x.numel())
    if scales is None:
        scales = torch.empty(n_seg, dtype=torch.float32, device=x.device)
    _dev(scales, torch.float32, "scales")
    if scales.numel() < n_seg:
        raise ValueError("scales too small")
    _enqueue(lib().dq8_absmax_segments, x.get_device(), x.data_ptr(), x.numel(), b.data_ptr(), n_seg, scales.data_ptr())
    return scales


def encode_segments(kind, x, bounds, scales=None, codes=None, scales_given=False):
    """Tensors back to back in x, one scale each.  Returns (codes, scales)."""
    done = _native.encode_segments(kind, x, bounds, scales, codes, scales_given)
    if done is not None:
        return done
    x = _dev(x, torch.float32, "x")
    n = x.numel()
    b, n_seg = _bounds(bounds, n)
    if scales is None:
        if scales_given:
            raise ValueError("scales_given needs scales")
        scales = torch.empty(n_seg, dtype=torch.float32, device=x.device)
    if codes is None:
        codes = torch.empty(n, dtype=torch.uint8, device=x.device)
    _dev(scales, torch.float32, "scales")
    _dev(codes, torch.uint8, "codes")
    if scales.numel() < n_seg or codes.numel() < n:
        raise ValueError("output buffers too small")
    _enqueue(lib().dq8_encode_segments, x.get_device(), int(kind), x.data_ptr(), n, b.data_ptr(), n_seg, scales.data_ptr(),
             codes.data_ptr(), SCALES_GIVEN if scales_given else 0)
    return codes, scales


def decode_segments(kind, codes, scales, bounds, out=None):
    done = _native.decode_segments(kind, codes, scales, bounds, out)
    if done is not None:
        return done
    codes = _dev(codes, torch.uint8, "codes")
    scales = _dev(scales, torch.float32, "scales")
    n = codes.numel()
    b, n_seg = _bounds(bounds, n)
    if scales.numel() < n_seg:
        raise ValueError("scales too small")
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=codes.device)
    _dev(out, torch.float32, "out")
    if out.numel() < n:
        raise ValueError("out too small")
    _enqueue(lib().dq8_decode_segments, codes.get_device(), int(kind), codes.data_ptr(), scales.data_ptr(), n, b.data_ptr(),
             n_seg, out.data_ptr())
    return out


def _workers(codes_list, scales_list, block, n=None):
    K = len(codes_list)
    if K != len(scales_list):
        raise ValueError("codes_list and scales_list differ in length")
    if n is None:
        if K == 0:
            raise ValueError("need at least one worker buffer")
        n = codes_list[0].numel()
    for c, s in zip(codes_list, scales_list):
        _dev(c, torch.uint8, "codes")
        _dev(s, torch.float32, "scales")
        if c.numel() != n or s.numel() < n_blocks(n, block):
            raise ValueError("worker buffers differ in size")
    cp = (ctypes.c_void_p * max(K, 1))(*[c.data_ptr() for c in codes_list])
    sp = (ctypes.c_void_p * max(K, 1))(*[s.data_ptr() for s in scales_list])
    return K, n, cp, sp


def decode_accumulate_avg(kind, codes_list, scales_list, block=0, out=None, local=None):
    """Mean of the K decoded buffers; with ``local`` (fp32) that array is the first of K + 1 terms."""
    done = _native.decode_accumulate_avg(kind, codes_list, scales_list, block, out, local)
    if done is not None:
        return done
    if local is not None:
        _dev(local, torch.float32, "local")
    K, n, cp, sp = _workers(codes_list, scales_list, block, None if local is None else local.numel())
    dev = local.device if local is not None else codes_list[0].device
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=dev)
    _dev(out, torch.float32, "out")
    if out.numel() < n:
        raise ValueError("out too small")
    if local is None:
        _enqueue(lib().dq8_decode_accumulate_avg, out.get_device(), int(kind), cp, sp, K, n, int(block), out.data_ptr())
    else:
        _enqueue(lib().dq8_decode_accumulate_avg_local, out.get_device(), int(kind), cp, sp, K, local.data_ptr(), n, int(block),
                 out.data_ptr())
    return out


def decode_accumulate_avg_segments(kind, codes_list, scales_list, bounds, out=None, local=None):
    """Mean of the K decoded buffers of tensors back to back, one scale per tensor and worker."""
    done = _native.decode_accumulate_avg_segments(kind, codes_list, scales_list, bounds, out, local)
    if done is not None:
        return done
    if local is not None:
        _dev(local, torch.float32, "local")
    K = len(codes_list)
    if K != len(scales_list) or (K == 0 and local is None):
        raise ValueError("need as many scale arrays as code arrays, and at least one worker or local")
    n = local.numel() if local is not None else codes_list[0].numel()
    b, n_seg = _bounds(bounds, n)
    for c, s in zip(codes_list, scales_list):
        _dev(c, torch.uint8, "codes")
        _dev(s, torch.float32, "scales")
        if c.numel() != n or s.numel() < n_seg:
            raise ValueError("worker buffers differ in size")
    cp = (ctypes.c_void_p * max(K, 1))(*[c.data_ptr() for c in codes_list])
    sp = (ctypes.c_void_p * max(K, 1))(*[s.data_ptr() for s in scales_list])
    if out is None:
        out = torch.empty(n, dtype=torch.float32, device=b.device)
    _dev(out, torch.float32, "out")
    if out.numel() < n:
        raise ValueError("out too small")
    _enqueue(lib().dq8_decode_accumulate_avg_segments, out.get_device(), int(kind), cp, sp, K,
             None if local is None else local.data_ptr(), n, b.data_ptr(), n_seg, out.data_ptr())
    return out


def decode_avg_encode(kind, codes_list, scales_list, block=0, local=None, scales=None, codes=None):
    """Average the K buffers (with ``local`` as first term if given) and compress the average: (codes, scales)."""
    done = _native.decode_avg_encode(kind, codes_list, scales_list, block, local, scales, codes)
    if done is not None:
        return done
    if local is not None:
        _dev(local, torch.float32, "local")
    K, n, cp, sp = _workers(codes_list, scales_list, block, None if local is None else local.numel())
    dev = local.device if local is not None else codes_list[0].device
    if scales is None:
        scales = torch.empty(n_blocks(n, block), dtype=torch.float32, device=dev)
    if codes is None:
        codes = torch.empty(n, dtype=torch.uint8, device=dev)
    _dev(scales, torch.float32, "scales")
    _dev(codes, torch.uint8, "codes")
    if scales.numel() < n_blocks(n, block) or codes.numel() < n:
        raise ValueError("output buffers too small")
    _enqueue(lib().dq8_decode_avg_encode, codes.get_device(), int(kind), cp, sp, K, None if local is None else local.data_ptr(),
             n, int(block), scales.data_ptr(), codes.data_ptr())
    return codes, scales


def error_stats(kind, x, block=0, scales=None, scales_given=False, stats=None, means=None):
    """Approximation error of compress-then-decompress (Sec. 3.4, Table 2).

    Returns (stats float64[nb, 4], means float64[2]) on the device: per block the sum of absolute errors,
    the sum of relative errors over non-zero inputs, the number of non-zero inputs and the largest absolute
    error; means = (mean absolute error, mean relative error over non-zero inputs)."""
    done = _native.error_stats(kind, x, block, scales, scales_given, stats, means)
    if done is not None:
        return done
    x = _dev(x, torch.float32, "x")
    n = x.numel()
    nb = n_blocks(n, block)
    if scales is None:
        if scales_given:
            raise ValueError("scales_given needs scales")
        scales = torch.empty(nb, dtype=torch.float32, device=x.device)
    if stats is None:
        stats = torch.zeros((nb, 4), dtype=torch.float64, device=x.device)
    if means is None:
        means = torch.zeros(2, dtype=torch.float64, device=x.device)
    _dev(scales, torch.float32, "scales")
    _dev(stats, torch.float64, "stats")
    _dev(means, torch.float64, "means")
    if scales.numel() < nb or stats.numel() < 4 * nb or means.numel() < 2:
        raise ValueError("output buffers too small")
    _enqueue(lib().dq8_error_stats, x.get_device(), int(kind), x.data_ptr(), n, int(block), scales.data_ptr(),
             SCALES_GIVEN if scales_given else 0, stats.data_ptr(), means.data_ptr())
    return stats, means


# types of keys, values and queries (include/dq8_cache.h)
_TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


def cache_buffers(pages, kv_heads, page_size, dim, device="cuda"):
    """(codes, scales) of an empty paged cache: uint8[2, pages, kv_heads, page_size, dim] and float32[2, pages, kv_heads, page_size],
    keys before values, every row a zero."""
    shape = (2, int(pages), int(kv_heads), int(page_size), int(dim))
    return torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(shape[:-1], dtype=torch.float32, device=device)


def _int32(v, what):
    """v as an int that a field of 32 bits holds (ctypes takes any other modulo 2^32)."""
    v = int(v)
    if not -2 ** 31 <= v < 2 ** 31:
        raise ValueError("%s does not fit 32 bits: %d" % (what, v))
    return v


def _cache(codes, scales):
    _dev(codes, torch.uint8, "codes")
    _dev(scales, torch.float32, "scales")
    if codes.dim() != 5 or codes.shape[0] != 2 or scales.shape != codes.shape[:-1]:
        raise ValueError("codes must be [2, pages, kv_heads, page_size, dim] and scales the same without the last axis")
    if scales.device != codes.device:
        raise ValueError("codes and scales are on different devices")
    return _Cache(codes.data_ptr(), scales.data_ptr(), codes.shape[1], *(_int32(n, "an axis of codes") for n in codes.shape[2:]))


def _on(device, t, dtype, shape, what):
    """A contiguous tensor of exactly this type, shape and device."""
    _dev(t, dtype, what)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s must have shape %s, got %s" % (what, tuple(shape), tuple(t.shape)))
    if t.device != device:
        raise ValueError("%s is on another device than the cache" % what)
    return t.data_ptr()


def _rows(t, what, device, dtype, tokens, heads, dim):
    """[tokens, heads, dim] with the elements of a row side by side, any other strides: (address, token stride, head stride)."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError("%s must be a CUDA tensor" % what)
    if t.dtype != dtype:
        raise TypeError("%s must be %s, got %s" % (what, dtype, t.dtype))
    if t.dim() != 3 or (tokens is not None and t.shape[0] != tokens) or (heads is not None and t.shape[1] != heads) or t.shape[2] != dim:
        raise ValueError("%s must have shape [tokens, heads, dim] = [%s, %s, %d], got %s"
                         % (what, "any" if tokens is None else tokens, "any" if heads is None else heads, dim, tuple(t.shape)))
    if t.stride(2) != 1 and t.numel():
        raise ValueError("the elements of a row of %s must lie side by side" % what)
    if t.device != device:
        raise ValueError("%s is on another device than the cache" % what)
    return t.data_ptr(), t.stride(0), t.stride(1)


def cache_append(kind, k, v, slots, codes, scales, positions=None, rotation=None, interleaved=False, q=None, q_weight=None,
                 k_weight=None, eps=1e-6, q_out=None):
    """Compresses keys and values [tokens, kv_heads, dim] into the cache rows that ``slots`` (int64, slot = page * page_size +
    place; any other number: padding) name, after the norm (``k_weight``) and the rotation (``rotation`` float32[n, 2, half]: cosines
    and sines of every position, ``positions`` int64) of the keys.  Queries [tokens, heads, dim] get theirs in the same pass.

    k, v and q may be views whose rows are contiguous (parts of a projection's output).  Returns the queries (``q_out``, a new tensor
    or q itself), None without q.  For serving: as with every call here no gradient passes through it."""
    done = _native.cache_append(kind, k, v, slots, codes, scales, positions, rotation, interleaved, q, q_weight, k_weight, eps, q_out)
    if done is not None:
        return None if done is False else done
    c = _cache(codes, scales)
    dev, dim = codes.device, c.dim
    if not isinstance(k, torch.Tensor) or k.dtype not in _TYPES:
        raise TypeError("k must be a float32, bfloat16 or float16 tensor")
    tokens = k.shape[0] if k.dim() == 3 else None
    a = _Append()
    a.type = _TYPES[k.dtype]
    a.k, a.k_token_stride, a.k_head_stride = _rows(k, "k", dev, k.dtype, tokens, c.kv_heads, dim)
    a.v, a.v_token_stride, a.v_head_stride = _rows(v, "v", dev, k.dtype, tokens, c.kv_heads, dim)
    a.tokens = tokens
    a.slots = _on(dev, slots, torch.int64, (tokens,), "slots")
    if q is not None:
        a.q, a.q_token_stride, a.q_head_stride = _rows(q, "q", dev, k.dtype, tokens, None, dim)
        a.heads = _int32(q.shape[1], "the number of query heads")
        if q_out is None:
            q_out = torch.empty(q.shape, dtype=q.dtype, device=dev)
        a.q_out, a.q_out_token_stride, a.q_out_head_stride = _rows(q_out, "q_out", dev, k.dtype, tokens, a.heads, dim)
    elif q_out is not None or q_weight is not None:
        raise ValueError("q_out and q_weight need q")
    if rotation is not None:
        if not isinstance(rotation, torch.Tensor) or rotation.dim() != 3 or rotation.shape[1] != 2:
            raise ValueError("rotation must be [positions, 2, half]")
        if positions is None:
            raise ValueError("rotation needs positions")
        a.rotation = _on(dev, rotation, torch.float32, rotation.shape, "rotation")
        a.positions = _on(dev, positions, torch.int64, (tokens,), "positions")
        a.n_positions, a.half, a.interleaved = rotation.shape[0], _int32(rotation.shape[2], "an axis of rotation"), bool(interleaved)
    elif positions is not None:
        raise ValueError("positions need a rotation")
    if q_weight is not None:
        a.q_weight = _on(dev, q_weight, torch.float32, (dim,), "q_weight")
    if k_weight is not None:
        a.k_weight = _on(dev, k_weight, torch.float32, (dim,), "k_weight")
    a.eps = float(eps)
    _enqueue(lib().dq8_cache_append, codes.get_device(), _int32(kind, "kind"), ctypes.byref(c), ctypes.byref(a))
    return q_out


def _attention(q, codes, scales, pages, lens, starts, max_new, softmax_scale, window, out):
    c = _cache(codes, scales)
    dev, dim = codes.device, c.dim
    if not isinstance(q, torch.Tensor) or q.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("q must be a bfloat16 or float16 tensor")
    a = _Attention()
    a.type = _TYPES[q.dtype]
    a.q, a.q_token_stride, a.q_head_stride = _rows(q, "q", dev, q.dtype, None, None, dim)
    a.tokens, a.heads = q.shape[0], _int32(q.shape[1], "the number of query heads")
    if not isinstance(pages, torch.Tensor) or pages.dim() != 2:
        raise ValueError("pages must be [sequences, pages of the longest]")
    a.batch, a.max_pages = pages.shape
    a.pages = _on(dev, pages, torch.int32, pages.shape, "pages")
    a.lens = _on(dev, lens, torch.int32, (a.batch,), "lens")
    if starts is not None:
        a.starts = _on(dev, starts, torch.int32, (a.batch + 1,), "starts")
    if max_new is not None:
        if not 0 <= int(max_new) < 2 ** 63:
            raise ValueError("max_new must be a number of tokens, got %d" % int(max_new))
        a.max_new = int(max_new)
    a.window = _int32(window, "window")
    a.softmax_scale = dim ** -0.5 if softmax_scale is None else float(softmax_scale)
    if out is not None:
        a.out, a.out_token_stride, a.out_head_stride = _rows(out, "out", dev, q.dtype, a.tokens, a.heads, dim)
    return c, a


def cache_attention_workspace(q, codes, scales, pages, lens, starts=None, max_new=None):
    """Bytes of scratch memory that cache_attention can use for these arguments."""
    c, a = _attention(q, codes, scales, pages, lens, starts, max_new, None, 0, None)
    with torch.cuda.device(codes.device):
        return int(lib().dq8_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(a)))


def cache_attention(kind, q, codes, scales, pages, lens, starts=None, max_new=None, softmax_scale=None, window=0, out=None, workspace=None):
    """Causal attention of new tokens q [tokens, heads, dim] (bfloat16 or float16) over the cached keys and values of their
    sequences, several query heads per cached head.

    pages int32 [sequences, n]: the page numbers of each sequence in order; lens int32 [sequences]: its cached tokens, the new ones
    among them.  starts int32 [sequences + 1]: where each sequence's new tokens begin in q; None: every sequence has as many.
    max_new: the largest number of new tokens of a sequence, where the host knows it.  window > 0: a query sees that many tokens at most.
    workspace: a uint8 tensor of cache_attention_workspace() bytes; None: taken from torch's allocator, and not while the stream is
    captured into a graph (hand one in there: without it one wavefront or workgroup reads the whole of a sequence's head).  For
    serving: as with every call here no gradient passes through it."""
    done = _native.cache_attention(kind, q, codes, scales, pages, lens, starts, max_new, softmax_scale, window, out, workspace)
    if done is not None:
        return done
    c, a = _attention(q, codes, scales, pages, lens, starts, max_new, softmax_scale, window, out)
    if out is None:
        out = torch.empty(q.shape, dtype=q.dtype, device=codes.device)
        a.out, a.out_token_stride, a.out_head_stride = out.data_ptr(), out.stride(0), out.stride(1)
    if workspace is None:
        with torch.cuda.device(codes.device):
            if not torch.cuda.is_current_stream_capturing():
                workspace = torch.empty(int(lib().dq8_cache_attention_workspace_bytes(ctypes.byref(c), ctypes.byref(a))), dtype=torch.uint8,
                                        device=codes.device)
    else:
        _dev(workspace, torch.uint8, "workspace")
        if workspace.device != codes.device:
            raise ValueError("workspace is on another device than the cache")
    _enqueue(lib().dq8_cache_attention, codes.get_device(), _int32(kind, "kind"), ctypes.byref(c), ctypes.byref(a),
             workspace.data_ptr() if workspace is not None and workspace.numel() else None, 0 if workspace is None else workspace.numel())
    return out


def model_speedup(n_gpus, total_ms, fc_ms, conv_penalty_ms, sub_batches, parallel_fc_ms, fc_penalty_ms):
    """Predicted speed-up of the single-node model (host arithmetic in the library)."""
    out = ctypes.c_double()
    _check(lib().dq8_model_speedup(int(n_gpus), total_ms, fc_ms, conv_penalty_ms, int(sub_batches), parallel_fc_ms,
                                   fc_penalty_ms, ctypes.byref(out)), "dq8_model_speedup")
    return out.value


def model_penalty(transfer_ms, compute_ms):
    """Sum of the parts of the transfers that their overlapping computations do not cover."""
    n = len(transfer_ms)
    if n != len(compute_ms):
        raise ValueError("transfer_ms and compute_ms differ in length")
    arr = ctypes.c_double * max(n, 1)
    out = ctypes.c_double()
    _check(lib().dq8_model_penalty(arr(*transfer_ms), arr(*compute_ms), n, ctypes.byref(out)), "dq8_model_penalty")
    return out.value
