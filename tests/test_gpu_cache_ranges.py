"""GPU: attention over the cache at the ends of the range of values.

The reference is that of the other cache tests, in 64 bits; its tolerance for weights below the normal range of binary16 goes by the
largest value that a query sees.  Here that term is the smaller one that include/dq8_cache.h states: a weight times its value's scale is off by
2^-30 of the largest such product of its query, whatever other queries see."""
import numpy as np
import pytest

import oracle
from tests.test_gpu_cache import attention_inputs, check_attention, dq8, host, to_gpu  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def attention_by_weight(kind, cache, q, pages, lens, starts, softmax_scale, window=0):
    """(out, tolerance) float64 as of cache_reference.attention, with the last term of the tolerance by each query's own products."""
    codes, scales = cache
    cb = oracle.codebook(kind).astype(np.float64)
    page, kv, dim = codes.shape[3], codes.shape[2], codes.shape[4]
    out, tol, u = np.zeros(q.shape), np.zeros(q.shape), 2.0 ** -11
    for b in range(len(lens)):
        first, n, length = int(starts[b]), int(starts[b + 1] - starts[b]), int(lens[b])
        j = np.arange(length)
        number, place = pages[b, j // page], j % page
        for h in range(kv):
            with np.errstate(invalid="ignore"):
                k, v = (cb[codes[part, number, h, place]] * scales[part, number, h, place].astype(np.float64)[:, None] for part in (0, 1))
            f = scales[1, number, h, place].astype(np.float64)
            for i in range(n):
                p = length - n + i
                see = (j <= p) & ((j > p - window) if window else True)
                for x in range(h * q.shape[1] // kv, (h + 1) * q.shape[1] // kv) if see.any() else ():
                    row = q[first + i, x].astype(np.float64)
                    s = k[see] @ row * softmax_scale
                    w = np.exp(s - s.max())
                    w /= w.sum()
                    e = (np.abs(k[see]) @ np.abs(row)).max() * abs(softmax_scale) * (u + (dim + 8) * 2.0 ** -24)
                    assert e < 2.0 ** -6, "inputs outside the derivation"
                    out[first + i, x] = w @ v[see]
                    tol[first + i, x] = (w @ np.abs(v[see]) * (2 * u + 2 * e + (8 + length) * 2.0 ** -24) * (1 + 2.0 ** -5)
                                         + see.sum() * 2.0 ** -30 * (w * f[see]).max())
    return out, tol


def check_both_kernels(dq8, kind, cache, q, pages, lens, starts, window=0, scale=None):
    """Both kernels (max_new chooses), their jobs cut or whole; all agree with the reference."""
    dim = q.shape[2]
    want, tol = attention_by_weight(kind, cache, host(q), pages, lens, starts, dim ** -0.5 if scale is None else scale, window)
    cuda = lambda a: torch.from_numpy(a).cuda()
    args = (kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens))
    for max_new in (1, q.shape[0]):
        for workspace in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            got = dq8.cache_attention(*args, starts=cuda(starts), max_new=max_new, window=window, workspace=workspace, softmax_scale=scale)
            check_attention(got, q, want, tol)


@pytest.mark.parametrize("n,cached", [(1, 3000), (5, 2000), (140, 1500)])
@pytest.mark.parametrize("size", [1e30, 1e34, 2e37])
def test_values_near_the_end_of_binary32(dq8, n, cached, size):
    """Outputs are finite whether or not the tokens are cut into parts that are joined: sums of weighted values need not be."""
    for dim in (64, 128):
        case = (0, "bf16", 4, 1, dim, 64, [(n, cached)], 0)
        cache, q, pages, lens, starts = attention_inputs(dq8, case)
        cache[1][1] *= np.float32(size)
        check_both_kernels(dq8, 0, cache, q, pages, lens, starts)
