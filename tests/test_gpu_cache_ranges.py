"""GPU: attention over the cache where the scales of values lie far apart, and what a query does not see.

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


#: (type, heads, kv_heads, dim, page, new tokens, cached): the largest max_new is more than 128 rows of a cached head
SHAPES = [("f16", 8, 2, 64, 16, 40, 140), ("bf16", 4, 1, 128, 32, 40, 1300), ("bf16", 2, 1, 256, 16, 70, 300), ("f16", 5, 1, 80, 16, 33, 33)]


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%s_d%d" % (s[0], s[3]))
@pytest.mark.parametrize("power", [20, 24, 28, 31, 60, 110])
def test_values_of_later_tokens_do_not_count(dq8, shape, power):
    """The new tokens' values grow from scales near one to scales near 2^power: an earlier query sees none of the large ones."""
    type_, heads, kv, dim, page, n, cached = shape
    case = (0, "bf16" if power > 16 else type_, heads, kv, dim, page, [(n, cached)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    j = np.arange(cached - n, cached)
    cache[1][1, pages[0, j // page], :, j % page] *= 2.0 ** np.linspace(0, power, n)[:, None].astype(np.float32)
    check_both_kernels(dq8, 0, cache, q, pages, lens, starts)


@pytest.mark.parametrize("power", [24, 60, 120])
def test_one_large_value_at_the_end(dq8, power):
    """Two new tokens, the second one's value larger by 2^power: the first query's output is that of a cache without it."""
    for n in (2, 140):
        case = (0, "bf16", 2, 2, 64, 16, [(n, n + 30)], 0)
        cache, q, pages, lens, starts = attention_inputs(dq8, case)
        last = n + 29
        cache[1][1, pages[0, last // 16], :, last % 16] = 2.0 ** power
        check_both_kernels(dq8, 0, cache, q, pages, lens, starts)


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "%s_d%d" % (s[0], s[3]))
@pytest.mark.parametrize("garbage", [1e30, 3.4e38, float("inf"), float("nan")])
def test_what_lies_below_a_window_may_be_anything(dq8, shape, garbage):
    """A window whose lower end lies inside a tile: scales of keys and values before it, in the same tile too."""
    type_, heads, kv, dim, page, n, cached = shape
    window = 21
    case = (2, type_, heads, kv, dim, page, [(n, cached)], window)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    j = np.arange(max(cached - n - window + 1, 0))
    cache[1][:, pages[0, j // page], :, j % page] = garbage
    check_both_kernels(dq8, 2, cache, q, pages, lens, starts, window)


@pytest.mark.parametrize("n", [2, 140])
@pytest.mark.parametrize("place", [0, 45, 99])
def test_a_large_value_with_hardly_any_weight(dq8, n, place):
    """A token that every query sees with a weight of about e^-28, its value larger by 2^30: both ends of the sum count."""
    kind, dim, page = 0, 64, 16
    case = (kind, "bf16", 2, 1, dim, page, [(n, n + 100)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    cb = oracle.codebook(kind)
    j = np.arange(n + 100)
    q = torch.full_like(q, 1.0)
    cache[0][0, pages[0, j // page], 0, j % page] = int(np.argmax(cb))  # every key the row's maximum
    cache[1][0, pages[0, j // page], 0, j % page] = 0.25 + 0.01 * (j % 7)
    at = pages[0, place // page], 0, place % page
    cache[0][(0,) + at] = int(np.argmin(cb))  # and this one its opposite
    cache[1][(0,) + at] = 3.25
    cache[1][(1,) + at] = 2.0 ** 30
    check_both_kernels(dq8, kind, cache, q, pages, lens, starts)


@pytest.mark.parametrize("shape", SHAPES[:3], ids=lambda s: "%s_d%d" % (s[0], s[3]))
@pytest.mark.parametrize("low,high", [(-36, 36), (-36, -30), (30, 38), (-4, 4)])
def test_scales_of_any_size_in_any_order(dq8, shape, low, high):
    _, heads, kv, dim, page, n, cached = shape
    case = (3, "bf16", heads, kv, dim, page, [(n, cached)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    rng = np.random.default_rng(dim + low)
    there = np.isfinite(cache[1][1])
    cache[1][1][there] = np.minimum(10.0 ** rng.uniform(low, high, there.sum()), 3e38).astype(np.float32)
    check_both_kernels(dq8, 3, cache, q, pages, lens, starts)


@pytest.mark.parametrize("n", [2, 140])
def test_values_of_zeros_under_the_largest_weights(dq8, n):
    """Rows of zeros have the scale zero.  Under most of the weight they leave the others' sum small, not empty."""
    kind, dim, page = 1, 128, 16
    case = (kind, "bf16", 1, 1, dim, page, [(n, n + 75)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    j = np.arange(n + 75)
    q = torch.full_like(q, 0.5)
    cache[0][0, pages[0, j // page], 0, j % page] = np.where(j % 3 == 0, 127, 255)[:, None]  # the row's maximum, or its opposite
    cache[1][0, pages[0, j // page], 0, j % page] = np.where(j % 3 == 0, 3.0, 2.0)
    cache[1][1, pages[0, j[::3] // page], 0, j[::3] % page] = 0.0
    check_both_kernels(dq8, kind, cache, q, pages, lens, starts)


@pytest.mark.parametrize("n", [2, 140])
def test_a_value_that_stands_for_nan_reaches_its_viewers_only(dq8, n):
    kind, dim, page = 0, 64, 16
    case = (kind, "bf16", 2, 1, dim, page, [(n, n + 60)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = attention_by_weight(kind, cache, host(q), pages, lens, starts, dim ** -0.5)
    bad = n + 60 - n // 2 - 1  # a new token in the middle
    cache[1][1, pages[0, bad // page], 0, bad % page] = np.nan
    cuda = lambda a: torch.from_numpy(a).cuda()
    for max_new in (1, n):
        got = dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(starts), max_new=max_new)
        first = bad - 60
        assert torch.isnan(got[first:]).all()
        check_attention(got[:first], q[:first], want[:first], tol[:first])


@pytest.mark.parametrize("n", [2, 140])
@pytest.mark.parametrize("scale", [3.4e38, -3.4e38, 1e38, 2.0 ** 98, 2.0 ** 101, 2.0 ** 102, -2.0 ** 103, 2.0 ** 104, 2.0 ** 106])
def test_the_largest_softmax_scales(dq8, n, scale):
    """Queries of about 2^-80, scores of about 2^20 to 2^50: they differ by far more than weights can say, and each output is one token's
    value.  A step between binary32 scores of this size is larger than the range of a product in binary16 leaves room for."""
    kind, dim, page = 0, 64, 16
    case = (kind, "bf16", 2, 1, dim, page, [(n, n + 100)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    q = (q.float() * 2.0 ** -80).to(q.dtype)
    cache[1][1] *= 2.0 ** np.random.default_rng(n).uniform(-20, 20, cache[1][1].shape).astype(np.float32)
    cb = oracle.codebook(kind).astype(np.float64)
    j = np.arange(n + 100)
    k, v = (cb[cache[0][part, pages[0, j // page], 0, j % page]] * cache[1][part, pages[0, j // page], 0, j % page][:, None] for part in (0, 1))
    cuda = lambda a: torch.from_numpy(a).cuda()
    for max_new in (1, n):
        got = host(dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(starts), max_new=max_new, softmax_scale=scale))
        for i in range(n):
            for h in range(2):
                s = k[:101 + i] @ host(q)[i, h].astype(np.float64) * np.sign(scale)
                best, second = np.argsort(s)[:-3:-1]
                # keys are off by 2^-11, sums by (dim + 8) 2^-24 of the sum of magnitudes; a closer second is not told apart
                if s[best] - s[second] > 2 * (2.0 ** -11 + (dim + 8) * 2.0 ** -24) * (np.abs(k[:101 + i]) @ np.abs(host(q)[i, h])).max():
                    assert (np.abs(got[i, h] - v[best]) <= (2.0 ** -8 + 2.0 ** -10) * np.abs(v[best])).all()


@pytest.mark.parametrize("n", [1, 5, 140])
@pytest.mark.parametrize("power", [0, 18, 24, 26, 60])
def test_ties_of_large_scores(dq8, n, power):
    """All keys alike: every token has the same weight whatever the size of the scores, also where the tokens are cut into parts."""
    kind, dim, page, cached = 0, 64, 64, 2001
    case = (kind, "bf16", 4, 1, dim, page, [(n, cached)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    cache[0][0] = cache[0][0, 0, 0, 0]
    cache[1][0][np.isfinite(cache[1][0])] = 1.5
    q = (q.float() * 2.0 ** power).to(q.dtype)
    j = np.arange(cached)
    v = oracle.codebook(kind).astype(np.float64)[cache[0][1, pages[0, j // page], 0, j % page]] * cache[1][1, pages[0, j // page], 0, j % page].astype(np.float64)[:, None]
    count = np.arange(cached - n + 1, cached + 1)[:, None]
    want, size = (np.cumsum(x, 0)[cached - n:] / count for x in (v, np.abs(v)))
    # a code's value and a weight times a scale are rounded once to 11 bits; sums of `cached` terms in binary32
    tol = size * (2 * 2.0 ** -11 + (8 + cached) * 2.0 ** -24) * (1 + 2.0 ** -5)
    cuda = lambda a: torch.from_numpy(a).cuda()
    for max_new in (1, n):
        for workspace in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            got = dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(starts), max_new=max_new, workspace=workspace)
            check_attention(got, q, np.repeat(want[:, None], 4, 1), np.repeat(tol[:, None], 4, 1))
