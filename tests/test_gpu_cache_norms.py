"""GPU: norms of queries and keys whose squares lie at the ends of binary32 or outside."""
import numpy as np
import pytest

from tests import cache_reference as ref
from tests.test_gpu_cache import TYPES, dq8, half_step, host, new_cache, to_gpu  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("type_", ["bf16", "f32"])
@pytest.mark.parametrize("eps", [0.0, 1e-30, 1e-12, 1e-6, 1e3, 1e30])
@pytest.mark.parametrize("dim", [64, 80, 256])
def test_norms_of_rows_of_any_size(dq8, type_, eps, dim):
    """Rows of 1e-36 to 3e37 in one call, neighbours in a wavefront; a row of zeros is 0 / 0 only with eps 0."""
    rng, t = np.random.default_rng(dim), TYPES[type_]
    sizes = 10.0 ** np.arange(-36, 38.0)
    tokens, heads, kv, page = len(sizes) + 1, 3, 2, 16
    cache = new_cache(0, rng, 6, kv, page, dim)
    gpu = to_gpu(cache)
    both = rng.normal(size=(tokens, heads + 2 * kv, dim)).clip(-2.9, 2.9)
    both[:-1] *= rng.permutation(sizes)[:, None, None]
    both[-1] = 0.0
    q, k, v = torch.from_numpy(both).to(t).cuda().split([heads, kv, kv], 1)
    slots, w = np.arange(tokens, dtype=np.int64), rng.uniform(0.5, 1.5, dim).astype(np.float32)
    cuda = lambda a: torch.from_numpy(a).cuda()
    got = host(dq8.cache_append(0, k, v, cuda(slots), *gpu, q=q, q_weight=cuda(w), k_weight=cuda(w), eps=eps))
    with np.errstate(invalid="ignore"):
        want = ref.append(0, cache, host(k), host(v), slots, host(q), w, w, eps)
    nan = np.isnan(want)
    assert nan[-1].all() == (eps == 0.0) and not nan[:-1].any()
    # binary32 inside: the sum (dim + 2 roundings, halved by the root), the quotient, two products; below the normal range of binary32 the
    # first product is off by half of the least step, 2^-150, which the weight multiplies by 1.5 at most, and the result by half a step of
    # its own type
    tol = (half_step(t) * np.abs(want) * (1 + 2.0 ** -10) + ((dim + 2) / 2 + 6) * 2.0 ** -24 * np.abs(want)
           + 1.5 * 2.0 ** -150 + torch.finfo(t).tiny * half_step(t))
    assert np.array_equal(np.isnan(got), nan)
    assert (np.abs(got - want)[~nan] <= tol[~nan]).all()
    there = np.isfinite(cache[1])
    assert np.array_equal(gpu[1].cpu().numpy()[there], cache[1][there]) and np.array_equal(gpu[0].cpu().numpy()[there], cache[0][there])
