"""GPU: calls for the cache whose numbers do not fit the fields of the C interface."""
import pytest

from tests.test_gpu_cache import dq8  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def test_numbers_that_do_not_fit_are_refused(dq8):
    codes, scales = dq8.cache_buffers(4, 2, 16, 64)
    k = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.arange(3, device="cuda")
    pages, lens = torch.zeros((3, 1), dtype=torch.int32, device="cuda"), torch.ones(3, dtype=torch.int32, device="cuda")
    out = torch.full_like(q, 3.0)
    attend = lambda kind=0, q=q, **other: dq8.cache_attention(kind, q, codes, scales, pages, lens, out=out, **other)
    bad = [lambda w=w: attend(window=w) for w in (-2 ** 32, -2 ** 32 + 5, -2 ** 31 - 1, 2 ** 31, 2 ** 32, 2 ** 40 + 1)]
    bad += [lambda m=m: attend(max_new=m) for m in (-1, -2 ** 64, -2 ** 64 + 3, 2 ** 64 + 3)]
    bad += [lambda m=m: dq8.cache_attention_workspace(q, codes, scales, pages, lens, max_new=m) for m in (-1, 2 ** 64 + 3)]
    bad += [lambda: attend(kind=2 ** 32), lambda: attend(kind=-2 ** 32 + 1), lambda: dq8.cache_append(2 ** 32, k, k, slots, codes, scales)]
    many = q[:, :1].expand(3, 2 ** 32 + 4, 64)  # a view: no memory behind it
    bad += [lambda: attend(q=many), lambda: dq8.cache_append(0, k, k, slots, codes, scales, q=many, q_out=many)]
    for i, call in enumerate(bad):
        with pytest.raises(ValueError):
            call()
            pytest.fail("refusal %d" % i)
    torch.cuda.synchronize()
    assert (out == 3.0).all() and not codes.any() and not scales.any()
    assert attend(window=2 ** 31 - 1, max_new=2 ** 63 - 1) is out and not out.any()
