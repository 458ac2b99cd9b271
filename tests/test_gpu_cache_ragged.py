"""GPU: batches of more than 64 sequences with different numbers of new tokens, where a lane counts several of them: both kernels, jobs cut
and whole, against float64 on the GPU."""
import numpy as np
import pytest

from tests.test_gpu_cache import dq8, half_step  # noqa: F401

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu


def ragged_reference(dq8, kind, codes, scales, q, pages, lens, starts, window):
    """(out, tolerance) as of cache_reference.attention, per sequence and cached head."""
    values, (kv, page, dim) = dq8.codebook(kind).double().cuda(), codes.shape[2:]
    group = q.shape[1] // kv
    out, tol, u = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda"), 2.0 ** -11
    for b in range(len(lens)):
        first, end, length = starts[b], starts[b + 1], lens[b]
        if first == end or length == 0:
            continue
        j, pos = torch.arange(length, device="cuda"), torch.arange(length - (end - first), length, device="cuda").repeat_interleave(group)[:, None]
        hidden = (j > pos) | (j <= pos - window) if window else j > pos
        sees = ~hidden.all(1, keepdim=True)
        number = pages[b, : -(-length // page)].long()
        k, v = (values[codes[p, number].transpose(0, 1).reshape(kv, -1, dim)[:, :length].int()]
                * scales[p, number].transpose(0, 1).reshape(kv, -1)[:, :length, None].double() for p in (0, 1))
        rows = q[first:end].view(-1, kv, group, dim).transpose(0, 1).reshape(kv, -1, dim).double()
        s = torch.matmul(rows, k.transpose(1, 2).contiguous()) * dim ** -0.5
        w = torch.nan_to_num(torch.softmax(s.masked_fill(hidden, float("-inf")), 2))
        e = torch.matmul(rows.abs(), k.abs().transpose(1, 2).contiguous()).amax(2, keepdim=True) * dim ** -0.5 * (u + (dim + 8) * 2.0 ** -24)
        assert e.max() < 2.0 ** -6
        t = (torch.matmul(w, v.abs()) * (2 * u + 2 * e + (8 + length) * 2.0 ** -24) * (1 + 2.0 ** -5) + length * 2.0 ** -30 * v.abs().amax()) * sees
        put = lambda x: x.view(kv, end - first, group, dim).transpose(0, 1).reshape(end - first, kv * group, dim)
        out[first:end], tol[first:end] = put(torch.matmul(w, v)), put(t)
    return out, tol


@pytest.mark.parametrize("window", [0, 37])
@pytest.mark.parametrize("batch,most,longest,heads,kv,dim", [(65, 9, 400, 8, 2, 128), (130, 40, 150, 4, 1, 64), (130, 3, 90, 4, 4, 256),
                                                              (300, 70, 100, 6, 2, 80), (300, 5, 2000, 16, 1, 128), (4500, 3, 20, 2, 1, 16)])
def test_many_sequences_of_unequal_numbers_of_new_tokens(dq8, batch, most, longest, heads, kv, dim, window):
    g, rng, page = torch.Generator(device="cuda").manual_seed(batch + dim), np.random.default_rng(batch + dim), 16
    new = rng.integers(0, most + 1, batch)
    new[rng.integers(0, batch, batch // 8)] = 0  # sequences without a new token, some in a row
    new[batch // 2: batch // 2 + 5] = 0
    new[0], new[-1] = most, most
    lens = np.where(rng.random(batch) < 0.1, rng.integers(0, 3, batch), rng.integers(1, longest + 1, batch))  # some shorter than their new tokens
    lens[1], lens[-1] = 0, longest
    starts = np.concatenate([[0], np.cumsum(new)])
    per = -(-longest // page)
    pool = batch * per + 1
    codes = torch.randint(0, 256, (2, pool, kv, page, dim), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.rand((2, pool, kv, page), device="cuda", generator=g) + 0.5
    pages = torch.randperm(pool, device="cuda", generator=g)[:batch * per].to(torch.int32).view(batch, per)
    tokens, behind = int(starts[-1]), 7
    q = (torch.randn((tokens + behind, heads, dim), device="cuda", generator=g) * 0.7).to(torch.bfloat16)
    want, tol = ragged_reference(dq8, 0, codes, scales, q[:tokens], pages, lens.tolist(), starts.tolist(), window)
    i32 = lambda a: torch.from_numpy(a.astype(np.int32)).cuda()
    step = half_step(q.dtype)
    allowed = tol + step * (want.abs() + tol) + torch.finfo(q.dtype).tiny * step
    for max_new in (1, most, 0, None, tokens):
        for workspace in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
            out = torch.full_like(q, 5.0)
            dq8.cache_attention(0, q, codes, scales, pages, i32(lens), starts=i32(starts), max_new=max_new, window=window, out=out, workspace=workspace)
            off = (out[:tokens].double() - want).abs()
            assert (off <= allowed).all(), (max_new, workspace is None, (off / allowed).max())
            assert (out[tokens:] == 5.0).all()
