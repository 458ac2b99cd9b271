"""Verification behind a plan that refused sequences: their rows hold no tokens, and the drop that they were refused with goes on to the next plan."""
import numpy as np
import pytest
import torch

from paper_1511_04561_amd import dq8

from .serve_refused import verify_of_plan
from .test_gpu_serve import dev, drafts

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64


# vocabularies of one launch and of two
@pytest.mark.parametrize("dtype,vocab", [(torch.float32, 501), (torch.bfloat16, 501), (torch.float32, 70001), (torch.float16, 150000)])
@pytest.mark.parametrize("sure", [False, True])
def test_verifications_of_refused_sequences(dtype, vocab, sure):
    rows = [1, 6, 2, 0, 9, 1, 3, 70, 2]
    p, q, ids, uniform, rng = drafts(sum(rows), vocab, vocab, dtype, sure)
    starts = np.concatenate([[0], np.cumsum(rows)]).astype(np.int32)
    args = [p.cuda(), dev(ids, I64), dev(uniform), dev(rng.random(len(rows)).astype(np.float32))]
    given = {"starts": dev(starts), "draft": None if q is None else q.cuda()}
    n = dq8.draft_verify_workspace(*args, **given)
    assert (n != 0) == (vocab > 60000)
    drop = np.array([3, -7, 10 ** 9, 4, 0, 2 ** 31 - 1, 1, 5, -(2 ** 31)], np.int32)
    for granted in ([-1] * 9, [1, -1, 2, -1, -1, 1, -5, -1, 2], [0] * 9, [-(2 ** 31), 6, -1, 0, 9, -1, 3, 70, -1]):
        granted = np.array(granted, np.int32)
        for d in (None, drop):
            want = verify_of_plan(p.double().numpy(), ids, uniform, args[3].cpu().numpy(), starts, None if q is None else q.double().numpy(), granted, d)
            for space in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
                got = dq8.draft_verify(*args, **given, workspace=space, granted=dev(granted), drop=None if d is None else dev(d))
                assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
        # in place: what the plan was given becomes what the next one is given
        state = dev(drop)
        got = dq8.draft_verify(*args, **given, granted=dev(granted), drop=state, rejected=state)
        assert got[2] is state and all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
    # without granted the plan refused nobody, and drop is not looked at
    want = dq8.draft_verify(*args, **given)
    assert all(torch.equal(a, b) for a, b in zip(dq8.draft_verify(*args, **given, drop=dev(drop)), want))


def test_the_python_path_gives_the_same(monkeypatch):
    p, q, ids, uniform, rng = drafts(8, 300, 5, torch.float16)
    args = [p.cuda(), dev(ids, I64), dev(uniform), dev(rng.random(2).astype(np.float32))]
    more = {"draft": q.cuda(), "granted": dev([-1, 4], I32), "drop": dev([3, 2], I32)}
    want = dq8.draft_verify(*args, **more)
    assert want[1][0] == -1 and want[2][0] == 3 and (want[0][:4] == -1).all() and want[1][1] >= 0
    monkeypatch.setattr(dq8, "_native", dq8._Unbound())
    assert all(torch.equal(a, b) for a, b in zip(dq8.draft_verify(*args, **more), want))
    for error, wrong in ((ValueError, {"granted": dev([1], I32)}), (TypeError, {"granted": dev([1, 1], I64)}), (TypeError, {"drop": [1, 2]}), (ValueError, {"drop": dev([1] * 3, I32)}),
                         (TypeError, {"granted": torch.ones(2, dtype=I32)})):
        with pytest.raises(error):
            dq8.draft_verify(*args, **{**more, **wrong})


def test_steps_of_decoding_with_refusals():
    """Steps of a batch whose cache is too small for all: sequences are refused for lack of pages and granted later, when others have ended.  `rejected` is the next
    plan's `drop` throughout, captured into a graph.  A row of the cache depends on its token and position only, so that every cached row is compared bit for bit
    with that of the same tokens appended at once."""
    kv, dim, page, vocab, batch, wide, n_pages, most = 2, 64, 16, 97, 5, 5, 14, 3
    torch.manual_seed(4)
    gen = np.random.default_rng(4)
    keys = torch.randn(vocab, kv, dim, device="cuda").bfloat16()
    table = torch.softmax(2 * torch.randn(vocab, vocab, device="cuda"), 1)
    angle = torch.arange(128, device="cuda")[:, None] * 100.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))
    rotation = torch.stack([angle.cos(), angle.sin()], 1).contiguous()
    codes, scales = dq8.cache_buffers(n_pages, kv, page, dim)
    free, n_free = dq8.cache_free_list(n_pages)
    pages, lens, drop = (torch.zeros(s, dtype=I32, device="cuda") for s in ((batch, wide), batch, batch))
    ids, new = torch.zeros(batch * most, dtype=I64, device="cuda"), torch.full((batch,), most, dtype=I32, device="cuda")
    uniform, sample, noise = (torch.rand(s, device="cuda") for s in (batch * most, batch, (batch * most, vocab)))

    def step(codes, scales, pages, lens, free, n_free, drop):
        slots, positions, starts, _, granted, _ = dq8.cache_plan(lens, new, pages, free, n_free, page, len(ids), drop=drop, lens_out=lens, n_free_out=n_free)
        dq8.cache_append(dq8.DYNAMIC_TREE, keys[ids], keys[ids].flip(2).contiguous(), slots, codes, scales, positions=positions, rotation=rotation)
        # behind rows without a place there is anything at all
        target = torch.where((slots < 0)[:, None], noise, table[ids])
        draft = torch.full_like(target, 0.5 / vocab)
        draft[:-1] += torch.nn.functional.one_hot(ids[1:], vocab) * 0.5
        out, accepted, _ = dq8.draft_verify(target, ids, uniform, sample, starts=starts, draft=draft, granted=granted, drop=drop, rejected=drop)
        return granted, out, accepted, starts

    state = (codes, scales, pages, lens, free, n_free, drop)
    so_far = [gen.integers(0, vocab, gen.integers(4, 30)).tolist() for _ in range(batch)]
    # prompts come in by an eager plan, as many as fit
    for b in range(batch):
        so_far[b] = so_far[b][:25]
    prompt = torch.tensor(sum((s[:-1] for s in so_far), []), device="cuda")
    slots, positions, _, _, granted, _ = dq8.cache_plan(lens, dev([len(s) - 1 for s in so_far], I32), pages, free, n_free, page, len(prompt), lens_out=lens, n_free_out=n_free)
    assert (granted >= 0).all()
    dq8.cache_append(dq8.DYNAMIC_TREE, keys[prompt], keys[prompt].flip(2).contiguous(), slots, codes, scales, positions=positions, rotation=rotation)

    kept = [t.clone() for t in state]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(*[t.clone() for t in state])
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        granted, out, accepted, starts = step(*state)
    assert all(torch.equal(a, b) for a, b in zip(state, kept))
    refused, ended = np.zeros(batch, int), 0
    for turn in range(60):
        fed = [[s[-1], (7 * s[-1] + turn) % vocab, (3 * s[-1] + 1) % vocab] for s in so_far]
        ids.copy_(torch.tensor(sum(fed, [])))
        uniform.copy_(torch.from_numpy(gen.random(batch * most).astype(np.float32) ** 3))
        sample.copy_(torch.from_numpy(gen.random(batch).astype(np.float32)))
        noise.copy_(torch.from_numpy(gen.random((batch * most, vocab)).astype(np.float32)))
        before, owed = lens.tolist(), drop.tolist()
        graph.replay()
        torch.cuda.synchronize()
        for b in range(batch):
            rows = out[most * b : most * b + most].tolist()
            if int(granted[b]) < 0:
                refused[b] += 1
                assert rows == [-1] * most and int(accepted[b]) == -1 and int(drop[b]) == owed[b] and int(lens[b]) == before[b]
            else:
                so_far[b] += rows[: int(accepted[b]) + 1]
            assert int(lens[b]) - int(drop[b]) == len(so_far[b]) - 1
        # the longest ends where somebody was refused: its places go back with the next plan, and it begins anew with one token
        if (granted < 0).any():
            b = max(range(batch), key=lambda b: len(so_far[b]))
            so_far[b], drop[b] = [int(gen.integers(0, vocab))], 10 ** 9
            dq8.cache_plan(lens, torch.zeros_like(new), pages, free, n_free, page, 0, drop=torch.where(torch.arange(batch, device="cuda") == b, drop, 0), lens_out=lens,
                           n_free_out=n_free)
            drop[b] = 0
            ended += 1
    assert refused.sum() > 2 and ended > 2  # that this happened at all
    # the same tokens at once into another cache
    codes2, scales2 = dq8.cache_buffers(batch * wide, kv, page, dim)
    for b in range(batch):
        n = len(so_far[b]) - 1
        if n == 0:
            continue
        tokens = torch.tensor(so_far[b][:-1], device="cuda")
        dq8.cache_append(dq8.DYNAMIC_TREE, keys[tokens], keys[tokens].flip(2).contiguous(), torch.arange(n, device="cuda"), codes2, scales2,
                         positions=torch.arange(n, device="cuda"), rotation=rotation)
        for j in range(n):
            p = int(pages[b, j // page])
            assert torch.equal(codes[:, p, :, j % page], codes2[:, j // page, :, j % page]) and torch.equal(scales[:, p, :, j % page], scales2[:, j // page, :, j % page])
    used = [p for b in range(batch) for p in pages[b, : -(-int(lens[b]) // page)].tolist()]
    assert sorted(used + free[: int(n_free)].tolist()) == list(range(n_pages))
