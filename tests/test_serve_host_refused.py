"""Verification behind a plan that refused sequences, as far as it needs no device: refusals of the call, and the chain of both in plain Python."""
import ctypes

import numpy as np
import pytest

from . import serve_reference as ref
from .serve_refused import verify_of_plan
from .test_serve_host import L, at, verify  # noqa: F401 (L is a fixture)


@pytest.mark.parametrize("status,change", [
    (3, {"granted": at(9, 2)}), (3, {"drop": at(10, 1)}), (3, {"out": at(9)}), (3, {"accepted": at(9)}), (3, {"rejected": at(9, 4)}), (3, {"out": at(10)}),
    (3, {"accepted": at(10)}), (3, {"drop": at(8, 4)}), (3, {"granted": at(8)}), (3, {"drop": at(7)})])
def test_refused_verifications_of_plans(L, status, change):  # noqa: F811
    v = verify(**{"granted": at(9), "drop": at(10), **change})
    assert L.dq8_draft_verify(ctypes.byref(v), None, 0, None) == status and L.dq8_last_error()


def test_workspaces_over_what_the_plan_wrote_are_refused(L):  # noqa: F811
    v = verify(granted=at(9), drop=at(10))
    for i in (9, 10):
        assert L.dq8_draft_verify(ctypes.byref(v), at(i), 64, None) == 3


@pytest.mark.parametrize("seed", range(20))
def test_a_chain_with_refusals_keeps_every_token_that_stayed(seed):
    """Random steps over too few pages.  What is cached of a sequence, less what the next plan takes back, is always all of its tokens but the last."""
    rng = np.random.default_rng(seed)
    batch, page, vocab, wide = 4, 16, 11, 6
    pages, free, n_free = np.zeros((batch, wide), np.int32), np.arange(9, dtype=np.int32), 9
    lens, drop, refused = np.zeros(batch, np.int32), np.zeros(batch, np.int32), 0
    so_far = [list(rng.integers(0, vocab, rng.integers(1, 30))) for _ in range(batch)]
    fed = [list(s) for s in so_far]  # a prompt is fed as a whole: none of its tokens is a draft
    prompt = [True] * batch
    for _ in range(40):
        ids = np.concatenate(fed)
        slots, positions, starts, lens, granted, n_free = ref.plan(lens, [len(f) for f in fed], pages, free, n_free, page, len(ids), drop)
        target = rng.dirichlet(np.ones(vocab), len(ids)).astype(np.float32).astype(np.float64)
        uniform = rng.random(len(ids)).astype(np.float32)
        for b in range(batch):
            if prompt[b]:
                uniform[starts[b] : starts[b + 1]] = -1.0
        out, accepted, rejected = verify_of_plan(target, ids, uniform, rng.random(batch).astype(np.float32), starts, None, granted, drop)
        refused += int((granted < 0).sum())
        for b in range(batch):
            if granted[b] < 0:
                assert accepted[b] == -1 and rejected[b] == drop[b] and (out[starts[b] : starts[b + 1]] == -1).all()
            else:
                new = out[starts[b] : starts[b] + accepted[b] + 1].tolist()
                so_far[b] += new[-1:] if prompt[b] else new
                prompt[b] = False
            if len(so_far[b]) > 60:  # ends: a new request takes its place, whose prompt waits until everything is given back
                so_far[b], prompt[b] = list(rng.integers(0, vocab, rng.integers(1, 30))), True
                rejected[b] = 10 ** 6
            fed[b] = list(so_far[b]) if prompt[b] else [so_far[b][-1]] + list(rng.integers(0, vocab, rng.integers(0, 4)))
            if not prompt[b]:
                assert lens[b] - rejected[b] == len(so_far[b]) - 1
        drop = rejected
        used = [int(p) for b in range(batch) for p in pages[b, : -(-int(lens[b]) // page)]]
        assert sorted(used + free[:n_free].tolist()) == list(range(9))
    assert refused > 0
