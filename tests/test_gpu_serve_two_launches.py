"""Verification of vocabularies that take two launches: ragged, empty and long sequences, starts out of range, rows that lie apart and start between words."""
import numpy as np
import pytest
import torch

from paper_1511_04561_amd import dq8

from . import serve_reference as ref
from .test_gpu_serve import both, dev, drafts

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64
CASES = [(torch.float32, 70001, False), (torch.bfloat16, 65537, False), (torch.float16, 80002, True)]


def two_launches(p, q, batch):
    rows = p.shape[0]
    return dq8.draft_verify_workspace(p, torch.zeros(rows, dtype=I64, device="cuda"), torch.zeros(rows, device="cuda"), torch.zeros(batch, device="cuda"),
                                      starts=torch.zeros(batch + 1, dtype=I32, device="cuda"), draft=q) > 0


@pytest.mark.parametrize("dtype,vocab,sure", CASES)
def test_ragged_sequences(dtype, vocab, sure):
    rows = [1, 6, 0, 2, 0, 9, 1, 3, 0]
    p, q, ids, uniform, rng = drafts(sum(rows), vocab, vocab, dtype, sure)
    assert two_launches(p.cuda(), None if q is None else q.cuda(), len(rows))
    starts = np.concatenate([[0], np.cumsum(rows)])
    for power in (0, 1, 3):
        want = both(p, q, ids, uniform * 0.5 ** power, rng.random(len(rows)), starts)
        assert (want[1][[2, 4, 8]] == -1).all() and (want[2][[2, 4, 8]] == 0).all()


@pytest.mark.parametrize("dtype,vocab,sure", CASES)
def test_starts_out_of_range_and_rows_of_no_sequence(dtype, vocab, sure):
    p, q, ids, uniform, rng = drafts(12, vocab, 1, dtype, sure)
    for starts in ([0, 3, 3, 7], [-5, 4, 9, 100], [2, 5, 8, 10], [0, 12, 12, 12], [12, 12, 12, 12], [5, 3, 3, 8], [-9, -3, 0, 2 ** 31 - 1]):
        want = both(p, q, ids, uniform, rng.random(3), starts)
        covered = np.zeros(12, bool)
        for a, b in zip(starts, starts[1:]):
            covered[max(a, 0) : max(min(b, 12), 0)] = True
        assert (want[0][~covered] == -55).all()


@pytest.mark.parametrize("dtype,vocab,sure", CASES)
def test_long_drafts(dtype, vocab, sure):
    """More rows than a wavefront has lanes; the row that refuses in the first and in the second of its turns, and behind all."""
    p, q, ids, uniform, rng = drafts(70, vocab, 2, dtype, sure)
    for refuse in (0, 63, 64, 67, None):
        u = np.zeros(70, np.float32)
        if refuse is not None:
            u[refuse] = np.nan
        want = both(p, q, ids, u, [0.7], [0, 70])
        if sure:  # (the likeliest token always has a probability; a drawn one may have rounded to none)
            assert want[1][0] == (69 if refuse is None else refuse)


@pytest.mark.parametrize("dtype,vocab,sure", CASES)
def test_rows_that_lie_apart(dtype, vocab, sure):
    p, q, ids, uniform, rng = drafts(12, vocab, 9, dtype, sure)
    sample = rng.random(4).astype(np.float32)
    big = torch.full((13, vocab + 9), float("nan"), dtype=dtype, device="cuda")
    big[1:, 3 : vocab + 3] = p.cuda()
    other = torch.full((24, vocab + 6), float("nan"), dtype=dtype, device="cuda")
    if q is not None:
        other[::2, 5 : vocab + 5] = q.cuda()
    args = [big[1:, 3 : vocab + 3], dev(ids, I64), dev(uniform), dev(sample)]
    draft = None if q is None else other[::2, 5 : vocab + 5]
    assert two_launches(args[0], draft, 4)
    want = ref.verify(p.double().numpy(), ids, uniform, sample, [0, 3, 6, 9, 12], None if q is None else q.double().numpy())
    got = dq8.draft_verify(*args, draft=draft)
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
    # one row for all
    same = p[:1].expand(12, vocab)
    want = ref.verify(same.double().numpy(), ids, uniform, sample, [0, 3, 6, 9, 12])
    got = dq8.draft_verify(p[:1].cuda().expand(12, vocab), *args[1:])
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
