"""Steps padded to a fixed number of rows: rows of no sequence hold no token in an `out` that the call makes, and stay as they were in one that it is given."""
import numpy as np
import pytest
import torch

from paper_1511_04561_amd import dq8

from .test_gpu_serve import dev, drafts
from . import serve_reference as ref

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64


# a vocabulary of one launch and one of two
@pytest.mark.parametrize("dtype,vocab", [(torch.bfloat16, 77), (torch.float32, 70001)])
@pytest.mark.parametrize("rows", [12, 300])
def test_rows_of_no_sequence(dtype, vocab, rows, monkeypatch):
    p, q, ids, uniform, rng = drafts(12, vocab, 1, dtype)
    big = torch.zeros(rows, vocab, dtype=dtype)
    big[:12] = p
    ids = np.concatenate([ids, np.zeros(rows - 12, np.int64)])
    uniform = np.concatenate([uniform, np.zeros(rows - 12, np.float32)])
    sample = rng.random(3).astype(np.float32)
    args = [big.cuda(), dev(ids, I64), dev(uniform), dev(sample)]
    native = dq8._native
    for starts in ([0, 3, 3, 7], [2, 5, 8, 10], [4, 4, 4, 4], [0, 0, 0, 0], [rows] * 4, [-5, 4, 9, rows + 7], [1, 1, 6, rows]):
        want = ref.verify(big.double().numpy(), ids, uniform, sample, starts)  # (its own `out` begins as -1)
        for path in (native, dq8._Unbound()):
            monkeypatch.setattr(dq8, "_native", path)
            # what the call takes from the allocator is what was just given back, and not zeros
            for n in (rows * 8, rows * 8 + 32, rows * 8 + 512):
                spoiled = [torch.full((n // 8,), 0x5555555555555555, dtype=I64, device="cuda") for _ in range(8)]
                del spoiled
            for space in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
                got = dq8.draft_verify(*args, starts=dev(starts, I32), workspace=space)
                assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))
                given = torch.full((rows,), -55, dtype=I64, device="cuda")
                assert dq8.draft_verify(*args, starts=dev(starts, I32), out=given, workspace=space)[0] is given
                s0, s1 = (min(max(s, 0), rows) for s in (starts[0], starts[-1]))
                kept = np.full(rows, -55)
                kept[s0:s1] = want[0][s0:s1]
                assert np.array_equal(given.cpu().numpy(), kept)


def test_a_call_without_sequences_or_rows():
    p, ids, u = torch.rand(6, 50, device="cuda"), torch.zeros(6, dtype=I64, device="cuda"), torch.rand(6, device="cuda")
    spoiled = torch.full((6,), 0x5555555555555555, dtype=I64, device="cuda")
    del spoiled
    out, accepted, rejected = dq8.draft_verify(p, ids, u, torch.rand(0, device="cuda"), starts=torch.zeros(1, dtype=I32, device="cuda"))
    assert out.tolist() == [-1] * 6 and accepted.numel() == 0 and rejected.numel() == 0
