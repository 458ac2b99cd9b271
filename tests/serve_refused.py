"""Verification of the rows of a plan from its definition: what serve_reference has, and for refused sequences nothing but the drop they still owe."""
import numpy as np

from . import serve_reference as ref


def verify_of_plan(target, ids, uniform, sample, starts, draft, granted, drop=None, out=None):
    """granted, drop: the plan's (drop None: it had none).  Returns (out, accepted, rejected)."""
    tokens = len(ids)
    out, accepted, rejected = ref.verify(target, ids, uniform, sample, starts, draft, out)
    for b in range(len(sample)):
        if granted[b] < 0:
            s0, s1 = (min(max(int(s), 0), tokens) for s in (starts[b], starts[b + 1]))
            out[s0:s1] = -1
            accepted[b], rejected[b] = -1, 0 if drop is None else max(int(drop[b]), 0)
    return out, np.asarray(accepted, np.int32), np.asarray(rejected, np.int32)
