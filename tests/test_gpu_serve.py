"""Plans of decoding steps and verification of drafted tokens against plain implementations, and a run of both with the cache between them."""
import numpy as np
import pytest
import torch

from paper_1511_04561_amd import dq8

from . import serve_reference as ref

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64


def dev(a, dtype=None):
    return torch.as_tensor(a, dtype=dtype).cuda()


# ---------------------------------------------------------------- plan


class State:
    """Requests in a random state: pages of the sequences and free ones are all different."""

    def __init__(self, batch, wide, page, seed, spare=5, longest=None):
        rng = np.random.default_rng(seed)
        self.page = page
        longest = wide * page if longest is None else longest
        self.lens = rng.integers(0, longest + 1, batch).astype(np.int32)
        had = -(-self.lens // page)
        order = rng.permutation(int(had.sum()) + spare).astype(np.int32)
        self.pages = np.full((batch, wide), -7, np.int32)
        at = 0
        for b, n in enumerate(had):
            self.pages[b, :n] = order[at : at + n]
            at += n
        self.free = np.full(len(order) + 3, -9, np.int32)
        self.free[:spare] = order[at:]
        self.n_free = np.array([spare], np.int32)
        self.rng = rng

    def both(self, new, drop, tokens, inplace=False):
        """The call and the reference on copies of the state; what differs fails."""
        pages, free = self.pages.copy(), self.free.copy()
        want = ref.plan(self.lens, new, pages, free, self.n_free[0], self.page, tokens, drop)
        t = {k: dev(v) for k, v in (("lens", self.lens), ("pages", self.pages), ("free", self.free), ("n_free", self.n_free))}
        more = {"lens_out": t["lens"], "n_free_out": t["n_free"]} if inplace else {}
        got = dq8.cache_plan(t["lens"], dev(np.asarray(new, np.int32)), t["pages"], t["free"], t["n_free"], self.page, tokens,
                             drop=None if drop is None else dev(np.asarray(drop, np.int32)), **more)
        for name, a, b in zip(("slots", "positions", "starts", "lens", "granted", "n_free"), got, want):
            assert np.array_equal(a.cpu().numpy(), b if name != "n_free" else [b]), name
        assert np.array_equal(t["pages"].cpu().numpy(), pages)
        # entries of the stack behind its end hold what was there or was given back for a moment
        assert np.array_equal(t["free"].cpu().numpy()[: want[5]], free[: want[5]])
        if inplace:
            assert got[3] is t["lens"] and got[5] is t["n_free"]
        self.lens, self.pages, self.n_free = want[3], pages, np.array([want[5]], np.int32)
        self.free = t["free"].cpu().numpy()
        return got, want


@pytest.mark.parametrize("page", [16, 64, 1024])
@pytest.mark.parametrize("batch", [1, 2, 7, 64, 65, 256, 1000, 1025, 2500, 4096])
def test_plans(batch, page):
    s = State(batch, 6, page, batch + page, spare=batch // 2 + 3)
    rng = s.rng
    for step in range(4):
        new = rng.integers(0, 2 * page if step == 1 else 6, batch)
        drop = None if step == 0 else np.where(rng.random(batch) < 0.1, 10 ** 6, rng.integers(-2, 8, batch))
        total = int(new.sum())
        got, want = s.both(new, drop, total + (0, 5, -min(total, 9), 1)[step], inplace=step % 2 == 1)


def test_plans_of_prompts_that_take_a_second_launch():
    s = State(9, 300, 16, 5, spare=2000, longest=50)
    new = [4097, 0, 1, 17, 3000, 2, 900, 33, 1234]
    got, want = s.both(new, None, sum(new) + 77)
    assert (want[4] >= 0).all()
    s.both([1] * 9, [5000, 0, 0, 17, 10 ** 9, 0, -3, 1, 1235], 9)
    s.both([4700, 4700, 9, 0, 9, 0, 0, 0, 0], None, 4700)  # the second ends behind the tokens, the first fits


def test_plans_without_room():
    s = State(5, 4, 16, 1, spare=2, longest=16)
    s.lens[:] = [16, 0, 10, 64, 3]
    s.pages[:] = np.arange(20).reshape(5, 4)
    got, want = s.both([17, 17, 6, 1, 14], None, 55)
    # two pages for the first, none left for the second, the third needs none, the fourth is full, the last finds none
    assert want[4].tolist() == [17, -1, 6, -1, -1] and want[5] == 0
    # pages given back in the same step are there
    s.both([0, 5, 0, 0, 14], [33, 0, 16, 1, 0], 19)
    # an empty stack, a stack whose count is out of range
    s.n_free[:] = 0
    s.both([40, 40, 40, 40, 40], None, 200)
    s.n_free[:] = -5
    s.both([1] * 5, [1] * 5, 5)
    s.n_free[:] = 1000
    s.both([1] * 5, None, 5)


def test_plans_of_lengths_out_of_range():
    s = State(6, 3, 16, 2, spare=9)
    s.lens[:] = [-5, 1000, 48, 2 ** 31 - 1, 0, 5]
    s.pages[:] = np.arange(18).reshape(6, 3)
    s.both([3, 1, 0, 0, -4, 2 ** 31 - 1], [0, 1, 2 ** 31 - 1, -(2 ** 31), 3, 0], 5)
    s.both([2 ** 31 - 1] * 6, None, 100)
    s.both([1] * 6, [2 ** 31 - 1] * 6, 0)


def test_a_stack_without_room_loses_pages():
    s = State(3, 4, 16, 3, spare=1)
    s.lens[:] = [64, 64, 64]
    s.pages[:] = np.arange(12).reshape(3, 4)
    s.free = np.array([99, -1, -1], np.int32)
    got, want = s.both([0, 0, 20], [64, 30, 64], 20)
    assert want[5] == 3


def test_plan_leaves_guards_and_keeps_what_it_does_not_need():
    lens, new = dev([20, 5], I32), dev([4, 0], I32)
    big = torch.full((4, 5), -3, dtype=I32, device="cuda")
    pages = big[1:3]
    pages.copy_(dev([[3, 4, 7, 8, 9], [5, 6, 6, 6, 6]], I32))
    band = {n: torch.full((k + 4,), -77, dtype=d, device="cuda") for n, k, d in
            (("slots", 6, I64), ("positions", 6, I64), ("starts", 3, I32), ("lens_out", 2, I32), ("granted", 2, I32), ("n_free_out", 1, I32))}
    free = dev([-1, -1, 30, 31, -1, -1], I32)
    dq8.cache_plan(lens, new, pages, free[2:4], dev([2], I32), 16, 6, **{n: v[2:-2] for n, v in band.items()})
    assert all((v[:2] == -77).all() and (v[-2:] == -77).all() for v in band.values())
    assert big[0].eq(-3).all() and big[3].eq(-3).all() and pages.tolist() == [[3, 4, 7, 8, 9], [5, 6, 6, 6, 6]]
    assert free.tolist() == [-1, -1, 30, 31, -1, -1]
    assert band["slots"][2:-2].tolist() == [68, 69, 70, 71, -1, -1] and band["starts"][2:-2].tolist() == [0, 4, 4]


# ---------------------------------------------------------------- verification


def drafts(rows, vocab, seed, dtype, sure=False, flat=1.0):
    rng = np.random.default_rng(seed)
    logits = 3 * flat * rng.standard_normal((rows, vocab))
    p = np.exp(logits - logits.max(1, keepdims=True))
    q = np.exp(0.8 * logits + 0.5 * rng.standard_normal((rows, vocab)))
    p, q = torch.from_numpy(p / p.sum(1, keepdims=True)).to(dtype), torch.from_numpy(q / q.sum(1, keepdims=True)).to(dtype)
    ids = np.array([0] + [int(q[i].float().argmax()) if sure else int(rng.choice(vocab, p=q[i].double().numpy() / q[i].double().sum().item())) for i in range(rows - 1)])
    return p, None if sure else q, ids, rng.random(rows).astype(np.float32), rng


def both(p, q, ids, uniform, sample, starts, **more):
    out = np.full(len(ids), -55, np.int64)
    uniform, sample = np.asarray(uniform, np.float32), np.asarray(sample, np.float32)
    want = ref.verify(p.double().numpy(), ids, uniform, sample, starts, None if q is None else q.double().numpy(), out)
    args = [p.cuda(), dev(ids, I64), dev(uniform), dev(sample)]
    for space in (True, False):
        given = {"draft": None if q is None else q.cuda(), "starts": dev(np.asarray(starts, np.int32)), "out": dev(out), **more}
        if not space:
            given["workspace"] = torch.empty(0, dtype=torch.uint8, device="cuda")
        got = dq8.draft_verify(*args, **given)
        for a, b in zip(got, want):
            assert np.array_equal(a.cpu().numpy(), b)
    return want


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16, torch.float16])
@pytest.mark.parametrize("vocab", [1, 2, 63, 1000, 1024, 1025, 5003, 20000])
@pytest.mark.parametrize("sure", [False, True])
def test_verifications(dtype, vocab, sure):
    rows = [1, 6, 2, 0, 9, 1, 3]
    p, q, ids, uniform, rng = drafts(sum(rows), vocab, vocab, dtype, sure)
    starts = np.concatenate([[0], np.cumsum(rows)])
    for _ in range(3):
        want = both(p, q, ids, uniform * 0.8 ** rng.integers(0, 4), rng.random(len(rows)), starts)
        assert want[1][3] == -1 and want[2][3] == 0


def test_verification_of_many_sequences_and_long_drafts():
    rng = np.random.default_rng(3)
    rows = np.concatenate([rng.integers(1, 5, 300), [200, 65, 66, 129]])
    p, q, ids, uniform, _ = drafts(int(rows.sum()), 50, 4, torch.float32)
    starts = np.concatenate([[0], np.cumsum(rows)])
    both(p, q, ids, uniform, rng.random(len(rows)), starts)
    want = both(p, q, ids, uniform * 0.0, rng.random(len(rows)), starts)  # all drafts stay
    assert (want[2] == 0).all()
    uniform = uniform * 0
    uniform[starts[-2] + 100] = np.nan  # ... but for one in the middle of a long one
    assert both(p, q, ids, uniform, rng.random(len(rows)), starts)[1][-1] == 100


@pytest.mark.parametrize("dtype,vocab", [(torch.float32, 300001), (torch.bfloat16, 131072), (torch.float16, 2500000)])
def test_large_vocabularies(dtype, vocab):
    g = torch.Generator().manual_seed(vocab)
    p, q = (torch.rand(5, vocab, generator=g).div_(vocab).mul_(3000 if dtype == torch.float16 else 1).to(dtype) for _ in range(2))
    ids = torch.randint(0, vocab, (5,), generator=g).numpy()
    for u in (0.0, 0.9):
        for draft in (q, None):
            both(p, draft, ids, np.full(5, u, np.float32), [0.0, 0.37, 0.9999999], [0, 2, 4, 5])
            both(p, draft, ids, np.full(5, u, np.float32), [1.0, 0.5, 0.25, float("nan"), 0.75], [0, 1, 2, 3, 4, 5])


def test_large_vocabularies_with_few_weights():
    """Whole chunks without a weight, before, between and behind those that have some."""
    vocab = 200000
    for some in ([199999], [0], [1024, 1023], [5000, 150000, 150001], [2047, 2048, 199998], []):
        p, q = torch.zeros(3, vocab), torch.zeros(3, vocab)
        p[:, some] = 0.25
        q[:, :70000] = 1e-6
        q[1, some] = 0.25
        for ids in ([0, 7, 100], [0, (some or [3])[0], 5]):
            for r in (0.0, 0.3, 0.5, 0.99999994, 1.0):
                both(p, q, np.array(ids), np.full(3, 0.5, np.float32), [r], [0, 3])
                both(p, None, np.array(ids), np.full(3, 0.1, np.float32), [r, r], [0, 2, 3])


def test_random_numbers_at_their_ends():
    p = torch.tensor([[0.0, 0.5, 0.0, 0.5, 0.0]] * 2)
    for r, token in ((0.0, 1), (0.25, 1), (0.49999997, 1), (0.5, 3), (0.99999994, 3), (1.0, 3), (7.0, 3), (float("inf"), 3), (float("nan"), 1), (-1.0, 1)):
        assert both(p[:1], None, np.array([0]), np.zeros(1, np.float32), [r], [0, 1])[0].tolist() == [token]
    # u q < p: equality refuses
    q = torch.tensor([[0.0, 1.0, 0.0, 0.0, 0.0]] * 2)
    for u, accepted in ((0.5, 0), (0.49999997, 1), (float("nan"), 0), (-1.0, 1), (1.0, 0)):
        assert both(p, q, np.array([0, 1]), np.array([u, 0], np.float32), [0.1], [0, 2])[1].tolist() == [accepted]


def test_weights_that_are_no_probabilities():
    inf, nan = float("inf"), float("nan")
    p = torch.tensor([[nan, -1.0, inf, 0.25, 0.0], [0.0, 0.0, 0.0, 0.0, 0.0], [0.1, 0.2, 0.3, 0.2, 0.2], [nan, nan, nan, -inf, 0.0]])
    q = torch.tensor([[0.0, nan, 1.0, -5.0, inf], [0.2] * 5, [0.1, 0.2, 0.3, 0.2, 0.2], [0.2] * 5])
    for ids in ([0, 3, 1, 2], [0, 2, 4, 4], [0, -1, 5, 2 ** 40], [0, 1, -(2 ** 62), 3]):
        for u in (0.0, 0.5, 0.999):
            both(p, q, np.array(ids), np.full(4, u, np.float32), [0.6], [0, 4])
            both(p, None, np.array(ids), np.full(4, u, np.float32), [0.6], [0, 4])
            for row in range(4):
                both(p[row : row + 1], None, np.array(ids[:1]), np.zeros(1, np.float32), [0.6], [0, 1])
    # nothing is left of the difference: the target's own probabilities; a row of none: no token
    assert both(p[2:], q[2:], np.array([0, 9]), np.zeros(2, np.float32), [0.5], [0, 2])[0].tolist() == [2, -1]
    assert both(p[1:2], None, np.array([0]), np.zeros(1, np.float32), [0.5], [0, 1])[0].tolist() == [-1]


def test_starts_out_of_range_and_rows_behind_the_last_sequence():
    p, q, ids, uniform, rng = drafts(12, 77, 1, torch.float32)
    for starts in ([0, 3, 3, 7], [-5, 4, 9, 100], [2, 5, 8, 10], [0, 12, 12, 12], [12, 12, 12, 12], [5, 3, 3, 8], [-9, -3, 0, 2 ** 31 - 1]):
        want = both(p, q, ids, uniform, rng.random(3), starts)
        covered = np.zeros(12, bool)
        for a, b in zip(starts, starts[1:]):
            covered[max(a, 0) : max(min(b, 12), 0)] = True
        assert (want[0][~covered] == -55).all()


def test_verification_with_strides_and_even_rows():
    p, q, ids, uniform, rng = drafts(12, 501, 9, torch.bfloat16)
    big = torch.full((13, 1100), float("nan"), dtype=torch.bfloat16, device="cuda")
    big[1:, 3:504], big[1:, 601:1102] = p.cuda(), 0
    other = torch.full((24, 507), float("nan"), dtype=torch.bfloat16, device="cuda")
    other[::2, 5:506] = q.cuda()
    sample = rng.random(4).astype(np.float32)
    want = ref.verify(p.double().numpy(), ids, uniform, sample, [0, 3, 6, 9, 12], q.double().numpy())
    got = dq8.draft_verify(big[1:, 3:504], dev(ids, I64), dev(uniform), dev(sample), draft=other[::2, 5:506])
    assert all(np.array_equal(a.cpu().numpy(), b) for a, b in zip(got, want))


def test_verification_workspaces_and_graphs():
    p, q, ids, uniform, rng = drafts(20, 50000, 2, torch.float32)
    args = [p.cuda(), dev(ids, I64), dev(uniform), dev(rng.random(5).astype(np.float32))]
    starts, draft = dev([0, 4, 8, 12, 16, 20], I32), q.cuda()
    n = dq8.draft_verify_workspace(*args, starts=starts, draft=draft)
    assert n == 5 * (24 + 49 * 8)
    want = dq8.draft_verify(*args, starts=starts, draft=draft)
    for bytes_ in (n, n - 1, n + 100):
        space = torch.full((n + 160,), 0xA5, dtype=torch.uint8, device="cuda")
        got = dq8.draft_verify(*args, starts=starts, draft=draft, workspace=space[16 : 16 + bytes_])
        assert all(torch.equal(a, b) for a, b in zip(got, want))
        assert (space[:16] == 0xA5).all() and (space[16 + n :] == 0xA5).all()
    # two graphs of the same inputs, each with its own workspace, replayed in turn with changing inputs, one without any
    graphs, spaces = [], [torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda"), None]
    for workspace in spaces:
        outs = [torch.zeros_like(w) for w in want]
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dq8.draft_verify(*args, starts=starts, draft=draft, out=outs[0], accepted=outs[1], rejected=outs[2], workspace=workspace)
        graphs.append((graph, outs))
    for seed in range(4):
        g = torch.Generator().manual_seed(seed)
        args[2].copy_(torch.rand(20, generator=g))
        args[3].copy_(torch.rand(5, generator=g))
        want = dq8.draft_verify(*args, starts=starts, draft=draft)
        for graph, outs in graphs:
            graph.replay()
        torch.cuda.synchronize()
        for _, outs in graphs:
            assert all(torch.equal(a, b) for a, b in zip(outs, want))


def test_the_python_path_gives_the_same(monkeypatch):
    p, q, ids, uniform, rng = drafts(8, 3000, 5, torch.float16)
    args = [p.cuda(), dev(ids, I64), dev(uniform), dev(rng.random(2).astype(np.float32))]
    lens, new, pages, free, n_free = dev([20, 5], I32), dev([4, 40], I32), dev([[3, 4, 0, 0], [5, 0, 0, 0]], I32), dev([8, 9, 2, 0], I32), dev([3], I32)

    def calls():
        f, t = free.clone(), pages.clone()
        return (*dq8.draft_verify(*args, draft=q.cuda()), *dq8.cache_plan(lens, new, t, f, n_free, 16, 50, drop=new), f, t)

    want = calls()
    monkeypatch.setattr(dq8, "_native", dq8._Unbound())
    assert all(torch.equal(a, b) for a, b in zip(calls(), want))
    # without sequences' rows
    out, accepted, rejected = dq8.draft_verify(args[0][:0], args[1][:0], args[2][:0], args[3])
    assert out.numel() == 0 and accepted.tolist() == [-1, -1] and rejected.tolist() == [0, 0]
    got = dq8.cache_plan(lens, new * 0, pages, free, n_free, 16, 0)
    assert got[0].numel() == 0 and got[3].tolist() == [20, 5]


def test_refusals():
    lens, pages, free, n_free = dev([20, 5], I32), torch.zeros(2, 4, dtype=I32, device="cuda"), torch.zeros(3, dtype=I32, device="cuda"), dev([3], I32)
    p, ids, u, r = torch.rand(6, 50, device="cuda"), torch.zeros(6, dtype=I64, device="cuda"), torch.rand(6, device="cuda"), torch.rand(2, device="cuda")
    bad = [
        (ValueError, lambda: dq8.cache_plan(lens[:1], lens, pages, free, n_free, 16, 4)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages, free, lens, 16, 4)),
        (TypeError, lambda: dq8.cache_plan(lens.long(), lens, pages, free, n_free, 16, 4)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages[0], free, n_free, 16, 4)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages.T, free, n_free, 16, 4)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 16, -1)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 16, 2 ** 31)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 2 ** 32 + 16, 4)),
        (dq8.Dq8Error, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 17, 4)),
        (dq8.Dq8Error, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 16, 4, granted=lens)),
        (ValueError, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 16, 4, slots=torch.zeros(5, dtype=I64, device="cuda"))),
        (TypeError, lambda: dq8.cache_plan(lens, lens, pages, free, n_free, 16, 4, drop=[1, 2])),
        (TypeError, lambda: dq8.draft_verify(p.double(), ids, u, r)),
        (TypeError, lambda: dq8.draft_verify(p, ids.int(), u, r)),
        (ValueError, lambda: dq8.draft_verify(p, ids[:5], u, r)),
        (ValueError, lambda: dq8.draft_verify(p, ids, u, r, draft=p[:, :49])),
        (TypeError, lambda: dq8.draft_verify(p, ids, u, r, draft=p.half())),
        (ValueError, lambda: dq8.draft_verify(p, ids, u, r, starts=lens)),
        (dq8.Dq8Error, lambda: dq8.draft_verify(p, ids, u, torch.rand(4, device="cuda"))),
        (dq8.Dq8Error, lambda: dq8.draft_verify(p, ids, u, r, out=ids)),
        (ValueError, lambda: dq8.draft_verify(p.T, ids, u, r)),
        (TypeError, lambda: dq8.draft_verify(p, ids, u, r, workspace=u)),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()


# ---------------------------------------------------------------- all together


def test_steps_of_decoding_with_drafts():
    """Prompts, then steps of three fed rows each (the last accepted token and two drafts): plan, projection, append, attention, logits, verification, whose
    `rejected` is the next plan's `drop`.  What is cached has to be what a run without drafts of the tokens that stayed would have cached, and the
    lengths those of the sequences so far."""
    heads, kv, dim, page, vocab, width, batch, group = 8, 2, 64, 16, 199, 256, 3, 32
    torch.manual_seed(11)
    embed = torch.randn(vocab, width, device="cuda").bfloat16()
    qkv_w, head_w = (dq8.weights_encode(torch.randn(n, m, device="cuda") * m ** -0.5, group) for n, m in (((heads + 2 * kv) * dim, width), (vocab, heads * dim)))
    angle = torch.arange(512, device="cuda")[:, None] * 10000.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))
    rotation = torch.stack([angle.cos(), angle.sin()], 1).contiguous()
    codes, scales = dq8.cache_buffers(40, kv, page, dim)
    free, n_free = dq8.cache_free_list(40)
    pages, lens = torch.zeros((batch, 12), dtype=I32, device="cuda"), torch.zeros(batch, dtype=I32, device="cuda")

    def forward(ids, new, drop, codes, scales, pages, lens, free, n_free, most):
        slots, positions, starts, _, granted, _ = dq8.cache_plan(lens, new, pages, free, n_free, page, len(ids), drop=drop, lens_out=lens, n_free_out=n_free)
        qkv = dq8.weights_product(embed[ids], *qkv_w).view(len(ids), -1, dim)
        q, k, v = qkv.split([heads, kv, kv], 1)
        q = dq8.cache_append(dq8.DYNAMIC_TREE, k, v, slots, codes, scales, positions=positions, rotation=rotation, q=q)
        y = dq8.cache_attention(dq8.DYNAMIC_TREE, q, codes, scales, pages, lens, starts=starts, max_new=most)
        logits = dq8.weights_product(y.view(len(ids), -1), *head_w, rows=vocab, dtype=torch.float32)
        return torch.softmax(logits * 4, 1), starts, granted

    prompts = [[5, 9, 17] * 7, [100] * 16, [33, 2]]
    so_far = [list(p) for p in prompts]
    ids = dev(sum(prompts, []), I64)
    new = dev([len(p) for p in prompts], I32)
    target, starts, granted = forward(ids, new, None, codes, scales, pages, lens, free, n_free, 21)
    assert lens.tolist() == [len(p) for p in prompts] and torch.equal(granted, new)
    out, _, _ = dq8.draft_verify(target[starts[1:].long() - 1], ids[:batch], torch.zeros(batch, device="cuda"), torch.rand(batch, device="cuda"))
    for b in range(batch):
        so_far[b].append(int(out[b]))
    drop = None
    for step in range(8):
        fed = [[s[-1], (7 * s[-1] + step) % vocab, (3 * s[-1] + 1) % vocab] for s in so_far]
        ids = dev(sum(fed, []), I64)
        target, starts, granted = forward(ids, dev([3] * batch, I32), drop, codes, scales, pages, lens, free, n_free, 3)
        assert granted.tolist() == [3] * batch
        draft = torch.full((3 * batch, vocab), 0.2 / vocab, device="cuda")
        draft[torch.arange(3 * batch - 1), ids[1:]] += 0.8
        uniform, sample = torch.rand(3 * batch, device="cuda") ** 3, torch.rand(batch, device="cuda")
        want = ref.verify(target.double().cpu().numpy(), ids.cpu().numpy(), uniform.cpu().numpy(), sample.cpu().numpy(), starts.tolist(), draft.double().cpu().numpy())
        out, accepted, drop = dq8.draft_verify(target, ids, uniform, sample, starts=starts, draft=draft)
        assert all(np.array_equal(a.cpu().numpy(), w) for a, w in zip((out, accepted, drop), want))
        for b in range(batch):
            so_far[b] += out[3 * b : 3 * b + int(accepted[b]) + 1].tolist()
            # cached: all but the token that was drawn last, and the rejected drafts
            assert int(lens[b]) - int(drop[b]) == len(so_far[b]) - 1
    # the same tokens at once into another cache
    codes2, scales2 = dq8.cache_buffers(40, kv, page, dim)
    free2, n_free2 = dq8.cache_free_list(40)
    pages2, lens2 = torch.zeros_like(pages), torch.zeros_like(lens)
    ids = dev(sum((s[:-1] for s in so_far), []), I64)
    forward(ids, dev([len(s) - 1 for s in so_far], I32), None, codes2, scales2, pages2, lens2, free2, n_free2, 60)
    used = []
    for b in range(batch):
        n = len(so_far[b]) - 1
        one, two = ([(int(t[b, j // page]), j % page) for j in range(n)] for t in (pages, pages2))
        for (pa, ia), (pb, ib) in zip(one, two):
            # scales and keys depend on the projection's rounding only: equal calls on other batches may differ in a sum's order
            a, c = (dq8.decode(dq8.DYNAMIC_TREE, x[:, p, :, i].contiguous().view(-1), y[:, p, :, i].contiguous().view(-1), dim) for x, y, p, i in
                    ((codes, scales, pa, ia), (codes2, scales2, pb, ib)))
            assert (a - c).abs().max() <= 0.1 * c.abs().max()
        had = -(-int(lens[b]) // page)
        used += pages[b, :had].tolist()
    # every page is either a sequence's or free, once
    assert sorted(used + free[: int(n_free)].tolist()) == list(range(40))
    # all of them end
    got = dq8.cache_plan(lens, torch.zeros_like(lens), pages, free, n_free, page, 0, drop=lens.clone())
    assert got[3].tolist() == [0] * batch and int(got[5]) == 40 and sorted(free.tolist()) == list(range(40))
