"""GPU: the paged cache of 8-bit keys and values against its definition in 64 bits (tests/cache_reference.py).

Codes and scales are compared bit for bit: the rows that are compressed are binary32 roundings of binary64 results.  Queries and
outputs of attention have the tolerances derived in the reference, plus half a step of their own type."""
import numpy as np
import pytest

import oracle
from tests import cache_reference as ref

torch = pytest.importorskip("torch")
pytestmark = pytest.mark.gpu

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}


@pytest.fixture(scope="module")
def dq8():
    if not torch.cuda.is_available():
        pytest.fail("these tests need a GPU (select them with -m gpu on a GPU box)")
    from paper_1511_04561_amd import dq8 as mod
    mod.lib()  # a missing library is an error, not a skip
    mod.init()
    return mod


def half_step(t):
    return torch.finfo(t).eps / 2


def host(t):
    return t.float().cpu().numpy()


def new_cache(kind, rng, pages, kv_heads, page, dim, spread=0.3):
    """A cache of random rows (numpy): any code, scales of some sizes."""
    codes = rng.integers(0, 256, (2, pages, kv_heads, page, dim), dtype=np.uint8)
    scales = np.exp(rng.normal(0, spread, codes.shape[:-1])).astype(np.float32)
    return codes, scales


def to_gpu(cache):
    return tuple(torch.from_numpy(a).cuda() for a in cache)


def angle_table(rng, n, half):
    a = rng.uniform(0, 6.3, (n, half))
    return np.stack([np.cos(a), np.sin(a)], 1).astype(np.float32)


# ---------------------------------------------------------------- append

APPENDS = [
    # kind, type, tokens, heads, kv_heads, dim, page, half, interleaved, norm
    (0, "bf16", 1, 8, 2, 128, 16, 64, False, True),
    (1, "f16", 5, 4, 4, 64, 32, 16, True, False),
    (2, "f32", 37, 0, 3, 80, 16, 40, False, False),
    (3, "bf16", 64, 6, 2, 16, 16, 8, False, True),
    (0, "f32", 33, 3, 1, 96, 64, 20, False, True),    # partners that are no whole eight away
    (0, "f16", 9, 2, 2, 48, 16, 11, True, True),      # pairs that end inside a lane's eight
    (2, "bf16", 19, 5, 5, 256, 128, 128, False, True),
    (3, "f32", 21, 2, 1, 144, 16, 0, False, True),
    (0, "f16", 130, 1, 3, 112, 1024, 1, False, False),
    (1, "bf16", 1000, 16, 8, 128, 16, 64, False, True),
]


@pytest.mark.parametrize("kind,type_,tokens,heads,kv_heads,dim,page,half,interleaved,norm", APPENDS)
def test_append(dq8, kind, type_, tokens, heads, kv_heads, dim, page, half, interleaved, norm):
    rng = np.random.default_rng(1000 * tokens + dim)
    t = TYPES[type_]
    pages = -(-tokens // page) + 2
    cache = new_cache(kind, rng, pages, kv_heads, page, dim)
    gpu = to_gpu(cache)
    both = torch.from_numpy((rng.normal(size=(tokens, heads + 2 * kv_heads, dim)) * np.exp(rng.normal(size=(tokens, 1, 1)))).astype(np.float32)).to(t).cuda()
    both[0, heads] = 0.0  # a row of zeros
    both[-1, -1, :] = -0.0
    q, k, v = both.split([heads, kv_heads, kv_heads], 1)
    slots = rng.permutation(pages * page)[:tokens].astype(np.int64)
    table = angle_table(rng, 50, half) if half else None
    positions = rng.integers(0, 50, tokens) if half else None
    if tokens > 4:
        slots[1], slots[3] = -1, pages * page  # padding
        if half:
            positions[2], positions[4] = 50, -1  # no angles
    qw, kw = ((rng.uniform(0.5, 1.5, dim)).astype(np.float32) for _ in range(2)) if norm else (None, None)
    cuda = lambda a: None if a is None else torch.from_numpy(a).cuda()
    got = dq8.cache_append(kind, k, v, cuda(slots), *gpu, positions=cuda(positions), rotation=cuda(table), interleaved=interleaved,
                           q=q if heads else None, q_weight=cuda(qw) if heads else None, k_weight=cuda(kw))
    want_q = ref.append(kind, cache, host(k), host(v), slots, host(q) if heads else None, qw, kw, 1e-6, table, positions, interleaved)
    finite = np.isfinite(cache[1])
    assert np.array_equal(gpu[1].cpu().numpy()[finite], cache[1][finite]) and np.array_equal(np.isfinite(gpu[1].cpu().numpy()), finite)
    assert np.array_equal(gpu[0].cpu().numpy()[finite], cache[0][finite])
    if not heads:
        assert got is None
        return
    assert got.dtype == t and got.shape == q.shape
    # binary32 inside: the row's sum (dim + 2 roundings, halved by the root), the quotient, two products, two more and a sum
    # around a pair, relative to the pair's larger products; then one rounding to the type
    pair = np.abs(host(q).astype(np.float64))
    if qw is not None:
        x = host(q).astype(np.float64)
        pair = np.abs(x / np.sqrt((x * x).mean(-1, keepdims=True) + 1e-6) * qw)
    size = pair.copy()
    if half:
        ia, ib = (np.arange(0, 2 * half, 2), np.arange(1, 2 * half, 2)) if interleaved else (np.arange(half), np.arange(half, 2 * half))
        size[..., ia] = size[..., ib] = pair[..., ia] + pair[..., ib]
    tiny = torch.finfo(t).tiny * half_step(t)
    tol = half_step(t) * np.abs(want_q) * (1 + 2.0 ** -10) + ((dim + 2) / 2 + 8) * 2.0 ** -24 * size + tiny
    nan = np.isnan(want_q)
    assert np.array_equal(np.isnan(host(got)), nan)
    assert (np.abs(host(got) - want_q)[~nan] <= tol[~nan]).all()


def test_append_rows_that_are_not_finite_and_in_place(dq8):
    rng = np.random.default_rng(7)
    kind, tokens, heads, kv, dim, page = 0, 6, 3, 2, 64, 16
    cache = new_cache(kind, rng, 2, kv, page, dim)
    gpu = to_gpu(cache)
    both = torch.from_numpy(rng.normal(size=(tokens, heads + 2 * kv, dim)).astype(np.float32)).cuda()
    q, k, v = both.split([heads, kv, kv], 1)
    k[1, 0, 5], k[2, 1, 63], v[3, 0, 0] = float("nan"), float("inf"), float("-inf")
    slots = np.arange(tokens, dtype=np.int64) * 3
    table, positions = angle_table(rng, tokens, dim // 2), np.arange(tokens)
    want = ref.append(kind, cache, host(k), host(v), slots, host(q), None, None, 1e-6, table, positions)
    kept = host(both[:, heads:])
    apart = dq8.cache_append(kind, k, v, torch.from_numpy(slots).cuda(), *gpu, positions=torch.from_numpy(positions).cuda(),
                             rotation=torch.from_numpy(table).cuda(), q=q)
    again = dq8.cache_append(kind, k, v, torch.from_numpy(slots).cuda(), *gpu, positions=torch.from_numpy(positions).cuda(),
                             rotation=torch.from_numpy(table).cuda(), q=q, q_out=q)
    assert again is q and torch.equal(apart, q)  # in place, inside the projection's output, whose other parts stay
    assert np.array_equal(host(both[:, heads:]), kept, equal_nan=True)
    assert np.abs(host(q) - want).max() < 1e-5
    assert np.isnan(cache[1]).sum() == 3
    assert np.array_equal(np.isnan(gpu[1].cpu().numpy()), np.isnan(cache[1]))
    good = np.isfinite(cache[1])
    assert np.array_equal(gpu[0].cpu().numpy()[good], cache[0][good]) and np.array_equal(gpu[1].cpu().numpy()[good], cache[1][good])
    values = dq8.decode(kind, *gpu, dim).view(gpu[0].shape)
    assert np.array_equal(torch.isnan(values).all(-1).cpu().numpy(), ~good) and np.array_equal(torch.isnan(values).any(-1).cpu().numpy(), ~good)


def test_append_equals_the_codec_on_rows(dq8):
    """Without norm and rotation a cache row is dq8_encode of that row, whatever its size."""
    rng = np.random.default_rng(11)
    for kind in range(4):
        x = torch.from_numpy((rng.normal(size=(200, 4, 128)) * 10.0 ** rng.uniform(-40, 36, (200, 4, 1))).astype(np.float32)).cuda()
        codes, scales = dq8.cache_buffers(13, 4, 16, 128)
        slots = torch.randperm(13 * 16)[:200].cuda()
        assert dq8.cache_append(kind, x, x.flip(0).contiguous(), slots, codes, scales) is None
        c, s = dq8.encode(kind, x.reshape(-1), 128)
        c, s = c.view(200, 4, 128), s.view(200, 4)
        for part, order in ((0, slice(None)), (1, torch.arange(199, -1, -1))):
            assert torch.equal(codes[part][slots // 16, :, slots % 16], c[order]) and torch.equal(scales[part][slots // 16, :, slots % 16], s[order])
        rest = torch.ones(13 * 16, dtype=torch.bool)
        rest[slots.cpu()] = False
        rest = rest.nonzero().squeeze(1).cuda()
        assert not codes[:, rest // 16, :, rest % 16].any() and not scales[:, rest // 16, :, rest % 16].any()


# ---------------------------------------------------------------- attention

# kind, type, heads, kv_heads, dim, page, [(new tokens, cached tokens)], window
ATTENTIONS = [
    (0, "bf16", 4, 1, 128, 16, [(1, 1)], 0),
    (0, "bf16", 8, 2, 128, 16, [(1, 37), (1, 0), (1, 16), (1, 257), (1, 1000)], 0),
    (1, "f16", 3, 3, 64, 32, [(1, 31), (1, 32), (1, 33), (1, 500)], 0),
    (2, "bf16", 10, 2, 80, 16, [(3, 3), (0, 70), (5, 100), (2, 1), (4, 0)], 0),      # queries that see nothing
    (3, "f16", 40, 1, 96, 64, [(1, 129), (1, 700)], 0),                                # more than 32 rows of one token
    (0, "f16", 4, 4, 256, 16, [(1, 300), (7, 40), (20, 21)], 0),
    (2, "bf16", 6, 2, 16, 16, [(9, 50), (1, 5)], 0),
    (0, "bf16", 2, 1, 144, 128, [(33, 200), (1, 129)], 0),
    (0, "f16", 4, 2, 48, 16, [(70, 70), (3, 500)], 0),
    (0, "bf16", 8, 2, 128, 32, [(1, 600), (1, 30), (4, 300), (90, 250)], 64),
    (3, "bf16", 2, 2, 64, 16, [(100, 130)], 1),                                        # every query sees itself
    (1, "bf16", 8, 1, 112, 16, [(65, 400)], 33),
    (0, "f16", 12, 4, 128, 16, [(130, 513)], 0),
    (0, "bf16", 1, 1, 128, 1024, [(1, 3000)], 0),
    # the kernel for many query rows: every head length it is compiled for, rows that end inside a wavefront, sequences without rows,
    # queries that see nothing, windows that begin and end inside a tile
    (0, "bf16", 8, 2, 256, 16, [(70, 300), (1, 20), (0, 5), (40, 33)], 0),
    (2, "f16", 3, 3, 240, 32, [(300, 300)], 100),
    (1, "bf16", 4, 1, 64, 16, [(65, 600), (17, 17), (200, 250)], 0),
    (3, "f16", 4, 4, 32, 64, [(257, 400), (100, 64)], 70),
    (0, "bf16", 5, 1, 128, 16, [(64, 1000), (0, 0), (90, 60), (1, 1)], 0),
    (0, "f16", 16, 2, 96, 16, [(33, 63), (40, 64), (41, 65), (9, 0)], 31),
    # some rows of a few sequences that are not short: the same kernel, jobs cut into parts, of which some lie behind a window
    (0, "bf16", 4, 1, 128, 64, [(5, 1500)], 0),
    (1, "f16", 6, 2, 64, 32, [(9, 1100), (11, 1030), (0, 700), (7, 3)], 200),
    (2, "bf16", 8, 2, 112, 128, [(8, 1025), (8, 2049)], 0),
]


def attention_inputs(dq8, case, seed=0, spare=3):
    kind, type_, heads, kv, dim, page, each, window = case
    rng = np.random.default_rng(100 * dim + len(each) + seed)
    per = [-(-max(m, 1) // page) for _, m in each]
    total = sum(per) + spare
    cache = new_cache(kind, rng, total, kv, page, dim)
    order = rng.permutation(total).astype(np.int32)
    pages = np.full((len(each), max(per)), total + 5, np.int32)  # entries behind a sequence's last page are no pages
    at = 0
    used = np.zeros((total, page), bool)
    for b, p in enumerate(per):
        pages[b, :p] = order[at:at + p]
        for j in range(each[b][1]):
            used[pages[b, j // page], j % page] = True
        at += p
    cache[1][:, ~used.any(1)] = np.nan
    for n, place in zip(*np.nonzero(~used)):
        cache[1][:, n, :, place] = np.nan  # what no query sees
    starts = np.concatenate([[0], np.cumsum([n for n, _ in each])]).astype(np.int32)
    lens = np.array([m for _, m in each], np.int32)
    q = torch.from_numpy(rng.normal(0, 0.7, (int(starts[-1]), heads, dim)).astype(np.float32)).to(TYPES[type_])
    return cache, q, pages, lens, starts


def check_attention(got, q, want, tol, rows=None):
    t = q.dtype
    got = host(got)
    rows = np.isfinite(want).all((1, 2)) if rows is None else rows
    allowed = tol + half_step(t) * (np.abs(want) + tol) + torch.finfo(t).tiny * half_step(t)
    off = np.abs(got - want)[rows]
    assert np.isfinite(got[rows]).all()
    assert (off <= allowed[rows]).all(), (off / allowed[rows]).max()


@pytest.mark.parametrize("case", ATTENTIONS, ids=lambda c: "k%d_%s_h%d_%d_d%d_p%d_w%d" % (c[:6] + (c[7],)))
def test_attention(dq8, case):
    kind, _, heads, kv, dim, page, each, window = case
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = ref.attention(kind, cache, host(q), pages, lens, starts, dim ** -0.5, window)
    gpu, cuda = to_gpu(cache), lambda a: torch.from_numpy(a).cuda()
    args = (kind, q.cuda(), *gpu, cuda(pages), cuda(lens))
    got = dq8.cache_attention(*args, starts=cuda(starts), window=window)
    check_attention(got, q, want, tol)
    again = dq8.cache_attention(*args, starts=cuda(starts), window=window)
    assert torch.equal(got, again)
    known = dq8.cache_attention(*args, starts=cuda(starts), window=window, max_new=max(n for n, _ in each))
    check_attention(known, q, want, tol)
    wrong = dq8.cache_attention(*args, starts=cuda(starts), window=window, max_new=1)  # a bad guess of the host's is right too
    check_attention(wrong, q, want, tol)
    if len({n for n, _ in each}) == 1:
        check_attention(dq8.cache_attention(*args, window=window), q, want, tol)
    # without scratch memory
    whole = dq8.cache_attention(*args, starts=cuda(starts), window=window, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    check_attention(whole, q, want, tol)


def test_attention_strides_and_rows_behind_the_last_sequence(dq8):
    case = (0, "bf16", 6, 2, 80, 16, [(2, 50), (3, 41)], 0)
    kind, _, heads, kv, dim, page, each, _ = case
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = ref.attention(kind, cache, host(q), pages, lens, starts, 0.2)
    wide = torch.zeros((9, heads + 1, dim + 3), dtype=q.dtype, device="cuda")  # odd strides: rows at any multiple of two bytes
    wide[:5, 1:, 3:] = q.cuda()
    wide[5:] = float("nan")
    out = torch.full((heads, 9, dim + 1), 7.0, dtype=q.dtype, device="cuda")
    cuda = lambda a: torch.from_numpy(a).cuda()
    got = dq8.cache_attention(kind, wide[:, 1:, 3:], *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(starts), softmax_scale=0.2,
                              out=out.transpose(0, 1)[:, :, 1:])
    check_attention(got[:5], q, want, tol)
    out = out.transpose(0, 1)
    assert (out[5:] == 7.0).all() and (out[:, :, 0] == 7.0).all()


def test_attention_of_bad_pages_lengths_and_starts(dq8):
    """Page numbers outside the cache are not seen, lengths and starts count as the nearest possible ones; nothing else is touched."""
    case = (0, "f16", 4, 2, 64, 16, [(1, 100), (1, 90), (1, 33), (2, 64)], 0)
    kind, _, heads, kv, dim, page, each, _ = case
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    pages[0, 2], pages[1, 0], pages[2, :] = -1, 2 ** 31 - 1, 1 << 20
    lens[1], lens[3] = 90, 10 ** 9
    cache[1][np.isnan(cache[1])] = 1.0
    pages[3, 4:] = -5
    cuda = lambda a: torch.from_numpy(a).cuda()
    want, tol = ref.attention(kind, cache, host(q), pages, lens, starts, dim ** -0.5)
    got = dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(starts))
    check_attention(got, q, want, tol)
    assert not got[2].any()  # none of its pages is one
    # starts outside the range count as its nearer end
    bad = starts.copy()
    bad[0], bad[4] = -7, 2 ** 31 - 1
    check_attention(dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(bad)), q, want, tol)
    negative = dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(np.full(4, -3, np.int32)), starts=cuda(starts))
    assert not negative.any()


@pytest.mark.parametrize("max_new", [1, 40])
@pytest.mark.parametrize("sequences", [2, 64, 300])
def test_attention_of_descending_starts_writes_nothing(dq8, sequences, max_new):
    """Sequences that lie over each other: far more work than as many tokens can be, so that none of it is begun.  One descent
    anywhere is enough."""
    case = (0, "f16", 8, 2, 64, 16, [(40, 300)], 0)
    kind, _, heads, kv, dim, page, _, _ = case
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    cuda = lambda a: torch.from_numpy(a).cuda()
    many = (np.repeat(pages, sequences, 0), np.repeat(lens, sequences))
    over = np.where(np.arange(sequences + 1) % 2, 40, 0).astype(np.int32)
    last = np.full(sequences + 1, 40, np.int32)
    last[0], last[-1] = 0, 39
    for bad in (over, last):
        out = torch.full_like(q, 7.0, device="cuda")
        got = dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(many[0]), cuda(many[1]), starts=cuda(bad), max_new=max_new, out=out)
        assert got is out and (out == 7.0).all()


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("n", [5, 60, 300])
@pytest.mark.parametrize("window", [1, 2 ** 31 - 1])
def test_attention_of_windows_where_the_first_queries_see_nothing(dq8, dim, n, window):
    """Sequences with fewer cached tokens than new ones under the smallest and the largest window."""
    case = (0, "f16", 2, 1, dim, 16, [(n, 2), (n, 0), (n, n - 1), (n, n + 40)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = ref.attention(0, cache, host(q), pages, lens, starts, dim ** -0.5, window)
    cuda = lambda a: torch.from_numpy(a).cuda()
    for max_new in (1, n):
        got = dq8.cache_attention(0, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), starts=cuda(starts), max_new=max_new, window=window)
        check_attention(got, q, want, tol)
        assert not got[:n - 2].any()


@pytest.mark.parametrize("scale", [0.0, -0.3, 1e-30, 1e-44])
@pytest.mark.parametrize("n", [2, 140])
def test_attention_of_any_softmax_scale(dq8, n, scale):
    case = (0, "f16", 4, 2, 128, 16, [(n, n + 100), (n, n)], 0)
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = ref.attention(0, cache, host(q), pages, lens, starts, scale)
    cuda = lambda a: torch.from_numpy(a).cuda()
    got = dq8.cache_attention(0, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens), softmax_scale=scale)
    check_attention(got, q, want, tol)


@pytest.mark.parametrize("n", [1, 50])
def test_attention_of_values_of_very_different_sizes(dq8, n):
    """Scales over thirty-six decades: weights follow the largest so far, whatever the order."""
    case = (0, "f16", 2, 1, 64, 16, [(n, 400)], 0)
    kind, _, heads, kv, dim, page, each, _ = case
    for order in (1, -1):
        cache, q, pages, lens, starts = attention_inputs(dq8, case)
        j = np.arange(400)
        size = 10.0 ** np.linspace(-32, 4, 400)[::order]
        cache[1][1, pages[0, j // page], 0, j % page] = size.astype(np.float32)
        want, tol = ref.attention(kind, cache, host(q), pages, lens, starts, dim ** -0.5)
        cuda = lambda a: torch.from_numpy(a).cuda()
        check_attention(dq8.cache_attention(kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens)), q, want, tol)


@pytest.mark.parametrize("n", [3, 40])
def test_attention_of_nan_and_extreme_queries_stays_in_its_rows(dq8, n):
    case = (0, "bf16", 4, 1, 128, 16, [(n, 197 + n)], 0)
    kind, _, heads, kv, dim, page, each, _ = case
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = ref.attention(kind, cache, host(q), pages, lens, starts, dim ** -0.5)
    bad = q.clone()
    bad[0, 1, 3], bad[1, 2, 7] = float("nan"), float("inf")
    bad[2, 0] *= 1e30
    cuda = lambda a: torch.from_numpy(a).cuda()
    got = dq8.cache_attention(kind, bad.cuda(), *to_gpu(cache), cuda(pages), cuda(lens))
    for i, h in ((0, 1), (1, 2)):
        assert torch.isnan(got[i, h]).all()
    # a row whose weights are all on one token
    cb = oracle.codebook(kind).astype(np.float64)
    j = np.arange(200)  # (the query's position is 199)
    kk = cb[cache[0][0, pages[0, j // page], 0, j % page]] * cache[1][0, pages[0, j // page], 0, j % page][:, None]
    best = int(np.argmax(kk @ host(bad)[2, 0].astype(np.float64)))
    vv = cb[cache[0][1, pages[0, best // page], 0, best % page]] * cache[1][1, pages[0, best // page], 0, best % page]
    assert np.abs(host(got)[2, 0] - vv).max() <= 2.0 ** -7 * np.abs(vv).max()
    got[0, 1], got[1, 2], got[2, 0] = (torch.from_numpy(want[i]).cuda().to(got.dtype) for i in ((0, 1), (1, 2), (2, 0)))
    check_attention(got, q, want, tol)


def dense(dq8, kind, gpu, q, pages, lens, n):
    """(out, tolerance) of sequences of n new tokens each in float64 on the GPU, for sizes that numpy is slow at: see
    cache_reference.attention."""
    values = dq8.codebook(kind).double().cuda()
    page, dim, kv = gpu[0].shape[3], gpu[0].shape[4], gpu[0].shape[2]
    out, tol, u = torch.zeros(q.shape, dtype=torch.float64, device="cuda"), torch.zeros(q.shape, dtype=torch.float64, device="cuda"), 2.0 ** -11
    for b in range(len(lens)):
        length = int(lens[b])
        number = pages[b, : -(-length // page)].long()
        hidden = torch.arange(length, device="cuda") > torch.arange(length - n, length, device="cuda")[:, None]
        for h in range(kv):
            k, v = (values[gpu[0][p, number, h].reshape(-1, dim)[:length].long()] * gpu[1][p, number, h].reshape(-1)[:length, None].double() for p in (0, 1))
            for x in range(h * q.shape[1] // kv, (h + 1) * q.shape[1] // kv):
                row = q[b * n:(b + 1) * n, x].double()
                w = torch.softmax(((row @ k.T) * dim ** -0.5).masked_fill(hidden, float("-inf")), 1)
                e = (row.abs() @ k.abs().T).amax(1, keepdim=True) * dim ** -0.5 * (u + (dim + 8) * 2.0 ** -24)
                assert e.max() < 2.0 ** -6
                out[b * n:(b + 1) * n, x] = w @ v
                tol[b * n:(b + 1) * n, x] = w @ v.abs() * (2 * u + 2 * e + (8 + length) * 2.0 ** -24) * (1 + 2.0 ** -5) + length * 2.0 ** -31 * v.abs().max()
    return out, tol


def near(got, want):
    out, tol = want
    step = half_step(got.dtype)
    return bool(((got.double() - out).abs() <= tol + step * (out.abs() + tol) + torch.finfo(got.dtype).tiny * step).all())


def test_attention_of_long_sequences_and_many(dq8):
    """Work cut over the token axis: one long history, many short ones, and more sequences than a workgroup has threads."""
    g = torch.Generator(device="cuda").manual_seed(3)
    for batch, longest, heads, kv, dim, page in ((1, 70001, 8, 1, 128, 64), (600, 90, 4, 2, 64, 16), (701, 70, 8, 4, 80, 16), (3, 9000, 32, 8, 128, 128)):
        per = -(-longest // page)
        pool = batch * per + 1
        codes = torch.randint(0, 256, (2, pool, kv, page, dim), dtype=torch.uint8, device="cuda", generator=g)
        scales = torch.rand((2, pool, kv, page), device="cuda", generator=g) + 0.5
        pages = torch.randperm(pool, device="cuda", generator=g)[:batch * per].to(torch.int32).view(batch, per)
        lens = torch.randint(1, longest + 1, (batch,), device="cuda", generator=g, dtype=torch.int32)
        lens[0] = longest
        q = torch.randn((batch, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
        got = dq8.cache_attention(0, q, codes, scales, pages, lens)
        assert near(got, dense(dq8, 0, (codes, scales), q, pages, lens.cpu(), 1))


def test_attention_and_append_beyond_32_bits(dq8):
    """A cache of over 4 GiB of codes: pages at its end."""
    pages, kv, page, dim = 4200, 4, 1024, 128  # 2 x 2.05 GiB of codes
    codes = torch.empty((2, pages, kv, page, dim), dtype=torch.uint8, device="cuda")
    scales = torch.empty((2, pages, kv, page), device="cuda")
    assert codes.numel() > 2 ** 32
    g = torch.Generator(device="cuda").manual_seed(4)
    k, v = (torch.randn((1500, kv, dim), device="cuda", generator=g) for _ in range(2))
    table = torch.tensor([pages - 1, pages - 2], dtype=torch.int32, device="cuda").view(1, 2)
    j = torch.arange(1500, device="cuda")
    slots = table[0].long()[j // page] * page + j % page
    dq8.cache_append(0, k, v, slots, codes, scales)
    for part, x in ((0, k), (1, v)):
        c, s = dq8.encode(0, x.reshape(-1), dim)
        assert torch.equal(codes[part][slots // page, :, slots % page].reshape(-1), c) and torch.equal(scales[part][slots // page, :, slots % page].reshape(-1), s)
    q = torch.randn((2, 8, dim), device="cuda", generator=g).to(torch.float16)
    lens = torch.tensor([1500], dtype=torch.int32, device="cuda")
    got = dq8.cache_attention(0, q, codes, scales, table, lens)
    assert near(got, dense(dq8, 0, (codes, scales), q, table, [1500], 2))


# ---------------------------------------------------------------- as they are used


def test_prompt_chunks_and_decoding_equal_one_pass(dq8):
    """Two sequences: a prompt in chunks, then tokens one by one, each step an append and the attention that reads it; and the
    whole at once.  The cache ends up the same, bit for bit, and the outputs agree."""
    kind, heads, kv, dim, page, total = 0, 8, 2, 64, 16, 75
    g = torch.Generator(device="cuda").manual_seed(9)
    x = torch.randn((2, total, heads + 2 * kv, dim), device="cuda", generator=g).to(torch.bfloat16)
    a = torch.arange(total, device="cuda", dtype=torch.float64)[:, None] * 100.0 ** (-torch.arange(dim // 2, device="cuda") / (dim // 2))
    table = torch.stack([a.cos(), a.sin()], 1).float()
    w = torch.rand(dim, device="cuda", generator=g) + 0.5
    pages = torch.randperm(10, device="cuda", generator=g).to(torch.int32).view(2, 5)

    def step(buffers, first, last):
        rows = x[:, first:last].reshape(-1, heads + 2 * kv, dim)
        q, k, v = rows.split([heads, kv, kv], 1)
        j = torch.arange(first, last, device="cuda")
        slots = (pages.long()[:, j // page] * page + j % page).reshape(-1)
        q = dq8.cache_append(kind, k, v, slots, *buffers, positions=j.repeat(2), rotation=table, q=q, q_weight=w, k_weight=w)
        lens = torch.full((2,), last, dtype=torch.int32, device="cuda")
        return q, dq8.cache_attention(kind, q, *buffers, pages, lens).view(2, last - first, heads, dim)

    one, parts = dq8.cache_buffers(10, kv, page, dim), dq8.cache_buffers(10, kv, page, dim)
    q, whole = step(one, 0, total)
    edges = [0, 33, 34, 60] + list(range(61, total + 1))
    pieces = torch.cat([step(parts, i, j)[1] for i, j in zip(edges, edges[1:])], 1)
    assert torch.equal(one[0], parts[0]) and torch.equal(one[1], parts[1])
    want = dense(dq8, kind, one, q, pages, [total, total], total)
    assert near(whole.reshape(-1, heads, dim), want) and near(pieces.reshape(-1, heads, dim), want)
    values = dq8.decode(kind, *one, dim)
    assert torch.isfinite(values).all() and values.abs().max() > 0


@pytest.mark.parametrize("n,most", [(1, 320), (12, 1280)])
def test_cache_calls_recorded_in_a_graph(dq8, n, most):
    """A step of one or more tokens captured once and replayed with new inputs and lengths, eager work and synchronisations between."""
    kind, batch, heads, kv, dim, page = 0, 3, 8, 2, 128, 16
    g = torch.Generator(device="cuda").manual_seed(5)
    codes, scales = dq8.cache_buffers(batch * most // page, kv, page, dim)
    codes.random_(0, 256, generator=g)
    scales.uniform_(0.5, 1.5, generator=g)
    pages = torch.randperm(batch * most // page, device="cuda", generator=g).to(torch.int32).view(batch, -1)
    x = torch.zeros((batch * n, heads + 2 * kv, dim), dtype=torch.bfloat16, device="cuda")
    q, k, v = x.split([heads, kv, kv], 1)
    slots, lens = torch.zeros(batch * n, dtype=torch.int64, device="cuda"), torch.zeros(batch, dtype=torch.int32, device="cuda")
    q2, out = (torch.empty((batch * n, heads, dim), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    space = torch.empty(dq8.cache_attention_workspace(q, codes, scales, pages, lens), dtype=torch.uint8, device="cuda")
    stream = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=stream):
        dq8.cache_append(kind, k, v, slots, codes, scales, q=q, q_out=q2)
        dq8.cache_attention(kind, q2, codes, scales, pages, lens, out=out, workspace=space)
    for rep in range(4):
        x.copy_(torch.randn(x.shape, device="cuda", generator=g))
        length = torch.randint(n, most + 1, (batch,), device="cuda", generator=g)
        lens.copy_(length)
        j = length[:, None] - n + torch.arange(n, device="cuda")
        slots.copy_((pages.long().gather(1, j // page) * page + j % page).reshape(-1))
        other = codes.clone(), scales.clone()
        dq8.cache_append(kind, k, v, slots, *other)
        eager = dq8.cache_attention(kind, q, *other, pages, lens, workspace=torch.empty(space.numel(), dtype=torch.uint8, device="cuda"))
        out.fill_(float("nan"))
        space.fill_(0xFF)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, eager) and torch.equal(codes, other[0]) and torch.equal(scales, other[1]) and torch.equal(q2, q)


def test_capture_without_a_workspace_allocates_nothing_and_is_right(dq8):
    case = (0, "bf16", 8, 2, 128, 16, [(1, 300), (1, 41)], 0)
    kind = case[0]
    cache, q, pages, lens, starts = attention_inputs(dq8, case)
    want, tol = ref.attention(kind, cache, host(q), pages, lens, starts, 128 ** -0.5)
    cuda = lambda a: torch.from_numpy(a).cuda()
    args = (kind, q.cuda(), *to_gpu(cache), cuda(pages), cuda(lens))
    out = torch.empty_like(args[1])
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        dq8.cache_attention(*args, out=out)
        after = torch.cuda.memory_stats()["allocation.all.allocated"]
    assert after == before
    for _ in range(3):
        out.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        check_attention(out, q, want, tol)


def test_two_streams_at_once(dq8):
    """Calls on two streams, each with scratch memory of its own from torch's allocator."""
    g = torch.Generator(device="cuda").manual_seed(6)
    codes = torch.randint(0, 256, (2, 300, 4, 16, 128), dtype=torch.uint8, device="cuda", generator=g)
    scales = torch.rand((2, 300, 4, 16), device="cuda", generator=g) + 0.5
    pages = torch.arange(300, dtype=torch.int32, device="cuda").view(2, 150)
    lens = torch.tensor([2400, 1999], dtype=torch.int32, device="cuda")
    qs = [torch.randn((2, 16, 128), device="cuda", generator=g).to(torch.bfloat16) for _ in range(2)]
    want = [dq8.cache_attention(0, q, codes, scales, pages, lens) for q in qs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in range(2)], [[], []]
    for _ in range(20):
        for i, s in enumerate(streams):
            with torch.cuda.stream(s):
                got[i].append(dq8.cache_attention(0, qs[i], codes, scales, pages, lens))
    torch.cuda.synchronize()
    assert all(torch.equal(o, want[i]) for i in range(2) for o in got[i])


def test_empty_calls(dq8):
    codes, scales = dq8.cache_buffers(2, 2, 16, 64)
    none = torch.empty((0, 2, 64), dtype=torch.bfloat16, device="cuda")
    dq8.cache_append(0, none, none, torch.empty(0, dtype=torch.int64, device="cuda"), codes, scales, q=none)
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    assert dq8.cache_attention(0, none, codes, scales, i32(0, 1), i32(0)).shape == (0, 2, 64)
    assert dq8.cache_attention(0, none, codes, scales, i32(3, 1), i32(3), starts=i32(4)).shape == (0, 2, 64)
    q = torch.ones((2, 2, 64), dtype=torch.bfloat16, device="cuda")
    out = torch.full_like(q, 3.0)
    dq8.cache_attention(0, q, codes, scales, i32(3, 1), i32(3), starts=i32(4), out=out)  # no sequence has a new token
    assert (out == 3.0).all()
    assert not codes.any() and not scales.any()


def test_refusals(dq8):
    codes, scales = dq8.cache_buffers(4, 2, 16, 64)
    k = torch.ones((3, 2, 64), dtype=torch.bfloat16, device="cuda")
    q = torch.ones((3, 4, 64), dtype=torch.bfloat16, device="cuda")
    slots, pos = torch.arange(3, device="cuda"), torch.arange(3, device="cuda")
    table, w = torch.ones((8, 2, 32), device="cuda"), torch.ones(64, device="cuda")
    bad = [
        (TypeError, lambda: dq8.cache_append(0, k.cpu(), k, slots, codes, scales)),
        (TypeError, lambda: dq8.cache_append(0, k.double(), k, slots, codes, scales)),
        (TypeError, lambda: dq8.cache_append(0, k, k.half(), slots, codes, scales)),
        (TypeError, lambda: dq8.cache_append(0, k, k, slots.int(), codes, scales)),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots[:2], codes, scales)),
        (ValueError, lambda: dq8.cache_append(0, k[:, :1], k, slots, codes, scales)),
        (ValueError, lambda: dq8.cache_append(0, k.transpose(1, 2), k, slots, codes, scales)),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots, codes[:1], scales)),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots, codes, scales[:, :2])),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots, codes, scales, rotation=table)),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots, codes, scales, positions=pos)),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots, codes, scales, q_weight=w)),
        (ValueError, lambda: dq8.cache_append(0, k, k, slots, codes, scales, k_weight=w[:32])),
        (dq8.Dq8Error, lambda: dq8.cache_append(0, k, k, slots, codes, scales, positions=pos, rotation=torch.ones((8, 2, 33), device="cuda"))),
        (dq8.Dq8Error, lambda: dq8.cache_append(4, k, k, slots, codes, scales)),
        (dq8.Dq8Error, lambda: dq8.cache_append(0, k, k, slots, codes, scales, k_weight=w, eps=float("nan"))),
        (dq8.Dq8Error, lambda: dq8.cache_append(0, k, k, slots, codes, scales, q=q, q_out=q[:, :, :].as_strided(q.shape, (256, 32, 1)))),
        (dq8.Dq8Error, lambda: dq8.cache_append(0, k, k, slots, codes, scales, q=q, q_out=torch.empty_like(q[:1]).expand(3, 4, 64))),
        (dq8.Dq8Error, lambda: dq8.cache_append(0, q[:, 2:], k, slots, codes, scales, q=q, q_out=q)),
        (dq8.Dq8Error, lambda: dq8.cache_append(0, k[:, :, :40], k[:, :, :40], slots, codes[..., :40].contiguous(), scales)),
    ]
    i32 = lambda *s: torch.zeros(s, dtype=torch.int32, device="cuda")
    pages, lens = i32(3, 1), i32(3)
    bad += [
        (TypeError, lambda: dq8.cache_attention(0, q.float(), codes, scales, pages, lens)),
        (TypeError, lambda: dq8.cache_attention(0, q, codes, scales, pages.long(), lens)),
        (ValueError, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens[:2])),
        (ValueError, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, starts=i32(3))),
        (ValueError, lambda: dq8.cache_attention(0, q[:, :, :32], codes, scales, pages, lens)),
        (ValueError, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, out=q[:2])),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q[:, :3], codes, scales, pages, lens)),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q[:2], codes, scales, pages, lens)),  # two tokens of three sequences
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, out=q)),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, out=torch.empty_like(q[:, :1]).expand(3, 4, 64))),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, window=-1)),
        (ValueError, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, window=2 ** 32 + 5)),
        (ValueError, lambda: dq8.cache_attention(0, q, codes, scales, torch.zeros((3, 2), dtype=torch.int32, device="cuda")[:, :1], lens)),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, softmax_scale=float("inf"))),
        (dq8.Dq8Error, lambda: dq8.cache_attention(9, q, codes, scales, pages, lens)),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q, codes, scales, i32(3, 0), lens)),
        (dq8.Dq8Error, lambda: dq8.cache_attention(0, q, codes, scales, pages, lens, workspace=torch.empty(100, dtype=torch.uint8, device="cuda")[1:])),
    ]
    for i, (error, call) in enumerate(bad):
        with pytest.raises(error):
            call()
            pytest.fail("refusal %d" % i)
    torch.cuda.synchronize()
    assert not codes.any() and not scales.any()


def test_work_of_2_to_the_31_tiles_is_refused(dq8):
    """64 heads of one sequence whose pages would hold 2^30 tokens; the sequence itself has one."""
    codes, scales = dq8.cache_buffers(1, 64, 1024, 16)
    q = torch.ones((1, 64, 16), dtype=torch.float16, device="cuda")
    pages, lens = torch.zeros((1, 1 << 20), dtype=torch.int32, device="cuda"), torch.ones(1, dtype=torch.int32, device="cuda")
    with pytest.raises(dq8.Dq8Error, match="too much work"):
        dq8.cache_attention(0, q, codes, scales, pages, lens)
    assert not dq8.cache_attention(0, q, codes, scales, pages[:, :1 << 18], lens).any()
