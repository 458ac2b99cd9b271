"""Weights in 4 bits and their products against plain implementations in 64 bits."""
import numpy as np
import pytest
import torch

from paper_1511_04561_amd import dq8

from . import serve_reference as ref

pytestmark = pytest.mark.gpu
DTYPES = [torch.bfloat16, torch.float16]
STEP = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # half a step, relative


def array(t):
    return t.detach().cpu().double().numpy()


def weights(rows, cols, seed):
    rng = np.random.default_rng(seed)
    w = (rng.standard_normal((rows, cols)) * np.exp(rng.standard_normal((rows, 1)))).astype(np.float32)
    w[rng.random(w.shape) < 0.02] = 0.0
    return w


def compressed(rows, cols, group, seed):
    codes, scales = ref.encode(weights(rows, cols, seed), group)
    return torch.from_numpy(codes).cuda(), torch.from_numpy(scales).to(torch.bfloat16).cuda(), ref.decode(codes, scales, rows, cols)


def within(got, want, size, group, cols, dtype, bias=0.0):
    """got against want: sums in binary32 of cols products of size `size` in all, one rounding to dtype.

    A product is exact.  Each of the at most 128 additions in a group, of the additions of groups (one fused with the scale) and of the eight parts and the bias
    is off by at most 2^-23 (whichever way the matrix unit rounds) of a sum of absolute values: (128 + cols / group + 10) 2^-23 size.  Results
    below the type's normal numbers are off by half of its smallest one."""
    tiny = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}[dtype]
    bound = (min(group, cols) + -(-cols // group) + 10) * 2.0 ** -23 * (size + np.abs(bias))
    bound = bound + STEP[dtype] * (np.abs(want) + bound) + tiny
    assert (np.abs(got - want) <= bound).all(), (np.abs(got - want) / bound).max()


SHAPES = [(1, 1), (16, 128), (5, 31), (17, 129), (33, 1000), (100, 257), (64, 2048), (48, 136)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("rows,cols", SHAPES)
@pytest.mark.parametrize("dtype", [torch.float32] + DTYPES)
def test_encode_and_decode(rows, cols, group, dtype):
    w = torch.from_numpy(weights(rows, cols, rows + cols)).to(dtype)
    codes, scales = ref.encode(w.float().numpy(), group)
    c, s = dq8.weights_encode(w.cuda(), group)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(array(s), scales)
    want = ref.decode(codes, scales, rows, cols)
    for to in [torch.float32] + DTYPES:
        got = dq8.weights_decode(c, s, rows, cols, dtype=to)
        assert got.dtype == to and torch.equal(got.cpu(), torch.from_numpy(want).to(torch.float32).to(to))
    # whole tiles: zeros behind the last row and column
    whole = array(dq8.weights_decode(c, s))
    assert np.array_equal(whole[:rows, :cols], want) and not whole[rows:].any() and not whole[:, cols:].any()


def test_encode_on_and_next_to_every_border():
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0], np.float32)
    w = np.zeros((16, 128), np.float32)
    for r, scale in enumerate([1.0, 3.0, 2.0 ** -126, 2.0 ** -132, 1.5 * 2.0 ** -133, 170 * 2.0 ** 118, 2.0 ** 100, 255.0]):
        for i, b in enumerate(borders):
            at = np.float32(b * scale)
            w[r, 4 * i : 4 * i + 3] = np.nextafter(at, np.float32(0)), at, -np.nextafter(at, np.float32(np.inf))
        w[r, 31] = 6 * scale
    codes, scales = ref.encode(w, 32)
    c, s = dq8.weights_encode(torch.from_numpy(w).cuda(), 32)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(array(s), scales)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("group", [32, 128])
def test_encode_16_bits_on_and_next_to_borders(dtype, group):
    """Every 16-bit number next to every border of many scales: mantissas of the scale, exponents to the ends of the type."""
    borders = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    rng = np.random.default_rng(5)
    exps = [-133, -130, -126, -120, -1, 0, 5, 100, 118] if dtype == torch.bfloat16 else [-26, -24, -15, -3, 0, 6, 12]
    rows = []
    for e in exps:
        for m in [1.0, 255 / 128, 129 / 128, 170 / 128] + list(rng.integers(128, 256, 20) / 128):
            s = m * 2.0 ** e
            top = torch.tensor(6 * s, dtype=torch.float64).float().to(dtype)  # the group's largest makes the scale
            if not torch.isfinite(top):
                continue
            scale = float(ref.bf16(np.float32(float(top.float())) / np.float32(6)))
            near = torch.from_numpy(borders * scale).float().to(dtype).view(torch.int16)
            row = torch.cat([near - 1, near, near + 1]).clamp(min=0).view(dtype)
            row = torch.where(torch.arange(21) % 2 == 0, row, -row)
            row = torch.where(row.abs() > top, top, row)
            rows.append(torch.cat([top.view(1), row, torch.zeros(group - 22, dtype=dtype)]))
    w = torch.stack(rows)
    codes, scales = ref.encode(w.float().numpy(), group)
    c, s = dq8.weights_encode(w.cuda(), group)
    assert np.array_equal(array(s), scales) and np.array_equal(c.cpu().numpy(), codes)


@pytest.mark.parametrize("dtype", DTYPES)
def test_encode_16_bits_extremes(dtype):
    top = torch.finfo(dtype).max
    w = torch.zeros((16, 256), dtype=dtype)
    w[0, :5] = torch.tensor([top, -top, top / 2, 1.0, -0.0])
    w[1, 3], w[1, 40], w[1, 70], w[1, 100] = float("inf"), float("-inf"), float("nan"), 1.0
    w[2, :] = -0.0
    w[3, :3] = torch.tensor([1, -32767, 3], dtype=torch.int16).view(dtype)  # subnormal numbers
    w[4, :64:2] = torch.arange(1, 33, dtype=torch.int16).view(dtype)
    codes, scales = ref.encode(w.float().numpy(), 32)
    c, s = dq8.weights_encode(w.cuda(), 32)
    assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(array(s), scales, equal_nan=True)


def test_encode_extremes():
    top = np.finfo(np.float32).max
    w = np.zeros((16, 256), np.float32)
    w[0, :5] = top, -top, top / 2, 1.0, -0.0
    w[1, 3], w[1, 40], w[1, 70], w[1, 100] = np.inf, -np.inf, np.nan, 1.0
    w[2, :] = -0.0
    w[3, :3] = 1e-45, -1e-45, 5e-39
    w[4, :2] = 6 * 2.0 ** -134, 6 * 2.0 ** -135  # the scale between zero and the smallest bfloat16 number
    codes, scales = ref.encode(w, 32)
    c, s = dq8.weights_encode(torch.from_numpy(w).cuda(), 32)
    assert np.array_equal(c.cpu().numpy(), codes)
    assert np.array_equal(array(s), scales, equal_nan=True)
    got = array(dq8.weights_decode(c, s))
    assert np.array_equal(got, ref.decode(codes, scales, 16, 256), equal_nan=True)
    assert np.isnan(got[1, :96]).all() and np.isfinite(got[[0, 2, 3, 4]]).all() and np.array_equal(np.signbit(got[2]), np.ones(256, bool))


@pytest.mark.parametrize("dtype", [torch.float32] + DTYPES)
def test_encode_and_decode_with_strides_and_guards(dtype):
    rows, cols = 37, 203
    big = torch.from_numpy(weights(rows + 2, cols + 14, 3)).to(dtype).cuda()
    view = big[1 : rows + 1, 5 : 5 + cols]
    c, s = dq8.weights_encode(view, 64)
    c2, s2 = dq8.weights_encode(view.contiguous(), 64)
    assert torch.equal(c, c2) and torch.equal(s, s2)
    out = torch.full((rows + 2, cols + 9), 77.0, dtype=dtype, device="cuda")
    got = dq8.weights_decode(c, s, rows, cols, dtype=dtype, out=out[1 : rows + 1, 3 : 3 + cols])
    assert torch.equal(got, dq8.weights_decode(c, s, rows, cols, dtype=dtype))
    assert (out[0] == 77).all() and (out[-1] == 77).all() and (out[:, :3] == 77).all() and (out[:, 3 + cols :] == 77).all()
    # outputs handed in, inside guard bands
    band = torch.full((c.numel() + 64,), 9, dtype=torch.uint8, device="cuda")
    sband = torch.full((s.numel() + 32,), 9.0, dtype=torch.bfloat16, device="cuda")
    dq8.weights_encode(view, 64, codes=band[32:-32].view(c.shape), scales=sband[16:-16].view(s.shape))
    assert torch.equal(band[32:-32].view(c.shape), c) and torch.equal(sband[16:-16].view(s.shape), s)
    assert (band[:32] == 9).all() and (band[-32:] == 9).all() and (sband[:16] == 9).all() and (sband[-16:] == 9).all()


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("rows,cols,stride,offset", [(40, 128, 129, 0), (33, 128, 128, 1), (16, 256, 257, 1), (50, 127, 127, 0), (20, 8, 9, 1), (35, 131, 133, 3), (17, 391, 392, 5), (3, 1, 1, 1)])
def test_encode_of_rows_that_start_between_words(rows, cols, stride, offset, dtype):
    flat = torch.randn(offset + (rows - 1) * stride + cols, device="cuda").to(dtype)
    view = flat[offset:].as_strided((rows, cols), (stride, 1))
    for group in (32, 64, 128):
        c, s = dq8.weights_encode(view, group)
        codes, scales = ref.encode(array(view).astype(np.float32), group)
        assert np.array_equal(c.cpu().numpy(), codes) and np.array_equal(array(s), scales)


@pytest.mark.parametrize("tokens", [1, 2, 3, 4, 5, 8, 13, 16, 17, 31, 32, 33, 48, 64, 65, 130])
@pytest.mark.parametrize("rows,cols,group", [(16, 128, 32), (37, 300, 32), (130, 1025, 64), (200, 2048, 128), (5, 7, 64)])
def test_products(tokens, rows, cols, group):
    codes, scales, w = compressed(rows, cols, group, tokens)
    rng = np.random.default_rng(rows)
    bias = torch.from_numpy(rng.standard_normal(rows).astype(np.float32)).cuda()
    for dtype in DTYPES:
        x = torch.from_numpy(rng.standard_normal((tokens, cols)).astype(np.float32)).to(dtype).cuda()
        want, size = array(x) @ w.T, np.abs(array(x)) @ np.abs(w).T
        for to in (dtype, torch.float32):
            got = dq8.weights_product(x, codes, scales, rows=rows, dtype=to)
            assert got.dtype == to
            within(array(got), want, size, group, cols, to)
            got = dq8.weights_product(x, codes, scales, rows=rows, dtype=to, bias=bias)
            within(array(got), want + array(bias), size, group, cols, to, array(bias))


@pytest.mark.parametrize("rows,cols,group,tokens", [(4096, 4096, 32, 1), (8200, 1000, 64, 4), (1024, 14336, 128, 16), (20000, 640, 32, 9), (2048, 2048, 64, 300),
                                                    (512, 28672, 32, 40), (12345, 999, 128, 64)])
def test_large_products(rows, cols, group, tokens):
    g = torch.Generator(device="cuda").manual_seed(rows)
    w = torch.randn(rows, cols, generator=g, device="cuda") * cols ** -0.5
    codes, scales = dq8.weights_encode(w, group)
    w = dq8.weights_decode(codes, scales, rows, cols).double()
    for dtype in DTYPES:
        x = torch.randn(tokens, cols, generator=g, device="cuda").to(dtype)
        want, size = x.double() @ w.T, x.double().abs() @ w.abs().T
        for to in (dtype, torch.float32):
            within(array(dq8.weights_product(x, codes, scales, rows=rows, dtype=to)), array(want), array(size), group, cols, to)


@pytest.mark.parametrize("rows", [4096 + 7, 8192 + 16, 16384 + 1, 4 * 4096 + 33, 32768 + 17])
def test_products_on_both_sides_of_the_choices(rows):
    """Row counts on the sides of every choice between forms, tokens too; a rest of the columns in most forms' last chunk."""
    g = torch.Generator(device="cuda").manual_seed(rows)
    for cols in (200, 1310):
        codes, scales = dq8.weights_encode(torch.randn(rows, cols, generator=g, device="cuda"), 32)
        w = dq8.weights_decode(codes, scales, rows, cols).double()
        for tokens in (1, 2, 3, 4, 7, 8, 11, 16, 30, 33, 70, 190):
            x = torch.randn(tokens, cols, generator=g, device="cuda").half()
            want, size = x.double() @ w.T, x.double().abs() @ w.abs().T
            within(array(dq8.weights_product(x, codes, scales, rows=rows, dtype=torch.float32)), array(want), array(size), 32, cols, torch.float32)


@pytest.mark.parametrize("rows,tokens", [(28400, 200), (8200, 300), (8200, 700), (14300, 300), (5000, 1000), (5000, 2000)])
def test_products_of_many_tokens(rows, tokens):
    """Each of the forms that the turns of the compute units choose between; a rest of the columns, rows and tokens behind the last tile."""
    for cols, group in ((300, 32), (640, 128)):
        codes, scales = dq8.weights_encode(torch.randn(rows, cols, device="cuda"), group)
        w = dq8.weights_decode(codes, scales, rows, cols).double()
        x = torch.randn(tokens, cols, device="cuda").bfloat16()
        want, size = array(x.double() @ w.T), array(x.double().abs() @ w.abs().T)
        within(array(dq8.weights_product(x, codes, scales, rows=rows)), want, size, group, cols, torch.bfloat16)


@pytest.mark.parametrize("rows,tokens", [(28401, 200), (8203, 301), (8203, 700)])
@pytest.mark.parametrize("to", [torch.float32, torch.float16])
def test_results_of_many_tokens_with_strides_and_guards(rows, tokens, to):
    cols, group = 200, 64
    codes, scales = dq8.weights_encode(torch.randn(rows, cols, device="cuda"), group)
    w = dq8.weights_decode(codes, scales, rows, cols).double()
    bias = torch.randn(rows, device="cuda")
    x = torch.randn(tokens, cols + 3, device="cuda").half()[:, 1 : cols + 1]
    want, size = array(x.double() @ w.T) + array(bias), array(x.double().abs() @ w.abs().T)
    for left, right in ((0, 0), (1, 4), (8, 5)):
        out = torch.full((tokens + 2, left + rows + right), 7.0, dtype=to, device="cuda")
        dq8.weights_product(x, codes, scales, rows=rows, bias=bias, out=out[1 : tokens + 1, left : left + rows])
        within(array(out[1 : tokens + 1, left : left + rows]), want, size, group, cols, to, array(bias))
        assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, :left] == 7).all() and (out[:, left + rows :] == 7).all()


@pytest.mark.parametrize("rows", [8300, 12287, 24600, 30001, 45000, 53300, 70001])
def test_products_of_evenly_divided_rows(rows):
    """Workgroups with three row tiles or any number from 5 to 13, and behind the last row."""
    cols = 1330 if rows < 20000 else 330
    codes, scales = dq8.weights_encode(torch.randn(rows, cols, device="cuda"), 32)
    w = dq8.weights_decode(codes, scales, rows, cols).double()
    bias = torch.randn(rows, device="cuda")
    for tokens in (3, 8, 15, 32):
        x = torch.randn(tokens, cols, device="cuda").half()
        out = torch.full((tokens + 1, rows + 3), 7.0, device="cuda")
        dq8.weights_product(x, codes, scales, rows=rows, bias=bias, out=out[:tokens, :rows])
        want, size = array(x.double() @ w.T) + array(bias), array(x.double().abs() @ w.abs().T)
        within(array(out[:tokens, :rows]), want, size, 32, cols, torch.float32, array(bias))
        assert (out[tokens] == 7).all() and (out[:, rows:] == 7).all()


def test_long_rows():
    """Rows of activations around what is staged whole, and columns divided over workgroups with a rest."""
    for rows, cols, tokens in ((20, 32640, 1), (20, 32760, 1), (4100, 32512, 1), (17000, 16256, 2), (20, 32768, 1), (33, 16300, 2), (33, 16400, 2), (40, 40001, 20), (70, 9999, 64), (40, 40001, 16), (3000, 12300, 9), (16, 70000, 1), (300, 5000, 100)):
        codes, scales = dq8.weights_encode(torch.randn(rows, cols, device="cuda"), 64)
        w = dq8.weights_decode(codes, scales, rows, cols).double()
        x = torch.randn(tokens, cols, device="cuda").bfloat16()
        want, size = array(x.double() @ w.T), array(x.double().abs() @ w.abs().T)
        within(array(dq8.weights_product(x, codes, scales, rows=rows, dtype=torch.float32)), want, size, 64, cols, torch.float32)
        none = torch.empty(0, dtype=torch.uint8, device="cuda")
        within(array(dq8.weights_product(x, codes, scales, rows=rows, dtype=torch.float32, workspace=none)), want, size, 64, cols, torch.float32)


def test_workspaces_of_products():
    codes, scales, w = compressed(200, 9000, 32, 4)
    x = torch.randn(40, 9000, device="cuda").half()
    bias = torch.randn(200, device="cuda")
    n = dq8.weights_product_workspace(x, codes, scales, rows=200)
    assert n and n % (200 * 40 * 4) == 0 and dq8.weights_product_workspace(x[:16], codes, scales, rows=200) == 0
    want = dq8.weights_product(x, codes, scales, rows=200, bias=bias)
    alone = dq8.weights_product(x, codes, scales, rows=200, bias=bias, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
    for bytes_, same in ((n, want), (n - 1, alone), (n + 100, want)):
        space = torch.full((n + 160,), 0xFF, dtype=torch.uint8, device="cuda")
        got = dq8.weights_product(x, codes, scales, rows=200, bias=bias, workspace=space[16 : 16 + bytes_])
        assert torch.equal(got, same)
        assert (space[:16] == 0xFF).all() and (space[16 + n :] == 0xFF).all()
    # two graphs with a workspace each, one without, replayed in turn
    graphs = []
    for space in (torch.empty(n, dtype=torch.uint8, device="cuda"), torch.empty(n, dtype=torch.uint8, device="cuda"), None):
        out = torch.zeros_like(want)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            dq8.weights_product(x, codes, scales, rows=200, bias=bias, out=out, workspace=space)
        graphs.append((graph, out, space))
    for seed in range(4):
        x.copy_(torch.randn(40, 9000, generator=torch.Generator().manual_seed(seed)).half())
        want = dq8.weights_product(x, codes, scales, rows=200, bias=bias)
        alone = dq8.weights_product(x, codes, scales, rows=200, bias=bias, workspace=torch.empty(0, dtype=torch.uint8, device="cuda"))
        for graph, _, _ in graphs:
            graph.replay()
        torch.cuda.synchronize()
        assert [torch.equal(out, alone if space is None else want) for _, out, space in graphs] == [True] * 3


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("tokens", [1, 3, 20, 70])
def test_products_with_strides_and_guards(dtype, tokens):
    rows, cols, group = 53, 333, 32
    codes, scales, w = compressed(rows, cols, group, 5)
    big = torch.randn(tokens + 2, cols + 40, device="cuda").to(dtype)
    big[:, :7] = float("nan")
    big[:, 7 + cols :] = float("nan")  # what lies beside the rows is not read into them
    big[0], big[-1] = float("nan"), float("nan")
    x = big[1:-1, 7 : 7 + cols]
    want, size = array(x) @ w.T, np.abs(array(x)) @ np.abs(w).T
    for to in (dtype, torch.float32):
        out = torch.full((tokens + 2, rows + 5), 7.0, dtype=to, device="cuda")
        got = dq8.weights_product(x, codes, scales, rows=rows, out=out[1:-1, 3 : 3 + rows])
        within(array(got), want, size, group, cols, to)
        assert (out[0] == 7).all() and (out[-1] == 7).all() and (out[:, :3] == 7).all() and (out[:, 3 + rows :] == 7).all()
    # every row the same one (a stride of zero), every second row
    same = big[1:2, 7 : 7 + cols].expand(tokens, cols)
    assert torch.equal(dq8.weights_product(same, codes, scales, rows=rows), dq8.weights_product(same.contiguous(), codes, scales, rows=rows))
    half = torch.randn(2 * tokens, cols, device="cuda").to(dtype)[::2]
    assert torch.equal(dq8.weights_product(half, codes, scales, rows=rows), dq8.weights_product(half.contiguous(), codes, scales, rows=rows))


@pytest.mark.parametrize("dtype", DTYPES)
def test_rows_of_infinities_and_nan_stay_by_themselves(dtype):
    rows, cols, tokens = 40, 200, 21
    codes, scales, w = compressed(rows, cols, 32, 8)
    x = torch.randn(tokens, cols, device="cuda").to(dtype)
    clean = dq8.weights_product(x, codes, scales, rows=rows)
    x[3, 5], x[17, 199] = float("nan"), float("inf")
    got = dq8.weights_product(x, codes, scales, rows=rows)
    others = [i for i in range(tokens) if i not in (3, 17)]
    assert torch.equal(got[others], clean[others])
    assert got[3].isnan().all() and not got[17].isfinite().any()
    zero = torch.from_numpy(w[:, 199] == 0).cuda()
    assert torch.equal(got[17].isnan(), zero)


def test_products_of_the_largest_and_smallest_activations():
    """A group's sum of products leaves binary32 for no bfloat16 activations whose result is finite."""
    rows, cols = 16, 256
    w = np.full((rows, cols), 6e-3, np.float32)
    codes, scales = ref.encode(w, 128)
    w = ref.decode(codes, scales, rows, cols)
    c, s = torch.from_numpy(codes).cuda(), torch.from_numpy(scales).to(torch.bfloat16).cuda()
    for size in (2.0 ** 127, 2.0 ** 100, 2.0 ** -100, 2.0 ** -120):
        x = torch.full((2, cols), size, dtype=torch.bfloat16, device="cuda")
        x[1, ::2] *= -1
        got = array(dq8.weights_product(x, c, s, dtype=torch.float32))
        within(got, array(x) @ w.T, np.abs(array(x)) @ w.T, 128, cols, torch.float32)
    # the smallest: an activation times a magnitude is a multiple of 2^-134, and 2^-10 of that one of 2^-144: exact in binary32's subnormal numbers
    for size in (2.0 ** -125, 2.0 ** -129, 2.0 ** -133):
        x = torch.full((2, cols), size, dtype=torch.bfloat16, device="cuda")
        x[1, ::2] *= 3
        for scale in (1.0, 2.0 ** 60):
            s2 = torch.full(s.shape, scale).to(torch.bfloat16).cuda()
            w2 = ref.decode(codes, array(s2), rows, cols)
            within(array(dq8.weights_product(x, c, s2, dtype=torch.float32)), array(x) @ w2.T, np.abs(array(x)) @ np.abs(w2).T, 128, cols, torch.float32)
    # scales at the ends of their range
    for scale in (170 * 2.0 ** 118, 2.0 ** -133):
        s2 = torch.full(s.shape, scale, dtype=torch.float64).to(torch.bfloat16).cuda()
        w2 = ref.decode(codes, array(s2), rows, cols)
        x = torch.full((1, cols), 2.0 ** -9 if scale > 1 else 2.0 ** 100, dtype=torch.bfloat16, device="cuda")
        x[:, ::2] *= -0.5
        within(array(dq8.weights_product(x, c, s2, dtype=torch.float32)), array(x) @ w2.T, np.abs(array(x)) @ np.abs(w2).T, 128, cols, torch.float32)


def test_a_group_of_nan_weights_is_one_row_s_nan():
    w = weights(20, 256, 1)
    w[7, 130] = np.inf
    c, s = dq8.weights_encode(torch.from_numpy(w).cuda(), 64)
    x = torch.randn(3, 256, device="cuda").bfloat16()
    got = dq8.weights_product(x, c, s, rows=20)
    assert got[:, 7].isnan().all() and got[:, [i for i in range(20) if i != 7]].isfinite().all()


def test_parts_of_weights_are_weights():
    """Tiles of rows by themselves: what one rank of several has of a layer."""
    w = torch.randn(96, 512, device="cuda")
    c, s = dq8.weights_encode(w, 32)
    x = torch.randn(5, 512, device="cuda").half()
    whole = dq8.weights_product(x, c, s)
    parts = [dq8.weights_product(x, c[a:b], s[a:b]) for a, b in ((0, 2), (2, 3), (3, 6))]
    assert torch.equal(torch.cat(parts, 1), whole)


def test_products_on_another_stream_and_in_a_graph():
    codes, scales, w = compressed(300, 700, 64, 2)
    x = torch.randn(7, 700, device="cuda").bfloat16()
    want = dq8.weights_product(x, codes, scales, rows=300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        got = dq8.weights_product(x, codes, scales, rows=300)
    side.synchronize()
    assert torch.equal(got, want)
    out, new, values = torch.empty_like(want), x.clone(), torch.empty(300, 700, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        dq8.weights_product(new, codes, scales, rows=300, out=out)
        dq8.weights_decode(codes, scales, 300, 700, out=values)
    for seed in range(4):
        new.copy_(torch.randn(7, 700, generator=torch.Generator().manual_seed(seed)).bfloat16())
        out.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, dq8.weights_product(new, codes, scales, rows=300))
        assert torch.equal(values, dq8.weights_decode(codes, scales, 300, 700))


def test_the_python_path_gives_the_same(monkeypatch):
    w = torch.randn(50, 400, device="cuda")
    x = torch.randn(6, 400, device="cuda").half()
    bias = torch.randn(50, device="cuda")

    def calls():
        c, s = dq8.weights_encode(w, 64)
        return c, s, dq8.weights_decode(c, s, 50, 400, dtype=torch.float16), dq8.weights_product(x, c, s, rows=50, bias=bias, dtype=torch.float32)

    want = calls()
    monkeypatch.setattr(dq8, "_native", dq8._Unbound())
    assert all(torch.equal(a, b) for a, b in zip(calls(), want))
    # nothing to do
    empty = dq8.weights_product(x[:0], want[0], want[1], rows=50)
    assert empty.shape == (0, 50)


def test_refusals():
    w = torch.randn(40, 300, device="cuda")
    c, s = dq8.weights_encode(w, 32)
    x = torch.randn(2, 300, device="cuda").bfloat16()
    bad = [
        (ValueError, lambda: dq8.weights_encode(w, 48)),
        (ValueError, lambda: dq8.weights_encode(w.T, 32)),
        (TypeError, lambda: dq8.weights_encode(w.double(), 32)),
        (ValueError, lambda: dq8.weights_encode(w, 64, scales=s)),
        (ValueError, lambda: dq8.weights_encode(w, 32, codes=c[:2])),
        (TypeError, lambda: dq8.weights_decode(c, s.float())),
        (ValueError, lambda: dq8.weights_decode(c, s, rows=32)),
        (ValueError, lambda: dq8.weights_decode(c, s, cols=385)),
        (ValueError, lambda: dq8.weights_decode(c, s[:, :2])),
        (TypeError, lambda: dq8.weights_decode(c, s, out=torch.empty(48, 384, dtype=torch.bfloat16, device="cuda"))),
        (TypeError, lambda: dq8.weights_product(x.float(), c, s, rows=40)),
        (ValueError, lambda: dq8.weights_product(x[:, :200], c, s, rows=40)),
        (ValueError, lambda: dq8.weights_product(x, c, s, rows=49)),
        (TypeError, lambda: dq8.weights_product(x, c, s, rows=40, dtype=torch.float16)),
        (ValueError, lambda: dq8.weights_product(x, c, s, rows=40, bias=torch.zeros(48, device="cuda"))),
        (TypeError, lambda: dq8.weights_product(x, c, s, rows=40, bias=torch.zeros(40, device="cuda").half())),
        (ValueError, lambda: dq8.weights_product(x, c, s, rows=40, out=torch.empty(2, 48, device="cuda").bfloat16())),
        (ValueError, lambda: dq8.weights_product(x[0], c, s, rows=40)),
        (dq8.Dq8Error, lambda: dq8.weights_product(x, c, s, rows=40, out=x[:, :40])),
        (dq8.Dq8Error, lambda: dq8.weights_product(x, c, s, rows=40, out=torch.empty(40, device="cuda").bfloat16().expand(2, 40))),
    ]
    for error, call in bad:
        with pytest.raises(error):
            call()
