"""Products in every form that row and token counts choose, with the groups and types that have loads and scales of their own."""
import pytest
import torch

from paper_1511_04561_amd import dq8

from .test_gpu_weights import array, within

pytestmark = pytest.mark.gpu


# row tiles: up to 3 for each of 256 compute units, up to 4, up to 8, up to 13, more
@pytest.mark.parametrize("rows", [8203, 12309, 20011, 40005, 60001])
@pytest.mark.parametrize("dtype,group", [(torch.bfloat16, 32), (torch.bfloat16, 64), (torch.bfloat16, 128), (torch.float16, 64), (torch.float16, 128)])
def test_forms_of_many_rows(rows, dtype, group):
    """With whole chunks of columns and without, with a rest and without."""
    g = torch.Generator(device="cuda").manual_seed(rows + group)
    bias = torch.randn(rows, generator=g, device="cuda")
    for cols in (1030, 512, 100) if rows < 30000 else (650, 256, 90):
        codes, scales = dq8.weights_encode(torch.randn(rows, cols, generator=g, device="cuda"), group)
        w = dq8.weights_decode(codes, scales, rows, cols).double()
        for tokens in (1, 4, 8, 15, 32):
            x = torch.randn(tokens, cols, generator=g, device="cuda").to(dtype)
            want, size = array(x.double() @ w.T) + array(bias), array(x.double().abs() @ w.abs().T)
            for to in (dtype, torch.float32):
                out = torch.full((tokens + 1, rows + 3), 7.0, dtype=to, device="cuda")
                dq8.weights_product(x, codes, scales, rows=rows, bias=bias, out=out[:tokens, :rows])
                within(array(out[:tokens, :rows]), want, size, group, cols, to, array(bias))
                assert (out[tokens] == 7).all() and (out[:, rows:] == 7).all()


@pytest.mark.parametrize("rows,cols,tokens", [(4096, 2049, 40), (5000, 1100, 40), (8192, 1300, 60), (9000, 700, 100), (6000, 900, 100)])
@pytest.mark.parametrize("dtype,group", [(torch.float16, 32), (torch.bfloat16, 64), (torch.bfloat16, 128)])
def test_forms_of_middling_tokens(rows, cols, tokens, dtype, group):
    g = torch.Generator(device="cuda").manual_seed(rows + group)
    codes, scales = dq8.weights_encode(torch.randn(rows, cols, generator=g, device="cuda"), group)
    w = dq8.weights_decode(codes, scales, rows, cols).double()
    x = torch.randn(tokens, cols, generator=g, device="cuda").to(dtype)
    within(array(dq8.weights_product(x, codes, scales, rows=rows)), array(x.double() @ w.T), array(x.double().abs() @ w.abs().T), group, cols, dtype)


@pytest.mark.parametrize("rows,cols,tokens", [(500, 13000, 13), (3000, 12300, 9), (500, 7000, 20), (500, 12800, 31), (300, 9001, 100)])
@pytest.mark.parametrize("dtype,group", [(torch.float16, 32), (torch.bfloat16, 32), (torch.bfloat16, 128)])
def test_divided_columns(rows, cols, tokens, dtype, group):
    g = torch.Generator(device="cuda").manual_seed(rows + group)
    codes, scales = dq8.weights_encode(torch.randn(rows, cols, generator=g, device="cuda"), group)
    w = dq8.weights_decode(codes, scales, rows, cols).double()
    x, bias = torch.randn(tokens, cols, generator=g, device="cuda").to(dtype), torch.randn(rows, generator=g, device="cuda")
    assert dq8.weights_product_workspace(x, codes, scales, rows=rows) > 0
    want, size = array(x.double() @ w.T) + array(bias), array(x.double().abs() @ w.abs().T)
    for space in (None, torch.empty(0, dtype=torch.uint8, device="cuda")):
        for to in (dtype, torch.float32):
            within(array(dq8.weights_product(x, codes, scales, rows=rows, bias=bias, dtype=to, workspace=space)), want, size, group, cols, to, array(bias))
