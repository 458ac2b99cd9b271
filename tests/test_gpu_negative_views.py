"""Tensors whose memory holds the negatives of their elements: no call takes their address as if it did not."""
import pytest
import torch

from paper_1511_04561_amd import dq8

pytestmark = pytest.mark.gpu
I32, I64 = torch.int32, torch.int64


def negative(t):
    """t with its elements' negatives in memory."""
    v = torch._neg_view(t.neg().contiguous())
    assert v.is_neg() and torch.equal(v, t) and v.stride() == t.stride()
    return v


def refused(call):
    with pytest.raises(ValueError, match="resolve_neg"):
        call()


def test_an_imaginary_part():
    z = torch.complex(torch.zeros(20, 1), torch.ones(20, 1)).cuda()
    w = z.conj().imag
    assert w.is_neg() and (w == -1).all()
    refused(lambda: dq8.weights_encode(w))
    codes, scales = dq8.weights_encode(w.resolve_neg())
    assert (dq8.weights_decode(codes, scales, 20, 1) < 0).all()


@pytest.mark.parametrize("bound", [True, False])
def test_negative_views_are_refused(bound, monkeypatch):
    if not bound:
        monkeypatch.setattr(dq8, "_native", dq8._Unbound())
    x, w = torch.randn(512, device="cuda"), torch.randn(32, 128, device="cuda")
    h = torch.randn(3, 128, device="cuda").bfloat16()
    codes, scales = dq8.encode(0, x)
    wc, ws = dq8.weights_encode(w)
    p, ids, u, r = torch.rand(4, 50, device="cuda"), torch.ones(4, dtype=I64, device="cuda"), torch.rand(4, device="cuda"), torch.rand(2, device="cuda")
    kc, ks = dq8.cache_buffers(4, 2, 16, 64)
    k = torch.randn(5, 2, 64, device="cuda").bfloat16()
    slots, pages, lens = torch.arange(5, device="cuda"), torch.ones(1, 4, dtype=I32, device="cuda"), torch.full((1,), 5, dtype=I32, device="cuda")
    calls = [
        lambda n: dq8.absmax(n(x)), lambda n: dq8.encode(0, n(x)), lambda n: dq8.decode(0, codes, n(scales)), lambda n: dq8.decode(0, codes, scales, out=n(x.clone())),
        lambda n: dq8.error_stats(0, n(x)), lambda n: dq8.decode_accumulate_avg(0, [codes], [n(scales)]), lambda n: dq8.decode_accumulate_avg(0, [codes], [scales], local=n(x)),
        lambda n: dq8.decode_avg_encode(0, [codes], [n(scales)]), lambda n: dq8.absmax_segments(n(x), [0, 512]),
        lambda n: dq8.weights_encode(n(w)), lambda n: dq8.weights_encode(w, scales=n(ws.clone())), lambda n: dq8.weights_decode(wc, n(ws)),
        lambda n: dq8.weights_decode(wc, ws, out=n(w.clone())), lambda n: dq8.weights_product(n(h), wc, ws), lambda n: dq8.weights_product(h, wc, ws, bias=n(torch.ones(32, device="cuda"))),
        lambda n: dq8.weights_product(h, wc, ws, out=n(torch.zeros(3, 32, device="cuda"))), lambda n: dq8.weights_product_workspace(n(h), wc, ws),
        lambda n: dq8.draft_verify(n(p), ids, u, r), lambda n: dq8.draft_verify(p, n(ids), u, r), lambda n: dq8.draft_verify(p, ids, n(u), r),
        lambda n: dq8.draft_verify(p, ids, u, n(r)), lambda n: dq8.draft_verify(p, ids, u, r, draft=n(p)), lambda n: dq8.draft_verify(p, ids, u, r, out=n(ids.clone())),
        lambda n: dq8.cache_plan(n(lens), lens, pages, pages[0], lens.clone(), 16, 5), lambda n: dq8.cache_plan(lens, lens, pages, pages[0], lens.clone(), 16, 5, drop=n(lens)),
        lambda n: dq8.cache_append(0, n(k), k, slots, kc, ks), lambda n: dq8.cache_append(0, k, n(k), slots, kc, ks), lambda n: dq8.cache_append(0, k, k, n(slots), kc, ks),
        lambda n: dq8.cache_append(0, k, k, slots, kc, ks, q=n(k)), lambda n: dq8.cache_append(0, k, k, slots, kc, ks, q=k, q_weight=n(torch.ones(64, device="cuda"))),
        lambda n: dq8.cache_attention(0, n(k), kc, ks, pages, lens), lambda n: dq8.cache_attention(0, k, kc, n(ks), pages, lens),
        lambda n: dq8.cache_attention(0, k, kc, ks, pages, lens, out=n(k.clone())), lambda n: dq8.cache_attention(0, k, kc, ks, n(pages), lens),
    ]
    for i, call in enumerate(calls):
        refused(lambda: call(negative))
