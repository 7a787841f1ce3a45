"""Calls that autograd does not record say so, and stand where a torch.autograd.Function makes them."""
import pytest
import torch

from test_gpu_reader_attention import BF, DEV, _off, pl  # noqa: F401 (pl is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", ["q", "k", "v", "key_bias"])
def test_inputs_that_require_a_gradient_are_refused(pl, which):  # noqa: F811
    g = torch.Generator().manual_seed(1)
    x = {n: torch.randn(s, generator=g).to(BF).to(DEV) for n, s in (("q", (5, 4, 64)), ("k", (40, 2, 64)), ("v", (40, 2, 64)), ("key_bias", (40,)))}
    offsets = dict(q_offsets=_off([5]), k_offsets=_off([40]))
    want = pl.plaid_cross_attention(**x, **offsets)
    x[which].requires_grad_()
    with pytest.raises(ValueError, match=which + " requires a gradient"):
        pl.plaid_cross_attention(**x, **offsets)
    with torch.no_grad():
        assert torch.equal(pl.plaid_cross_attention(**x, **offsets), want)

    class Recorded(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, bias):
            out, lse = pl.plaid_cross_attention(q, k, v, key_bias=bias, return_lse=True, **offsets)
            ctx.save_for_backward(q, k, v, bias, out, lse)
            return out

        @staticmethod
        def backward(ctx, d_out):
            q, k, v, bias, out, lse = ctx.saved_tensors
            return pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, key_bias=bias, **offsets)

    out = Recorded.apply(x["q"], x["k"], x["v"], x["key_bias"])
    assert torch.equal(out, want)
    out.float().sum().backward()
    assert x[which].grad is not None and torch.isfinite(x[which].grad).all()
