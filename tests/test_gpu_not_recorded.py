"""What autograd would lose without a word is refused: the calls carry no forward-mode tangents, and the gradients' calls record nothing of what the
forward ones gave either."""
import pytest
import torch
from torch.autograd import forward_ad

pytestmark = pytest.mark.gpu
DEV, BF = torch.device("cuda", 0), torch.bfloat16


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl
    pl.load_library()
    return pl


def _calls(pl):
    """name -> (call of a dict of its tensors, that dict, names of those that could be differentiated)"""
    g = torch.Generator(device=DEV).manual_seed(5)
    new = lambda *shape: torch.randn(*shape, generator=g, device=DEV).to(BF)  # noqa: E731
    ids, rng = torch.arange(6, device=DEV), torch.tensor([1, 2], device=DEV)
    offsets = torch.tensor([0, 6], device=DEV)
    x, w, b, table = new(6, 64), new(64), new(64), new(40, 64)
    with torch.no_grad():
        statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)[1]
        lse = pl.plaid_cross_entropy(x, table, ids, return_lse=True)[1]
    return {
        "embedding": (lambda a: pl.plaid_embedding(a["table"], ids), {"table": table}),
        "embedding_backward": (lambda a: pl.plaid_embedding_backward(a["d_out"], ids, 40, add_to=a["add_to"]), {"d_out": x, "add_to": table.clone()}),
        "dropout": (lambda a: pl.plaid_dropout(a["x"], 0.1, rng, residual=a["residual"]), {"x": x, "residual": new(6, 64)}),
        "layer_norm": (lambda a: pl.plaid_layer_norm(a["x"], a["weight"], a["bias"]), {"x": x, "weight": w, "bias": b}),
        "layer_norm_backward": (lambda a: pl.plaid_layer_norm_backward(a["d_out"], a["x"], a["weight"], a["bias"], a["statistics"]),
                                {"d_out": new(6, 64), "x": x, "weight": w, "bias": b, "statistics": statistics}),
        "cross_entropy": (lambda a: pl.plaid_cross_entropy(a["hidden"], a["weight"], ids), {"hidden": x, "weight": table}),
        "cross_entropy_backward": (lambda a: pl.plaid_cross_entropy_backward(a["d_loss"], a["hidden"], a["weight"], ids, a["lse"]),
                                   {"d_loss": torch.ones(6, device=DEV), "hidden": x, "weight": table, "lse": lse}),
        "cross_attention": (lambda a: pl.plaid_cross_attention(a["q"], a["k"], a["v"], offsets, offsets, key_bias=a["key_bias"]),
                            {"q": new(6, 2, 64), "k": new(6, 2, 64), "v": new(6, 2, 64), "key_bias": new(6)}),
    }


NAMES = ["embedding", "embedding_backward", "dropout", "layer_norm", "layer_norm_backward", "cross_entropy", "cross_entropy_backward", "cross_attention"]


@pytest.mark.parametrize("name", NAMES)
def test_forward_mode_tangents_are_refused(pl, name):
    call, tensors = _calls(pl)[name]
    with forward_ad.dual_level():
        call(tensors)  # none has a tangent
        for which, t in tensors.items():
            dual = dict(tensors, **{which: forward_ad.make_dual(t, torch.ones_like(t))})
            for grad in (True, False):
                with torch.set_grad_enabled(grad), pytest.raises(ValueError, match=f"{which} has a forward-mode tangent"):
                    call(dual)
    call(tensors)


@pytest.mark.parametrize("name,which", [("layer_norm_backward", "statistics"), ("cross_entropy_backward", "lse")])
def test_gradients_of_what_the_forward_call_gave_are_refused(pl, name, which):
    call, tensors = _calls(pl)[name]
    tensors = dict(tensors, **{which: tensors[which].clone().requires_grad_()})
    with pytest.raises(ValueError, match=f"{which} requires a gradient"):
        call(tensors)
    with torch.no_grad():
        call(tensors)
