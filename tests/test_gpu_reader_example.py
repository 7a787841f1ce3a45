"""The example of a reader: it trains, gives the scores a gradient, and answers token by token as it does all at once."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "reader.py")
    spec = importlib.util.spec_from_file_location("reader_example", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_example_trains_and_answers(example):
    losses, grad, out, last, answers = example.main(steps=6)
    assert losses[-1] < losses[0]
    assert torch.isfinite(grad).all() and float(grad.abs().max()) > 0
    assert torch.isfinite(out).all() and torch.isfinite(last).all()
    assert answers.lengths.tolist() == [24 - 3 * r + 4 for r in range(6)]


def test_token_by_token_and_at_once(example):
    """The same tokens one at a time and all at once read the same cache: what differs is the order of sums and which kernel forms
    them, so two results are a few roundings to bfloat16 apart (each at most 2^-8 of the layer's values, which are below 8)."""
    torch.manual_seed(1)
    device = torch.device("cuda", 0)
    layer, n, m = example.Layer(device), 3, 21
    keys, values = (torch.randn(100, example.KV_HEADS, example.DIM, device=device, dtype=example.DTYPE) for _ in range(2))
    bias, k_offsets = torch.randn(100, device=device, dtype=example.DTYPE), torch.tensor([0, 40, 41, 100], device=device)
    x = torch.randn(n, m, example.WIDTH, device=device, dtype=example.DTYPE)
    with torch.no_grad():
        whole = layer.answer(x.view(n * m, -1), example.Answers(n, 32, 16, device), torch.full((n,), m, dtype=torch.int32, device=device),
                             keys, values, bias, k_offsets).view(n, m, -1)
        answers, one = example.Answers(n, 32, 16, device), torch.ones(n, dtype=torch.int32, device=device)
        for t in range(m):
            y = layer.answer(x[:, t].contiguous(), answers, one, keys, values, bias, k_offsets)
            assert float((y.float() - whole[:, t].float()).abs().max()) <= 4 * 8 * 2.0 ** -8
