"""Every form of a training step's kernels: that the shapes here get the form that they are here for, as the profiler names it, and that it is
right there."""
import pytest
import torch

from test_gpu_cross_entropy import BF, DEV, HALF, _check as check_loss, _inputs as loss_inputs, pl  # noqa: F401 (pl is a fixture)
from test_gpu_embedding import _inputs as embed_inputs
from test_gpu_layer_norm import _check as check_norm, _inputs as norm_inputs
from training_util import close, embed, embed_bound, embed_grad

pytestmark = pytest.mark.gpu


def _kernels(f):
    """Names of the kernels that f launches, without their arguments."""
    from torch.profiler import ProfilerActivity, profile
    with profile(activities=[ProfilerActivity.CUDA, ProfilerActivity.CPU]) as p:
        f()
        torch.cuda.synchronize()
    names = {e.key.split("(")[0] for e in p.key_averages()}
    if not any("_kernel" in n for n in names):
        pytest.skip("no kernels from torch's profiler here")
    return names


# rows, vocabulary, width -> kernel of the scores (bf16) forward, backward
SCORES = {
    "16 rows, 64 entries": (9, 500, 72, "loss_few_kernel<0, 4, 1, 1, false>", "loss_few_kernel<0, 4, 1, 4, true>"),
    "32 rows, 64 entries": (30, 500, 72, "loss_few_kernel<0, 4, 1, 2, false>", "loss_few_kernel<0, 4, 1, 4, true>"),
    "48 rows, 64 entries": (40, 500, 72, "loss_few_kernel<0, 4, 1, 3, false>", "loss_few_kernel<0, 4, 1, 4, true>"),
    "64 rows, 64 entries": (64, 500, 72, "loss_few_kernel<0, 4, 1, 4, false>", "loss_few_kernel<0, 4, 1, 4, true>"),
    "96 rows, 64 entries": (90, 500, 72, "loss_few_kernel<0, 4, 1, 6, false>", "loss_few_kernel<0, 4, 1, 8, true>"),
    "128 rows, 64 entries": (100, 500, 72, "loss_few_kernel<0, 4, 1, 8, false>", "loss_few_kernel<0, 4, 1, 8, true>"),
    "16 rows, 128 entries": (9, 90_001, 72, "loss_few_kernel<0, 4, 2, 1, false>", "loss_few_kernel<0, 4, 2, 4, true>"),
    "32 rows, 128 entries": (30, 70_001, 72, "loss_few_kernel<0, 4, 2, 2, false>", "loss_few_kernel<0, 4, 2, 4, true>"),
    "48 rows, 128 entries": (40, 50_001, 72, "loss_few_kernel<0, 4, 2, 3, false>", "loss_few_kernel<0, 4, 2, 4, true>"),
    "64 rows, 128 entries": (64, 50_001, 72, "loss_few_kernel<0, 4, 2, 4, false>", "loss_few_kernel<0, 4, 2, 4, true>"),
    "96 rows, 256 entries": (90, 40_001, 72, "loss_few_kernel<0, 8, 2, 6, false>", "loss_few_kernel<0, 8, 2, 8, true>"),
    "128 rows, 256 entries": (128, 40_001, 72, "loss_few_kernel<0, 8, 2, 8, false>", "loss_few_kernel<0, 8, 2, 8, true>"),
    "more rows, 64 entries": (300, 3000, 72, "loss_few_kernel<0, 4, 1, 8, false>", "loss_few_kernel<0, 4, 1, 8, true>"),
    "more rows, 256 entries": (500, 12_000, 72, "loss_few_kernel<0, 8, 2, 8, false>", "loss_few_kernel<0, 8, 2, 8, true>"),
    "large tiles": (700, 15_000, 72, "loss_mm_kernel<0, 0>", "loss_mm_kernel<0, 1>"),
    "wide rows begin at different columns": (60, 3000, 2056, "loss_few_kernel<0, 4, 1, 4, false>", "loss_few_kernel<0, 4, 1, 4, true>"),
    "large tiles, one step": (700, 15_000, 64, "loss_mm_kernel<0, 0>", "loss_mm_kernel<0, 1>"),
    "large tiles, three steps": (700, 15_000, 192, "loss_mm_kernel<0, 0>", "loss_mm_kernel<0, 1>"),
    "large tiles, four steps": (700, 15_000, 200, "loss_mm_kernel<0, 0>", "loss_mm_kernel<0, 1>"),
    "large tiles, six steps": (700, 15_000, 360, "loss_mm_kernel<0, 0>", "loss_mm_kernel<0, 1>"),
}


@pytest.mark.parametrize("name", SCORES)
def test_scores(pl, name):  # noqa: F811
    rows, vocabulary, width, forward, backward = SCORES[name]
    h, w, t, d = loss_inputs(rows, vocabulary, width, BF, seed=rows)
    check_loss(pl, h, w, t, d, width ** -0.5, name)
    lse = pl.plaid_cross_entropy(h, w, t, scale=width ** -0.5, return_lse=True)[1]
    assert any(forward in n for n in _kernels(lambda: pl.plaid_cross_entropy(h, w, t, scale=width ** -0.5)))
    assert any(backward in n for n in _kernels(lambda: pl.plaid_cross_entropy_backward(d, h, w, t, lse, scale=width ** -0.5)))
    h, w, t, d = loss_inputs(rows, vocabulary, width, HALF, seed=rows)
    check_loss(pl, h, w, t, d, width ** -0.5, name + " fp16")


@pytest.mark.parametrize("rows,vocabulary,width", [
    (64, 700, 64), (200, 700, 64),     # one and four steps of d_weight, eleven of d_hidden, whole
    (300, 30_000, 64),                 # d_hidden in parts, d_weight whole
    (3000, 700, 64), (5000, 300, 264),  # d_weight in parts
    (4000, 6000, 520),                 # both
])
def test_parts_of_the_gradients(pl, rows, vocabulary, width):  # noqa: F811
    h, w, t, d = loss_inputs(rows, vocabulary, width, BF, seed=rows)
    check_loss(pl, h, w, t, d, width ** -0.5, "parts")


# width, rows -> forward, backward
NORMS = [(5, 300, "1, 1", "1, 1"), (60, 300, "8, 1", "8, 1"), (120, 300, "16, 1", "16, 1"), (250, 300, "32, 1", "32, 1"), (500, 300, "64, 1", "64, 1"), (1000, 300, "64, 2", "64, 2"),
         (1500, 300, "256, 1", "64, 3"), (1500, 2500, "64, 3", "64, 3"), (2000, 300, "256, 1", "256, 1"), (2000, 2500, "64, 4", "256, 1"), (2500, 2500, "64, 5", "256, 2"),
         (2900, 2500, "64, 6", "256, 2"), (2500, 300, "256, 2", "256, 2"), (4000, 2500, "256, 2", "256, 2"), (6000, 300, "256, 4", "256, 4"), (9000, 300, "1024, 2", "1024, 2")]


@pytest.mark.parametrize("width,rows,forward,backward", NORMS)
def test_layer_norm(pl, width, rows, forward, backward):  # noqa: F811
    x, w, b, d = norm_inputs(rows, width, BF, seed=width)
    check_norm(pl, x, w, b, d, 1e-5, str(width))
    statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)[1]
    assert any(f"norm_kernel<0, {forward}>" in n for n in _kernels(lambda: pl.plaid_layer_norm(x, w, b)))
    assert any(f"norm_grad_kernel<0, {backward}>" in n for n in _kernels(lambda: pl.plaid_layer_norm_backward(d, x, w, b, statistics)))


@pytest.mark.parametrize("n,vocabulary,width,forward,backward", [
    (300, 500, 40, "embed_kernel<0, 1>", ("sort_one_kernel", "embed_grad_kernel<0, false>", "embed_grad_join_kernel")),
    (300, 500, 600, "embed_kernel<0, 1>", ("sort_one_kernel", "embed_grad_kernel<0, true>")),
    (9000, 500, 1030, "embed_kernel<0, 4>", ("sort_count_kernel", "sort_scan_kernel", "sort_place_kernel", "embed_grad_kernel<0, true>", "embed_grad_join_kernel")),
    (9000, 300_000, 8, "embed_kernel<0, 1>", ("sort_place_kernel", "embed_grad_kernel<0, false>")),
])
def test_embedding(pl, n, vocabulary, width, forward, backward):  # noqa: F811
    table, ids, d = embed_inputs(n, vocabulary, width, BF, seed=n, frequent=0.2)
    want = embed(table, ids, 2.0)
    close(pl.plaid_embedding(table, ids, scale=2.0), want, embed_bound(want, BF), "rows")
    close(pl.plaid_embedding_backward(d, ids, vocabulary), *embed_grad(d, ids, vocabulary, 1.0), "gradient")
    assert any(forward in k for k in _kernels(lambda: pl.plaid_embedding(table, ids)))
    names = _kernels(lambda: pl.plaid_embedding_backward(d, ids, vocabulary))
    for kernel in backward:
        assert any(kernel in k for k in names), kernel
