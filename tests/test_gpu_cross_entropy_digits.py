"""Cross entropy's gradients where the digits are at stake: targets whose probability is almost one, by scales that are no power of two and scores that are
not exact; in fp16, rows whose gradients of the loss are far apart; scores whose size leaves their differences few digits."""
import pytest
import torch

from loss_bounds import relative
from training_util import close, half_step

pytestmark = pytest.mark.gpu
DEV, BF, HALF = torch.device("cuda", 0), torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl
    pl.load_library()
    return pl


def _gradients(pl, h, w, t, d, scale):
    loss, lse = pl.plaid_cross_entropy(h, w, t, scale=scale, return_lse=True)
    return (loss,) + pl.plaid_cross_entropy_backward(d, h, w, t, lse, scale=scale)


def _check(pl, h, w, t, d, scale):
    want, got = relative(h, w, t, scale, d), _gradients(pl, h, w, t, d, scale)
    for x, name in zip(got, ("loss", "d_hidden", "d_weight")):
        close(x, want[name], want[name + "_bound"], name)
    return want, got


# a row, few rows of both tiles, more rows by small tiles, large tiles, more rows than one launch prepares
SHAPES = [(1, 900, 264), (30, 900, 264), (64, 50_001, 264), (300, 3000, 264), (700, 15_000, 264), (2050, 15_000, 264)]


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("scale", [1.1, 1.3, -1.3, 264 ** -0.5, 768 ** -0.5])
@pytest.mark.parametrize("rows,vocabulary,width", SHAPES)
def test_targets_near_one(pl, rows, vocabulary, width, scale, dtype):
    """States that point at their target: its score is 18 to 32, the others' are 1 to 2 about zero, and 1 - p is 1e-4 to 1e-10.  A score's rounding, 2^-20,
    is far more than that."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    w = torch.randn(vocabulary, width, generator=g, device=DEV).to(dtype)
    t = torch.randint(0, vocabulary, (rows,), generator=g, device=DEV)
    score = 18 + 14 * torch.rand(rows, 1, generator=g, device=DEV)
    h = (score / (scale * width) * w[t].float()).to(dtype)
    _check(pl, h, w, t, torch.full((rows,), 2.0 ** 20, device=DEV), scale)


def _pointed(rows, vocabulary, width, dtype, seed):
    """States that point at another entry than their target, with a score of about 40, so that a target's row of d_weight is its own rows' alone."""
    g = torch.Generator(device=DEV).manual_seed(seed)
    w = torch.randn(vocabulary, width, generator=g, device=DEV).to(dtype)
    h = 40 * width ** -0.5 * w[:1].float() + torch.randn(rows, width, generator=g, device=DEV)
    return h.to(dtype), w, torch.arange(rows, device=DEV) % (vocabulary - 1) + 1


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("rows,vocabulary,width", [(29, 900, 264), (300, 3000, 136), (700, 15_000, 136), (2050, 3000, 72)])
def test_rows_whose_gradients_are_far_apart(pl, rows, vocabulary, width, dtype):
    """2^-28 between the largest and the smallest: each target's row of d_weight has the digits that its own row's states have."""
    h, w, t = _pointed(rows, vocabulary, width, dtype, rows)
    d = torch.exp2(13 - torch.arange(rows, device=DEV) % 29.0) * (1 if rows < 100 else 29 / rows)
    want, (_, _, dw) = _check(pl, h, w, t, d, width ** -0.5)
    mine = want["d_weight"][t]
    normal = mine.abs() > 2.0 ** -14
    # the result's rounding, the states' (2^-25 of what is 2^-28 + 11 or more: less than another), and r
    assert ((dw[t].double() - mine).abs() <= 2.5 * half_step(dtype) * mine.abs())[normal].all()
    assert normal.any(1).sum() > 0.6 * rows


@pytest.mark.parametrize("rows,vocabulary,width", [(30, 900, 72), (700, 15_000, 72)])
def test_a_row_of_zeros_and_rows_without_a_target_scale_nothing(pl, rows, vocabulary, width):
    """Neither a row whose states are zero nor one that takes no part says by what power of two the others' states are scaled."""
    h, w, t = _pointed(rows, vocabulary, width, HALF, rows)
    d = torch.ones(rows, device=DEV)
    h[3] = 0.0
    d[3] = 0.0
    t[5] = -1
    want = _gradients(pl, h, w, t, d, width ** -0.5)
    d[3], d[5] = 1e30, 1e30
    h[5] = 65504.0
    got = _gradients(pl, h, w, t, d, width ** -0.5)
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    keep = torch.arange(rows, device=DEV) != 3
    assert torch.equal(got[1][keep], want[1][keep])


@pytest.mark.parametrize("rows,vocabulary,width", [(30, 900, 72), (700, 15_000, 72)])
@pytest.mark.parametrize("size", [2.0 ** -20, 3e4])
def test_states_at_the_ends_of_fp16(pl, rows, vocabulary, width, size):
    """Subnormal states, and states next to the largest number of fp16."""
    h, w, t = _pointed(rows, vocabulary, width, HALF, rows)
    h = (h.float() / h.float().abs().amax() * size * 2).to(HALF)
    d = torch.exp2(-(torch.arange(rows, device=DEV) % 5.0))
    scale = 1e-4 if size > 1 else 1.0
    _check(pl, h, w, t, d * (2.0 ** 12 if size < 1 else 2.0 ** -4), scale)


@pytest.mark.parametrize("rows,vocabulary,width", [(30, 900, 72), (2050, 3000, 72)])
def test_captured_and_replayed(pl, rows, vocabulary, width):
    h, w, t = _pointed(rows, vocabulary, width, HALF, 0)
    scale, d = width ** -0.5, torch.ones(rows, device=DEV)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        _gradients(pl, h, w, t, d, scale)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = _gradients(pl, h, w, t, d, scale)
    for seed in (1, 2, 3):
        h.copy_(_pointed(rows, vocabulary, width, HALF, seed)[0] * seed)
        d.copy_(torch.exp2(-(torch.arange(rows, device=DEV) * seed % 20.0)))
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, _gradients(pl, h, w, t, d, scale)))


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("sign", [1, -1])
@pytest.mark.parametrize("rows,vocabulary", [(20, 900), (64, 50_001), (300, 3000), (700, 15_000)])
def test_scores_far_from_zero(pl, rows, vocabulary, sign, dtype):
    """All scores are 2^20 (or that less than zero) and a number of eighths below eight: each is exact, and so are their differences."""
    g = torch.Generator(device=DEV).manual_seed(rows)
    w = torch.zeros(vocabulary, 64, device=DEV)
    w[:, 0], w[:, 1] = 1024.0, torch.randint(0, 64, (vocabulary,), generator=g, device=DEV) / 8
    h = torch.zeros(rows, 64, device=DEV)
    h[:, 0], h[:, 1] = 1024.0 * sign, 1.0
    t = torch.randint(0, vocabulary, (rows,), generator=g, device=DEV)
    for scale in (1.0, 0.5):
        h, w, d = h.to(dtype), w.to(dtype), torch.rand(rows, generator=g, device=DEV) + 0.5
        want, got = relative(h, w, t, scale, d, exact=True), _gradients(pl, h, w, t, d, scale)
        for x, name in zip(got, ("loss", "d_hidden", "d_weight")):
            close(x, want[name], want[name + "_bound"], name)
