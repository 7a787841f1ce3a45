"""Cross entropy's gradients where the digits are at stake: targets whose probability is almost one, by scales that are no power of two and scores that are
not exact."""
import pytest
import torch

from loss_bounds import relative
from training_util import close

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
