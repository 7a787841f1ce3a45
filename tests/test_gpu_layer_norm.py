"""Layer norm and its gradients against the definitions in 64 bits, and against differences."""
import pytest
import torch

from training_util import close, norm

pytestmark = pytest.mark.gpu
DEV, BF, HALF = torch.device("cuda", 0), torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl
    pl.load_library()
    return pl


def _inputs(rows, width, dtype, seed=0, mean=0.3, spread=1.0):
    g = torch.Generator(device=DEV).manual_seed(seed)
    x = torch.randn(rows, width, generator=g, device=DEV) * spread * torch.exp(0.7 * torch.randn(width, generator=g, device=DEV)) + mean
    return (x.to(dtype), (1 + 0.2 * torch.randn(width, generator=g, device=DEV)).to(dtype), (0.1 * torch.randn(width, generator=g, device=DEV)).to(dtype),
            torch.randn(rows, width, generator=g, device=DEV).to(dtype))


def _check(pl, x, weight, bias, d, eps, what):
    want = norm(x, weight, bias, eps, d)
    out, statistics = pl.plaid_layer_norm(x, weight, bias, eps=eps, return_statistics=True)
    close(out, want["out"], want["out_bound"], what + " out")
    close(statistics[:, 0], want["mean"], want["mean_bound"], what + " mean")
    close(statistics[:, 1], want["inverse"], want["inverse_bound"], what + " inverse")
    got = pl.plaid_layer_norm_backward(d, x, weight, bias, statistics)
    for name, value, there in (("dx", got[0], True), ("dweight", got[1], weight is not None), ("dbias", got[2], bias is not None)):
        assert (value is not None) == there
        if there:
            close(value, want[name], want[name + "_bound"], f"{what} {name}")
    again = pl.plaid_layer_norm_backward(d, x, weight, bias, statistics)
    assert all(a is None or torch.equal(a, b) for a, b in zip(got, again))
    return out


WIDTHS = [1, 2, 7, 8, 9, 64, 65, 128, 130, 200, 256, 257, 511, 512, 520, 765, 1024, 1025, 1500, 1537, 2048, 2056, 4096, 4100, 8192, 8193, 16384]


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("width", WIDTHS)
@pytest.mark.parametrize("rows", [1, 5, 130])
def test_widths(pl, rows, width, dtype):
    x, w, b, d = _inputs(rows, width, dtype, seed=rows + width)
    _check(pl, x, w, b, d, 1e-5, "all")


@pytest.mark.parametrize("rows,width", [(4001, 765), (9000, 64), (70_000, 7), (40_000, 120), (20_000, 250), (6000, 1500), (5000, 1024), (3000, 2048), (2100, 4096), (1300, 9000)])
def test_more_rows_than_workers(pl, rows, width):
    x, w, b, d = _inputs(rows, width, BF, seed=rows)
    _check(pl, x, w, b, d, 1e-5, "all")


@pytest.mark.parametrize("weight", [False, True])
@pytest.mark.parametrize("bias", [False, True])
def test_without_weight_or_bias(pl, weight, bias):
    x, w, b, d = _inputs(50, 200, HALF)
    _check(pl, x, w if weight else None, b if bias else None, d, 1e-3, "some")


def test_far_means_constant_rows_and_small_values(pl):
    x, w, b, d = _inputs(40, 768, HALF, mean=1000.0)  # a variance of differences of large numbers
    x[7] = 3.0
    x[8] = 0.0
    _check(pl, x, w, b, d, 1e-5, "far")
    x, w, b, d = _inputs(40, 768, BF, mean=0.0, spread=1e-12)
    _check(pl, x, w, b, d, 1e-5, "below eps")
    x, w, b, d = _inputs(40, 768, BF, mean=0.0, spread=1e15)
    _check(pl, x, w, b, d, 0.0, "large")


def test_strided_and_misaligned_rows(pl):
    x, w, b, d = _inputs(90, 300, BF)
    wide, other = torch.zeros(90, 401, device=DEV, dtype=BF), torch.zeros(90, 333, device=DEV, dtype=BF)
    wide[:, 1:301], other[:, 3:303] = x, d
    want = _check(pl, x, w, b, d, 1e-5, "contiguous")
    assert torch.equal(_check(pl, wide[:, 1:301], w, b, other[:, 3:303], 1e-5, "views"), want)
    assert torch.equal(_check(pl, x.T.contiguous().T, w, b, d, 1e-5, "transposed"), want)
    one = d[:1].expand(90, 300)  # a gradient that all rows share
    _check(pl, x, w, b, one, 1e-5, "expanded")
    _check(pl, x[::2], w, b, d[::2], 1e-5, "every other row")
    odd = torch.zeros(301, device=DEV, dtype=BF)
    odd[1:] = w
    assert torch.equal(pl.plaid_layer_norm(x, odd[1:], b), want)


def test_a_row_that_is_not_finite_keeps_to_itself(pl):
    x, w, b, d = _inputs(30, 512, BF)
    clean, statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)
    dx = pl.plaid_layer_norm_backward(d, x, w, b, statistics)[0]
    y = x.clone()
    y[3, 100], y[11, 0] = float("inf"), float("nan")
    out, statistics = pl.plaid_layer_norm(y, w, b, return_statistics=True)
    keep = [i for i in range(30) if i not in (3, 11)]
    assert torch.equal(out[keep], clean[keep]) and torch.isnan(out[[3, 11]]).all()
    assert torch.equal(pl.plaid_layer_norm_backward(d, y, w, b, statistics)[0][keep], dx[keep])


def test_no_rows(pl):
    x, w, b, d = _inputs(1, 40, BF)
    out, statistics = pl.plaid_layer_norm(x[:0], w, b, return_statistics=True)
    assert out.shape == (0, 40) and statistics.shape == (0, 2)
    dx, dw, db = pl.plaid_layer_norm_backward(d[:0], x[:0], w, b, statistics)
    assert dx.shape == (0, 40) and not dw.any() and not db.any()


def test_gradients_against_differences(pl):
    """Central differences of the 64-bit formula, which the forward test ties the kernel to, at a few elements."""
    x, w, b, d = _inputs(6, 33, HALF, seed=4)
    _, statistics = pl.plaid_layer_norm(x, w, b, eps=1e-2, return_statistics=True)
    dx, dw, db = pl.plaid_layer_norm_backward(d, x, w, b, statistics)
    want = norm(x, w, b, 1e-2, d)

    def value(x, w, b):
        x = x - x.mean(1, keepdim=True)
        return ((x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-2) * w + b) * d.double()).sum()

    arrays, h = [x.double(), w.double(), b.double()], 1e-5
    for which, got, name in ((0, dx, "dx"), (1, dw, "dweight"), (2, db, "dbias")):
        for at in (0, 5, 32):
            changed = []
            for sign in (1, -1):
                moved = [t.clone() for t in arrays]
                moved[which].view(-1)[at] += sign * h
                changed.append(value(*moved))
            slope = (changed[0] - changed[1]) / (2 * h)  # error h^2 third derivative / 6 and 1e-16 / h: below 1e-7
            assert abs(float(slope) - float(got.view(-1)[at])) <= float(want[name + "_bound"].view(-1)[at]) + 1e-6


def test_refusals(pl):
    x, w, b, d = _inputs(10, 24, BF)
    _, statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)
    for f in (lambda: pl.plaid_layer_norm(x.float(), w, b), lambda: pl.plaid_layer_norm(x, w[:8], b), lambda: pl.plaid_layer_norm(x, w.half(), b),
              lambda: pl.plaid_layer_norm(x[0], w, b), lambda: pl.plaid_layer_norm_backward(d[:5], x, w, b, statistics),
              lambda: pl.plaid_layer_norm_backward(d, x, w, b, statistics[:5]), lambda: pl.plaid_layer_norm_backward(d, x, w, b, statistics.double())):
        with pytest.raises(ValueError):
            f()
    with pytest.raises(pl.PlaidError):
        pl.plaid_layer_norm(x, w, b, eps=-1e-5)
    with pytest.raises(pl.PlaidError):
        pl.plaid_layer_norm(torch.zeros(2, 16385, device=DEV, dtype=BF))
    w.requires_grad_()
    with pytest.raises(ValueError, match="weight requires a gradient"):
        pl.plaid_layer_norm(x, w, b)


def test_rows_beyond_four_gigabytes(pl):
    """The same thousand rows again and again: every thousand of the result is the first, bit for bit, and the first is right."""
    rows, width = 1_100_000, 2048
    few, w, b, d = _inputs(1000, width, BF)
    x = torch.empty(rows, width, dtype=BF, device=DEV)
    x.view(1100, 1000, width)[:] = few
    out, statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)
    want = norm(few, w, b, 1e-5, d)
    close(out[:1000], want["out"], want["out_bound"], "out")
    d = d.expand(1100, 1000, width).reshape(rows, width)
    dx, _, _ = pl.plaid_layer_norm_backward(d, x, w, b, statistics)
    close(dx[:1000], want["dx"], want["dx_bound"], "dx")
    for t in (out, statistics, dx):
        for block in t.view(1100, 1000, -1).split(100):
            assert (block == t[:1000]).all()


def test_more_threads_than_one_axis_of_a_grid_has(pl):
    """One row, expanded: each row of the result is the first, and the first is right."""
    rows, width = 2 ** 29 + 3, 16
    few, w, b, d = _inputs(1, width, BF)
    out = pl.plaid_layer_norm(few.expand(rows, width), w, b)
    want = norm(few, w, b, 1e-5, d)
    close(out[:1], want["out"], want["out_bound"], "out")
    for block in out.split(2 ** 26):
        assert (block == out[:1]).all()


def test_gradients_of_gradients_are_refused(pl):
    x, w, b, d = _inputs(10, 24, BF)
    _, statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)
    for t, name in ((d, "d_out"), (x, "x"), (w, "weight"), (b, "bias")):
        t.requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            pl.plaid_layer_norm_backward(d, x, w, b, statistics)
        with torch.no_grad():
            pl.plaid_layer_norm_backward(d, x, w, b, statistics)
        t.requires_grad_(False)
