"""Dropout from a counter-based generator: the mask bit for bit, the values, and that both directions have one mask."""
import pytest
import torch

from training_util import E, TINY, close, half_step, kept

pytestmark = pytest.mark.gpu
DEV, BF, HALF = torch.device("cuda", 0), torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl
    pl.load_library()
    return pl


def _rng(seed, call):
    return torch.tensor([seed, call], device=DEV)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("shape", [(1,), (7,), (8,), (9,), (3, 5, 11), (64, 63), (41, 100)])
@pytest.mark.parametrize("p", [0.0, 0.1, 0.5, 0.99999, 1.0])
def test_mask_and_values(pl, shape, dtype, p):
    x, residual = torch.randn(*shape, device=DEV).to(dtype), torch.randn(*shape, device=DEV).to(dtype)
    for seed, call in ((0, 0), (-3, 2 ** 40 + 5), (2 ** 63 - 1, -1)):
        mask, factor = kept(0, x.numel(), p, seed, call)
        mask = mask.view(shape).to(DEV)
        want = torch.where(mask, x.double() * factor, 0.0)
        u, tiny = half_step(dtype), TINY[dtype]
        close(pl.plaid_dropout(x, p, _rng(seed, call)), want, (u + 4 * E) * want.abs() + tiny, "without residual")
        both = want + residual.double()
        close(pl.plaid_dropout(x, p, _rng(seed, call), residual=residual), both, u * both.abs() + 4 * E * (want.abs() + residual.double().abs()) + tiny, "with residual")


def test_what_is_dropped_leaves_no_trace(pl):
    x = torch.tensor([float("inf"), float("nan"), -float("inf")], device=DEV).to(BF).repeat(500)
    mask = kept(0, 1500, 0.5, 11, 12)[0].to(DEV)
    out = pl.plaid_dropout(x, 0.5, _rng(11, 12))
    assert (out[~mask] == 0).all() and torch.equal(torch.isnan(out[mask]), torch.isnan(x[mask])) and not torch.isfinite(out[mask]).any()
    assert not pl.plaid_dropout(x, 1.0, _rng(11, 12)).any()
    residual = torch.randn(1500, device=DEV).to(BF)
    assert torch.equal(pl.plaid_dropout(x, 0.5, _rng(11, 12), residual=residual)[~mask], residual[~mask])


def test_both_directions_share_the_mask(pl):
    """out is linear in x: the gradient of sum(out c) is dropout of c, by differences of single elements too."""
    x, c = torch.randn(300, device=DEV).to(HALF), torch.randn(300, device=DEV).to(HALF)
    grad = pl.plaid_dropout(c, 0.3, _rng(5, 6))
    base = pl.plaid_dropout(x, 0.3, _rng(5, 6))
    assert torch.equal(grad == 0, base == 0)
    for i in (0, 7, 8, 150, 299):
        y = x.clone()
        y[i] += 1
        slope = (pl.plaid_dropout(y, 0.3, _rng(5, 6)).double() - base.double()) @ c.double()
        # two results and the changed input, each off by half a step of at most 8, times c; and grad's own rounding
        assert abs(float(slope - grad[i])) <= 3 * half_step(HALF) * 8 * abs(float(c[i])) * 1.5 + half_step(HALF) * abs(float(grad[i]))


def test_share_of_what_is_kept_and_unlike_calls(pl):
    n = 1 << 20
    x = torch.ones(n, device=DEV, dtype=BF)
    a, b, c = (pl.plaid_dropout(x, 0.1, _rng(*s)) != 0 for s in ((1, 1), (1, 2), (2, 1)))
    for m in (a, b, c):
        assert abs(int(m.sum()) / n - 0.9) < 6 * (0.09 / n) ** 0.5 + 2.0 ** -17
    for m in (b, c):  # independent masks agree on 0.82 of the places
        assert abs(int((a == m).sum()) / n - 0.82) < 6 * (0.82 * 0.18 / n) ** 0.5 + 2.0 ** -15


def test_elements_beyond_32_bits(pl):
    n = 2 ** 32 + 8 * 3 + 5
    x = torch.ones(n, device=DEV, dtype=BF)
    out = pl.plaid_dropout(x, 0.5, _rng(77, 78))
    for first in (0, 2 ** 31 - 24, 2 ** 32 - 24, n - 29):
        mask, factor = kept(first, 29, 0.5, 77, 78)
        assert torch.equal(out[first:first + 29].double().cpu(), mask * factor), first


def test_in_place_shapes_and_views(pl):
    x = torch.randn(30, 40, device=DEV).to(BF)
    want = pl.plaid_dropout(x.T.contiguous(), 0.2, _rng(3, 4))
    assert torch.equal(pl.plaid_dropout(x.T, 0.2, _rng(3, 4)), want)
    flat = torch.randn(1001, device=DEV).to(BF)
    odd = flat[1:]  # not 16-byte aligned
    assert torch.equal(pl.plaid_dropout(odd, 0.2, _rng(3, 4)), pl.plaid_dropout(odd.clone(), 0.2, _rng(3, 4)))
    assert pl.plaid_dropout(x[:0], 0.2, _rng(3, 4)).shape == (0, 40)
    two = torch.tensor([[3, 9], [4, 9]], device=DEV)[:, 0]  # rng with a stride
    assert torch.equal(pl.plaid_dropout(x.T, 0.2, two), want)


def test_a_captured_graph_draws_new_masks(pl):
    x, rng = torch.randn(64, 256, device=DEV).to(BF), _rng(9, 0)
    stream = torch.cuda.Stream()
    with torch.cuda.stream(stream):
        pl.plaid_dropout(x, 0.4, rng)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = pl.plaid_dropout(x, 0.4, rng, residual=x)
        grad = pl.plaid_dropout(out, 0.4, rng)
        rng[1] += 1
    rng.copy_(_rng(9, 0))
    seen = []
    for call in range(4):
        graph.replay()
        torch.cuda.synchronize()
        want = pl.plaid_dropout(x, 0.4, _rng(9, call), residual=x)
        assert torch.equal(out, want) and torch.equal(grad, pl.plaid_dropout(want, 0.4, _rng(9, call)))
        seen.append(out.clone())
    assert not torch.equal(seen[0], seen[1])


def test_refusals(pl):
    x = torch.randn(4, 4, device=DEV).to(BF)
    for bad in (dict(rng=_rng(1, 2).int()), dict(rng=torch.zeros(3, dtype=torch.int64, device=DEV)), dict(residual=x.half()), dict(residual=x[:2]), dict(x=x.float())):
        with pytest.raises(ValueError):
            pl.plaid_dropout(**{**dict(x=x, p=0.1, rng=_rng(1, 2)), **bad})
    for p in (-0.1, 1.5, float("nan")):
        with pytest.raises(pl.PlaidError):
            pl.plaid_dropout(x, p, _rng(1, 2))
    x.requires_grad_()
    with pytest.raises(ValueError, match="x requires a gradient"):
        pl.plaid_dropout(x, 0.1, _rng(1, 2))


def test_more_threads_than_one_axis_of_a_grid_has(pl):
    """2^32 groups of eight elements and some more: the counter's second word is used too."""
    n = 2 ** 35 + 2048 + 5
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info()[0] < 5 * n:
        pytest.skip("the arrays do not fit beside what else the card holds")
    x = torch.ones(n, device=DEV, dtype=BF)
    out = pl.plaid_dropout(x, 0.5, _rng(5, 6))
    del x
    for first in (0, 2 ** 34, 2 ** 35 - 2048 - 16, 2 ** 35 - 16, n - 37):
        first = first // 8 * 8
        mask, factor = kept(first, 29, 0.5, 5, 6)
        assert torch.equal(out[first:first + 29].double().cpu(), mask * factor), first
