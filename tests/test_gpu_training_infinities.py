"""What is not finite in a training step's operators: the right infinity, or no number, where the definition has one, and nothing beside it."""
import pytest
import torch

from training_util import close, embed, embed_bound, embed_grad, kept, norm

pytestmark = pytest.mark.gpu
DEV, BF, HALF = torch.device("cuda", 0), torch.bfloat16, torch.float16
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl
    pl.load_library()
    return pl


def _strict(got, want, bound, what):
    """What is finite within its bound, what is not the same; beyond the type's largest number (by more than the bound) is an infinity, and at that border
    either is right."""
    most = torch.finfo(got.dtype).max
    beyond = torch.isfinite(want) & (want.abs() - bound > most)
    border = torch.isfinite(want) & (want.abs() + bound > most) & ~beyond
    want = torch.where(beyond, torch.copysign(torch.full_like(want, INF), want), want)
    g, out = got.double(), ~torch.isfinite(want)
    assert out.any(), what
    assert ((g == want) | (torch.isnan(g) & torch.isnan(want)))[out].all(), what + ", not finite"
    rest = ~out & ~border
    close(g[rest], want[rest], bound[rest], what)


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("scale", [2.0, -2.0])
@pytest.mark.parametrize("width", [5, 64, 2050])
def test_embedding(pl, width, scale, dtype):
    g = torch.Generator(device=DEV).manual_seed(width)
    table = torch.randn(40, width, generator=g, device=DEV).to(dtype)
    table[3, 0], table[4, -1], table[5, 1], table[6, 2] = INF, -INF, NAN, torch.finfo(dtype).max
    ids = torch.randint(-2, 42, (700,), generator=g, device=DEV)
    want = embed(table, ids, scale)
    _strict(pl.plaid_embedding(table, ids, scale=scale), want, embed_bound(want, dtype), "rows")


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("n,width", [(300, 5), (300, 64), (300, 2050), (9000, 8), (9000, 520)])
def test_embedding_gradient(pl, n, width, dtype):
    """Sums with an infinity, with two opposite ones, and beyond the type's range; the tokens are so frequent that several chunks share them."""
    g = torch.Generator(device=DEV).manual_seed(n)
    ids = torch.randint(-1, 7, (n,), generator=g, device=DEV)
    d = torch.randn(n, width, generator=g, device=DEV).to(dtype)
    first, last = (ids == 2).nonzero()[0], (ids == 2).nonzero()[-1]
    d[first, 0], d[last, 1], d[first, 2], d[last, 2], d[first, 3] = INF, -INF, INF, -INF, NAN
    d[ids == 4, 0], d[ids == 4, 1] = torch.finfo(dtype).max / 8, -torch.finfo(dtype).max / 8
    d[ids < 0] = NAN
    size = embed_grad(d.nan_to_num(0.0, 0.0, 0.0), ids, 7, -0.5)[1]
    want = embed_grad(d, ids, 7, -0.5)[0]
    _strict(pl.plaid_embedding_backward(d, ids, 7, scale=-0.5), want, size, "gradient")
    before = torch.randn(7, width, generator=g, device=DEV).to(dtype)
    before[2, 0], before[2, 1], before[0, 4], before[6, 4] = INF, INF, -INF, NAN
    want = embed_grad(d, ids, 7, -0.5, before)[0]
    size = size + 2.0 ** -7 * before.double().abs().nan_to_num(0.0, 0.0, 0.0)
    _strict(pl.plaid_embedding_backward(d, ids, 7, scale=-0.5, add_to=before.clone()), want, size, "added")


@pytest.mark.parametrize("dtype", [BF, HALF])
def test_dropout(pl, dtype):
    n = 1000
    g = torch.Generator(device=DEV).manual_seed(3)
    x, r = torch.randn(n, generator=g, device=DEV).to(dtype), torch.randn(n, generator=g, device=DEV).to(dtype)
    x[::5], x[1::7], x[2::11] = INF, -INF, NAN
    r[::3], r[1::13] = -INF, NAN
    keep, factor = kept(0, n, 0.4, 11, 12)
    keep = keep.to(DEV)
    rng = torch.tensor([11, 12], device=DEV)
    part = torch.where(keep, x.double() * factor, 0.0)
    for residual in (None, r):
        want = part if residual is None else part + residual.double()
        bound = 2.0 ** -7 * (part.abs() + (0 if residual is None else residual.double().abs())).nan_to_num(0.0, 0.0, 0.0)
        _strict(pl.plaid_dropout(x, 0.4, rng, residual=residual), want, bound, "dropout")


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("rows,width", [(300, 5), (300, 64), (300, 765), (300, 2000), (2500, 1030), (300, 4000), (300, 9000)])
def test_layer_norm(pl, rows, width, dtype):
    g = torch.Generator(device=DEV).manual_seed(width)
    x, d = torch.randn(rows, width, generator=g, device=DEV).to(dtype), torch.randn(rows, width, generator=g, device=DEV).to(dtype)
    w, b = torch.randn(width, generator=g, device=DEV).to(dtype), torch.randn(width, generator=g, device=DEV).to(dtype)
    clean = norm(x, w, b, 1e-5, d)
    out, statistics = pl.plaid_layer_norm(x, w, b, return_statistics=True)
    close(out, clean["out"], clean["out_bound"], "out")
    # parameters
    w2, b2 = w.clone(), b.clone()
    w2[0], w2[1], b2[2], b2[3], w2[4] = INF, -INF, -INF, NAN, torch.finfo(dtype).max
    n = (x.double() - clean["mean"][:, None]) * clean["inverse"][:, None]
    want, bound = n * w2.double() + b2.double(), norm(x, w2.nan_to_num(0.0, 0.0, 0.0), b2.nan_to_num(0.0, 0.0, 0.0), 1e-5)["out_bound"]
    near = n.abs() < 2.0 ** -10  # whose sign is a rounding's, or whose product is at the range's end
    want[near] = 0.0
    got = pl.plaid_layer_norm(x, w2, b2)
    got[near] = 0.0
    _strict(got, want, bound, "parameters")
    # a row that holds an infinity has no numbers, the others what they had
    x2 = x.clone()
    x2[7, 2], x2[200, 0] = INF, NAN
    got, statistics2 = pl.plaid_layer_norm(x2, w, b, return_statistics=True)
    keep = torch.ones(rows, dtype=torch.bool, device=DEV)
    keep[7] = keep[200] = False
    assert torch.isnan(got[~keep]).all() and torch.equal(got[keep], out[keep]) and torch.equal(statistics2[keep], statistics[keep])
    # gradients: of a d_out that holds one, and sums beyond the range
    d2 = d.clone()
    d2[7, 0], d2[9, 1], d2[200, 1], d2[11, 2] = INF, INF, -INF, NAN
    d2[:, 3] = torch.finfo(dtype).max / 4
    d2[:, 4] = -torch.finfo(dtype).max / 4
    dx, dw, db = pl.plaid_layer_norm_backward(d, x, w, b, statistics)
    dx2, dw2, db2 = pl.plaid_layer_norm_backward(d2, x, w, b, statistics)
    assert not torch.isfinite(dx2[[7, 9, 11, 200]]).any()
    sign = torch.sign(n[7, 0])
    assert db2[0] == INF and torch.isnan(db2[1]) and torch.isnan(db2[2]) and db2[3] == INF and db2[4] == -INF
    assert dw2[0] == sign * INF and torch.isnan(dw2[2])
    assert torch.isnan(dw2[1]) if n[9, 1] * n[200, 1] > 0 else dw2[1] == torch.sign(n[9, 1]) * INF
    assert torch.equal(dw2[5:], dw[5:]) and torch.equal(db2[5:], db[5:])
