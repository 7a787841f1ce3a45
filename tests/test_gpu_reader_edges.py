"""Values that are not finite at a request's end, rows whose scores overflow, weights below the type's normal range, and offsets that do not ascend."""
import math

import pytest
import torch

import reader_util as ru
from test_gpu_reader_attention import BF, DEV, HF, _off, _randn, pl  # noqa: F401 (pl is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype", [BF, HF])
def test_small_weights_of_half_precision(pl, dtype):  # noqa: F811
    """A hundred thousand keys: a weight is 1e-5, which fp16 holds as a multiple of 2^-24.  dv keeps the type's relative precision."""
    n, m, dim = 100_000, 3, 64
    q, k, v = (_randn((x, 1, dim), i, dtype, g) for i, (x, g) in enumerate(((m, 0.25), (n, 1.0), (n, 1.0))))
    d_out = _randn((m, 1, dim), 9, dtype, 256.0)
    d = lambda t: t.to(DEV)  # noqa: E731
    out, lse = pl.plaid_cross_attention(d(q), d(k), d(v), _off([m]), _off([n]), return_lse=True)
    _, _, dv, _ = pl.plaid_cross_attention_backward(d(d_out), d(q), d(k), d(v), out, lse, _off([m]), _off([n]))
    s = q[:, 0].double() @ k[:, 0].double().T * dim ** -0.5
    p = torch.softmax(s, -1)
    want = p.T @ d_out[:, 0].double()
    u, e = ru.U[dtype], ru.E32 * (1 + float((q[:, 0].double().abs() @ k[:, 0].double().abs().T).max()) * dim ** -0.5 / 16)
    ru.close(dv[:, 0], want, u * want.abs() + (u + e) * (p.T @ d_out[:, 0].double().abs()) + ru.TINY[dtype], "dv")


# lengths that no tile divides; the key that is not finite is the last one, which has nothing behind it
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads", [2, 16])
@pytest.mark.parametrize("m,n", [(1, 83), (40, 83), (300, 83), (1, 3001), (300, 3001), (64, 1), (300, 1)])
def test_a_last_key_that_is_not_finite(pl, m, n, heads, dim, dtype):  # noqa: F811
    """An infinite value of the last key gives what one of the first key gives."""
    q, k, v = _randn((2 * m, heads, dim), 1, dtype).to(DEV), _randn((2 * n, 2, dim), 2, dtype).to(DEV), _randn((2 * n, 2, dim), 3, dtype).to(DEV)
    half, qo, ko = heads // 2, _off([m, m]), _off([n, n])
    for at in (0, n - 1):
        w = v.clone()
        w[at, 1, 7] = math.inf
        out = pl.plaid_cross_attention(q, k, w, qo, ko)
        assert torch.isinf(out[:m, half:, 7]).all() and torch.isfinite(out[m:]).all() and torch.isfinite(out[:, :half]).all()
        assert torch.isfinite(out[..., :7]).all() and torch.isfinite(out[..., 8:]).all()


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("m,n,heads", [(1, 40, 2), (41, 90, 2), (5, 700, 6), (301, 90, 8), (301, 20, 10)])
def test_a_last_row_that_is_not_finite(pl, m, n, heads, dtype):  # noqa: F811
    """An infinite d_out of the last row makes its dimension of dv infinite, as one of the first row does, and no other."""
    for dim in (64, 128):
        q, k, v, d_out = (_randn((x, h, dim), i, dtype).to(DEV) for i, (x, h) in enumerate(((2 * m, heads), (2 * n, 2), (2 * n, 2), (2 * m, heads))))
        out, lse = pl.plaid_cross_attention(q, k, v, _off([m, m]), _off([n, n]), return_lse=True)
        for token, head in ((0, 0), (m - 1, heads // 2 - 1)):
            o = d_out.clone()
            o[token, head, 9] = math.inf
            _, dk, dv, _ = pl.plaid_cross_attention_backward(o, q, k, v, out, lse, _off([m, m]), _off([n, n]))
            assert torch.isinf(dv[:n, 0, 9]).all() and torch.isfinite(dv[:, 1]).all() and torch.isfinite(dv[n:]).all() and torch.isfinite(dk[n:]).all()
            assert torch.isfinite(dv[..., :9]).all() and torch.isfinite(dv[..., 10:]).all()


@pytest.mark.parametrize("low", [-1000.0, 3000.0, -3e38])
@pytest.mark.parametrize("m,n,heads", [(3, 40, 2), (3, 3000, 2), (40, 90, 4), (300, 200, 8), (300, 2000, 8)])
def test_a_row_whose_scores_overflow(pl, m, n, heads, low):  # noqa: F811
    """The first row's products are -infinity throughout, so no weight is left there.  The other rows of its request, whose biases are all
    far from zero, have their gradients all the same."""
    dim = 64
    q, k, v, d_out = (_randn((x, h, dim), i, BF) for i, (x, h) in enumerate(((m, heads), (n, 2), (n, 2), (m, heads))))
    q[..., 0], k[..., 0] = 0.0, 1e10
    q[0, 0, 0] = -1e32
    d_out[0, 0] = 0.0
    bias = (torch.randn(n, generator=torch.Generator().manual_seed(4)) * 8 + low).to(BF)
    d = lambda t: t.to(DEV)  # noqa: E731
    out, lse = pl.plaid_cross_attention(d(q), d(k), d(v), _off([m]), _off([n]), key_bias=d(bias), return_lse=True)
    assert not out[0, 0].any() and float(lse[0, 0].sum()) == -math.inf
    got = pl.plaid_cross_attention_backward(d(d_out), d(q), d(k), d(v), out, lse, _off([m]), _off([n]), key_bias=d(bias))
    assert not got[0][0, 0].any()
    want = ru.cross(q, k, v, [m], [n], dim ** -0.5, bias, d_out)
    keep = torch.ones(m, heads, dtype=torch.bool)
    keep[0, 0] = False
    for name, x in zip(("out", "dq"), (out, got[0])):
        ru.close(x.cpu()[keep], want[name][keep], want[name + "_bound"][keep], name)
    for name, x in zip(("dk", "dv", "dbias"), got[1:]):
        ru.close(x[..., 1:] if x.dim() == 3 else x, *(want[name + e][..., 1:] if x.dim() == 3 else want[name + e] for e in ("", "_bound")), name)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("m,n,heads", [(1, 40, 2), (3, 3000, 2), (40, 90, 4), (300, 200, 8), (300, 2000, 8)])
def test_a_key_that_is_not_finite_beside_the_lowest_biases(pl, m, n, heads, dtype):  # noqa: F811
    """Scores vanish beside biases of the type's lowest value; a key that is not a number makes its rows so all the same."""
    q, k, v, d_out = (_randn((x, h, 64), i, dtype).to(DEV) for i, (x, h) in enumerate(((2 * m, heads), (2 * n, 2), (2 * n, 2), (2 * m, heads))))
    k[n // 2, 1, 3] = math.nan
    bias = torch.full((2 * n,), torch.finfo(dtype).min, dtype=dtype, device=DEV)
    out, lse = pl.plaid_cross_attention(q, k, v, _off([m, m]), _off([n, n]), key_bias=bias, return_lse=True)
    half = heads // 2
    assert torch.isnan(out[:m, half:]).all() and torch.isfinite(out[:m, :half]).all() and torch.isfinite(out[m:]).all()
    dq, dk, dv, _ = pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, _off([m, m]), _off([n, n]), key_bias=bias)
    for x, at in ((dq, m), (dk, n), (dv, n)):
        first = x.shape[1] // 2
        assert torch.isnan(x[:at, first:]).all() and torch.isfinite(x[:at, :first]).all() and torch.isfinite(x[at:]).all()


def test_offsets_that_claim_rows_many_times(pl):  # noqa: F811
    """Offsets that do not ascend: half of 3000 requests claim all of 40 000 tokens and 131 072 keys, 3.8e9 steps of work, which 32 bits do
    not hold.  What they get is unspecified; the call ends, touches nothing else, and the next one is right."""
    n, nq, nk = 3000, 40_000, 131_072
    q, k = _randn((nq, 1, 64), 1, BF).to(DEV), _randn((nk, 1, 64), 2, BF).to(DEV)
    off = lambda x: torch.tensor([0, x], device=DEV).repeat(n // 2 + 1)[:n + 1].contiguous()  # noqa: E731
    want = pl.plaid_cross_attention(q[:3], k, k, _off([1, 1, 1]), _off([nk, 0, 0]))
    for _ in range(2):
        pl.plaid_cross_attention(q, k, k, off(nq), off(nk))
        torch.cuda.synchronize()
    assert torch.equal(q.cpu(), _randn((nq, 1, 64), 1, BF)) and torch.equal(k.cpu(), _randn((nk, 1, 64), 2, BF))
    assert torch.equal(pl.plaid_cross_attention(q[:3], k, k, _off([1, 1, 1]), _off([nk, 0, 0])), want)
