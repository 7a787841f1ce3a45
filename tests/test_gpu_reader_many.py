"""The kernels of many rows at the sizes that reach them: sums of whole tiles, requests that are taken in the order of their work or
(more than 64 of them) as they come, splits over long keys, masks and scales."""
import pytest
import torch

import reader_util as ru
from test_gpu_reader_attention import BF, HF, _bias, _check_cached, _check_cross, pl  # noqa: F401 (pl is a fixture)

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 16, 2), (128, 16, 2), (128, 9, 1), (64, 15, 5)])
def test_long_and_short_requests(pl, dim, heads, kv_heads, dtype, with_bias):  # noqa: F811
    k_lengths = [64, 0, 331, 1, 130]
    bias = _bias(sum(k_lengths), 5, dtype) if with_bias else None
    _check_cross(pl, [300, 40, 257, 512, 1], k_lengths, heads, kv_heads, dim, dtype, bias, seed=3)


@pytest.mark.parametrize("n", [64, 65, 130])
def test_numbers_of_requests(pl, n):  # noqa: F811
    lengths = [(7 * r) % 40 for r in range(n)]
    keys = [(11 * r + 3) % 150 for r in range(n)]
    _check_cross(pl, lengths, keys, 16, 2, 64, BF, _bias(sum(keys), 1, BF), seed=n)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_requests_of_few_and_of_many_keys(pl, dtype):  # noqa: F811
    _check_cross(pl, [200, 333, 128], [3000, 32, 33], 8, 4, 128, dtype, _bias(3065, 2, dtype), seed=9)


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.5])
@pytest.mark.parametrize("with_bias", [False, True])
def test_scales(pl, scale, with_bias):  # noqa: F811
    _check_cross(pl, [300, 290], [200, 101], 16, 2, 64, BF, _bias(301, 4, BF) if with_bias else None, scale=scale, seed=6)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_masks_of_the_lowest_value(pl, dtype):  # noqa: F811
    keys = [150, 200, 70]
    lowest = torch.finfo(dtype).min
    bias = _bias(sum(keys), 8, dtype, masked=0.0)
    bias[:150] = lowest                                                  # all of the first request's
    bias[150 + 64:150 + 128] = lowest                                    # a whole tile of the second's
    bias[350 + 3] = -float("inf")
    _check_cross(pl, [280, 270, 300], keys, 16, 2, 64, dtype, bias, seed=10)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dim,bs,heads,kv_heads", [(BF, 128, 16, 16, 2), (HF, 64, 64, 16, 2), (BF, 64, 32, 9, 3), (HF, 128, 128, 12, 4)])
def test_prompts_behind_contexts(pl, dtype, dim, bs, heads, kv_heads, causal):  # noqa: F811
    _check_cached(pl, [400, 1, 0, 513, 257], [1200, 700, 30, 513, 100], heads, kv_heads, dim, bs, dtype, causal=causal, hide=((0, 1), (3, 0)), seed=12)


def test_many_prompts(pl):  # noqa: F811
    n = 70
    q = [(13 * r) % 45 for r in range(n)]
    _check_cached(pl, q, [x + (29 * r) % 200 for r, x in enumerate(q)], 16, 2, 64, 16, BF, seed=13)


def test_long_keys_in_splits(pl):  # noqa: F811
    _check_cross(pl, [330], [9000], 8, 1, 128, BF, _bias(9000, 3, BF), seed=14)


def test_numbers_that_are_not_finite_in_masked_keys(pl):  # noqa: F811
    bias = _bias(500, 6, BF, masked=0.4)

    def change(q, k, v):
        for t, x in ((k, float("nan")), (v, float("inf"))):
            t[(bias == -float("inf")).nonzero().flatten()] = x

    _check_cross(pl, [300, 320], [300, 200], 16, 2, 64, BF, bias, change=change, seed=15)


@pytest.mark.parametrize("dim", [64, 128])
def test_scores_of_hundreds(pl, dim):  # noqa: F811
    _check_cross(pl, [300, 270], [700, 333], 16, 2, dim, BF, gain=20.0, train=False)
    _check_cross(pl, [300, 270], [700, 333], 16, 2, dim, HF, _bias(1033, 2, HF), gain=20.0, train=False)


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("heads,m", [(2, 5), (2, 40), (16, 600)])
def test_what_is_not_finite_reaches_later_tokens_only(pl, dim, heads, m):  # noqa: F811
    """A key or a value of a prompt's token that is not finite: earlier tokens do not see it, later ones do, where it is."""
    kv, bs, n = 2, 16, m + 70
    g = torch.Generator().manual_seed(m)
    q, k, v = (torch.randn(x, h, dim, generator=g).to(BF).to("cuda:0") for x, h in ((m, heads), (n, kv), (n, kv)))
    at_k, at_v = n - m + m // 2, n - m + 2 * m // 3
    k[at_k, 0, 3] = float("nan")
    v[at_v, 1, dim - 1] = float("inf")
    blocks = -(-n // bs)
    cache = pl.PagedCache.empty(blocks, bs, kv, dim, BF)
    slots = torch.arange(n, device="cuda:0")
    table, lengths = torch.arange(blocks, device="cuda:0", dtype=torch.int32)[None], torch.tensor([n], device="cuda:0", dtype=torch.int32)
    offsets = torch.tensor([0, m], device="cuda:0")
    pl.plaid_cache_write(cache, k, v, slots)
    out = pl.plaid_cached_attention(q, cache, table, lengths, offsets).float()
    clean = k.clone(), v.clone()
    clean[0][at_k, 0, 3] = 0.0
    clean[1][at_v, 1, dim - 1] = 0.0
    pl.plaid_cache_write(cache, *clean, slots)
    want = pl.plaid_cached_attention(q, cache, table, lengths, offsets).float()
    first, second = heads // kv, slice(heads // kv, heads)
    assert torch.equal(out[:m // 2, :first], want[:m // 2, :first]) and torch.isnan(out[m // 2:, :first]).all()
    seen = 2 * m // 3
    assert torch.equal(out[:seen, second], want[:seen, second])
    assert torch.isnan(out[seen:, second, dim - 32:]).all() and torch.equal(out[:, second, :dim - 32], want[:, second, :dim - 32])


@pytest.mark.parametrize("m", [3, 300])
def test_a_row_without_keys_has_no_gradient(pl, m):  # noqa: F811
    """Every key of the first request is masked and its queries are not finite: zeros, and nothing of it reaches the second request."""
    g = torch.Generator().manual_seed(m)
    q, k, v = (torch.randn(n, 4, 64, generator=g).to(BF).to("cuda:0") for n in (2 * m, 130, 130))
    d_out = torch.randn(2 * m, 4, 64, generator=g).to(BF).to("cuda:0")
    bias = torch.zeros(130, dtype=BF, device="cuda:0")
    bias[:50] = -float("inf")
    offsets = torch.tensor([0, m, 2 * m], device="cuda:0"), torch.tensor([0, 50, 130], device="cuda:0")
    results = []
    for value in (0.0, float("nan"), float("inf")):
        q[:m] = value
        out, lse = pl.plaid_cross_attention(q, k, v, *offsets, key_bias=bias, return_lse=True)
        results.append((out, *pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, *offsets, key_bias=bias)))
    for got in results:
        for x, y in zip(got, results[0]):
            assert torch.equal(x, y) and torch.isfinite(x).all()
        assert (got[0][:m] == 0).all() and (got[1][:m] == 0).all() and all((x[:50] == 0).all() for x in got[2:])
