"""Where the definition makes the scores' gradient zero, and where it is small beside what it is a difference of: one key, one key that is not
masked, few keys that are not masked, a softmax with nearly all of its weight on one key."""
import ctypes as ct
import itertools
import math

import pytest
import torch

import reader_util as ru
from test_gpu_reader_attention import BF, DEV, HF, _bias, _off, _randn, pl  # noqa: F401 (pl is a fixture)

pytestmark = pytest.mark.gpu


def _inputs(q_lengths, k_lengths, heads, kv_heads, dim, dtype, seed, gain=0.25):
    nq, nk = sum(q_lengths), sum(k_lengths)
    return (_randn((nq, heads, dim), seed + 1, dtype), _randn((nk, kv_heads, dim), seed + 2, dtype), _randn((nk, kv_heads, dim), seed + 3, dtype),
            _randn((nq, heads, dim), seed + 4, dtype, gain))


def _gradients(pl, q, k, v, d_out, bias, q_lengths, k_lengths):  # noqa: F811
    d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    out, lse = pl.plaid_cross_attention(d(q), d(k), d(v), _off(q_lengths), _off(k_lengths), key_bias=d(bias), return_lse=True)
    return out, pl.plaid_cross_attention_backward(d(d_out), d(q), d(k), d(v), out, lse, _off(q_lengths), _off(k_lengths), key_bias=d(bias))


# keys of the request, the place of the one that is not masked (None: no bias), queries: every kernel and both ways to cut its work
ONE = [(1, None, 1), (1, None, 40), (1, None, 700), (1, 0, 5), (2, 1, 33), (32, 31, 300), (33, 0, 7), (40, 39, 64), (100, 50, 300), (700, 333, 3),
       (3000, 2999, 1), (3000, 64, 200)]


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 3, 3), (128, 8, 2)])
@pytest.mark.parametrize("n,at,m", ONE)
def test_one_key_that_counts(pl, n, at, m, dim, heads, kv_heads, dtype):  # noqa: F811
    """P is 1 and dP = delta: dq, dk and dbias are zero, not nearly so.  dv is the sum of d_out."""
    q, k, v, d_out = _inputs([m], [n], heads, kv_heads, dim, dtype, n + m)
    bias = None
    if at is not None:
        bias = torch.full((n,), -math.inf, dtype=dtype)
        bias[at] = -1.25
    out, (dq, dk, dv, dbias) = _gradients(pl, q, k, v, d_out, bias, [m], [n])
    assert torch.equal(out.cpu(), v[at or 0].repeat_interleave(heads // kv_heads, 0).expand(m, heads, dim))
    assert not dq.any() and not dk.any() and (dbias is None or not dbias.any())
    want = ru.cross(q, k, v, [m], [n], dim ** -0.5, bias, d_out)
    ru.close(dv, want["dv"], want["dv_bound"], "dv")


@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 3, 3), (128, 8, 2)])
@pytest.mark.parametrize("n,at,m", [c for c in ONE if c[1] is not None])
def test_one_key_beside_masks_of_the_lowest_value(pl, n, at, m, dim, heads, kv_heads):  # noqa: F811
    """Beside a key of an ordinary bias those of bfloat16's lowest value have weights of zero: the gradients are zero as well."""
    q, k, v, d_out = _inputs([m], [n], heads, kv_heads, dim, BF, n + m)
    bias = torch.full((n,), torch.finfo(BF).min, dtype=BF)
    bias[at] = 0.75
    out, (dq, dk, dv, dbias) = _gradients(pl, q, k, v, d_out, bias, [m], [n])
    assert torch.equal(out.cpu(), v[at].repeat_interleave(heads // kv_heads, 0).expand(m, heads, dim))
    assert not dq.any() and not dk.any() and not dbias.any()


@pytest.mark.parametrize("dtype", [BF, HF])
def test_one_key_beside_other_requests(pl, dtype):  # noqa: F811
    """A request with one key that counts among others, in both orders of requests (up to 64 of them and more)."""
    for times in (1, 20):
        q_lengths, k_lengths = [5, 40, 0, 70] * times, [1, 70, 3, 45] * times
        nq, nk = sum(q_lengths), sum(k_lengths)
        q, k, v, d_out = _inputs(q_lengths, k_lengths, 4, 2, 64, dtype, times)
        bias = _bias(nk, 3, dtype)
        for r in range(times):
            bias[r * 119] = 0.5
            bias[r * 119 + 74:r * 119 + 119] = -math.inf
            bias[r * 119 + 74 + 37] = 2.0
        _, (dq, dk, dv, dbias) = _gradients(pl, q, k, v, d_out, bias, q_lengths, k_lengths)
        want = ru.cross(q, k, v, q_lengths, k_lengths, 0.125, bias, d_out)
        for name, x in zip(("dq", "dk", "dv", "dbias"), (dq, dk, dv, dbias)):
            ru.close(x, want[name], want[name + "_bound"], name)
        dq, dk, dbias = dq.view(times, nq // times, -1), dk.view(times, nk // times, -1), dbias.view(times, -1)
        assert not dq[:, :5].any() and not dq[:, 45:].any() and dq[:, 5:45].any()
        assert not dk[:, 0].any() and not dk[:, 74:].any() and not dbias[:, 0].any() and not dbias[:, 74:].any() and dk[:, 1:71].any()


def _close_in_scores(pl, q, k, v, d_out, bias, m, n, dtype):  # noqa: F811
    """Bounds that grow with the scores' gradient dS and not with d_out . out: dS rounds to the type (u), delta is known to u / 2 of the sum
    of |dS| over a row, and the arithmetic in 32 bits is allowed E32 of what is subtracted."""
    u, (_, heads, dim), kv_heads = ru.U[dtype], q.shape, k.shape[1]
    _, (dq, dk, _, dbias) = _gradients(pl, q, k, v, d_out, bias, [m], [n])
    want = {x: torch.zeros(y.shape, dtype=torch.float64) for x, y in (("dq", q), ("dk", k), ("db", k[:, 0, 0]))}
    off = {x: torch.zeros_like(y) for x, y in want.items()}
    scale = dim ** -0.5
    for h in range(heads):
        g = h * kv_heads // heads
        x, y, z, o = q[:, h].double(), k[:, g].double(), v[:, g].double(), d_out[:, h].double()
        p = torch.softmax(x @ y.T * scale + (0.0 if bias is None else bias.double()), -1)
        dp = o @ z.T
        ds = p * (dp - (p * dp).sum(-1, keepdim=True))
        rough = (o.abs() @ z.abs().T).amax(-1, keepdim=True)
        err = (u + ru.E32) * ds.abs() + p * (u / 2 * ds.abs().sum(-1, keepdim=True) + ru.E32 * rough) + (2.0 ** -25 if dtype == HF else 0.0)
        want["dq"][:, h], off["dq"][:, h] = ds @ y * scale, err @ y.abs() * scale
        want["dk"][:, g] += ds.T @ x * scale
        off["dk"][:, g] += err.T @ x.abs() * scale
        want["db"] += ds.sum(0)
        off["db"] += err.sum(0)
    for name, got in (("dq", dq), ("dk", dk), ("db", dbias)):
        if got is not None:
            ru.close(got, want[name], off[name] + u * want[name].abs() + ru.TINY[dtype], name)


# queries: rows that one workgroup has, and rows that are shared among several keys' parts
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("m,n,live", [(40, 40, 2), (300, 40, 2), (5, 40, 3), (64, 1000, 2), (3, 4000, 2), (200, 3000, 4), (33, 20, 2)])
def test_few_keys_that_count(pl, m, n, live, dtype):  # noqa: F811
    for dim, heads, kv_heads in ((64, 4, 4), (128, 4, 1)):
        q, k, v, d_out = _inputs([m], [n], heads, kv_heads, dim, dtype, m * n)
        bias = torch.full((n,), -math.inf, dtype=dtype)
        bias[torch.randperm(n, generator=torch.Generator().manual_seed(n))[:live]] = 0.25
        _close_in_scores(pl, q, k, v, d_out, bias, m, n, dtype)


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("m,n", [(40, 50), (300, 333), (3, 4000), (200, 3000), (20, 31)])
def test_weight_on_one_key(pl, m, n, with_bias, dtype):  # noqa: F811
    """One key's score is far above the others: its weight is about 0.99, and dS a hundredth of what it is a difference of."""
    for dim, heads, kv_heads in ((64, 2, 2), (128, 4, 1)):
        q, k, v, d_out = _inputs([m], [n], heads, kv_heads, dim, dtype, m + n)
        bias = _bias(n, 5, dtype, 0.1) if with_bias else None
        if with_bias:
            bias[n // 2] = 2.0
        lift = math.log(99 * n * math.e ** 0.5) * dim ** 0.5 / 16       # q's first dimension is 16: the score of that key rises by log(99 n e^1/2)
        q[..., 0], k[..., 0] = 16.0, 0.0
        k[n // 2, :, 0] = lift
        _close_in_scores(pl, q, k, v, d_out, bias, m, n, dtype)


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("q_lengths,k_lengths", [([5, 40], [2, 31]), ([300, 7], [40, 90]), ([3], [3000]), ([700], [20])])
def test_gradients_do_not_depend_on_which_are_asked_for(pl, q_lengths, k_lengths, with_bias):  # noqa: F811
    from paper_2205_09707_amd import plaid, reader
    lib = pl.load_library()
    q, k, v, d_out = (t.to(DEV) for t in _inputs(q_lengths, k_lengths, 4, 2, 64, BF, 7))
    bias = _bias(sum(k_lengths), 2, BF).to(DEV) if with_bias else None
    qo, ko = _off(q_lengths), _off(k_lengths)
    out, lse = pl.plaid_cross_attention(q, k, v, qo, ko, key_bias=bias, return_lse=True)
    whole = pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, qo, ko, key_bias=bias)
    a = reader._attention(reader._rows(q), reader._rows(k), reader._rows(v), bias, qo, ko, 2, None, out, lse)
    need = ct.c_int64(0)
    assert lib.plaid_cross_attention_workspace(ct.byref(a), 1, ct.byref(need)) == plaid.PLAID_OK
    for asked in itertools.product((False, True), repeat=4 if with_bias else 3):
        work = torch.full((need.value,), 0x7f, dtype=torch.uint8, device=DEV)
        got = [torch.full_like(t, 3.0) if yes else None for t, yes in zip(whole, asked)] + [None] * (4 - len(asked))
        assert lib.plaid_cross_attention_backward(ct.byref(a), d_out.data_ptr(), *[None if t is None else t.data_ptr() for t in got], work.data_ptr(),
                                                  need.value, 0, torch.cuda.current_stream().cuda_stream) == plaid.PLAID_OK
        torch.cuda.synchronize()
        for x, y in zip(got, whole):
            assert x is None or torch.equal(x, y), asked
