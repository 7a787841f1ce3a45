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
