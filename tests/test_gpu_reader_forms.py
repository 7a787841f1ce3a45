"""Every form of the kernels of many rows and of the gradients: workgroups of four and of eight waves, axes whole and in parts, dense keys,
biases and the cache, both head sizes.  test_reader_plans.py checks, without a GPU, that these shapes get the forms that they are here for."""
import random

import pytest
import torch

import reader_util as ru
from test_gpu_reader_attention import BF, DEV, HF, _bias, _check_cached, _check_cross, _filled_cache, _off, _randn, pl  # noqa: F401 (pl is a fixture)

pytestmark = pytest.mark.gpu


def _spread(n, lo, hi, seed):
    rng = random.Random(seed)
    return [rng.randint(lo, hi) for _ in range(n - 1)] + [lo]


# name: queries, keys, heads, key heads, head_dim; forward's waves and whether its keys are in parts; backward's waves of dk and dv, whether the
# keys of dq and the rows of dk and dv are in parts
CROSS = {
    "four 128": (_spread(64, 5, 20, 1), _spread(64, 0, 300, 2), 8, 2, 128, 4, False, 4, False, False),
    "four 64": (_spread(100, 0, 12, 3), _spread(100, 1, 200, 4), 16, 4, 64, 4, False, 4, False, False),
    "four 128 in parts": ([10, 3, 17, 9, 12, 0], [9000, 4000, 12000, 7000, 8001, 7000], 16, 4, 128, 4, True, 4, True, False),
    "four 64 in parts": ([16, 5, 18], [11000, 12000, 10003], 16, 8, 64, 4, True, 4, True, False),
    "eight 128": ([150, 300, 80, 333, 290, 70, 201, 170], [700, 64, 65, 900, 0, 130, 333, 400], 16, 4, 128, 8, False, 8, False, True),
    "eight 64": ([150, 300, 80, 333] * 4, [700, 64, 1300, 411] * 4, 16, 8, 64, 8, False, 4, False, False),
    "eight 128 in parts": ([330], [9000], 4, 1, 128, 8, True, 8, True, True),
    "eight 64 in parts": ([330], [9000], 4, 1, 64, 8, True, 4, True, True),
    "rows in parts 128": ([1500], [200], 4, 1, 128, 8, False, 8, False, True),
    "rows in parts 64": ([3, 1200], [90, 130], 8, 2, 64, 0, False, 4, False, True),
}
# queries, keys, heads, key heads, head_dim, block size, table's width in blocks; waves, whether the keys are in parts
CACHED = {
    "four 128": (_spread(100, 3, 15, 5), _spread(100, 3, 200, 6), 8, 4, 128, 16, 13, 4, False),
    "four 64": (_spread(100, 3, 15, 7), _spread(100, 3, 200, 8), 8, 4, 64, 32, 7, 4, False),
    "four 128 in parts": ([10, 3, 17, 9], [2500, 300, 17, 64], 16, 4, 128, 16, 2900, 4, True),
    "four 64 in parts": ([10, 3, 17, 9], [2500, 300, 17, 64], 16, 4, 64, 64, 730, 4, True),
    "eight 128": ([300, 70, 513, 200] * 4, [700, 70, 513, 201] * 4, 8, 4, 128, 16, 45, 8, False),
    "eight 64": ([300, 70, 513, 200] * 4, [700, 70, 513, 201] * 4, 8, 4, 64, 16, 45, 8, False),
    "eight 128 in parts": ([300], [3000], 8, 1, 128, 256, 90, 8, True),
    "eight 64 in parts": ([300], [3000], 8, 1, 64, 128, 180, 8, True),
}


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("name", CROSS)
def test_cross_attention(pl, name, dtype, with_bias):  # noqa: F811
    q, k, heads, kv_heads, dim = CROSS[name][:5]
    _check_cross(pl, q, k, heads, kv_heads, dim, dtype, _bias(sum(k), 4, dtype) if with_bias else None, seed=21)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("name", CACHED)
def test_cached_attention(pl, name, dtype, causal):  # noqa: F811
    q, k, heads, kv_heads, dim, bs, width = CACHED[name][:7]
    k = [max(a, b) for a, b in zip(q, k)] if causal else k
    _check_cached(pl, q, k, heads, kv_heads, dim, bs, dtype, causal, hide=((0, 1),), width=width, seed=22)
