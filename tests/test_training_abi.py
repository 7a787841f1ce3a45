"""What the entry points of a reader's training step refuse on the host, before a device is touched, and the sizes that they tell.  No GPU."""
import ctypes as ct

import pytest
import torch

import paper_2205_09707_amd as pl
from paper_2205_09707_amd import plaid, training

from test_library_abi import _struct_fields
from training_util import philox

E, OK = plaid.PLAID_EINVAL, plaid.PLAID_OK
A, ODD = 4096, 4097  # an aligned address and an odd one; neither is read


@pytest.fixture(scope="module")
def lib():
    return pl.load_library()


def test_struct_mirrors_the_header():
    kinds = {"int32_t": ct.c_int32, "int64_t": ct.c_int64, "float": ct.c_float}
    fields = _struct_fields("plaid_token_loss")
    assert [f for _, f in fields] == [f for f, _ in training.plaid_token_loss._fields_]
    for (kind, field), (_, have) in zip(fields, training.plaid_token_loss._fields_):
        assert have is (ct.c_void_p if kind.endswith("*") else kinds[kind]), field


def _call(f, defaults, over):
    a = dict(defaults)
    assert set(over) <= set(a)
    a.update(over)
    return f(*a.values())


EMBED = dict(table=A, table_stride=64, vocabulary=100, width=64, ids=A, n=5, scale=1.0, out=A, dtype=0, device=0, stream=None)
EMBED_BACK = dict(d_out=A, d_out_stride=64, vocabulary=100, width=64, ids=A, n=5, scale=1.0, add=0, d_table=A, dtype=0, work=A, bytes=1 << 30, device=0, stream=None)
TABLES = [dict(dtype=2), dict(dtype=-1), dict(n=-1), dict(n=(1 << 30) + 1), dict(vocabulary=0), dict(vocabulary=(1 << 30) + 1), dict(width=0), dict(width=(1 << 20) + 1),
          dict(ids=None), dict(ids=4100), dict(vocabulary=1 << 30, width=1 << 11), dict(n=1 << 30, width=1 << 11)]


@pytest.mark.parametrize("over", TABLES + [dict(table=None), dict(table=ODD), dict(table_stride=-1), dict(table_stride=1 << 32), dict(out=None), dict(out=4098)])
def test_embedding_refusals(lib, over):
    assert _call(lib.plaid_embedding, EMBED, over) == E
    assert pl.plaid_last_error()


@pytest.mark.parametrize("over", TABLES + [dict(d_out=None), dict(d_out=ODD), dict(d_out_stride=-1), dict(d_table=None), dict(d_table=ODD), dict(work=None), dict(work=4104), dict(bytes=8)])
def test_embedding_backward_refusals(lib, over):
    assert _call(lib.plaid_embedding_backward, EMBED_BACK, over) == E


def test_embedding_workspace(lib):
    need = ct.c_int64(-1)

    def of(n, vocabulary, width):
        assert lib.plaid_embedding_backward_workspace(n, vocabulary, width, ct.byref(need)) == OK
        return need.value

    assert 0 < of(0, 100, 64) < of(8, 100, 64) < of(9, 100, 64) < of(5000, 100, 64)
    for bad in ((-1, 100, 64), (1, 0, 64), (1, 100, 0), (1 << 31, 100, 64), (1, 1 << 30, 1 << 11)):
        assert lib.plaid_embedding_backward_workspace(*bad, ct.byref(need)) == E
    assert lib.plaid_embedding_backward_workspace(1, 1, 1, None) == E
    assert _call(lib.plaid_embedding, EMBED, dict(n=0, ids=None, table=None, out=None)) == OK  # nothing is launched


DROP = dict(x=A, residual=A, n=100, p=0.1, rng=A, out=A, dtype=1, device=0, stream=None)


@pytest.mark.parametrize("over", [dict(x=None), dict(x=ODD), dict(residual=ODD), dict(out=None), dict(out=ODD), dict(n=-1), dict(n=(1 << 40) + 1), dict(p=-0.01), dict(p=1.01),
                                  dict(p=float("nan")), dict(rng=None), dict(rng=4100), dict(dtype=3)])
def test_dropout_refusals(lib, over):
    assert _call(lib.plaid_dropout, DROP, over) == E


def test_dropout_of_nothing(lib):
    assert _call(lib.plaid_dropout, DROP, dict(n=0, x=None, out=None, rng=None)) == OK


NORM = dict(x=A, x_stride=64, weight=A, bias=A, rows=5, width=64, eps=1e-5, out=A, statistics=A, dtype=0, device=0, stream=None)
NORM_BACK = dict(d_out=A, d_out_stride=64, x=A, x_stride=64, weight=A, statistics=A, rows=5, width=64, dx=A, dweight=A, dbias=A, dtype=0, work=A, bytes=1 << 30, device=0, stream=None)
NORMS = [dict(x=None), dict(x=ODD), dict(x_stride=-1), dict(x_stride=1 << 32), dict(weight=ODD), dict(rows=-1), dict(rows=(1 << 30) + 1), dict(width=0), dict(width=16385),
         dict(statistics=4100), dict(dtype=2)]


@pytest.mark.parametrize("over", NORMS + [dict(bias=ODD), dict(out=None), dict(out=ODD), dict(eps=-1.0), dict(eps=float("nan"))])
def test_layer_norm_refusals(lib, over):
    assert _call(lib.plaid_layer_norm, NORM, over) == E


@pytest.mark.parametrize("over", NORMS + [dict(d_out=None), dict(d_out=ODD), dict(d_out_stride=-1), dict(statistics=None), dict(dx=ODD), dict(dweight=ODD), dict(dbias=ODD),
                                          dict(weight=None), dict(work=None), dict(work=4104), dict(bytes=8)])
def test_layer_norm_backward_refusals(lib, over):
    assert _call(lib.plaid_layer_norm_backward, NORM_BACK, over) == E


def test_layer_norm_of_nothing(lib):
    assert _call(lib.plaid_layer_norm, NORM, dict(rows=0, x=None, out=None)) == OK
    assert _call(lib.plaid_layer_norm_backward, NORM_BACK, dict(rows=0, x=None, d_out=None, statistics=None, dweight=None, dbias=None, work=None, bytes=0)) == OK
    need = ct.c_int64(-1)
    assert lib.plaid_layer_norm_backward_workspace(5, 64, ct.byref(need)) == OK and need.value > 0
    assert lib.plaid_layer_norm_backward_workspace(5, 0, ct.byref(need)) == E and lib.plaid_layer_norm_backward_workspace(5, 64, None) == E


def _loss(**over):
    a = dict(dtype=0, width=64, rows=100, vocabulary=1000, scale=1.0, hidden=A, weight=A, hidden_stride=64, weight_stride=64, targets=A, loss=A, lse=A)
    assert set(over) <= set(a)
    a.update(over)
    return training.plaid_token_loss(*a.values())


BAD_SHAPES = [dict(dtype=2), dict(width=0), dict(width=68), dict(width=16392), dict(rows=-1), dict(rows=(1 << 24) + 1), dict(vocabulary=0), dict(vocabulary=(1 << 27) + 1)]
BAD_ARRAYS = [dict(hidden=None), dict(hidden=4104), dict(hidden_stride=60), dict(hidden_stride=-64), dict(hidden_stride=1 << 24), dict(weight=None), dict(weight=4104),
              dict(weight_stride=60), dict(weight_stride=1 << 24), dict(targets=None), dict(targets=4100), dict(loss=4098), dict(lse=4100)]


@pytest.mark.parametrize("over", BAD_SHAPES + BAD_ARRAYS)
def test_cross_entropy_refusals(lib, over):
    a, big = _loss(**over), 1 << 40
    assert lib.plaid_cross_entropy(ct.byref(a), A, big, 0, None) == E
    assert lib.plaid_cross_entropy_backward(ct.byref(a), A, 1, A, A, A, big, 0, None) == E
    need = ct.c_int64(-1)
    for backward in (0, 1):
        assert lib.plaid_cross_entropy_workspace(ct.byref(a), backward, ct.byref(need)) == (E if over in BAD_SHAPES else OK)


@pytest.mark.parametrize("rows", [3, 100])
def test_cross_entropy_workspace_and_gradient_refusals(lib, rows):
    a, need = _loss(rows=rows), ct.c_int64(-1)
    assert lib.plaid_cross_entropy_workspace(ct.byref(a), 0, ct.byref(need)) == OK and need.value > 0
    assert lib.plaid_cross_entropy(ct.byref(a), A, need.value - 1, 0, None) == E and "workspace" in pl.plaid_last_error()
    assert lib.plaid_cross_entropy(ct.byref(a), 4104, need.value, 0, None) == E and lib.plaid_cross_entropy(ct.byref(a), None, need.value, 0, None) == E
    assert lib.plaid_cross_entropy(ct.byref(_loss(rows=rows, loss=None)), A, need.value, 0, None) == E
    assert lib.plaid_cross_entropy(None, A, need.value, 0, None) == E and lib.plaid_cross_entropy_workspace(None, 0, ct.byref(need)) == E
    assert lib.plaid_cross_entropy_workspace(ct.byref(a), 0, None) == E
    assert lib.plaid_cross_entropy_workspace(ct.byref(a), 1, ct.byref(need)) == OK and need.value > 0
    back = lambda a=a, d=A, stride=1, dh=A, dw=A, work=A, size=need.value: lib.plaid_cross_entropy_backward(ct.byref(a), d, stride, dh, dw, work, size, 0, None)  # noqa: E731
    assert back(size=need.value - 1) == E and back(work=None) == E and back(work=4104) == E
    assert back(d=None) == E and back(d=4098) == E and back(stride=2) == E and back(stride=-1) == E and back(dh=4104) == E and back(dw=4104) == E
    assert back(a=_loss(rows=rows, lse=None)) == E
    assert back(dh=None, dw=None) == OK  # nothing is asked for


def test_no_rows(lib):
    need = ct.c_int64(-1)
    a = _loss(rows=0, hidden=None, targets=None, loss=None, lse=None)
    assert lib.plaid_cross_entropy_workspace(ct.byref(a), 0, ct.byref(need)) == OK and need.value == 0
    assert lib.plaid_cross_entropy(ct.byref(a), None, 0, 0, None) == OK


def test_generator_of_the_tests_has_the_published_values():
    """Known answers of Philox4x32-10 that its authors published with the paper."""
    full = 0xFFFFFFFF
    assert philox((0, 0, 0, 0), (0, 0)) == [0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8]
    assert philox((full,) * 4, (full,) * 2) == [0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD]


def test_binding_refuses_what_is_not_on_a_gpu():
    x, i = torch.zeros(4, 64, dtype=torch.bfloat16), torch.zeros(4, dtype=torch.int64)
    for f in (lambda: pl.plaid_embedding(x, i), lambda: pl.plaid_embedding_backward(x, i, 10), lambda: pl.plaid_dropout(x, 0.1, i[:2]), lambda: pl.plaid_layer_norm(x),
              lambda: pl.plaid_layer_norm_backward(x, x, None, None, torch.zeros(4, 2)), lambda: pl.plaid_cross_entropy(x, x, i),
              lambda: pl.plaid_cross_entropy_backward(torch.zeros(4), x, x, i, torch.zeros(4, 2))):
        with pytest.raises(ValueError):
            f()
