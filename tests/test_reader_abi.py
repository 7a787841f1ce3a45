"""What the reader's entry points refuse on the host, before a device is touched, and the sizes that they tell.  No GPU."""
import ctypes as ct

import pytest
import torch

import paper_2205_09707_amd as pl
from paper_2205_09707_amd import plaid, reader

from test_library_abi import _struct_fields

E = plaid.PLAID_EINVAL
A, ODD = 4096, 4104  # an aligned address and one that is aligned to 8 bytes; neither is read


@pytest.fixture(scope="module")
def lib():
    return pl.load_library()


def test_structs_mirror_the_header():
    kinds = {"int32_t": ct.c_int32, "int64_t": ct.c_int64, "float": ct.c_float}
    for name, cls in (("plaid_paged_cache", reader.plaid_paged_cache), ("plaid_attention", reader.plaid_attention)):
        fields = _struct_fields(name)
        assert [f for _, f in fields] == [f for f, _ in cls._fields_]
        for (kind, field), (_, have) in zip(fields, cls._fields_):
            assert have is (ct.c_void_p if kind.endswith("*") else kinds[kind]), (name, field)


def _tables(lib, **over):
    a = dict(lengths=A, added=A, n=4, table=A, table_stride=8, max_blocks=8, free_blocks=A, n_free=10, block_size=16, offsets=A, totals=A,
             positions=A, slots=A, capacity=64, wanted=A, workspace=None, bytes=0, device=0, stream=None)
    a.update(over)
    return lib.plaid_block_tables(*a.values())


@pytest.mark.parametrize("over", [dict(n=0), dict(n=-1), dict(lengths=None), dict(added=None), dict(table=None), dict(offsets=None), dict(totals=None),
                                  dict(wanted=None), dict(block_size=0), dict(block_size=24), dict(block_size=512), dict(max_blocks=0),
                                  dict(max_blocks=1 << 27, table_stride=1 << 27), dict(table_stride=7), dict(n_free=-1), dict(free_blocks=None), dict(capacity=-1),
                                  dict(positions=None), dict(slots=None), dict(slots=ODD), dict(positions=ODD), dict(offsets=4100), dict(n=3000)])
def test_block_tables_refusals(lib, over):
    assert _tables(lib, **over) == E
    assert pl.plaid_last_error()


def _cache(**over):
    a = dict(data=A, num_blocks=8, block_size=16, kv_heads=2, head_dim=128, dtype=0)
    a.update(over)
    return reader.plaid_paged_cache(*a.values())


BAD_CACHES = [dict(block_size=8), dict(block_size=48), dict(head_dim=96), dict(head_dim=0), dict(dtype=2), dict(kv_heads=0), dict(num_blocks=-1),
              dict(data=None), dict(data=ODD), dict(num_blocks=1 << 32)]


@pytest.mark.parametrize("over", BAD_CACHES)
def test_cache_refusals(lib, over):
    c = _cache(**over)
    assert lib.plaid_cache_write(ct.byref(c), A, A, 256, 128, 256, 128, A, 4, 0, None) == E
    assert lib.plaid_cache_read(ct.byref(c), A, 4, A, A, 0, None) == E


def test_cache_call_refusals(lib):
    c = ct.byref(_cache())

    def write(k=A, v=A, ks=256, kh=128, vs=256, vh=128, slots=A, n=4):
        return lib.plaid_cache_write(c, k, v, ks, kh, vs, vh, slots, n, 0, None)

    for over in (dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD), dict(ks=12), dict(kh=4), dict(vs=-256), dict(vh=1 << 24), dict(slots=None), dict(slots=4100), dict(n=-1)):
        assert write(**over) == E, over
    assert write(n=0) == plaid.PLAID_OK  # nothing to write: nothing is launched
    assert lib.plaid_cache_write(None, A, A, 256, 128, 256, 128, A, 4, 0, None) == E
    assert lib.plaid_cache_read(c, None, 4, A, A, 0, None) == E
    assert lib.plaid_cache_read(c, A, 4, ODD, A, 0, None) == E
    assert lib.plaid_cache_read(c, A, 0, A, A, 0, None) == plaid.PLAID_OK


def _args(**over):
    a = dict(dtype=0, n=2, heads=8, kv_heads=2, head_dim=128, scale=0.1, num_queries=6, num_keys=40, q=A, k=A, v=A, key_bias=None, q_token_stride=1024,
             q_head_stride=128, k_token_stride=256, k_head_stride=128, v_token_stride=256, v_head_stride=128, q_offsets=A, k_offsets=A, out=A, lse=A)
    a.update(over)
    return reader.plaid_attention(*a.values())


BAD_SHAPES = [dict(dtype=3), dict(n=0), dict(heads=7), dict(heads=0), dict(kv_heads=0), dict(head_dim=80), dict(num_queries=-1), dict(num_keys=-1),
              dict(num_keys=(1 << 30) + 1), dict(num_queries=1 << 31), dict(heads=1 << 14, kv_heads=2), dict(heads=8192, kv_heads=2, num_queries=1 << 20)]
BAD_QUERIES = [dict(q=None), dict(q=ODD), dict(q_token_stride=1020), dict(q_head_stride=4), dict(q_token_stride=1 << 24), dict(q_head_stride=-128),
               dict(q_offsets=None), dict(q_offsets=4100), dict(out=None), dict(out=ODD), dict(lse=4100)]
BAD_KEYS = [dict(k=None), dict(v=None), dict(k=ODD), dict(v=ODD), dict(k_token_stride=4), dict(v_head_stride=4), dict(k_offsets=None), dict(key_bias=4097)]


@pytest.mark.parametrize("over", BAD_SHAPES + BAD_QUERIES + BAD_KEYS)
def test_cross_attention_refusals(lib, over):
    a = _args(**over)
    big = 1 << 30
    assert lib.plaid_cross_attention(ct.byref(a), A, big, 0, None) == E
    assert lib.plaid_cross_attention_backward(ct.byref(a), A, A, A, A, None, A, big, 0, None) == E
    need = ct.c_int64(-1)
    for backward in (0, 1):
        assert lib.plaid_cross_attention_workspace(ct.byref(a), backward, ct.byref(need)) == (E if over in BAD_SHAPES else plaid.PLAID_OK)


@pytest.mark.parametrize("over", BAD_SHAPES[:-1] + BAD_QUERIES)
def test_cached_attention_refusals(lib, over):
    a = _args(**over)
    if over in BAD_SHAPES and ("num_keys" in over):
        return
    assert lib.plaid_cached_attention(ct.byref(a), ct.byref(_cache()), A, 8, 8, A, 1, A, 1 << 30, 0, None) == E


def test_cached_attention_refuses_what_does_not_fit_together(lib):
    def call(a=None, c=None, table=A, stride=8, blocks=8, lengths=A, work=A, size=1 << 30):
        return lib.plaid_cached_attention(ct.byref(a or _args()), ct.byref(c or _cache()), table, stride, blocks, lengths, 1, work, size, 0, None)

    assert call(c=_cache(kv_heads=4)) == E and call(c=_cache(head_dim=64)) == E and call(c=_cache(dtype=1)) == E
    assert call(table=None) == E and call(lengths=None) == E and call(stride=7) == E and call(blocks=0) == E and call(blocks=1 << 27, stride=1 << 27) == E
    for over in BAD_CACHES:
        assert call(c=_cache(**over)) == E


def test_backward_refusals_and_workspace(lib):
    a = _args(key_bias=A)
    need = ct.c_int64(-1)
    assert lib.plaid_cross_attention_workspace(ct.byref(a), 1, ct.byref(need)) == plaid.PLAID_OK and need.value > 0
    bw = lib.plaid_cross_attention_backward
    assert bw(ct.byref(a), None, A, A, A, A, A, need.value, 0, None) == E            # no d_out
    assert bw(ct.byref(_args(lse=None)), A, A, A, A, None, A, need.value, 0, None) == E
    assert bw(ct.byref(a), ODD, A, A, A, A, A, need.value, 0, None) == E
    assert bw(ct.byref(a), A, ODD, A, A, A, A, need.value, 0, None) == E
    assert bw(ct.byref(_args()), A, A, A, A, A, A, need.value, 0, None) == E          # dbias without a bias
    assert bw(ct.byref(a), A, A, A, A, A, A, need.value - 1, 0, None) == E            # the workspace is a byte short
    assert bw(ct.byref(a), A, A, A, A, A, ODD, need.value, 0, None) == E
    assert bw(ct.byref(a), A, A, A, A, A, None, need.value, 0, None) == E
    assert "workspace" in pl.plaid_last_error()
    assert lib.plaid_cross_attention_workspace(ct.byref(a), 0, None) == E
    assert lib.plaid_cross_attention_workspace(None, 0, ct.byref(need)) == E


def test_workspaces_hold_partial_sums_only_where_work_is_split(lib):
    need = ct.c_int64(-1)

    def forward(**over):
        assert lib.plaid_cross_attention_workspace(ct.byref(_args(**over)), 0, ct.byref(need)) == plaid.PLAID_OK
        return need.value

    assert forward(n=64, num_queries=64 * 512, num_keys=64 * 4000) == 0         # enough tiles for every compute unit
    assert forward(n=1, num_queries=1, num_keys=60_000) > 0                     # one token: cut along the keys
    assert forward(n=1, num_queries=1, num_keys=60_000) == forward(n=1, num_queries=1, num_keys=600_000)
    assert lib.plaid_cached_attention_workspace(ct.byref(_args(n=1, num_queries=1)), 1, 16, ct.byref(need)) == plaid.PLAID_OK
    assert lib.plaid_block_tables_workspace(16, 100, ct.byref(need)) == plaid.PLAID_OK and need.value == 0
    assert lib.plaid_block_tables_workspace(5000, 100, ct.byref(need)) == plaid.PLAID_OK and need.value == 2 * 5001 * 8


def test_binding_refuses_what_is_not_on_a_gpu_or_of_another_type():
    f = torch.zeros(2, 1, 64, dtype=torch.bfloat16)
    i = torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):
        pl.plaid_cross_attention(f, f, f, i, i)
    with pytest.raises(ValueError):
        pl.PagedCache(torch.zeros(4, 1, 16 * 64 * 17 // 16, dtype=torch.uint8), 16, 64, torch.bfloat16)
    with pytest.raises(ValueError):
        pl.plaid_block_tables(torch.zeros(2, dtype=torch.int32), torch.zeros(2, dtype=torch.int32), torch.zeros(2, 4, dtype=torch.int32),
                              torch.zeros(4, dtype=torch.int32), 16, 8)
