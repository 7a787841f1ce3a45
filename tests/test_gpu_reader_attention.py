"""Attention over the cache and cross attention with its gradients on the GPU, against the definitions in 64 bits within bounds
that follow from what is rounded (reader_util)."""
import math

import pytest
import torch

import reader_util as ru

pytestmark = pytest.mark.gpu
DEV = "cuda:0"
BF, HF = torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl_
    pl_.load_library()
    return pl_


def _off(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int64).cumsum(0).to(DEV)


def _randn(shape, seed, dtype, gain=1.0):
    return (torch.randn(shape, generator=torch.Generator().manual_seed(seed)) * gain).to(dtype)


# ------------------------------------------------------------------------------------------------ over the cache
def _filled_cache(pl, lengths, bs, kv_heads, dim, dtype, width=None, seed=0, poison=True):
    """A cache with the requests' tokens at random blocks, and bytes that stand for values that are not finite everywhere else."""
    counts = [-(-n // bs) for n in lengths]
    blocks = sum(counts) + 3
    width = width or max(1, max(counts))
    g = torch.Generator().manual_seed(seed)
    ids = torch.randperm(blocks, generator=g)[:sum(counts)].int()
    table = torch.full((len(lengths), width), -1, dtype=torch.int32)
    cache = pl.PagedCache.empty(blocks, bs, kv_heads, dim, dtype, DEV)
    if poison:
        cache.data.fill_(255)
    at, keys, values = 0, [], []
    for r, (n, c) in enumerate(zip(lengths, counts)):
        table[r, :c] = ids[at:at + c]
        at += c
        t = torch.arange(n)
        slots = table[r, t // bs].long() * bs + t % bs
        k, v = _randn((n, kv_heads, dim), seed + 2 * r + 1, dtype, 1.5), _randn((n, kv_heads, dim), seed + 2 * r + 2, dtype)
        pl.plaid_cache_write(cache, k.to(DEV), v.to(DEV), slots.to(DEV))
        keys.append(ru.value_of(*ru.quantise(k)))
        values.append(ru.value_of(*ru.quantise(v)))
    return cache, table, keys, values


def _check_cached(pl, q_lengths, k_lengths, heads, kv_heads, dim, bs, dtype, causal=True, scale=None, hide=(), width=None, seed=0):
    cache, table, keys, values = _filled_cache(pl, k_lengths, bs, kv_heads, dim, dtype, width, seed)
    for r, b in hide:
        table[r, b] = -1 if (r + b) % 2 else cache.num_blocks + 5       # a block that is not there
    q = _randn((sum(q_lengths), heads, dim), seed + 99, dtype)
    scale = dim ** -0.5 if scale is None else scale
    out, lse = pl.plaid_cached_attention(q.to(DEV), cache, table.to(DEV), torch.tensor(k_lengths, dtype=torch.int32, device=DEV), _off(q_lengths),
                                         scale=scale, causal=causal, return_lse=True)
    again = pl.plaid_cached_attention(q.to(DEV), cache, table.to(DEV), torch.tensor(k_lengths, dtype=torch.int32, device=DEV), _off(q_lengths),
                                      scale=scale, causal=causal)
    assert torch.equal(out, again)                                       # the same bits, with lse or without
    a = 0
    for r, (m, n) in enumerate(zip(q_lengths, k_lengths)):
        place = torch.arange(n)
        there = torch.ones(n, dtype=torch.bool)
        for rr, b in hide:
            if rr == r:
                there &= place // bs != b
        seen = there[None].expand(m, n)
        if causal:
            seen = seen & (place[None] < n - m + torch.arange(m)[:, None] + 1)
        for h in range(heads):
            g = h * kv_heads // heads
            x = ru.attend(q[a:a + m, h], keys[r][:, g], values[r][:, g], scale, None, seen, None, dtype)
            ru.close(out[a:a + m, h], x["out"], x["out_bound"], f"out of request {r} head {h}")
            ru.close(lse[a:a + m, h].double().sum(-1), x["lse"], x["lse_bound"], f"lse of request {r} head {h}")
        a += m


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,bs,heads,kv_heads", [(128, 16, 8, 2), (64, 16, 3, 1), (128, 64, 4, 4), (64, 256, 6, 3), (128, 32, 16, 1), (64, 128, 40, 2)])
def test_cached_single_tokens(pl, dtype, dim, bs, heads, kv_heads):
    lengths = [1, 2, 15, 16, 17, 31, 33, 127, 129, 300, 0, 64]
    _check_cached(pl, [1] * len(lengths), lengths, heads, kv_heads, dim, bs, dtype)


@pytest.mark.parametrize("length", [0, 1, 128, 129, 700, 2000, 5001])
def test_cached_one_request(pl, length):
    _check_cached(pl, [1], [length], 8, 2, 128, 16, BF)
    _check_cached(pl, [1], [length], 4, 4, 64, 64, HF, width=200)        # a table far wider than the request


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype", [BF, HF])
def test_cached_few_tokens(pl, dtype, causal):
    """Several tokens a request in the kernel for few rows: more rows than a tile, some before any key, requests without tokens."""
    _check_cached(pl, [3, 0, 7, 1, 12, 2], [40, 9, 7, 0, 5, 333], 6, 2, 128, 16, dtype, causal)
    _check_cached(pl, [9, 3], [9, 200], 2, 1, 64, 32, dtype, causal)


@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("dtype,dim,bs", [(BF, 128, 16), (HF, 64, 32), (BF, 64, 128), (HF, 128, 256)])
def test_cached_prompts(pl, dtype, dim, bs, causal):
    """Tiles of rows: whole prompts, pieces behind a context, lengths around the tiles' edges, more tokens than keys."""
    _check_cached(pl, [70, 33, 0, 129, 64], [70, 200, 50, 129, 63], 4, 2, dim, bs, dtype, causal)
    _check_cached(pl, [300], [450], 2, 1, dim, bs, dtype, causal)
    _check_cached(pl, [40], [1500], 4, 4, dim, bs, dtype, causal)        # split over the keys


def test_cached_hidden_blocks(pl):
    for m in (1, 40):
        _check_cached(pl, [m, m, m], [100, 64, 50], 4, 2, 128, 16, BF, False, hide=[(0, 1), (0, 6), (1, 0), (1, 1), (1, 2), (1, 3), (2, 3)])
        _check_cached(pl, [m], [700], 2, 2, 64, 32, HF, True, hide=[(0, 20), (0, 3), (0, 21)])


@pytest.mark.parametrize("scale", [0.0, -0.2, 1.0])
def test_cached_scales(pl, scale):
    _check_cached(pl, [1, 1], [77, 300], 4, 2, 128, 16, BF, scale=scale)
    _check_cached(pl, [50], [300], 4, 2, 64, 16, HF, scale=scale)


def test_cached_refusals(pl):
    cache = pl.PagedCache.empty(4, 16, 2, 64, BF, DEV)
    q = torch.zeros(2, 4, 64, dtype=BF, device=DEV)
    table, lengths, off = torch.zeros(2, 2, dtype=torch.int32, device=DEV), torch.ones(2, dtype=torch.int32, device=DEV), _off([1, 1])
    pl.plaid_cached_attention(q, cache, table, lengths, off)
    for bad in (dict(q=q.half()), dict(q=q[:, :3]), dict(q=torch.zeros(2, 4, 128, dtype=BF, device=DEV)), dict(q=q.cpu()), dict(table=table.long()),
                dict(table=table[:1]), dict(lengths=lengths.long()), dict(off=off[:2]), dict(off=off.int())):
        a = dict(q=q, table=table, lengths=lengths, off=off)
        a.update(bad)
        with pytest.raises(ValueError):
            pl.plaid_cached_attention(a["q"], cache, a["table"], a["lengths"], a["off"])
    with pytest.raises(ValueError):
        pl.plaid_cache_write(cache, torch.zeros(1, 3, 64, dtype=BF, device=DEV), torch.zeros(1, 2, 64, dtype=BF, device=DEV), torch.zeros(1, dtype=torch.int64, device=DEV))
    with pytest.raises(pl.PlaidError):
        pl.plaid_cached_attention(q, cache, torch.zeros(2, 0, dtype=torch.int32, device=DEV), lengths, off)


# ------------------------------------------------------------------------------------------------ cross attention
def _check_cross(pl, q_lengths, k_lengths, heads, kv_heads, dim, dtype, bias=None, train=True, scale=None, gain=1.0, change=None, seed=0):
    nq, nk = sum(q_lengths), sum(k_lengths)
    q, k, v = _randn((nq, heads, dim), seed + 1, dtype, gain), _randn((nk, kv_heads, dim), seed + 2, dtype), _randn((nk, kv_heads, dim), seed + 3, dtype)
    d_out = _randn((nq, heads, dim), seed + 4, dtype, 0.25) if train else None
    if change:
        change(q, k, v)
    scale = dim ** -0.5 if scale is None else scale
    d = lambda t: None if t is None else t.to(DEV)  # noqa: E731
    qo, ko = _off(q_lengths), _off(k_lengths)
    out, lse = pl.plaid_cross_attention(d(q), d(k), d(v), qo, ko, key_bias=d(bias), scale=scale, return_lse=True)
    want = ru.cross(q, k, v, q_lengths, k_lengths, scale, bias, d_out)
    ru.close(out, want["out"], want["out_bound"], "out")
    low = want["lse"] < -1e30                                            # beside such a reference the rest of the sum is a number of its own
    ru.close(lse.double().sum(-1).cpu()[~low], want["lse"][~low], want["lse_bound"][~low], "lse")
    if not train:
        return out
    grads = pl.plaid_cross_attention_backward(d(d_out), d(q), d(k), d(v), out, lse, qo, ko, key_bias=d(bias), scale=scale)
    for name, g in zip(("dq", "dk", "dv", "dbias"), grads):
        if g is not None:
            ru.close(g, want[name], want[name + "_bound"], name)
    assert (grads[3] is None) == (bias is None)
    again = pl.plaid_cross_attention_backward(d(d_out), d(q), d(k), d(v), out, lse, qo, ko, key_bias=d(bias), scale=scale)
    for x, y in zip(grads, again):
        assert x is None or torch.equal(x, y)                            # the same bits
    return grads


def _bias(n, seed, dtype, masked=0.2):
    g = torch.Generator().manual_seed(seed)
    b = torch.randn(n, generator=g) * 2
    return b.masked_fill(torch.rand(n, generator=g) < masked, -math.inf).to(dtype)


@pytest.mark.parametrize("with_bias", [False, True])
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,heads,kv_heads", [(64, 3, 3), (128, 4, 1), (128, 6, 2), (64, 8, 1)])
def test_cross_attention_and_gradients(pl, dim, heads, kv_heads, dtype, with_bias):
    q_lengths, k_lengths = [1, 17, 0, 33, 70, 5, 64], [3, 65, 12, 0, 129, 1, 64]
    bias = _bias(sum(k_lengths), 8, dtype) if with_bias else None
    _check_cross(pl, q_lengths, k_lengths, heads, kv_heads, dim, dtype, bias)


@pytest.mark.parametrize("m,n", [(1, 1), (1, 500), (2, 31), (31, 32), (33, 33), (200, 3), (300, 257), (1, 3000), (700, 40), (130, 1000)])
def test_cross_attention_shapes(pl, m, n):
    """One request: lengths around the tiles' edges, rows split over keys and keys over rows."""
    _check_cross(pl, [m], [n], 2, 1, 128, BF, _bias(n, 5, BF, 0.1))
    _check_cross(pl, [m], [n], 2, 2, 64, HF)


@pytest.mark.parametrize("heads,kv_heads", [(5, 5), (12, 4), (7, 1), (9, 3)])
def test_cross_attention_groups_that_do_not_divide_a_tile(pl, heads, kv_heads):
    _check_cross(pl, [40, 7, 21], [90, 130, 5], heads, kv_heads, 64, BF, _bias(225, 2, BF))
    _check_cross(pl, [1, 1, 1], [90, 130, 5], heads, kv_heads, 128, HF, train=False)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_masked_keys_may_hold_anything(pl, dtype):
    lengths = [50, 140, 33]
    bias = _bias(sum(lengths), 3, dtype, 0.3)
    bias[:50] = -math.inf                                                # a request with every key masked
    bias[sum(lengths) - 1] = -math.inf                                   # the last key, which others may stand in for

    def poison(q, k, v):
        for i in torch.nonzero(bias == -math.inf).flatten().tolist():
            k[i] = (math.nan, math.inf, -math.inf)[i % 3]
            v[i] = (math.inf, math.nan, -math.inf)[i % 3]

    for q_lengths in ([1, 1, 1], [40, 33, 64]):
        _check_cross(pl, q_lengths, lengths, 4, 2, 128, dtype, bias, change=poison)
        _check_cross(pl, q_lengths, lengths, 2, 2, 64, dtype, bias, change=poison)


@pytest.mark.parametrize("dtype", [BF, HF])
def test_masks_of_the_lowest_value(pl, dtype):
    """A finite mask: beside other keys it hides, a row of nothing else weighs its keys alike (bf16: the scores vanish beside it)."""
    lengths = [40, 70, 33]
    low = torch.finfo(dtype).min
    bias = _bias(sum(lengths), 3, dtype, 0.0)
    bias[::3] = low
    bias[:40] = low
    for q_lengths in ([1, 1, 1], [40, 33, 64]):
        _check_cross(pl, q_lengths, lengths, 4, 2, 128, dtype, bias)
        mixed = bias.clone()
        mixed[:40:2] = -math.inf
        _check_cross(pl, q_lengths, lengths, 2, 1, 64, dtype, mixed)


def test_values_that_are_not_finite_stay_visible(pl):
    """A key that is not masked and holds a value that is not finite makes its request's rows not finite, and no other's."""
    for m in (1, 40):
        q, k, v = _randn((2 * m, 2, 64), 1, BF).to(DEV), _randn((160, 2, 64), 2, BF).to(DEV), _randn((160, 2, 64), 3, BF).to(DEV)
        k[100, 0, 5] = math.nan
        v[30, 1, 7] = math.inf
        out = pl.plaid_cross_attention(q, k, v, _off([m, m]), _off([80, 80]))
        assert torch.isnan(out[m:, 0]).all() and torch.isfinite(out[m:, 1]).all() and torch.isfinite(out[:m, 0]).all()
        assert torch.isinf(out[:m, 1, 7]).all() and torch.isfinite(out[:m, 1, :7]).all()
        bias = torch.full((160,), -math.inf, dtype=BF, device=DEV)
        q[0, 0, 0] = math.nan                                            # not finite, but nothing to attend to
        out = pl.plaid_cross_attention(q, k, v, _off([m, m]), _off([80, 80]), key_bias=bias)
        assert (out == 0).all()


@pytest.mark.parametrize("scale", [0.0, -0.3, 2.0])
def test_cross_scales(pl, scale):
    for bias in (None, _bias(150, 4, BF)):
        _check_cross(pl, [40, 30], [90, 60], 4, 2, 64, BF, bias, scale=scale)
        _check_cross(pl, [1, 1], [90, 60], 4, 2, 128, BF, bias, scale=scale, train=False)


def test_scores_of_hundreds(pl):
    """Weights of one key alone, scores far beyond the exponential's range: maxima move, nothing overflows."""
    for dtype in (BF, HF):
        _check_cross(pl, [1, 40], [300, 333], 2, 1, 64, dtype, gain=20.0, train=False)
        _check_cross(pl, [1, 40], [300, 333], 2, 1, 128, dtype, _bias(633, 2, dtype), gain=20.0, train=False)


def test_gradients_against_differences(pl):
    """The gradients' products with random directions against differences of the plain forward pass in 64 bits.  The bound is what
    the gradients' elementwise bounds allow along the direction, and the differences' own error."""
    q_lengths, k_lengths, heads, kv_heads, dim, dtype = [9, 20], [30, 41], 4, 2, 64, HF
    q, k, v, d_out = (_randn(s, i, dtype) for i, s in enumerate([(29, heads, dim), (71, kv_heads, dim), (71, kv_heads, dim), (29, heads, dim)]))
    bias = _bias(71, 9, dtype, 0.0)
    d = lambda t: t.to(DEV)  # noqa: E731
    qo, ko = _off(q_lengths), _off(k_lengths)
    out, lse = pl.plaid_cross_attention(d(q), d(k), d(v), qo, ko, key_bias=d(bias), return_lse=True)
    grads = pl.plaid_cross_attention_backward(d(d_out), d(q), d(k), d(v), out, lse, qo, ko, key_bias=d(bias))
    want = ru.cross(q, k, v, q_lengths, k_lengths, dim ** -0.5, bias, d_out)

    def loss(q, k, v, b):
        total, a, c = 0.0, 0, 0
        for m, n in zip(q_lengths, k_lengths):
            for h in range(heads):
                s = q[a:a + m, h] @ k[c:c + n, h // 2].T * dim ** -0.5 + b[c:c + n]
                total += float((torch.softmax(s, -1) @ v[c:c + n, h // 2] * d_out[a:a + m, h].double()).sum())
            a, c = a + m, c + n
        return total

    at = [t.double() for t in (q, k, v, bias)]
    for i, name in enumerate(("dq", "dk", "dv", "dbias")):
        direction = torch.randn(at[i].shape, generator=torch.Generator().manual_seed(50 + i), dtype=torch.float64)
        step = 1e-4
        moved = [[t + (sign * step * direction if j == i else 0) for j, t in enumerate(at)] for sign in (1, -1)]
        slope = (loss(*moved[0]) - loss(*moved[1])) / (2 * step)
        got = float((grads[i].double().cpu() * direction).sum())
        assert abs(got - slope) <= float((want[name + "_bound"] * direction.abs()).sum()) + 1e-4 * abs(slope) + 1e-6, (name, got, slope)


def test_strided_inputs(pl):
    """Views of a fused projection, transposed heads, one tensor for all tokens (stride 0), rows that are not 16-byte aligned."""
    x = _randn((60, 8, 64), 1, BF).to(DEV)
    q, k, v = x[:, :4], x[:, 4:6], x[:, 6:]
    qo, ko = _off([20, 40]), _off([35, 25])
    want = pl.plaid_cross_attention(q.contiguous(), k.contiguous(), v.contiguous(), qo, ko)
    assert torch.equal(pl.plaid_cross_attention(q, k, v, qo, ko), want)
    t = lambda y: y.transpose(0, 1).contiguous().transpose(0, 1)  # noqa: E731
    assert torch.equal(pl.plaid_cross_attention(t(q), t(k), t(v), qo, ko), want)
    flat = torch.empty(60 * 4 * 64 + 1, dtype=BF, device=DEV)
    odd = flat[1:].view(60, 4, 64)
    odd.copy_(q)
    assert torch.equal(pl.plaid_cross_attention(odd, k, v, qo, ko), want)
    one = _randn((1, 2, 64), 5, BF).to(DEV).expand(60, 2, 64)
    assert torch.equal(pl.plaid_cross_attention(q, one, one, qo, ko), pl.plaid_cross_attention(q, one.contiguous(), one.contiguous(), qo, ko))
    d_out = _randn((60, 4, 64), 7, BF).to(DEV)
    out, lse = pl.plaid_cross_attention(q, k, v, qo, ko, return_lse=True)
    a = pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, qo, ko)
    b = pl.plaid_cross_attention_backward(t(d_out), t(q), t(k), t(v), t(out), lse, qo, ko)
    for y, z in zip(a[:3], b[:3]):
        assert torch.equal(y, z)


def test_rows_of_no_request_are_not_written(pl):
    q, k = _randn((50, 2, 64), 1, BF).to(DEV), _randn((80, 2, 64), 2, BF).to(DEV)
    off = torch.tensor([5, 20, 45], device=DEV)
    ko = torch.tensor([10, 40, 70], device=DEV)
    whole = pl.plaid_cross_attention(q[5:45].contiguous(), k[10:70].contiguous(), k[10:70].contiguous(), off - 5, ko - 10)
    part = pl.plaid_cross_attention(q, k, k, off, ko)
    assert torch.equal(part[5:45], whole)


def test_another_stream_and_graph_replay(pl):
    """Calls on a stream of their own, and captured: replays give the eager bits, with other work between them."""
    lengths = [40, 333, 1, 90]
    bias = _bias(sum(lengths), 3, BF).to(DEV)
    q, k, v, d_out = (_randn((n, h, 128), i, BF).to(DEV) for i, (n, h) in enumerate([(100, 4), (464, 2), (464, 2), (100, 4)]))
    qo, ko = _off([10, 60, 20, 10]), _off(lengths)
    cache = pl.PagedCache.empty(40, 16, 2, 128, BF, DEV)
    table = torch.full((4, 24), -1, dtype=torch.int32, device=DEV)
    old, new = torch.tensor([0, 0, 0, 0], dtype=torch.int32, device=DEV), torch.tensor([40, 100, 1, 90], dtype=torch.int32, device=DEV)
    free = torch.arange(40, dtype=torch.int32, device=DEV).flip(0).contiguous()
    single = _randn((4, 4, 128), 9, BF).to(DEV)
    one = _off([1, 1, 1, 1])

    def work():
        offsets, totals, _, slots, _ = pl.plaid_block_tables(old, new, table, free, 16, 231)
        pl.plaid_cache_write(cache, k[:231], v[:231], slots)
        step = pl.plaid_cached_attention(single, cache, table, totals, one)
        out, lse = pl.plaid_cross_attention(q, k, v, qo, ko, key_bias=bias, return_lse=True)
        return (step, out) + pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, qo, ko, key_bias=bias)

    eager = [t.clone() for t in work()]
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        there = work()
    torch.cuda.current_stream().wait_stream(side)
    for a, b in zip(eager, there):
        assert torch.equal(a, b)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = work()
    for i in range(4):
        for t in captured:
            t.fill_(i)
        cache.data.fill_(i)
        work()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(eager, captured):
            assert torch.equal(a, b), i
