"""The operators of a reader that answers from what a search has found, as cases that can be timed and compared.

A search returns passages, and plaid_decompress_passages their token vectors.  A reader is a decoder whose layers attend to the
tokens written so far and to the states of the passages found.  Its operators here:

* ``tables``: plaid_block_tables -- the blocks of a paged cache handed to each request, and the slot of every new token, from
  the requests' lengths;
* ``cache``: plaid_cache_write and plaid_cache_read -- new keys and values into that cache, which holds four bits a value, and back;
* ``cached``: plaid_cached_attention -- attention of a step's new tokens over that cache;
* ``cross``: plaid_cross_attention -- attention to the states of the passages found, one new token a request;
* ``train``: plaid_cross_attention and plaid_cross_attention_backward -- the same for whole answers, with all gradients, the
  retrieval bias's among them.

The cache's bytes: for every block and key head, the codes of the keys, the codes of the values, the scales of the keys, the
scales of the values.  A code is a 4-bit float (sign, 2 bits of exponent, 1 of mantissa: 0 0.5 1 1.5 2 3 4 6), a scale the biased
exponent of a power of two for 32 dimensions of one token and head, 255 for a group that is not finite.  Keys lie row by row, two
dimensions a byte, the even one in the low half.  Values lie in cells of 16 tokens as [token / 4][dim % 16][dim / 32][token % 4],
a byte's halves being dims 32 i + m and 32 i + 16 + m.
"""
import math
import random

import numpy as np
import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16}
GROUP = 32  # values under one scale
CELL = 16  # tokens of a cell of the value codes


# ------------------------------------------------------------------------------------------------ cases
def _tables(name, n, old, new, block_size, shorter=False):
    return {"name": name, "kind": "tables", "n": n, "old_lo": old[0], "old_hi": old[1], "new_lo": new[0], "new_hi": new[1],
            "block_size": block_size, "shorter": shorter}


def _cache(name, tokens, heads, dim, block_size, dtype):
    return {"name": name, "kind": "cache", "tokens": tokens, "kv_heads": heads, "dim": dim, "block_size": block_size, "dtype": dtype}


def _cached(name, n, q, keys, heads, kv_heads, dim, block_size, dtype, causal=True):
    return {"name": name, "kind": "cached", "n": n, "q_lo": q[0], "q_hi": q[1], "k_lo": keys[0], "k_hi": keys[1], "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "block_size": block_size, "dtype": dtype, "causal": causal}


def _cross(name, kind, n, q, keys, heads, kv_heads, dim, dtype, bias):
    return {"name": name, "kind": kind, "n": n, "q_lo": q[0], "q_hi": q[1], "k_lo": keys[0], "k_hi": keys[1], "heads": heads,
            "kv_heads": kv_heads, "dim": dim, "dtype": dtype, "bias": bias}


def listed():
    return [
        # a decode step of sixteen running requests: one token each, now and then a new block
        _tables("tables_step", 16, (1, 2000), (1, 1), 16),
        # a thousand questions admitted at once, each with the hundred passages found for it as its prompt
        _tables("tables_prompts", 1000, (0, 0), (3000, 10_000), 16),
        # a decode step's keys and values of 64 requests
        _cache("cache_step", 64, 8, 128, 16, "bf16"),
        # the keys and values of ten prompts of a hundred passages
        _cache("cache_prompts", 65_003, 8, 128, 32, "bf16"),
        # one user, one token, a context of ten passages: nothing to fill the chip with
        _cached("cached_one", 1, (1, 1), (677, 677), 32, 8, 128, 16, "bf16"),
        # a serving batch, one token a request, contexts of every length
        _cached("cached_batch", 64, (1, 1), (1, 8192), 32, 8, 128, 16, "fp16"),
        # few requests with very long contexts
        _cached("cached_long", 4, (1, 1), (100_000, 131_072), 32, 8, 128, 64, "bf16"),
        # prompts taken in pieces behind a context: many tokens a request, each seeing what is before it
        _cached("cached_prompts", 6, (200, 1500), (1500, 8000), 32, 8, 128, 32, "bf16"),
        # one token that attends to ten passages
        _cross("cross_one", "cross", 1, (1, 1), (605, 605), 12, 12, 64, "fp16", False),
        # one token a request that attends to a thousand passages
        _cross("cross_thousand", "cross", 4, (1, 1), (60_000, 70_000), 32, 8, 128, "bf16", True),
        # training on short answers to ten passages, with dropped tokens, requests without passages among them
        _cross("train_short", "train", 16, (1, 63), (0, 900), 12, 12, 64, "fp16", True),
        # training on long answers to a hundred passages
        _cross("train_long", "train", 16, (400, 512), (4500, 8000), 16, 4, 128, "bf16", True),
    ]


def _log_uniform(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["tables", "cache", "cached", "cached", "cross", "train", "train"])
    dtype, dim, block_size = rng.choice(["bf16", "fp16"]), rng.choice([64, 128]), rng.choice([16, 32, 64, 128])
    kv_heads = rng.choice([1, 2, 4, 5, 8, 12])
    heads = kv_heads * rng.choice([1, 1, 2, 3, 4, 8] if kv_heads <= 4 else [1, 1, 2, 3, 4])
    if kind == "tables":
        n = _log_uniform(rng, 1, 3000)
        old = _log_uniform(rng, 1, 20_000)
        if rng.random() < 0.5:
            c = _tables("", n, (0, old), (0, rng.choice([1, 1, 5])), block_size, rng.random() < 0.3)
        else:
            c = _tables("", n, (0, rng.choice([0, old])), (0, _log_uniform(rng, 2, min(20_000, 12_000_000 // n))), block_size, rng.random() < 0.3)
    elif kind == "cache":
        tokens = _log_uniform(rng, 1, 65_003)
        while tokens * kv_heads * dim > 65_003 * 8 * 128:
            kv_heads = max(1, kv_heads // 2)
        c = _cache("", tokens, kv_heads, dim, block_size, dtype)
    else:
        # rows of queries, keys of a request and requests within what the largest listed case of the kind has
        single = kind == "cross" or (kind == "cached" and rng.random() < 0.5)
        q_hi = 1 if single else _log_uniform(rng, 2, 600 if kind == "train" else 1500)
        k_hi = _log_uniform(rng, 1, 8000 if not single else 131_072)
        room = min(4 * 131_072 * 8 * 128 / (k_hi * kv_heads * dim), (4e8 if kind == "train" else 1.5e9) / (heads * q_hi * k_hi))
        if kind == "train":
            room = min(room, 16 * 512 * 8000 * 16 * 128 / (q_hi * k_hi * heads * dim))
        n = _log_uniform(rng, 1, max(1, min(64, int(room))))
        q = (1, 1) if single else (1, q_hi)
        keys = (k_hi // rng.choice([1, 2, 1000]), k_hi)
        if kind == "cached":
            causal = single or rng.random() < 0.8
            c = _cached("", n, q, (max(keys[0], q_hi) if causal else keys[0], max(k_hi, q_hi)), heads, kv_heads, dim, block_size, dtype, causal)
        else:
            c = _cross("", kind, n, q, keys, heads, kv_heads, dim, dtype, rng.random() < 0.6)
    del c["name"]
    return c


def _lengths(case, what):
    """The requests' lengths: the case's, whatever the seed; the first and the last are the ends of the range."""
    rng = random.Random("%s %d %d %d" % (what, case["n"], case[what + "_lo"], case[what + "_hi"]))
    lo, hi = case[what + "_lo"], case[what + "_hi"]
    got = [rng.randint(lo, hi) for _ in range(case["n"])]
    got[0] = hi
    if case["n"] > 1:
        got[-1] = lo
    return got


def _attention_lengths(case):
    q, k = _lengths(case, "q"), _lengths(case, "k")
    if case.get("causal"):  # the new tokens are in the cache
        k = [max(a, b) for a, b in zip(q, k)]
    return q, k


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed((seed * 1_000_003 + stream) & 0x7FFFFFFFFFFFFFFF)
    return g


def _normal(shape, seed, stream, dtype, spread=0.0):
    """Unit normal values; with a spread, the last axis's channels have gains around one, as keys have them."""
    g = _generator(seed, stream)
    x = torch.randn(shape, generator=g, device="cuda")
    if spread:
        x *= torch.exp(spread * torch.randn(shape[-1], generator=g, device="cuda"))
    return x.to(dtype)


def _offsets(lengths):
    return torch.tensor([0] + list(np.cumsum(lengths)), dtype=torch.int64, device="cuda")


def _tables_inputs(case, seed):
    old, new, bs = _lengths(case, "old"), _lengths(case, "new"), case["block_size"]
    have = [-(-a // bs) for a in old]
    want = [-(-(a + b) // bs) - h for a, b, h in zip(old, new, have)]
    width = max(1, max(h + w for h, w in zip(have, want)) - (1 if case["shorter"] else 0))  # a table one block too narrow
    ids = torch.randperm(sum(have) + sum(want) + 7, generator=_generator(seed, 1), device="cuda").int()
    table = torch.full((case["n"], width), -1, dtype=torch.int32, device="cuda")
    filled = torch.arange(width, device="cuda")[None] < torch.tensor(have, device="cuda")[:, None]
    table[filled] = ids[:int(filled.sum())]
    free = ids[sum(have):]
    if case["shorter"]:
        free = free[:max(1, sum(want) - 3)]  # and too few blocks
    i32 = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    return {"lengths": i32(old), "added": i32(new), "table": table, "free_blocks": free.contiguous(), "block_size": bs, "capacity": sum(new)}


def _cache_inputs(case, seed):
    tokens, heads, dim, bs, dtype = case["tokens"], case["kv_heads"], case["dim"], case["block_size"], DTYPES[case["dtype"]]
    blocks = -(-tokens // bs) + 3
    # the layer's projection gives keys and values side by side, so both are views with a stride
    kv = torch.cat([_normal((tokens, heads, dim), seed, 1, dtype, 0.5), _normal((tokens, heads, dim), seed, 2, dtype)], dim=1)
    order = torch.randperm(blocks, generator=_generator(seed, 3), device="cuda")
    if tokens <= 256:  # a step: each token is in a block of its own request
        slots = torch.randperm(blocks * bs, generator=_generator(seed, 4), device="cuda")[:tokens]
    else:
        t = torch.arange(tokens, device="cuda")
        slots = order[t // bs] * bs + t % bs
    data = torch.zeros((blocks, heads, bs * dim + bs * dim // 16), dtype=torch.uint8, device="cuda")
    return {"k": kv[:, :heads], "v": kv[:, heads:], "slots": slots, "data": data, "block_size": bs, "dim": dim, "dtype": dtype}


def _cached_inputs(case, seed):
    nq, nk = _attention_lengths(case)
    heads, kv_heads, dim, bs, dtype = case["heads"], case["kv_heads"], case["dim"], case["block_size"], DTYPES[case["dtype"]]
    counts = [-(-a // bs) for a in nk]
    blocks = sum(counts) + 2
    width = max(1, max(counts))
    held = torch.arange(width, device="cuda")[None] < torch.tensor(counts, device="cuda")[:, None]
    table = torch.full((case["n"], width), -1, dtype=torch.int32, device="cuda")
    table[held] = torch.randperm(blocks, generator=_generator(seed, 1), device="cuda").int()[:sum(counts)]
    # a cache as it is after the writes: codes of normal values under scales that follow the channels' gains
    g = _generator(seed, 2)
    data = torch.empty((blocks, kv_heads, bs * dim + bs * dim // 16), dtype=torch.uint8, device="cuda")
    pick = torch.tensor([0, 0, 1, 1, 1, 2, 2, 2, 3, 3, 4, 4, 5, 6, 7, 5] + [8, 8, 9, 9, 9, 10, 10, 10, 11, 11, 12, 12, 13, 14, 15, 13],
                        dtype=torch.uint8, device="cuda")
    for a in range(0, blocks, 4096):
        part = data[a:a + 4096]
        byte = torch.randint(0, 1024, (part.shape[0], kv_heads, bs * dim), generator=g, device="cuda", dtype=torch.int32)
        part[:, :, :bs * dim] = pick[byte & 31] | (pick[byte >> 5] << 4)
        part[:, :, bs * dim:] = torch.randint(124, 127, (part.shape[0], kv_heads, bs * dim // 16), generator=g, device="cuda", dtype=torch.uint8)
    return {"q": _normal((sum(nq), heads, dim), seed, 3, dtype), "data": data, "table": table,
            "lengths": torch.tensor(nk, dtype=torch.int32, device="cuda"), "q_offsets": _offsets(nq), "block_size": bs, "dim": dim,
            "dtype": dtype, "scale": dim ** -0.5, "causal": case["causal"], "longest_q": max(nq), "longest_k": width * bs}


def _cross_inputs(case, seed):
    nq, nk = _attention_lengths(case)
    heads, kv_heads, dim, dtype = case["heads"], case["kv_heads"], case["dim"], DTYPES[case["dtype"]]
    kv = torch.cat([_normal((sum(nk), kv_heads, dim), seed, 2, dtype, 0.3), _normal((sum(nk), kv_heads, dim), seed, 3, dtype)], dim=1)
    bias = None
    if case["bias"]:
        # the scores of the passages, sixty tokens each, and tokens that nothing attends to (punctuation)
        g = _generator(seed, 4)
        bias = torch.randn(sum(nk) // 60 + 1, generator=g, device="cuda").repeat_interleave(60)[:sum(nk)]
        bias = bias.masked_fill(torch.rand(sum(nk), generator=g, device="cuda") < 0.1, -math.inf).to(dtype)
    # a loss's gradient is small; in 16 bits with a short exponent the loss is scaled up
    d_out = _normal((sum(nq), heads, dim), seed, 5, torch.float32) * (1.0 if dtype == torch.float16 else 0.02) if case["kind"] == "train" else None
    return {"q": _normal((sum(nq), heads, dim), seed, 1, dtype), "k": kv[:, :kv_heads], "v": kv[:, kv_heads:], "key_bias": bias,
            "q_offsets": _offsets(nq), "k_offsets": _offsets(nk), "scale": dim ** -0.5, "d_out": None if d_out is None else d_out.to(dtype),
            "longest_q": max(nq), "longest_k": max(1, max(nk))}


_INPUTS = {"tables": _tables_inputs, "cache": _cache_inputs, "cached": _cached_inputs, "cross": _cross_inputs, "train": _cross_inputs}


def prepare(case, seed):
    state = _INPUTS[case["kind"]](case, seed)
    state["kind"] = case["kind"]
    return state


# ------------------------------------------------------------------------------------------------ one pass
def run(state):
    return (_OWN if own else _PLAIN)[state["kind"]](state)


def _own_tables(s):
    import paper_2205_09707_amd as pl
    got = pl.plaid_block_tables(s["lengths"], s["added"], s["table"], s["free_blocks"], s["block_size"], s["capacity"])
    return (s["table"],) + tuple(got)


def _own_cache(s):
    import paper_2205_09707_amd as pl
    cache = pl.PagedCache(s["data"], s["block_size"], s["dim"], s["dtype"])
    pl.plaid_cache_write(cache, s["k"], s["v"], s["slots"])
    return pl.plaid_cache_read(cache, s["slots"])


def _own_cached(s):
    import paper_2205_09707_amd as pl
    cache = pl.PagedCache(s["data"], s["block_size"], s["dim"], s["dtype"])
    return pl.plaid_cached_attention(s["q"], cache, s["table"], s["lengths"], s["q_offsets"], scale=s["scale"], causal=s["causal"])


def _own_cross(s):
    import paper_2205_09707_amd as pl
    return pl.plaid_cross_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], key_bias=s["key_bias"], scale=s["scale"])


def _own_train(s):
    import paper_2205_09707_amd as pl
    out, lse = pl.plaid_cross_attention(s["q"], s["k"], s["v"], s["q_offsets"], s["k_offsets"], key_bias=s["key_bias"], scale=s["scale"],
                                        return_lse=True)
    grads = pl.plaid_cross_attention_backward(s["d_out"], s["q"], s["k"], s["v"], out, lse, s["q_offsets"], s["k_offsets"],
                                              key_bias=s["key_bias"], scale=s["scale"])
    return (out,) + tuple(g for g in grads if g is not None)


_OWN = {"tables": _own_tables, "cache": _own_cache, "cached": _own_cached, "cross": _own_cross, "train": _own_train}


# ------------------------------------------------------------------------------------------------ the plain forms
def _plain_tables(s):
    old, new, bs, free = s["lengths"].long(), s["added"].long(), s["block_size"], s["free_blocks"]
    n, width = s["table"].shape
    zero = torch.zeros(1, dtype=torch.int64, device=old.device)
    offsets = torch.cat([zero, torch.cumsum(new, 0)])
    total = old + new
    have = torch.clamp((old + bs - 1) // bs, max=width)
    want = torch.clamp((total + bs - 1) // bs, max=width) - have
    column = torch.arange(width, device=old.device)[None]
    place = (torch.cumsum(want, 0) - want)[:, None] + column - have[:, None]
    ids = torch.where(place < free.shape[0], free[place.clamp(0, free.shape[0] - 1)], -1)
    table = torch.where((column >= have[:, None]) & (column < (have + want)[:, None]), ids, s["table"])
    token = torch.arange(s["capacity"], device=old.device)
    request = torch.repeat_interleave(new, output_size=s["capacity"])
    position = old[request] + token - offsets[request]
    block = position // bs
    held = torch.where(block < width, table[request, block.clamp(max=width - 1)].long(), -1)
    slots = torch.where(held >= 0, held * bs + position % bs, -1)
    return table, offsets, total.int(), position.int(), slots, want.sum().reshape(1)


def _regions(data, bs, dim):
    """Views of a cache's bytes: key codes [block, token, head, dim / 2], value codes [block, cell, token / 4, token % 4, head,
    dim % 16, dim / 32], scales [block, token, head, dim / 32]."""
    codes, scales = bs * dim // 2, bs * dim // GROUP
    k = data[:, :, :codes].unflatten(2, (bs, dim // 2)).transpose(1, 2)
    v = data[:, :, codes:2 * codes].unflatten(2, (bs // CELL, 4, 16, dim // GROUP, 4)).permute(0, 2, 3, 6, 1, 4, 5)
    ks = data[:, :, 2 * codes:2 * codes + scales].unflatten(2, (bs, dim // GROUP)).transpose(1, 2)
    vs = data[:, :, 2 * codes + scales:].unflatten(2, (bs, dim // GROUP)).transpose(1, 2)
    return k, v, ks, vs


def _quantise(x):
    """Codes [..., dim] and scale bytes [..., dim / 32] of values in 16 bits."""
    top, lowest = (14, -23) if x.dtype == torch.float16 else (126, -126)
    g = x.float().unflatten(-1, (-1, GROUP))
    a = g.abs()
    largest = a.amax(-1)
    finite = torch.isfinite(largest)
    fraction, exponent = torch.frexp(torch.where(finite, largest, 0) / 6)  # largest / 6 = fraction 2^exponent, 1/2 <= fraction < 1
    e = exponent - (fraction == 0.5).int()
    # the division rounds: the exponent is one off where 6 2^e is just below the largest value, or 6 2^(e-1) just holds it
    e = torch.where(largest > torch.ldexp(torch.full_like(largest, 6.0), e), e + 1, e)
    e = torch.where(largest <= torch.ldexp(torch.full_like(largest, 6.0), e - 1), e - 1, e)
    e = torch.where(largest == 0, lowest, e).clamp(lowest, top)
    u = torch.ldexp(a, -e[..., None])
    code = (u > 0.25).int() + (u >= 0.75).int() + (u > 1.25).int() + (u >= 1.75).int() + (u > 2.5).int() + (u >= 3.5).int() + (u > 5).int()
    code = torch.where(e[..., None] == top, code.clamp(max=5), code)  # 4 2^top is not finite in the type
    code = code | (torch.signbit(g).int() << 3)
    return code.flatten(-2), torch.where(finite, e + 127, 255)


def _values(code, scale):
    """What codes [..., dim] under scale bytes [..., dim / 32] stand for, in 32 bits."""
    code, b = code.int().unflatten(-1, (-1, GROUP)), scale.int()[..., None]
    m = code & 7
    magnitude = torch.where(m < 4, m.float() / 2, torch.where(m < 6, m.float() - 2, 2 * m.float() - 8))
    power = torch.where(b == 255, math.nan, (b << 23).view(torch.float32))
    return (torch.where(code >= 8, -magnitude, magnitude) * power).flatten(-2)


def _halves(byte):
    return byte & 15, byte >> 4


def _plain_cache(s):
    bs, dim = s["block_size"], s["dim"]
    k, v, ks, vs = _regions(s["data"], bs, dim)
    block, token = s["slots"] // bs, s["slots"] % bs
    where = (block, token // CELL, token % CELL // 4, token % 4)
    code, scale = _quantise(s["k"])
    k[block, token] = (code[..., 0::2] | (code[..., 1::2] << 4)).byte()
    ks[block, token] = scale.byte()
    code, scale = _quantise(s["v"])
    code = code.unflatten(-1, (dim // GROUP, 2, 16))
    v[where] = (code[..., 0, :] | (code[..., 1, :] << 4)).byte().transpose(-1, -2)
    vs[block, token] = scale.byte()
    back_k = torch.stack(_halves(k[block, token]), -1).flatten(-2)
    back_v = torch.stack(_halves(v[where].transpose(-1, -2)), -2).flatten(-3)
    return _values(back_k, ks[block, token]).to(s["dtype"]), _values(back_v, vs[block, token]).to(s["dtype"])


def _padded(offsets, longest):
    """[request, place] -> row of the packed tensor, and whether there is one."""
    place = torch.arange(longest, device=offsets.device)[None]
    return offsets[:-1, None] + place, place < (offsets[1:] - offsets[:-1])[:, None]


def _take(x, row, there):
    """Packed [rows, heads, dim] -> [request, heads, place, dim] in 32 bits, zero where there is no row."""
    y = x[row.clamp(max=max(0, x.shape[0] - 1))].float() if x.shape[0] else torch.zeros(row.shape + x.shape[1:], device=x.device)
    return torch.where(there[..., None, None], y, 0).transpose(1, 2)


def _grouped(q, kv_heads):
    """[request, heads, place, dim] -> [request, kv_heads, (heads / kv_heads) places, dim]"""
    return q.unflatten(1, (kv_heads, -1)).flatten(2, 3)


def _ungrouped(x, heads):
    n, kv_heads, rows, dim = x.shape
    group = heads // kv_heads
    return x.unflatten(2, (group, rows // group)).flatten(1, 2)


def _softmax(s):
    """Over the last axis, in place of the scores; a row of -inf alone gives zeros."""
    m = s.amax(-1, keepdim=True)
    p = torch.exp(s - torch.where(m == -math.inf, 0, m))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, 1, total)


def _plain_cached(s):
    bs, dim, heads = s["block_size"], s["dim"], s["q"].shape[1]
    n, width = s["table"].shape
    held = s["data"][s["table"].clamp(min=0).long().flatten()]
    k, v, ks, vs = _regions(held, bs, dim)
    key = torch.arange(width * bs, device=held.device)
    there = (key[None] < s["lengths"][:, None]) & (s["table"] >= 0).repeat_interleave(bs, 1)
    k = _values(torch.stack(_halves(k), -1).flatten(-2), ks)
    v = _values(torch.stack(_halves(v.transpose(-1, -2)), -2).flatten(-3).flatten(1, 3), vs)
    # [n width, bs, kv_heads, dim] -> [n, kv_heads, keys, dim]
    k = torch.where(there[..., None, None], k.unflatten(0, (n, width)).flatten(1, 2), 0).transpose(1, 2)
    v = torch.where(there[..., None, None], v.unflatten(0, (n, width)).flatten(1, 2), 0).transpose(1, 2)
    row, new = _padded(s["q_offsets"], s["longest_q"])
    q = _grouped(_take(s["q"], row, new), k.shape[1])
    score = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    seen = there[:, None, :]
    if s["causal"]:
        many = s["q_offsets"][1:] - s["q_offsets"][:-1]
        last = s["lengths"].long()[:, None] - many[:, None] + torch.arange(s["longest_q"], device=held.device)[None]
        seen = seen & (key[None, None] <= last[:, :, None])
    seen = seen.expand(-1, s["longest_q"], -1).repeat(1, heads // k.shape[1], 1)[:, None]
    p = _softmax(score.masked_fill_(~seen, -math.inf))
    out = _ungrouped(torch.matmul(p, v), heads).transpose(1, 2)
    return out[new].to(s["dtype"])


def _cross_scores(s):
    kv_heads = s["k"].shape[1]
    q_row, q_there = _padded(s["q_offsets"], s["longest_q"])
    k_row, k_there = _padded(s["k_offsets"], s["longest_k"])
    seen = k_there
    bias = None
    if s["key_bias"] is not None:
        b = s["key_bias"].float()
        bias = torch.where(k_there, b[k_row.clamp(max=max(0, b.shape[0] - 1))] if b.shape[0] else 0.0, -math.inf)
        seen = seen & (bias != -math.inf)
    q = _grouped(_take(s["q"], q_row, q_there), kv_heads)
    k, v = _take(s["k"], k_row, seen), _take(s["v"], k_row, seen)
    score = torch.matmul(q, k.transpose(2, 3)) * s["scale"]
    if bias is not None:
        score = score + bias[:, None, None, :]
    return q, k, v, score.masked_fill_(~seen[:, None, None, :], -math.inf), q_there, k_there, q_row


def _plain_cross(s):
    q, k, v, score, q_there, _, _ = _cross_scores(s)
    out = _ungrouped(torch.matmul(_softmax(score), v), s["q"].shape[1]).transpose(1, 2)
    return out[q_there].to(s["q"].dtype)


def _plain_train(s):
    heads, dtype = s["q"].shape[1], s["q"].dtype
    q, k, v, score, q_there, k_there, q_row = _cross_scores(s)
    p = _softmax(score)
    out = torch.matmul(p, v)
    d_out = _grouped(_take(s["d_out"], q_row, q_there), k.shape[1])
    dp = torch.matmul(d_out, v.transpose(2, 3))
    ds = p * (dp - (d_out * out).sum(-1, keepdim=True))
    dv = torch.matmul(p.transpose(2, 3), d_out)
    dk = torch.matmul(ds.transpose(2, 3), q) * s["scale"]
    dq = torch.matmul(ds, k) * s["scale"]
    packed = lambda x, there: x.transpose(1, 2)[there].to(dtype)  # noqa: E731
    got = (packed(_ungrouped(out, heads), q_there), packed(_ungrouped(dq, heads), q_there), packed(dk, k_there), packed(dv, k_there))
    if s["key_bias"] is not None:
        # rows that no token owns have a zero gradient, so they add nothing
        got += (ds.sum((1, 2))[k_there].to(dtype),)
    return got


_PLAIN = {"tables": _plain_tables, "cache": _plain_cache, "cached": _plain_cached, "cross": _plain_cross, "train": _plain_train}


# ------------------------------------------------------------------------------------------------ what a pass cannot do without
def work(case):
    if case["kind"] == "tables":
        old, new, bs = _lengths(case, "old"), _lengths(case, "new"), case["block_size"]
        want = sum(-(-(a + b) // bs) - -(-a // bs) for a, b in zip(old, new))
        n, tokens = case["n"], sum(new)
        return {"bytes": 8 * n + 4 * n + 8 * want + 8 * (n + 1) + 4 * n + 12 * tokens, "flops": 4 * tokens + 8 * n}
    if case["kind"] == "cache":
        values = 2 * case["tokens"] * case["kv_heads"] * case["dim"]
        held = values // 2 + values // GROUP
        return {"bytes": 2 * values + 2 * held + 2 * values + 16 * case["tokens"], "flops": 4 * values}
    nq, nk = _attention_lengths(case)
    heads, kv_heads, dim = case["heads"], case["kv_heads"], case["dim"]
    if case.get("causal"):  # query i of a sees b - a + i + 1 of b keys
        pairs = sum(a * (b - a) + a * (a + 1) // 2 for a, b in zip(nq, nk))
    else:
        pairs = sum(a * b for a, b in zip(nq, nk))
    rows, keys = sum(nq), sum(nk)
    if case["kind"] == "cached":
        held = keys * kv_heads * (dim + dim // 16)
        table = 4 * sum(-(-b // case["block_size"]) for b in nk)
        return {"bytes": held + table + 4 * rows * heads * dim + 12 * case["n"], "flops": 4 * pairs * heads * dim}
    bias = 2 * keys if case["bias"] else 0
    read = 2 * rows * heads * dim + 4 * keys * kv_heads * dim + bias + 16 * case["n"]
    if case["kind"] == "cross":
        return {"bytes": read + 2 * rows * heads * dim, "flops": 4 * pairs * heads * dim}
    # forward and the five products of the backward pass; d_out in, out, dq, dk, dv and the bias's gradient out
    return {"bytes": read + 6 * rows * heads * dim + 4 * keys * kv_heads * dim + bias, "flops": 14 * pairs * heads * dim}


# ------------------------------------------------------------------------------------------------ in 64 bits
def exact(case, seed):
    s = prepare(case, seed)
    return {"tables": _exact_tables, "cache": _exact_cache, "cached": _exact_cached, "cross": _exact_cross, "train": _exact_cross}[case["kind"]](s)


def _exact_tables(s):
    old, new, bs = s["lengths"].tolist(), s["added"].tolist(), s["block_size"]
    table, free = s["table"].cpu().numpy().copy(), s["free_blocks"].cpu().numpy()
    width, taken, offsets, positions, slots = table.shape[1], 0, [0], [], []
    for r, (a, b) in enumerate(zip(old, new)):
        for c in range(-(-a // bs), min(width, -(-(a + b) // bs))):
            table[r, c] = free[taken] if taken < len(free) else -1
            taken += 1
        at = np.arange(a, a + b, dtype=np.int64)
        ids = np.append(table[r].astype(np.int64), -1)[np.minimum(at // bs, width)]
        positions.append(at.astype(np.int32))
        slots.append(np.where(ids >= 0, ids * bs + at % bs, -1))
        offsets.append(offsets[-1] + b)
    total = np.array([a + b for a, b in zip(old, new)], dtype=np.int32)
    return (table, np.array(offsets, dtype=np.int64), total, np.concatenate(positions), np.concatenate(slots), np.array([taken], dtype=np.int64))


_E2M1 = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])


def _exact_cache(s):
    top, lowest = (14, -23) if s["dtype"] == torch.float16 else (126, -126)
    got = []
    for x in (s["k"], s["v"]):
        g = x.double().cpu().numpy().reshape(x.shape[0], x.shape[1], -1, GROUP)
        largest = np.abs(g).max(-1, keepdims=True)
        e = np.full(largest.shape, lowest)
        for power in range(-40, 40):  # the inputs' range
            e = np.where(largest > 6 * 2.0 ** power, max(lowest, min(top, power + 1)), e)
        u = np.abs(g) / 2.0 ** e
        # the nearest value; of two that are as near, the one with the even code
        nearest = np.zeros(u.shape, dtype=np.int64)
        for c in range(1, 8):
            if c < 6:
                fits = True
            else:
                fits = e != top
            d, best = np.abs(u - _E2M1[c]), np.abs(u - _E2M1[nearest])
            nearest = np.where(fits & ((d < best) | ((d == best) & (c % 2 == 0))), c, nearest)
        got.append((np.copysign(_E2M1[nearest], g) * 2.0 ** e).reshape(x.shape))
    return tuple(got)


def _exact_cached(s):
    """Request by request and head by head, from the bytes."""
    bs, dim, (rows, heads, _) = s["block_size"], s["dim"], s["q"].shape
    kv_heads, codes, scales = s["data"].shape[1], bs * dim // 2, bs * dim // GROUP
    if rows * heads * s["longest_k"] * dim > 2e12:
        return None
    values = torch.tensor(np.concatenate([_E2M1, -_E2M1]), device="cuda")
    out = torch.zeros((rows, heads, dim), dtype=torch.float64, device="cuda")
    at, lengths = s["q_offsets"].tolist(), s["lengths"].tolist()
    d = torch.arange(dim, device="cuda")
    for r, length in enumerate(lengths):
        if length == 0 or at[r + 1] == at[r]:
            continue
        place = torch.arange(length, device="cuda")
        block, t = s["table"][r].long()[place // bs][:, None], (place % bs)[:, None]
        k_byte = t * (dim // 2) + d // 2
        v_byte = codes + t // 16 * (8 * dim) + (t % 16 // 4 * 16 + d % 16) * (dim // 8) + d // 32 * 4 + t % 4
        scale_byte = 2 * codes + t * (dim // GROUP) + d // GROUP
        query = torch.arange(at[r + 1] - at[r], device="cuda")
        hidden = place[None] > (length - len(query) + query if s["causal"] else query * 0 + length)[:, None]
        for g in range(kv_heads):
            bytes_of = s["data"][:, g]
            power = lambda b: torch.pow(torch.tensor(2.0, dtype=torch.float64, device="cuda"), b.double() - 127)  # noqa: E731
            k = values[(bytes_of[block, k_byte].int() >> (d % 2 * 4)) & 15] * power(bytes_of[block, scale_byte])
            v = values[(bytes_of[block, v_byte].int() >> (d // 16 % 2 * 4)) & 15] * power(bytes_of[block, scale_byte + scales])
            for h in range(g * heads // kv_heads, (g + 1) * heads // kv_heads):
                score = (s["q"][at[r]:at[r + 1], h].double() @ k.T * s["scale"]).masked_fill(hidden, -math.inf)
                out[at[r]:at[r + 1], h] = torch.softmax(score, -1).nan_to_num(0) @ v
    return out


def _exact_cross(s):
    """Request by request and head by head; a masked key is left out of the request."""
    (rows, heads, dim), kv_heads = s["q"].shape, s["k"].shape[1]
    if rows * heads * s["longest_k"] * dim > 2e12:
        return None
    zeros = lambda x: torch.zeros(x.shape, dtype=torch.float64, device="cuda")  # noqa: E731
    out, dq, dk, dv = zeros(s["q"]), zeros(s["q"]), zeros(s["k"]), zeros(s["v"])
    db = torch.zeros(s["k"].shape[0], dtype=torch.float64, device="cuda")
    a, b = s["q_offsets"].tolist(), s["k_offsets"].tolist()
    for r in range(len(a) - 1):
        key = torch.arange(b[r], b[r + 1], device="cuda")
        if s["key_bias"] is not None:
            key = key[s["key_bias"][key] != -math.inf]
        if len(key) == 0 or a[r + 1] == a[r]:
            continue
        for h in range(heads):
            g, at = h * kv_heads // heads, slice(a[r], a[r + 1])
            q, k, v = s["q"][at, h].double(), s["k"][key, g].double(), s["v"][key, g].double()
            score = q @ k.T * s["scale"]
            if s["key_bias"] is not None:
                score = score + s["key_bias"][key].double()
            p = torch.softmax(score, -1)
            out[at, h] = p @ v
            if s["d_out"] is not None:
                do = s["d_out"][at, h].double()
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(-1, keepdim=True))
                dq[at, h] = ds @ k * s["scale"]
                dk[key, g] += ds.T @ q * s["scale"]
                dv[key, g] += p.T @ do
                db[key] += ds.sum(0)
    if s["d_out"] is None:
        return out
    return (out, dq, dk, dv) + ((db,) if s["key_bias"] is not None else ())
