"""Block tables and the cache in four bits on the GPU against plain implementations: whole numbers and held values are equal."""
import numpy as np
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


def _i32(x):
    return torch.tensor(x, dtype=torch.int32, device=DEV)


def _plain_tables(old, new, table, free, bs, capacity):
    old, new = [max(0, x) for x in old], [max(0, x) for x in new]
    table, taken, offsets, positions, slots = table.copy(), 0, [0], [], []
    width = table.shape[1]
    for r, (a, b) in enumerate(zip(old, new)):
        for c in range(min(width, -(-a // bs)), min(width, -(-(a + b) // bs))):
            table[r, c] = free[taken] if taken < len(free) else -1
            taken += 1
        for p in range(a, a + b):
            held = table[r, p // bs] if p // bs < width else -1
            positions.append(p)
            slots.append(int(held) * bs + p % bs if held >= 0 else -1)
        offsets.append(offsets[-1] + b)
    pad = lambda x: (x + [-1] * capacity)[:capacity]  # noqa: E731
    return table, offsets, [a + b for a, b in zip(old, new)], pad(positions), pad(slots), [taken]


def _check_tables(pl, old, new, bs, width, n_free, capacity=None, stride=None, seed=0):
    rng = np.random.default_rng(seed)
    n = len(old)
    ids = rng.permutation(n * width + n_free + 5).astype(np.int32)
    host = np.full((n, stride or width), -7, dtype=np.int32)
    host[:, :width] = -1
    k = n_free
    for r, a in enumerate(old):
        have = min(width, -(-max(0, a) // bs))
        host[r, :have] = ids[k:k + have]
        k += have
    free = ids[:n_free]
    capacity = sum(max(0, x) for x in new) if capacity is None else capacity
    wide = torch.from_numpy(host).to(DEV)
    table = wide[:, :width]
    got = pl.plaid_block_tables(_i32(old), _i32(new), table, torch.from_numpy(free).to(DEV), bs, capacity)
    torch.cuda.synchronize()
    want = _plain_tables(old, new, host[:, :width], free, bs, capacity)
    np.testing.assert_array_equal(table.cpu().numpy(), want[0])
    if stride:
        assert (wide[:, width:] == -7).all()
    for name, g, w in zip(("offsets", "totals", "positions", "slots", "wanted"), got, want[1:]):
        np.testing.assert_array_equal(g.cpu().numpy(), np.array(w), err_msg=name)


@pytest.mark.parametrize("bs", [16, 32, 64, 128, 256])
@pytest.mark.parametrize("n", [1, 2, 63, 64, 65, 257])
def test_block_tables(pl, n, bs):
    rng = np.random.default_rng(n * bs)
    old = rng.integers(0, 5 * bs, n).tolist()
    new = rng.integers(0, 3 * bs, n).tolist()
    old[0], new[-1] = 0, 0
    want = sum(-(-(a + b) // bs) - -(-a // bs) for a, b in zip(old, new))
    _check_tables(pl, old, new, bs, 8, want + 3)
    _check_tables(pl, old, [1] * n, bs, 8, n, stride=11)          # a decode step; rows of a wider table


def test_block_tables_where_something_is_missing(pl):
    old, new = [0, 15, 16, 17, 40, 0, 33], [70, 1, 1, 15, 0, 5, 100]
    _check_tables(pl, old, new, 16, 9, 3)                         # too few blocks
    _check_tables(pl, old, new, 16, 9, 0)                         # none
    _check_tables(pl, old, new, 16, 3, 50)                        # rows too short for the request, old tokens included
    _check_tables(pl, old, new, 16, 9, 50, capacity=64)           # room for some of the tokens
    _check_tables(pl, old, new, 16, 9, 50, capacity=0)
    _check_tables(pl, old, new, 16, 9, 50, capacity=203)          # more room than tokens, and odd
    _check_tables(pl, [-3, 5, 0], [4, -2, 0], 32, 2, 4, capacity=9)  # negative numbers count as 0
    _check_tables(pl, [0] * 5, [0] * 5, 64, 1, 1)                 # nothing at all


def test_block_tables_of_many_requests(pl):
    rng = np.random.default_rng(5)
    for n in (2048, 2049, 5003):                                  # the two-launch form from 2049 on
        old, new = rng.integers(0, 60, n).tolist(), rng.integers(0, 9, n).tolist()
        want = sum(-(-(a + b) // 16) - -(-a // 16) for a, b in zip(old, new))
        _check_tables(pl, old, new, 16, 6, want - 1)


def _special(dtype, n, dim, seed):
    """Tokens of every kind: wide ranges, ties between codes, subnormals, the largest value, groups that are not finite."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(n, dim, generator=g) * torch.exp2(torch.randint(-12, 12, (n, 1), generator=g).float())
    x = x.to(dtype)
    ties = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.0, -0.25, -2.5, 0.0, -0.0, 1e-3, 4.5, 5.5, 0.5])
    if n > 9:
        x[1, :16] = ties.to(dtype)
        x[1, 16:32] = -ties.to(dtype)
        x[2, :] = 0
        x[3, :32] = torch.finfo(dtype).max
        x[4, :32] = torch.finfo(dtype).tiny / 4
        x[5, 3] = float("inf")
        x[6, dim - 1] = float("nan")
        x[7, 0] = float("-inf")
        x[8, :32] = torch.finfo(dtype).smallest_normal * torch.arange(32).to(dtype)
        x[9, :32] = torch.finfo(dtype).max / 8
    return x


@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("dim,bs,heads", [(64, 16, 1), (64, 64, 3), (128, 16, 2), (128, 32, 1), (128, 256, 2)])
def test_cache_write_and_read(pl, dtype, dim, bs, heads):
    n, blocks = 75, 9 if bs == 16 else 3
    k = torch.stack([_special(dtype, n, dim, 10 * h) for h in range(heads)], 1)
    v = torch.stack([_special(dtype, n, dim, 10 * h + 5) for h in range(heads)], 1)
    g = torch.Generator().manual_seed(3)
    slots = torch.randperm(blocks * bs, generator=g)[:n]
    first = torch.arange(30) + 5                                   # a run of neighbours that begins inside a quad
    slots[~torch.isin(slots, first)][:0]
    rest = slots[~torch.isin(slots, first)][:n - 30]
    rest = torch.cat([rest, torch.full((n - 30 - len(rest),), -1)])
    slots = torch.cat([first, rest])
    slots[40] = -1
    slots[41] = blocks * bs                                        # past the end: left out
    cache = pl.PagedCache.empty(blocks, bs, heads, dim, dtype, DEV)
    cache.data.fill_(77)                                           # what is not written stays
    both = torch.cat([k, v], 1).to(DEV)                            # strided views of one tensor
    pl.plaid_cache_write(cache, both[:, :heads], both[:, heads:], slots.to(DEV))
    want = torch.full(cache.data.shape, 77, dtype=torch.uint8)
    kc, ks = ru.quantise(k)
    vc, vs = ru.quantise(v)
    for t, s in enumerate(slots.tolist()):
        if 0 <= s < blocks * bs:
            for h in range(heads):
                ru.put(want, s, h, kc[t, h], ks[t, h], vc[t, h], vs[t, h], bs, dim)
    got = cache.data.cpu()
    # the codes of a group that is not finite, and the sign of a zero code, are free: compared by value below, the rest byte by byte
    rk, rv = pl.plaid_cache_read(cache, slots.to(DEV))
    inside = (slots >= 0) & (slots < blocks * bs)
    for name, back, code, scale in (("k", rk, kc, ks), ("v", rv, vc, vs)):
        value = ru.value_of(code, scale)
        value[~inside] = 0
        ru.close(back, value, torch.zeros(value.shape, dtype=torch.float64), name)
    codes = bs * dim // 2
    assert torch.equal(got[:, :, 2 * codes:], want[:, :, 2 * codes:])                       # scales, and nothing else there
    finite_tokens = torch.ones(blocks * bs, dtype=torch.bool)
    for t, s in enumerate(slots.tolist()):
        if inside[t]:
            finite_tokens[s] = bool((ks[t] != 255).all() and (vs[t] != 255).all())
    rows = got[:, :, :codes].reshape(blocks, heads, bs, dim // 2).transpose(1, 2).reshape(blocks * bs, -1)
    rows_want = want[:, :, :codes].reshape(blocks, heads, bs, dim // 2).transpose(1, 2).reshape(blocks * bs, -1)
    assert torch.equal(rows[finite_tokens], rows_want[finite_tokens])
    cells = lambda x: x[:, :, codes:2 * codes].reshape(blocks, heads, bs // 16, 4, dim // 2 // 4 * 4 // (dim // 8) * 4, dim // 32, 4)  # noqa: E731
    tokens = lambda x: cells(x).permute(0, 2, 3, 6, 1, 4, 5).reshape(blocks * bs, -1)  # noqa: E731
    assert torch.equal(tokens(got)[finite_tokens], tokens(want)[finite_tokens])


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 33])
def test_cache_write_sizes(pl, n):
    for dtype, dim in ((BF, 128), (HF, 64)):
        x = _special(dtype, n, dim, n)[:, None].contiguous()
        cache = pl.PagedCache.empty(4, 16, 1, dim, dtype, DEV)
        slots = (torch.arange(n) + 3).to(DEV)
        pl.plaid_cache_write(cache, x.to(DEV), x.flip(0).contiguous().to(DEV), slots)
        k, v = pl.plaid_cache_read(cache, slots)
        want = ru.value_of(*ru.quantise(x))
        ru.close(k, want, torch.zeros(want.shape, dtype=torch.float64), "k")
        ru.close(v, want.flip(0), torch.zeros(want.shape, dtype=torch.float64), "v")
    cache = pl.PagedCache.empty(1, 16, 1, 64, BF, DEV)
    none = torch.zeros(0, dtype=torch.int64, device=DEV)
    pl.plaid_cache_write(cache, torch.zeros(0, 1, 64, dtype=BF, device=DEV), torch.zeros(0, 1, 64, dtype=BF, device=DEV), none)
    assert pl.plaid_cache_read(cache, none)[0].shape == (0, 1, 64)


def test_all_codes_are_read_as_their_values(pl):
    """Every byte under every scale that a type's values can have."""
    for dtype, scales in ((BF, [1, 2, 60, 126, 127, 128, 200, 252]), (HF, [104, 110, 120, 127, 130, 140])):
        for b in scales:
            data = torch.zeros(1, 1, 16 * 64 * 17 // 16, dtype=torch.uint8)
            data[0, 0, :512] = torch.arange(512) % 256
            data[0, 0, 512:1024] = torch.arange(512).flip(0) % 256
            data[0, 0, 1024:] = b
            cache = pl.PagedCache(data.to(DEV), 16, 64, dtype)
            k, _ = pl.plaid_cache_read(cache, torch.arange(16, device=DEV))
            byte = data[0, 0, :512].long().reshape(16, 32)
            code = torch.stack([byte & 15, byte >> 4], -1).flatten(1)
            want = ru.value_of(code, torch.full((16, 2), b))
            most = torch.finfo(dtype).max
            want = torch.where(want.abs() > most, torch.sign(want) * float("inf"), want)
            ru.close(k[:, 0], want, torch.zeros(want.shape, dtype=torch.float64), f"{dtype} {b}")


def test_a_cache_of_more_than_four_gigabytes(pl):
    blocks, bs, heads, dim = 66_000, 64, 8, 128                     # 4.6 GB
    cache = pl.PagedCache.empty(blocks, bs, heads, dim, BF, DEV)
    g = torch.Generator().manual_seed(1)
    n = 70
    k, v, q = (torch.randn(s, generator=g).to(BF).to(DEV) for s in ((n, heads, dim), (n, heads, dim), (1, heads, dim)))
    slots = (blocks - 2) * bs + torch.arange(n, device=DEV)
    pl.plaid_cache_write(cache, k, v, slots)
    rk, rv = pl.plaid_cache_read(cache, slots)
    want = ru.value_of(*ru.quantise(k.cpu()))
    ru.close(rk, want, torch.zeros(want.shape, dtype=torch.float64), "k")
    assert not cache.data[:blocks - 2].any()
    table = torch.tensor([[blocks - 2, blocks - 1]], dtype=torch.int32, device=DEV)
    off = torch.tensor([0, 1], device=DEV)
    out = pl.plaid_cached_attention(q, cache, table, _i32([n]), off)
    for h in range(heads):
        x = ru.attend(q[:, h].cpu(), rk[:, h].cpu(), rv[:, h].cpu(), dim ** -0.5)
        ru.close(out[:, h], x["out"], x["out_bound"], "out")
