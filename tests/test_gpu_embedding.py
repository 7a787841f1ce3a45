"""Embedding and the table's gradient by sorted tokens, against the definitions in 64 bits."""
import pytest
import torch

from training_util import close, embed, embed_bound, embed_grad

pytestmark = pytest.mark.gpu
DEV, BF, HALF = torch.device("cuda", 0), torch.bfloat16, torch.float16


@pytest.fixture(scope="module")
def pl():
    import paper_2205_09707_amd as pl
    pl.load_library()
    return pl


def _inputs(n, vocabulary, width, dtype, seed=0, frequent=0.0, outside=0.1):
    g = torch.Generator(device=DEV).manual_seed(seed)
    ids = torch.randint(0, vocabulary, (n,), generator=g, device=DEV)
    u = torch.rand(n, generator=g, device=DEV)
    ids = torch.where(u < frequent, vocabulary // 2, ids)
    ids = torch.where(u > 1 - outside, torch.tensor([-1, vocabulary, -100, 2 ** 40], device=DEV)[torch.arange(n, device=DEV) % 4], ids)
    return torch.randn(vocabulary, width, generator=g, device=DEV).to(dtype), ids, torch.randn(n, width, generator=g, device=DEV).to(dtype)


SIZES = [(1, 1, 1), (1, 5, 8), (2, 1, 64), (33, 10, 7), (64, 300, 765), (70, 1000, 2048), (200, 50, 2056), (257, 100_000, 16), (5000, 3, 40), (4096, 700, 128), (8192, 5000, 40), (8193, 70_000, 40), (1025, 300, 64),
         (4097, 700, 128), (20_011, 1000, 64), (30_000, 300_000, 24), (3, 70, 5000)]


@pytest.mark.parametrize("dtype", [BF, HALF])
@pytest.mark.parametrize("n,vocabulary,width", SIZES)
def test_rows_and_gradient(pl, n, vocabulary, width, dtype):
    table, ids, d = _inputs(n, vocabulary, width, dtype, seed=n, frequent=0.3 if n > 1 else 0.0, outside=0.1 if n > 1 else 0.0)
    scale = 1.7
    out = pl.plaid_embedding(table, ids, scale=scale)
    want = embed(table, ids, scale)
    close(out, want, embed_bound(want, dtype), "rows")
    got = pl.plaid_embedding_backward(d, ids, vocabulary, scale=scale)
    close(got, *embed_grad(d, ids, vocabulary, scale), "gradient")
    assert torch.equal(got, pl.plaid_embedding_backward(d, ids, vocabulary, scale=scale))
    before = torch.randn(vocabulary, width, device=DEV).to(dtype)
    held = before.clone()
    assert pl.plaid_embedding_backward(d, ids, vocabulary, scale=scale, add_to=held) is held
    close(held, *embed_grad(d, ids, vocabulary, scale, before), "gradient added")
    absent = torch.ones(vocabulary, dtype=torch.bool, device=DEV)
    absent[ids[(ids >= 0) & (ids < vocabulary)]] = False
    assert torch.equal(held[absent], before[absent])


@pytest.mark.parametrize("n", [31, 32, 33, 64, 65, 2048, 5000, 70_000])
def test_one_token_has_all_places(pl, n):
    """Whole chunks of one token, and chunks that it begins or ends in."""
    for at in (0, n // 3):
        ids = torch.full((n,), 4, device=DEV)
        ids[:at] = torch.arange(at, device=DEV) % 4
        d = torch.randn(n, 72, device=DEV).to(BF)
        close(pl.plaid_embedding_backward(d, ids, 6), *embed_grad(d, ids, 6, 1.0), f"{n} from {at}")


def test_no_tokens_and_no_known_tokens(pl):
    table = torch.randn(9, 16, device=DEV).to(BF)
    none = torch.empty(0, dtype=torch.int64, device=DEV)
    assert pl.plaid_embedding(table, none).shape == (0, 16)
    assert not pl.plaid_embedding_backward(table[:0], none, 9).any()
    held = table.clone()
    pl.plaid_embedding_backward(table[:0], none, 9, add_to=held)
    assert torch.equal(held, table)
    outside = torch.full((40,), -1, device=DEV)
    nan = torch.full((40, 16), float("nan"), device=DEV, dtype=BF)
    assert not pl.plaid_embedding(table, outside).any() and not pl.plaid_embedding_backward(nan, outside, 9).any()


def test_what_is_not_finite_stays_with_its_token(pl):
    table, ids, d = _inputs(3000, 50, 40, HALF, seed=5)
    d[ids == 7] = float("inf")
    d[ids == 9, 3] = float("nan")
    d[ids < 0] = float("nan")
    want, bound = embed_grad(d, ids, 50, 1.0)
    got = pl.plaid_embedding_backward(d, ids, 50)
    assert torch.isfinite(got[[i for i in range(50) if i not in (7, 9)]]).all()
    assert torch.isinf(got[7]).all() and torch.isnan(got[9, 3]) and torch.isfinite(got[9, 4:]).all()
    keep = [i for i in range(50) if i not in (7, 9)]
    close(got[keep], want[keep], bound[keep], "the others")


def test_strided_rows(pl):
    wide = torch.randn(40, 3 * 33, device=DEV).to(BF)
    table, ids = wide[:, 33:66], torch.arange(39, -1, -1, device=DEV).repeat_interleave(2)
    want = embed(table, ids[::2], 1.0)
    assert torch.equal(pl.plaid_embedding(table, ids[::2]).double(), want)
    d = torch.randn(80, 70, device=DEV).to(BF)
    close(pl.plaid_embedding_backward(d[:, 1:34], ids, 40), *embed_grad(d[:, 1:34], ids, 40, 1.0), "a view of d_out")
    every = torch.randn(33, 80, device=DEV).to(BF).T  # columns are not together: copied
    close(pl.plaid_embedding_backward(every, ids, 40), *embed_grad(every, ids, 40, 1.0), "transposed d_out")
    one = torch.randn(1, 33, device=DEV).to(BF).expand(80, 33)  # a broadcast gradient
    close(pl.plaid_embedding_backward(one, ids, 40), *embed_grad(one, ids, 40, 1.0), "expanded d_out")


def test_table_beyond_four_gigabytes(pl):
    rows, width = 1_100_000, 2048
    table = torch.empty(rows, width, dtype=BF, device=DEV)
    table[:] = (torch.arange(rows, device=DEV) % 251)[:, None].to(BF)
    ids = torch.tensor([0, rows - 1, rows // 2, 1_048_577, rows], device=DEV)
    assert pl.plaid_embedding(table, ids)[:, 5].tolist() == [0, (rows - 1) % 251, (rows // 2) % 251, 1_048_577 % 251, 0]
    d = torch.ones(5, width, dtype=BF, device=DEV)
    table.fill_(3.0)
    pl.plaid_embedding_backward(d, ids, rows, add_to=table)
    assert table[ids[:4]].eq(4).all() and int((table[:, 9] != 3).sum()) == 4
    got = pl.plaid_embedding_backward(d, ids, rows)
    assert got[ids[:4]].eq(1).all() and int(got[:, width - 1].float().sum()) == 4


def test_refusals(pl):
    table, ids, d = _inputs(10, 20, 16, BF)
    with pytest.raises(ValueError):
        pl.plaid_embedding(table, ids.int())
    with pytest.raises(ValueError):
        pl.plaid_embedding(table.float(), ids)
    with pytest.raises(ValueError):
        pl.plaid_embedding_backward(d, ids[:9], 20)
    with pytest.raises(ValueError):
        pl.plaid_embedding_backward(d, ids, 20, add_to=table[:, :8])
    with pytest.raises(ValueError):
        pl.plaid_embedding_backward(d, ids, 20, add_to=table.half())
    with pytest.raises(ValueError):
        pl.plaid_embedding_backward(d, ids, 20, add_to=torch.zeros(20, 32, dtype=BF, device=DEV)[:, :16])
    with pytest.raises(pl.PlaidError):
        pl.plaid_embedding_backward(d, ids, 0)
    table.requires_grad_()
    with pytest.raises(ValueError, match="table requires a gradient"):
        pl.plaid_embedding(table, ids)
    with torch.no_grad():
        pl.plaid_embedding(table, ids)


def test_gradients_of_gradients_are_refused(pl):
    d, ids, held = torch.randn(6, 16, device=DEV).to(BF), torch.arange(6, device=DEV), torch.zeros(9, 16, device=DEV, dtype=BF)
    for x, name in ((d, "d_out"), (held, "add_to")):
        x.requires_grad_()
        with pytest.raises(ValueError, match=f"{name} requires a gradient"):
            pl.plaid_embedding_backward(d, ids, 9, add_to=held)
        with torch.no_grad():
            pl.plaid_embedding_backward(d, ids, 9, add_to=held)
        x.requires_grad_(False)
