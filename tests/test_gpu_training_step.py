"""The operators of a training step one after another, as a reader has them: tokens in, dropout and layer norm between, cross attention to the
passages, a loss over the table that the tokens came from.  Gradients against autograd of the same step in 64 bits."""
import math
import importlib.util
import os

import pytest
import torch

from training_util import half_step, kept

pytestmark = pytest.mark.gpu
DEV = torch.device("cuda", 0)


@pytest.fixture(scope="module")
def example():
    path = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "reader.py")
    spec = importlib.util.spec_from_file_location("reader_example_of_a_step", path)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


HEADS, KV_HEADS, DIM, WIDTH, VOCABULARY, P = 4, 2, 64, 256, 900, 0.2


def _state(dtype, rows=(37, 0, 120), keys=(50, 9, 200)):
    g = torch.Generator().manual_seed(3)
    r = lambda *s, gain=1.0: (torch.randn(*s, generator=g) * gain).to(dtype)  # noqa: E731
    n = sum(rows)
    ids = torch.randint(0, 60, (n,), generator=g)  # few tokens, often: sums of many rows
    ids[5] = -1
    targets = torch.randint(0, VOCABULARY, (n,), generator=g)
    targets[[0, 36, 90]] = -100
    weights = {"table": r(VOCABULARY, WIDTH, gain=WIDTH ** -0.5), "w1": 1 + r(WIDTH, gain=0.1), "b1": r(WIDTH, gain=0.1), "w2": 1 + r(WIDTH, gain=0.1), "b2": r(WIDTH, gain=0.1),
               "k": r(sum(keys), KV_HEADS, DIM), "v": r(sum(keys), KV_HEADS, DIM)}
    off = lambda lengths: torch.tensor([0] + torch.tensor(lengths).cumsum(0).tolist())  # noqa: E731
    return {n: w.to(dtype) for n, w in weights.items()}, ids, targets, off(rows), off(keys)


def _own(example, weights, ids, targets, q_offsets, k_offsets, rng):
    w = weights
    x = example.Embedding.apply(w["table"], ids, WIDTH ** 0.5)
    x = example.Dropout.apply(x, None, P, rng[0])
    q = example.LayerNorm.apply(x, w["w1"], w["b1"]).view(-1, HEADS, DIM)
    bias = torch.zeros(w["k"].shape[0], dtype=x.dtype, device=DEV)
    y = example.CrossAttention.apply(q, w["k"], w["v"], bias, q_offsets, k_offsets).reshape(-1, WIDTH)
    x = example.Dropout.apply(y, x, P, rng[1])
    h = example.LayerNorm.apply(x, w["w2"], w["b2"])
    return example.CrossEntropy.apply(h, w["table"], targets, 1.0).sum() / (targets >= 0).sum()


def _exact(weights, ids, targets, q_offsets, k_offsets, rng):
    w = weights

    def drop(x, rng):
        mask, factor = kept(0, x.numel(), P, *rng.tolist())
        return torch.where(mask.view(x.shape), x * factor, 0.0)

    def norm(x, weight, bias):
        x = x - x.mean(1, keepdim=True)
        return x / torch.sqrt((x * x).mean(1, keepdim=True) + 1e-5) * weight + bias

    x = torch.where((ids >= 0)[:, None], w["table"][ids.clamp(min=0)] * WIDTH ** 0.5, 0.0)
    x = drop(x, rng[0])
    q = norm(x, w["w1"], w["b1"]).view(-1, HEADS, DIM)
    out = []
    for r in range(len(q_offsets) - 1):
        a, b = slice(q_offsets[r], q_offsets[r + 1]), slice(k_offsets[r], k_offsets[r + 1])
        k, v = (t[b].repeat_interleave(HEADS // KV_HEADS, 1) for t in (w["k"], w["v"]))
        p = torch.softmax(torch.einsum("qhd,khd->hqk", q[a], k) / math.sqrt(DIM), -1)
        out.append(torch.einsum("hqk,khd->qhd", p, v))
    x = x + drop(torch.cat(out).reshape(-1, WIDTH), rng[1])
    logp = torch.log_softmax(norm(x, w["w2"], w["b2"]) @ w["table"].T, 1)
    live = targets >= 0
    return -logp[live, targets[live]].mean()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float16])
def test_gradients_of_a_whole_step(example, dtype):
    """Six roundings to the type stand between the table and the loss and as many on the way back, each off by half a step at most and by a third
    of it or so in the mean square; a gradient is off by their root of squares times what layer norm and softmax make of them, about two each
    (the width's factor 1 / deviation is one here).  20 half steps, relative to the norm of each gradient, hold that with room."""
    weights, ids, targets, q_offsets, k_offsets = _state(dtype)
    scale = 1024.0 if dtype == torch.float16 else 1.0
    rng = [torch.tensor([5, 1]), torch.tensor([5, 2])]
    exact = {n: w.double().requires_grad_() for n, w in weights.items()}
    want = _exact(exact, ids, targets, q_offsets, k_offsets, rng)
    want.backward()
    own = {n: w.to(DEV).requires_grad_() for n, w in weights.items()}
    loss = _own(example, own, ids.to(DEV), targets.to(DEV), q_offsets.to(DEV), k_offsets.to(DEV), [r.to(DEV) for r in rng])
    (loss * scale).backward()
    assert abs(float(loss.detach()) - float(want.detach())) <= 20 * half_step(dtype) * float(want.detach())
    for n, w in own.items():
        off = (w.grad.double().cpu() / scale - exact[n].grad).norm() / exact[n].grad.norm()
        assert off <= 20 * half_step(dtype), (n, float(off))


def test_a_captured_step_is_the_eager_one(example):
    """Forward and backward of a whole step in one graph, replayed on new tokens with other masks; an eager step of the same weights lives
    beside it."""
    import paper_2205_09707_amd as pl
    dtype = torch.bfloat16
    weights, ids, targets, q_offsets, k_offsets = _state(dtype)
    w = {n: t.to(DEV) for n, t in weights.items()}
    ids, targets, q_offsets, k_offsets = (t.to(DEV) for t in (ids, targets, q_offsets, k_offsets))
    rng = torch.tensor([9, 1], device=DEV)

    def step():
        x = pl.plaid_dropout(pl.plaid_embedding(w["table"], ids, scale=WIDTH ** 0.5), P, rng)
        h, statistics = pl.plaid_layer_norm(x, w["w1"], w["b1"], return_statistics=True)
        q = h.view(-1, HEADS, DIM)
        out, lse = pl.plaid_cross_attention(q, w["k"], w["v"], q_offsets, k_offsets, return_lse=True)
        loss, top = pl.plaid_cross_entropy(out.view(-1, WIDTH), w["table"], targets, return_lse=True)
        dh, d_table = pl.plaid_cross_entropy_backward(torch.full_like(loss, 1e-2), out.view(-1, WIDTH), w["table"], targets, top)
        dq, dk, dv, _ = pl.plaid_cross_attention_backward(dh.view_as(q), q, w["k"], w["v"], out, lse, q_offsets, k_offsets)
        dx, dw, db = pl.plaid_layer_norm_backward(dq.view(-1, WIDTH), x, w["w1"], w["b1"], statistics)
        pl.plaid_embedding_backward(pl.plaid_dropout(dx, P, rng), ids, VOCABULARY, scale=WIDTH ** 0.5, add_to=d_table)
        return loss, d_table, dk, dv, dw, db

    with torch.no_grad():
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            step()
        torch.cuda.current_stream().wait_stream(side)
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            got = step()
        for call in (1, 2, 3, 4):
            rng[1] = call
            ids.copy_(torch.randint(-1, VOCABULARY, ids.shape, device=DEV))
            targets.copy_(torch.randint(-1, VOCABULARY, targets.shape, device=DEV))
            graph.replay()
            torch.cuda.synchronize()
            for a, b in zip(got, step()):
                assert torch.equal(a, b)


def test_on_a_side_stream_and_by_two_threads(example):
    """Calls of two threads on two streams give what they give alone."""
    import threading

    import paper_2205_09707_amd as pl
    weights, ids, targets, _, _ = _state(torch.bfloat16)
    table, ids, targets = weights["table"].to(DEV), ids.to(DEV), targets.to(DEV)
    w1, b1 = weights["w1"].to(DEV), weights["b1"].to(DEV)

    def step(i):
        x = pl.plaid_embedding(table, ids.roll(i), scale=3.0)
        y, statistics = pl.plaid_layer_norm(x, w1, b1, return_statistics=True)
        loss, lse = pl.plaid_cross_entropy(y, table, targets, return_lse=True)
        dy, d_table = pl.plaid_cross_entropy_backward(torch.ones_like(loss), y, table, targets, lse)
        dx, _, _ = pl.plaid_layer_norm_backward(dy, x, w1, b1, statistics)
        return loss, pl.plaid_embedding_backward(dx, ids.roll(i), VOCABULARY, scale=3.0, add_to=d_table)

    want = [step(i) for i in range(2)]
    torch.cuda.synchronize()
    got, failed = [None, None], []

    def work(i):
        try:
            with torch.no_grad(), torch.cuda.stream(torch.cuda.Stream()):
                for _ in range(10):
                    got[i] = step(i)
                torch.cuda.current_stream().synchronize()
        except Exception as e:  # noqa: BLE001 (a thread's failure has to reach the test)
            failed.append(e)

    threads = [threading.Thread(target=work, args=(i,)) for i in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    assert not failed, failed
    for a, b in zip(got, want):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
