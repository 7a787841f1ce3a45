"""One layer of a reader over the passages that a search finds, from tokens to the loss of the next ones, in training and in answering.

    python examples/reader.py            # on a GPU

A search gives the passages of each question and their scores; `plaid_decompress_passages` gives their token vectors, packed.  The
layer attends to its own tokens through a paged cache in four bits and to the passages' tokens by cross attention, with the
passage's score as the bias of its tokens' keys: what the answer's loss says about the bias is the gradient of the scores.  Tokens come
in through an embedding whose table is the vocabulary of the loss as well; dropout and layer norm stand between.
"""
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2205_09707_amd as pl  # noqa: E402

DTYPE, HEADS, KV_HEADS, DIM, WIDTH, VOCABULARY = torch.bfloat16, 8, 2, 64, 512, 1000


class CrossAttention(torch.autograd.Function):
    @staticmethod
    def forward(ctx, q, k, v, bias, q_offsets, k_offsets):
        out, lse = pl.plaid_cross_attention(q, k, v, q_offsets, k_offsets, key_bias=bias, return_lse=True)
        ctx.save_for_backward(q, k, v, bias, out, lse, q_offsets, k_offsets)
        return out

    @staticmethod
    def backward(ctx, d_out):
        q, k, v, bias, out, lse, q_offsets, k_offsets = ctx.saved_tensors
        dq, dk, dv, dbias = pl.plaid_cross_attention_backward(d_out, q, k, v, out, lse, q_offsets, k_offsets, key_bias=bias)
        return dq, dk, dv, dbias, None, None


class Embedding(torch.autograd.Function):
    @staticmethod
    def forward(ctx, table, ids, scale):
        ctx.save_for_backward(ids)
        ctx.rows, ctx.scale = table.shape[0], scale
        return pl.plaid_embedding(table, ids, scale=scale)

    @staticmethod
    def backward(ctx, d_out):
        return pl.plaid_embedding_backward(d_out, *ctx.saved_tensors, ctx.rows, scale=ctx.scale), None, None


class Dropout(torch.autograd.Function):
    """residual + dropout of x; rng [2]: a seed and the number of the call, of which the backward pass makes the same mask."""

    @staticmethod
    def forward(ctx, x, residual, p, rng):
        ctx.save_for_backward(rng)
        ctx.p = p
        return pl.plaid_dropout(x, p, rng, residual=residual)

    @staticmethod
    def backward(ctx, d_out):
        return pl.plaid_dropout(d_out, ctx.p, *ctx.saved_tensors), d_out if ctx.needs_input_grad[1] else None, None, None


class LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias):
        out, statistics = pl.plaid_layer_norm(x, weight, bias, return_statistics=True)
        ctx.save_for_backward(x, weight, bias, statistics)
        return out

    @staticmethod
    def backward(ctx, d_out):
        return pl.plaid_layer_norm_backward(d_out, *ctx.saved_tensors)


class CrossEntropy(torch.autograd.Function):
    @staticmethod
    def forward(ctx, hidden, weight, targets, scale):
        loss, lse = pl.plaid_cross_entropy(hidden, weight, targets, scale=scale, return_lse=True)
        ctx.save_for_backward(hidden, weight, targets, lse)
        ctx.scale = scale
        return loss

    @staticmethod
    def backward(ctx, d_loss):
        return pl.plaid_cross_entropy_backward(d_loss, *ctx.saved_tensors, scale=ctx.scale) + (None, None)


class Norm(torch.nn.Module):
    def __init__(self, device):
        super().__init__()
        self.weight = torch.nn.Parameter(torch.ones(WIDTH, dtype=DTYPE, device=device))
        self.bias = torch.nn.Parameter(torch.zeros(WIDTH, dtype=DTYPE, device=device))

    def forward(self, x):
        return LayerNorm.apply(x, self.weight, self.bias)


class Layer(torch.nn.Module):
    def __init__(self, device):
        super().__init__()
        linear = lambda n, m: torch.nn.Linear(n, m, bias=False, dtype=DTYPE, device=device)  # noqa: E731
        self.own_qkv, self.own_out = linear(WIDTH, (HEADS + 2 * KV_HEADS) * DIM), linear(HEADS * DIM, WIDTH)
        self.q, self.kv, self.out = linear(WIDTH, HEADS * DIM), linear(128, 2 * KV_HEADS * DIM), linear(HEADS * DIM, WIDTH)
        self.norm, self.last_norm = Norm(device), Norm(device)
        self.table = torch.nn.Parameter(torch.randn(VOCABULARY, WIDTH, dtype=DTYPE, device=device) * WIDTH ** -0.5)
        self.rng = torch.tensor([17, 0], device=device)  # a seed, and how many masks were made

    def tokens(self, ids):
        """States of packed tokens."""
        return Embedding.apply(self.table, ids, WIDTH ** 0.5)

    def dropout(self, x, residual, p):
        self.rng[1] += 1
        return Dropout.apply(x, residual, p, self.rng.clone())

    def loss(self, x, targets):
        """The mean of -log of the targets' probabilities, over the tokens that have one (not negative)."""
        return CrossEntropy.apply(self.last_norm(x), self.table, targets, 1.0).sum() / (targets >= 0).sum()

    def passages(self, vectors):
        """Keys and values of packed token vectors."""
        return self.kv(vectors.to(DTYPE)).view(-1, 2 * KV_HEADS, DIM).split(KV_HEADS, 1)

    def read(self, x, k, v, bias, q_offsets, k_offsets, p=0.0):
        """Cross attention of packed tokens x to their question's passages, with dropout of probability p."""
        q = self.q(self.norm(x)).view(-1, HEADS, DIM)
        return self.dropout(self.out(CrossAttention.apply(q, k, v, bias, q_offsets, k_offsets).view(-1, HEADS * DIM)), x, p)

    def answer(self, x, answers, added, k, v, bias, k_offsets):
        """The layer for the next tokens x, added[r] (int32, on the device) of every answer r, behind those that the cache holds."""
        q_offsets, slots = answers.extend(added, x.shape[0])
        q, own_k, own_v = self.own_qkv(self.norm(x)).view(-1, HEADS + 2 * KV_HEADS, DIM).split([HEADS, KV_HEADS, KV_HEADS], 1)
        pl.plaid_cache_write(answers.cache, own_k, own_v, slots)
        own = pl.plaid_cached_attention(q, answers.cache, answers.table, answers.lengths, q_offsets)
        return self.read(x + self.own_out(own.view(-1, HEADS * DIM)), k, v, bias, q_offsets, k_offsets)


class Answers:
    """The paged cache of n answers of at most `longest` tokens."""

    def __init__(self, n, longest, block_size, device):
        width = -(-longest // block_size)
        self.block_size = block_size
        self.cache = pl.PagedCache.empty(n * width, block_size, KV_HEADS, DIM, DTYPE, device)
        self.table = torch.full((n, width), -1, dtype=torch.int32, device=device)
        self.lengths = torch.zeros(n, dtype=torch.int32, device=device)
        self.free = torch.arange(n * width, dtype=torch.int32, device=device)

    def extend(self, added, count):
        """Room for added[r] more tokens of every answer, `count` in all: (offsets of the new tokens, their slots)."""
        offsets, self.lengths, _, slots, wanted = pl.plaid_block_tables(self.lengths, added, self.table, self.free, self.block_size, count)
        self.free = self.free[int(wanted):]
        return offsets, slots


def passages_of(index, questions, k):
    """Packed token vectors of every question's passages, the questions' offsets in them, and the token's passage, and the scores."""
    ids, scores = pl.plaid_search(index, questions, nprobe=2, t_cs=0.45, ndocs=64, k=k)
    capacity = int(pl.plaid_decompress_passages(index, ids.reshape(-1), 0, vectors=False, indices=False)[0][-1])
    offsets, vectors, _ = pl.plaid_decompress_passages(index, ids.reshape(-1), capacity, indices=False)
    passage = torch.repeat_interleave(torch.arange(ids.numel(), device=ids.device), offsets.diff(), output_size=capacity)
    return vectors, offsets[::k].contiguous(), passage, scores.reshape(-1)


def main(steps=8, tokens=24, k=10, seed=0):
    from synth import make_workload, tiny_config
    torch.manual_seed(seed)
    device = torch.device("cuda", 0)
    w = make_workload(tiny_config(C=256, P=2000, lo=5, hi=80, nbits=2, nq=6, seed=42), noise="calibrated")
    names = ("centroids", "doc_offsets", "codes", "residuals", "bucket_weights", "ivf_offsets", "ivf_pids")
    index = pl.plaid_index_from_view({n: getattr(w, n).to(device) for n in names}, w.cfg.nbits)
    vectors, k_offsets, passage, scores = passages_of(index, w.queries.to(device), k)
    n = w.queries.shape[0]
    layer = Layer(device)

    # training: answers of different lengths; the scores are learnt with the layer
    lengths = torch.tensor([tokens - 3 * r for r in range(n)])
    q_offsets = torch.cat([torch.zeros(1, dtype=torch.int64), lengths.cumsum(0)]).to(device)
    ids = torch.randint(0, VOCABULARY, (int(lengths.sum()),), device=device)
    targets = ids.roll(-1)
    targets[q_offsets[1:] - 1] = -1  # nothing comes after an answer's last token
    learnt = (scores - scores.mean()).requires_grad_()
    optimizer = torch.optim.Adam([*layer.parameters(), learnt], lr=1e-3)
    losses = []
    for _ in range(steps):
        optimizer.zero_grad()
        keys, values = layer.passages(vectors)
        loss = layer.loss(layer.read(layer.tokens(ids), keys, values, learnt[passage].to(DTYPE), q_offsets, k_offsets, p=0.1), targets)
        loss.backward()
        optimizer.step()
        losses.append(float(loss.detach()))

    # answering: prompts at once, then token by token
    with torch.no_grad():
        keys, values = layer.passages(vectors)
        bias = learnt[passage].to(DTYPE)
        answers = Answers(n, 2 * tokens, 16, device)
        out = layer.answer(layer.tokens(ids), answers, lengths.to(device, torch.int32), keys, values, bias, k_offsets)
        one = torch.ones(n, dtype=torch.int32, device=device)
        last = out[q_offsets[1:] - 1]
        for _ in range(4):
            best = torch.matmul(layer.last_norm(last), layer.table.T).argmax(1)
            last = layer.answer(layer.tokens(best), answers, one, keys, values, bias, k_offsets)
    pl.plaid_index_free(index)
    return losses, learnt.grad, out, last, answers


if __name__ == "__main__":
    losses, grad, out, last, answers = main()
    print("loss %.4f -> %.4f" % (losses[0], losses[-1]))
    print("gradient of the passages' scores: norm %.3g" % float(grad.norm()))
    print("answers hold", answers.lengths.tolist(), "tokens; the last ones' states have the norms", [round(float(t), 2) for t in last.float().norm(dim=1)])
