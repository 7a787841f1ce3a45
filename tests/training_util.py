"""What the operators of a reader's training step compute, in 64 bits, and how far a kernel that keeps its sums in 32 bits and rounds
what the header says may be from it.

u is the type's half step (2^-8 bf16, 2^-11 fp16: torch.finfo(t).eps / 2), e = 2^-24 that of 32 bits.  A sum of n terms in 32 bits in any
order is within n e of the sum of their magnitudes (to first order; twice that is allowed throughout); TINY is half the spacing where
the type's no longer shrinks.
"""
import math

import torch

E = 2.0 ** -24
TINY = {torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, bound, what):
    """Every element within its bound; what is not finite has to be the same."""
    got, want = got.detach().double().cpu(), want.detach().double().cpu()
    bound = bound.detach().double().cpu().expand_as(want) if isinstance(bound, torch.Tensor) else torch.full_like(want, float(bound))
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= bound) & ~same
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / bound.clamp(min=1e-300))[bad].max()):.3g} times the bound"


# ------------------------------------------------------------------------------------------------ embedding
def embed(table, ids, scale):
    there = (ids >= 0) & (ids < table.shape[0])
    return torch.where(there[:, None], table.double()[torch.where(there, ids, 0)] * scale, 0.0)


def embed_bound(out, dtype):
    return (half_step(dtype) + 2 * E) * out.abs() + TINY[dtype]


def embed_grad(d_out, ids, vocabulary, scale, before=None):
    """(gradient, bound); before: what it is added to."""
    dtype, width = d_out.dtype, d_out.shape[1]
    there = (ids >= 0) & (ids < vocabulary)
    want, size, count = (torch.zeros((vocabulary, w), dtype=torch.float64, device=d_out.device) for w in (width, width, 1))
    d = d_out[there].double()
    want.index_add_(0, ids[there], d)
    size.index_add_(0, ids[there], d.abs())
    count.index_add_(0, ids[there], torch.ones_like(d[:, :1]))
    want, size = want * scale, size * abs(scale)
    if before is not None:
        want = want + before.double()
    return want, half_step(dtype) * want.abs() + 2 * (count + 3) * E * (size + want.abs()) + TINY[dtype]


# ------------------------------------------------------------------------------------------------ dropout
def philox(counter, key):
    """Ten rounds of Philox4x32 on plain integers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57
        c = [b >> 32 ^ c[1] ^ k[0], b & 0xFFFFFFFF, a >> 32 ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(first, count, p, seed, call):
    """Whether elements first .. first + count - 1 are kept."""
    threshold, low = math.floor(65536 * p + 0.5), 0xFFFFFFFF
    seed, call = seed & 2 ** 64 - 1, call & 2 ** 64 - 1
    got, words, at = [], None, None
    for e in range(first, first + count):
        if e // 8 != at:
            at = e // 8
            words = philox((at & low, at >> 32, call & low, call >> 32), (seed & low, seed >> 32))
        got.append((words[e // 2 % 4] >> 16 * (e & 1)) & 0xFFFF >= threshold)
    return torch.tensor(got), 65536 / (65536 - threshold) if threshold < 65536 else 0.0


# ------------------------------------------------------------------------------------------------ layer norm
def norm(x, weight, bias, eps, d_out=None):
    """A dict of out, statistics and, with d_out, dx, dweight, dbias, and of their bounds.

    A row's sum goes through at most 64 additions of a thread and 10 joins: its mean is within 2^-16 / 2 of the mean magnitude, the
    variance about it and 1 / sqrt of that within the same, relative.  spread is what such an error of the mean is in units of x^."""
    dtype, u, e = x.dtype, half_step(x.dtype), 2.0 ** -16
    rows, width = x.shape
    tiny = TINY[dtype]
    x = x.double()
    w = torch.ones(width, dtype=torch.float64, device=x.device) if weight is None else weight.double()
    b = torch.zeros_like(w) if bias is None else bias.double()
    m = x.mean(1, keepdim=True)
    r = 1 / torch.sqrt(((x - m) ** 2).mean(1, keepdim=True) + eps)
    n = (x - m) * r
    spread = x.abs().mean(1, keepdim=True) * r
    off = e * (spread + n.abs())
    got = {"out": n * w + b, "mean": m[:, 0], "mean_bound": e * x.abs().mean(1), "inverse": r[:, 0], "inverse_bound": e * (1 + spread[:, 0]) * r[:, 0]}
    got["out_bound"] = u * got["out"].abs() + (1 + u) * (off * w.abs() + 4 * E * ((n * w).abs() + b.abs())) + tiny
    if d_out is None:
        return got
    d = d_out.double()
    g = d * w
    mean = lambda t: t.mean(1, keepdim=True)  # noqa: E731
    wide = n.abs() + spread
    got["dx"] = r * (g - mean(g) - n * mean(g * n))
    got["dx_bound"] = u * got["dx"].abs() + 2 * e * r * (1 + spread) * (g.abs() + mean(g.abs()) + wide * mean(g.abs() * wide)) + tiny
    got["dweight"], got["dbias"] = (d * n).sum(0), d.sum(0)
    got["dweight_bound"] = u * got["dweight"].abs() + ((d.abs() * off).sum(0) + 2 * (rows + 8) * E * (d * n).abs().sum(0)) * (1 + u) + tiny
    got["dbias_bound"] = u * got["dbias"].abs() + 2 * (rows + 8) * E * d.abs().sum(0) + tiny
    return got


# ------------------------------------------------------------------------------------------------ cross entropy
def cross_entropy(hidden, weight, targets, scale, d_loss=None):
    """A dict of loss, lse and, with d_loss, d_hidden and d_weight, and of their bounds.

    A score is a sum of `width` products in 32 bits; a probability is off by twice a score's error, relative; G rounds to the type once, its
    targets' entries twice as finely, in fp16 in steps of 2^-24 of 2^15 d_loss's power of two; the states that G is multiplied with carry that power, in fp16 in steps of 2^-24 of
    the largest one's.  What is below 2^-126, the least normal number of 32 bits and of bf16, may become zero, as the exponential's instruction
    and the matrix unit make it: a probability, and its product with the fraction of d_loss (in units of the power: 2^-125 for both), and a state."""
    dtype, u, (rows, width), vocabulary, dev = hidden.dtype, half_step(hidden.dtype), hidden.shape, weight.shape[0], hidden.device
    live = torch.nonzero((targets >= 0) & (targets < vocabulary))[:, 0]
    h, w, t = hidden[live].double(), weight.double(), targets[live]
    at = torch.arange(len(live), device=dev)
    s = h @ w.T * scale
    size = h.abs() @ w.abs().T * abs(scale)
    off = 2 * (width + 4) * E * size.amax(1, keepdim=True) if len(live) else torch.zeros((0, 1), dtype=torch.float64, device=dev)
    lse = torch.logsumexp(s, 1)
    loss = lse - s[at, t]
    full = lambda x, shape: torch.zeros(shape, dtype=torch.float64, device=dev).index_copy_(0, live, x)  # noqa: E731
    # the sum of exponentials: parts of 128, joined one after another
    sum_off = 2 * (vocabulary / 128 + 150) * E
    got = {"loss": full(loss, rows), "loss_bound": full(2 * off[:, 0] + sum_off + 4 * E * (s.abs().amax(1) + loss.abs()), rows) if len(live) else full(loss, rows),
           "lse": full(lse, rows)}
    if d_loss is None:
        return got
    c = d_loss[live].double()[:, None]
    p = torch.exp(s - lse[:, None])
    g = p.clone()
    g[at, t] = torch.expm1(-loss)
    g_off = p * (2 * off + sum_off + 4 * E * (1 + s.abs())) + u * g.abs() * (1 + 2 ** -6)
    # what the target's entry loses in rounding is multiplied too, itself rounded: u of u
    g_off[at, t] = p[at, t] * (2 * off + sum_off + 4 * E * (1 + s.abs()))[at, t] + u * u * g[at, t].abs() * (1 + 2 ** -6)
    power = torch.exp2(torch.where(c == 0, -math.inf, torch.floor(torch.log2(c.abs())) + 1))
    top = power.amax() if len(live) else torch.tensor(0.0, dtype=torch.float64, device=dev)
    if not top > 0:
        top = torch.ones_like(top)
    if dtype == torch.float16:
        g_off = g_off * c.abs() + 2.0 ** -40 * power
        # the packed states: what 2^(exponent - largest) takes below the type's range
        h_off = 2.0 ** -25 * top / power.clamp(min=1e-300) * (power < top)
    else:
        g_off = g_off * c.abs() + 2.0 ** -125 * power
        h_off = 2.0 ** -126 * top / power.clamp(min=1e-300) * (power < top)
    g = g * c
    got["d_hidden"] = full(g @ w * scale, (rows, width))
    got["d_hidden_bound"] = full((1 + u) * (g_off + 2 * (vocabulary / 64 + 100) * E * g.abs()) @ w.abs() * abs(scale), (rows, width))
    got["d_hidden_bound"] += u * got["d_hidden"].abs() + TINY[dtype]
    got["d_weight"] = g.T @ h * scale
    got["d_weight_bound"] = ((1 + u) * ((g_off + 2 * (rows + 8) * E * g.abs()).T @ h.abs() + (g.abs() * h_off).sum(0)[:, None]) * abs(scale)
                             + u * got["d_weight"].abs() + TINY[dtype])
    for name in ("d_hidden", "d_weight"):  # what is beyond the type's largest number rounds to an infinity
        beyond = got[name].abs() - got[name + "_bound"] > torch.finfo(dtype).max
        either = got[name].abs() + got[name + "_bound"] > torch.finfo(dtype).max  # at the border both are right
        got[name + "_bound"] = torch.where(either & ~beyond, math.inf, got[name + "_bound"])
        got[name] = torch.where(beyond, torch.copysign(torch.full_like(got[name], math.inf), got[name]), got[name])
    return got
