"""Cross entropy and its gradients in 64 bits with bounds that stay relative: to the distance of a probability from one where it is near one, and, for
d_weight, to each row's own d_loss.

u is the type's half step, e = 2^-24 that of 32 bits.  A score is off by `off`: a sum of `width` products in 32 bits, twice n e of their magnitudes.  With
the target's score the largest its loss is log1p of a sum of exponentials of differences, so that the loss, and 1 - p = -expm1(-loss) with it, is off by
r = 2 off + (what the sum of exponentials is off by) + (the exponents' roundings), relative; so is every other probability.  G of the target is expm1 of the
target's score less the maximum, which is nothing, and less the logarithm beside it, which is the loss: r, relative to G itself.  G rounds to the type
once, its targets' entries twice as finely; in fp16 both in steps of 2^-24 of 2^15 times the power of two above d_loss: 2^-40 of that.

In fp16 the states that G is multiplied with for d_weight are scaled so that the largest state times d_loss's power of all rows has 2^15 to 2^16; what rounds,
rounds by 2^-25: 2^-40 of that largest product.  In bf16 they carry the power itself: what is below 2^-126 of the largest may become zero."""
import torch

from training_util import E, TINY, half_step


def relative(hidden, weight, targets, scale, d_loss, exact=False):
    """A dict of loss, d_hidden and d_weight, and of their bounds.  exact: the scores are numbers of 32 bits, their products sums without a rounding and the
    scale a power of two, so that only their differences round."""
    dtype, u, (rows, width), vocabulary, dev = hidden.dtype, half_step(hidden.dtype), hidden.shape, weight.shape[0], hidden.device
    live = torch.nonzero((targets >= 0) & (targets < vocabulary))[:, 0]
    h, w, t, c = hidden[live].double(), weight.double(), targets[live], d_loss[live].double()[:, None]
    at = torch.arange(len(live), device=dev)
    s = h @ w.T * scale
    off = 2 * (width + 4) * E * (h.abs() @ w.abs().T * abs(scale)).amax(1, keepdim=True)
    own = s[at, t]
    others = s.clone()
    others[at, t] = -torch.inf
    # loss = log(1 + the sum of the others beside the target), without the loss of digits where that is nothing
    beside = torch.logsumexp(others, 1) - own
    loss = torch.nn.functional.softplus(beside, threshold=1e3)
    sum_off = 2 * (vocabulary / 128 + 150) * E
    r = 2 * off + sum_off + 8 * E * (1 + s.abs().amax(1, keepdim=True))
    if exact:
        r = sum_off + 8 * E * (1 + (s.amax(1, keepdim=True) - s).amax(1, keepdim=True))
    # near one the loss is the sum itself and off by r of it; far from one it is a difference of scores
    loss_off = r[:, 0] * torch.minimum(torch.exp(beside), torch.ones_like(loss)) + 4 * E * loss
    far = own < others.amax(1)
    loss_off = torch.where(far, r[:, 0] + 4 * E * loss, loss_off)
    full = lambda x, shape: torch.zeros(shape, dtype=torch.float64, device=dev).index_copy_(0, live, x)  # noqa: E731
    got = {"loss": full(loss, rows), "loss_bound": full(loss_off, rows)}
    g = torch.exp(s - own[:, None] - loss[:, None])
    g_off = g * (r + u * (1 + 2 ** -6))
    mine = torch.expm1(-loss)
    g[at, t] = mine
    g_off[at, t] = r[:, 0] * torch.where(far, 1 + mine, -mine) + u * u * (1 + 2 ** -6) * mine.abs()
    power = torch.exp2(torch.floor(torch.log2(c.abs())) + 1)
    g_off = g_off * c.abs() + (2.0 ** -40 if dtype == torch.float16 else 2.0 ** -125) * power
    g = g * c
    got["d_hidden"] = full(g @ w * scale, (rows, width))
    got["d_hidden_bound"] = full((1 + u) * (g_off + 2 * (vocabulary / 64 + 100) * E * g.abs()) @ w.abs() * abs(scale), (rows, width))
    got["d_hidden_bound"] += u * got["d_hidden"].abs() + TINY[dtype]
    got["d_weight"] = g.T @ h * scale
    lost = (2.0 ** -40 * (power * h.abs()).amax() if dtype == torch.float16 else 2.0 ** -126 * power.amax()) * (g.abs() / power).sum(0)[:, None]
    got["d_weight_bound"] = ((1 + u) * ((g_off + 2 * (rows + 8) * E * g.abs()).T @ h.abs() + lost) * abs(scale) + u * got["d_weight"].abs() + TINY[dtype])
    return got
