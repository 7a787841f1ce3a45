"""Plain implementations, in 64 bits and on the CPU, of what the reader's operators compute, and how far a kernel that keeps its
sums in 32 bits and rounds what the header says may be from them.

Bounds.  u is half a unit in the last place of the type (2^-8 bf16, 2^-11 fp16), e = 2e-5 stands for the arithmetic in 32 bits:
scores of a few tens have 2^-20 of relative error, their exponentials the same, sums of a few thousand terms less than that.
Weights round to the type before they multiply (relative u), results once more.  In fp16 a weight below 2^-14 is held to 2^-25
of the largest one.  delta = d_out . out is taken from the rounded out, whose error is that of the forward pass.
"""
import math

import torch

U = {torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}
TINY = {torch.bfloat16: 1e-38, torch.float16: 2.0 ** -24}  # where the type's spacing no longer shrinks
E32 = 2e-5
E2M1 = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], dtype=torch.float64)


# ------------------------------------------------------------------------------------------------ the cache
def quantise(x):
    """Codes [..., dim] and scale bytes [..., dim / 32] of a 16-bit tensor: the smallest power of two that keeps a group within 6,
    the nearest code, of two as near the even one."""
    top, lowest, most = (14, -23, 65504.0) if x.dtype == torch.float16 else (126, -126, 3.3895313892515355e38)
    g = x.double().unflatten(-1, (-1, 32))
    finite = torch.isfinite(g).all(-1)
    largest = torch.where(finite, g.abs().amax(-1), 0.0)
    e = torch.full(largest.shape, lowest)
    for p in range(lowest, top):
        e = torch.where(largest > 6 * 2.0 ** p, p + 1, e)
    power = torch.pow(torch.tensor(2.0, dtype=torch.float64), e.double())[..., None]
    distance = (g.abs()[..., None] - E2M1 * power[..., None]).abs()
    distance = torch.where(E2M1 * power[..., None] > most, math.inf, distance)
    best = distance.amin(-1, keepdim=True)
    code = torch.arange(8)
    rank = torch.where(distance == best, code % 2 * 8 + code, 99)  # even codes first
    code = rank.argmin(-1)
    code = code + 8 * torch.signbit(x.double().unflatten(-1, (-1, 32))).long()
    return code.flatten(-2), torch.where(finite, e + 127, 255)


def value_of(code, scale):
    power = torch.where(scale == 255, math.nan, torch.pow(torch.tensor(2.0, dtype=torch.float64), scale.double() - 127))
    c = code.unflatten(-1, (-1, 32))
    return (torch.where(c >= 8, -E2M1[c & 7], E2M1[c & 7]) * power[..., None]).flatten(-2)


def put(data, slot, head, k_code, k_scale, v_code, v_scale, block_size, dim):
    """One token's codes and scales of one head into the bytes of a cache [blocks, heads, region]."""
    region = data[slot // block_size, head]
    t, codes, groups = slot % block_size, block_size * dim // 2, dim // 32
    for d in range(dim // 2):
        region[t * dim // 2 + d] = int(k_code[2 * d]) | int(k_code[2 * d + 1]) << 4
    for i in range(groups):
        for m in range(16):
            at = codes + t // 16 * 8 * dim + (t // 4 % 4 * 16 + m) * (dim // 8) + i * 4 + t % 4
            region[at] = int(v_code[32 * i + m]) | int(v_code[32 * i + 16 + m]) << 4
    for i in range(groups):
        region[2 * codes + t * groups + i] = int(k_scale[i])
        region[2 * codes + block_size * groups + t * groups + i] = int(v_scale[i])


# ------------------------------------------------------------------------------------------------ attention
def attend(q, k, v, scale, bias=None, seen=None, d_out=None, dtype=torch.bfloat16):
    """Attention of rows q [m, D] to keys k, v [n, D] in 64 bits.  bias [n]; seen [m, n] hides keys from rows.  Returns a dict of
    values and, under the same name with "_bound", of how far a kernel may be off: out, lse and with d_out dq, dk, dv, dbias."""
    u, tiny = U[dtype], TINY[dtype]
    q, k, v = q.double(), k.double(), v.double()
    m, n = q.shape[0], k.shape[0]
    live = torch.ones(n, dtype=torch.bool) if bias is None else bias.double() != -math.inf
    k, v = torch.where(live[:, None], k, 0.0), torch.where(live[:, None], v, 0.0)
    s = q @ k.T * scale + (0.0 if bias is None else bias.double())
    s = s.masked_fill(~(live[None] if seen is None else live[None] & seen), -math.inf)
    top = s.amax(-1, keepdim=True) if n else torch.full((m, 1), -math.inf, dtype=torch.float64)
    w = torch.exp(s - torch.where(top == -math.inf, 0.0, top))
    total = w.sum(-1, keepdim=True)
    p = w / torch.where(total == 0, 1.0, total)
    out = p @ v
    spread = p @ v.abs()  # what relative errors of weights act on
    size = (q.abs() @ k.abs().T * abs(scale)).amax(-1) if n else torch.zeros(m, dtype=torch.float64)
    e = E32 * (1 + size / 16)[:, None]  # errors of 32-bit scores grow with their terms
    floor = n * 2.0 ** -25 * (v.abs().amax() if n else 0.0) if dtype == torch.float16 else 0.0
    r = {"out": out, "out_bound": u * out.abs() + (u + e) * spread + floor + tiny,
         "lse": (torch.where(top == -math.inf, 0.0, top) + torch.log(total)).squeeze(-1), "lse_bound": (e * (1 + top.abs().clamp(max=1e4))).squeeze(-1)}
    if d_out is None:
        return r
    d_out = d_out.double()
    dp = d_out @ v.T
    ds = p * (dp - (d_out * out).sum(-1, keepdim=True))
    off = ((u + u + e) * (d_out.abs() * spread)).sum(-1, keepdim=True) + floor * d_out.abs().sum(-1, keepdim=True)  # delta's error
    rough = d_out.abs() @ v.abs().T
    ds_off = u * ds.abs() + p * off + e * p * (rough + off)
    p_floor = 2.0 ** -25 if dtype == torch.float16 else 0.0  # weights and ds below the type's normal range
    p_off = (u + e) * p + p_floor
    ds_off = ds_off + p_floor
    r["dv"], r["dv_bound"] = p.T @ d_out, u * (p.T @ d_out).abs() + p_off.T @ d_out.abs() + tiny
    r["dq"], r["dq_bound"] = ds @ k * scale, u * (ds @ k * scale).abs() + ds_off @ k.abs() * abs(scale) + tiny
    r["dk"], r["dk_bound"] = ds.T @ q * scale, u * (ds.T @ q * scale).abs() + ds_off.T @ q.abs() * abs(scale) + tiny
    r["dbias"], r["dbias_off"] = ds.sum(0), ds_off.sum(0)
    return r


def cross(q, k, v, q_lengths, k_lengths, scale, bias=None, d_out=None):
    """plaid_cross_attention and its gradients over packed tensors [tokens, heads, D] on the CPU, with bounds."""
    dtype, (_, heads, dim), kv_heads = q.dtype, q.shape, k.shape[1]
    names = ["out", "lse"] + (["dq", "dk", "dv", "dbias"] if d_out is not None else [])
    like = {"out": q, "lse": q[..., 0], "dq": q, "dk": k, "dv": k, "dbias": k[:, 0, 0]}
    r = {}
    for n in names:
        r[n] = torch.zeros(like[n].shape, dtype=torch.float64)
        r[n + "_bound"] = torch.zeros(like[n].shape, dtype=torch.float64)
    r["lse"].fill_(-math.inf)
    a = b = 0
    for m, n in zip(q_lengths, k_lengths):
        rows, keys = slice(a, a + m), slice(b, b + n)
        a, b = a + m, b + n
        for h in range(heads):
            g = h * kv_heads // heads
            x = attend(q[rows, h], k[keys, g], v[keys, g], scale, None if bias is None else bias[keys], None, None if d_out is None else d_out[rows, h], dtype)
            for name in ("out", "lse") + (("dq",) if d_out is not None else ()):
                r[name][rows, h] = x[name]
                r[name + "_bound"][rows, h] = x[name + "_bound"]
            if d_out is not None:
                for name in ("dk", "dv"):  # heads that share keys add up; the sum is rounded once
                    r[name][keys, g] += x[name]
                    r[name + "_bound"][keys, g] += x[name + "_bound"]
                r["dbias"][keys] += x["dbias"]
                r["dbias_bound"][keys] += x["dbias_off"]
    if d_out is not None:
        r["dbias_bound"] += U[dtype] * r["dbias"].abs() + TINY[dtype]
    return r


def close(got, want, bound, what):
    got = got.double().cpu()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))
    off = torch.where(same, 0.0, (got - want).abs())
    bad = ~(off <= bound) & ~same
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.numel()} off, worst {float((off / bound.clamp(min=1e-300))[bad].max()):.3g} times the bound"
