"""The prompt's attention, the position rotation and the paged cache in plain 64-bit torch, one
sequence (and head) at a time, with what rounding errors are judged against.  Runs on any device;
pinned on the CPU by test_plain64.py."""
import math

import torch

BF16_HALF_STEP = 2.0 ** -8     # a bf16 rounding, relative to the value
FP32_STEP = 2.0 ** -23         # one step of an fp32 accumulation that may truncate


def attention(q, k, v, n_before):
    """q [n, Hq, d], k and v [m, Hkv, d]; query i sees keys j <= n_before + i.  Returns 64-bit
    out [n, Hq, d], lse [n, Hq], scale [n, Hq, d] (sum_j p_j |v_j|) and mag [n, Hq] (the largest
    sum_c |q_c k_c| / sqrt(d) among the keys a query sees).  No visible key: zeros, minus infinity."""
    n, Hq, d = q.shape
    m, Hkv, _ = k.shape
    out, scale = (torch.zeros(n, Hq, d, dtype=torch.float64, device=q.device) for _ in range(2))
    lse = torch.full((n, Hq), -math.inf, dtype=torch.float64, device=q.device)
    mag = torch.zeros(n, Hq, dtype=torch.float64, device=q.device)
    if n == 0 or m == 0:
        return out, lse, scale, mag
    see = torch.arange(m, device=q.device)[None] <= n_before + torch.arange(n, device=q.device)[:, None]
    some = see.any(1)
    for h in range(Hq):
        kh, vh, qh = k[:, h // (Hq // Hkv)].double(), v[:, h // (Hq // Hkv)].double(), q[:, h].double()
        s = (qh @ kh.T / math.sqrt(d)).masked_fill(~see, -math.inf)
        z = torch.logsumexp(s, -1)
        p = torch.where(see, torch.exp(s - torch.where(some, z, 0.0)[:, None]), 0.0)
        lse[:, h] = torch.where(some, z, -math.inf)
        out[:, h] = p @ vh
        scale[:, h] = p @ vh.abs()
        mag[:, h] = (qh.abs() @ kh.abs().T / math.sqrt(d)).masked_fill(~see, 0.0).amax(-1)
    return out, lse, scale, mag


def logit_error(mag, d):
    """How far an fp32 logit may be off: d products added one by one, then scaled."""
    return (d + 2) * FP32_STEP * mag


def lse_tolerance(lse, mag, d):
    # the logits' error, an exponential and a logarithm good to 2^-20 each, fp32 sums, the result's rounding
    return logit_error(mag, d) + 2.0 ** -19 + lse.abs().clamp(max=1e6) * 2.0 ** -22


def bf16_tolerance(out, scale, mag, d):
    # output rounding; probabilities rounded to bf16; logits and exponentials in fp32, numerator and sum
    return BF16_HALF_STEP * out.abs() + (BF16_HALF_STEP * 1.01 + 2 * logit_error(mag, d)[..., None] + 2.0 ** -18) * scale + 1e-30


def fp32_tolerance(scale, mag, d):
    # two bf16 terms of a probability leave 2^-17 of it at most; the rest as above
    return (2.0 ** -17 + 2 * logit_error(mag, d)[..., None] + 2.0 ** -18) * scale + 1e-30


def rotate(x, positions, inv_freq, interleaved):
    """x [T, H, d] turned by positions[t] * inv_freq[r], in 64 bits; and |x| + |y| of every element's pair."""
    x = x.double()
    r = inv_freq.numel()
    y, size = x.clone(), torch.zeros_like(x)
    angle = positions.double()[:, None] * inv_freq.double()
    for i in range(r):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + r)
        c, s = torch.cos(angle[:, i])[:, None], torch.sin(angle[:, i])[:, None]
        y[..., a] = x[..., a] * c - x[..., b] * s
        y[..., b] = x[..., a] * s + x[..., b] * c
        size[..., a] = size[..., b] = x[..., a].abs() + x[..., b].abs()
    return y, size


def rotate_tolerance(y, size):
    # one rounding to bf16; sine, cosine (2^-21 each), two products and a sum in fp32
    return BF16_HALF_STEP * y.abs() + 2.0 ** -19 * size


def read_paged(pool, row, length):
    """Rows 0 .. length - 1 of a sequence as [length, heads, d]; pages outside the pool read as zeros."""
    page = pool.shape[2]
    out = torch.zeros(length, pool.shape[1], pool.shape[3], dtype=pool.dtype, device=pool.device)
    for p in range(-(-length // page)):
        n = min(page, length - p * page)
        if 0 <= int(row[p]) < pool.shape[0]:
            out[p * page:p * page + n] = pool[int(row[p]), :, :n].transpose(0, 1)
    return out


def decode_paged(q, k_pool, v_pool, table, lens):
    """q [B, Hq, d] over rows 0 .. lens[b] - 1.  Returns what attention() does, for one query each."""
    got = []
    for b, n in enumerate(lens):
        n = max(0, min(int(n), table.shape[1] * k_pool.shape[2]))
        k, v = read_paged(k_pool, table[b].tolist(), n), read_paged(v_pool, table[b].tolist(), n)
        got.append(attention(q[b:b + 1], k, v, n - 1))
    return [torch.cat(x) for x in zip(*got)]


def append_paged(k, v, k_pool, v_pool, table, cache_lens, starts, counts):
    """Writes rows k, v (already [tokens, Hc, d]) into copies of the pools, token by token."""
    k_pool, v_pool = k_pool.clone(), v_pool.clone()
    pages, page = k_pool.shape[0], k_pool.shape[2]
    for b, (t0, n) in enumerate(zip(starts, counts)):
        for i in range(n):
            slot = int(cache_lens[b]) + i
            if not 0 <= slot < table.shape[1] * page:
                continue
            to = int(table[b, slot // page])
            if 0 <= to < pages:
                k_pool[to, :, slot % page] = k[t0 + i]
                v_pool[to, :, slot % page] = v[t0 + i]
    return k_pool, v_pool
