"""Plain definitions in 64 bits of the operators that a decoder answers with (include/ff_ops.h): what a paged cache holds and reads back,
attention over it with a bound of how far it may be off, and the choice of a word.  On the CPU or the GPU, one value after the other where that is plainest."""
import math

import torch

from operators_reference import U, half, tiny

E4M3 = [(-1 if c >> 7 else 1) * ((1 + (c & 7) / 8) * 2.0 ** ((c >> 3 & 15) - 7) if c >> 3 & 15 else (c & 7) / 8 * 2.0 ** -6) for c in range(256)]
E4M3[127] = E4M3[255] = math.nan
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]
POWERS = [2.0 ** (s - 127) for s in range(255)] + [math.nan]
TOP = {"e4m3": 448.0, "e2m1": 6.0}


def table(values, device):
    return torch.tensor(values, dtype=torch.float64, device=device)


def block(held, dim):
    return dim if held == "e4m3" else 32


def hold(x, held):
    """(codes as whole numbers [..., dim], scales [..., blocks]) of rows x: the least power, the nearest code, the even one of two as near"""
    t = x.dtype
    d = x.double().unflatten(-1, (-1, block(held, x.shape[-1])))
    fine = torch.isfinite(d).all(-1, keepdim=True)
    most = (15 / 8 if held == "e4m3" else 3 / 2) * 2.0 ** (15 if t == torch.float16 else 127)
    d = torch.where(fine, d, 0.0).clamp(-most, most)
    powers = table(POWERS[:255], x.device)
    # the first power that is large enough
    scale = torch.searchsorted(powers * TOP[held], d.abs().amax(-1).contiguous())
    values = table((E4M3 if held == "e4m3" else E2M1)[:127 if held == "e4m3" else 8], x.device)
    a = (d.abs() / powers[scale][..., None]).contiguous()
    hi = torch.searchsorted(values, a).clamp(1, len(values) - 1)
    up, down = values[hi] - a, a - values[hi - 1]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, hi - 1)
    code = code + torch.signbit(d) * (128 if held == "e4m3" else 8)
    return torch.where(fine, code, 0).flatten(-2), torch.where(fine[..., 0], scale, 255)


def codes_of(pages):
    """[..., dim] of pages: whole numbers"""
    if pages.dtype == torch.float8_e4m3fn:
        return pages.view(torch.uint8).long()
    return torch.stack([pages & 15, pages >> 4], -1).flatten(-2).long()


def stands_for(codes, scales, held, t):
    """values, rounded to the type, of codes [..., dim] with scales [..., blocks]"""
    values = table(E4M3 if held == "e4m3" else E2M1, codes.device)[codes].unflatten(-1, (scales.shape[-1], -1))
    return (values * table(POWERS, codes.device)[scales.long()][..., None]).flatten(-2).to(t).double()


def dense(pages, scales, tab, lengths, kv_len, t):
    """[batch, kv_heads, kv_len, dim] in 64 bits, zero behind the lengths, NaN where the table has no page"""
    if scales is None:
        x = pages.double()
    else:
        x = stands_for(codes_of(pages), scales.transpose(2, 3), "e4m3" if pages.dtype == torch.float8_e4m3fn else "e2m1", t)
    N, K, P, D = x.shape
    out = torch.zeros(tab.shape[0], K, kv_len, D, dtype=torch.float64, device=pages.device)
    for b, n in enumerate(lengths.tolist()):
        for i in range(min(n, kv_len, tab.shape[1] * P)):
            at = int(tab[b, i // P])
            out[b, :, i] = x[at, :, i % P] if 0 <= at < N else math.nan
    return out


def attention(q, k, v, nk, causal=False, q_lengths=None, scale=None):
    """(o, its bound, lse, its bound) over dense keys k, v [batch, kv_heads, kv_len, dim] (64 bits) of lengths nk"""
    t = q.dtype
    B, H, n, D = q.shape
    S = k.shape[2]
    k, v = (x.repeat_interleave(H // k.shape[1], 1) for x in (k, v))
    scale = D ** -0.5 if scale is None else scale
    i, j = torch.arange(n, device=q.device).view(1, 1, n, 1), torch.arange(S, device=q.device).view(1, 1, 1, S)
    nk = nk.long().clamp(0, S).view(B, 1, 1, 1)
    nq = (torch.full((B,), n, device=q.device) if q_lengths is None else q_lengths.long().clamp(0, n)).view(B, 1, 1, 1)
    see = ((j < nk) & (i < nq) & ((j <= i + nk - nq) if causal else True)).expand(B, H, n, S)
    rows = (i < nq)[..., 0].expand(B, 1, n)[..., None]
    qd = torch.where(rows, q.double(), 0.0)
    none = torch.isnan(k).all(3)[:, :, None] & see          # positions without a page
    k, v = torch.where(torch.isnan(k).all(3, keepdim=True), 0.0, k), torch.where(torch.isnan(v).all(3, keepdim=True), 0.0, v)
    z = torch.where(see, scale * (qd @ k.transpose(2, 3)), -math.inf)
    lse = torch.logsumexp(z, 3) if S else torch.full((B, H, n), -math.inf, dtype=torch.float64, device=q.device)
    p = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
    # a score: D / 4 + 4 additions at most and the roundings of the scale and of the exponent's argument, which is relative to a maximum that is up to 2^8 behind
    e_z = torch.where(see, U * ((D / 4 + 4) * scale * (qd.abs() @ k.abs().transpose(2, 3)) + 4 * z.abs().nan_to_num(posinf=0) + 16), 0.0)
    worst = e_z.amax(3) if S else torch.zeros_like(lse)
    # p as the products see it: rounded once; in bfloat16 cut off, which leaves less than a step, 2 half(t) of p, that is rounded and added.  Sums over a wave's share of the positions, four waves, and the runs
    once = half(t) if t == torch.float16 else 2 * half(t) ** 2
    c = once + 4 * worst[..., None] + (S / 8 + 128) * U
    o = p @ v
    top = v.abs().amax((2, 3), keepdim=True) if S else torch.zeros_like(o[:, :, :1, :1])
    bad = none.any(3)
    o, lse = torch.where(bad[..., None], math.nan, o), torch.where(bad, math.nan, lse)
    # probabilities of float16 end at 2^-25 of 2^8 times the row's largest
    low = S * 2.0 ** -33 * top if t == torch.float16 else S * 2.0 ** -126 * top
    return o, half(t) * o.abs() + 1.01 * c * (p @ v.abs()) + tiny(t) + low, lse, torch.where(torch.isinf(lse), 0.0, worst + (S / 8 + 128) * U + 4 * U * lse.abs())


def choose(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(word, logprob) of one row of logits: the list of words, cut and gone through; parameters are Python numbers (of a float's values where they are one)"""
    z = [float(x) + 0.0 for x in z.double().tolist()]
    if any(math.isnan(x) for x in (*z, u, top_p, min_p)) or max(z) == -math.inf or not 0 <= temperature < math.inf:
        return -1, math.nan
    order = sorted(range(len(z)), key=lambda i: (-z[i], i))
    if temperature == 0:
        return order[0], 0.0
    most = z[order[0]]
    w = [1.0 if z[i] == most else math.exp((z[i] - most) / temperature) for i in order]
    n = len(w) if top_k <= 0 else min(top_k, len(w))
    if top_p < 1:
        total, run, k = math.fsum(w[:n]), 0.0, 0
        while k < n and (k == 0 or run < top_p * total):
            run, k = run + w[k], k + 1
        n = k
    while n > 1 and w[n - 1] < min_p:
        n -= 1
    total, run = math.fsum(w[:n]), 0.0
    for k in range(n):
        run += w[k]
        if run > max(u, 0.0) * total:
            break
    while k > 0 and w[k] == 0:
        k -= 1
    return order[k], math.log(w[k] / total)
