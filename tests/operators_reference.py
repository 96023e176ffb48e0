"""Plain definitions in 64 bits of the training operators, with a bound for every output: how far a computation may be off
that holds its sums in 32 bits and rounds where include/ff_ops.h says so.

u = 2^-24 is half a step of a float, `half(t)` half a step of the type.  A sum of n terms in 32 bits is off by at most
(number of additions a term passes through) * u * sum |terms|; the kernels' longest chains are below the counts used here."""
import math

import torch

U = 2.0 ** -24


def half(t):
    return torch.finfo(t).eps / 2


def tiny(t):
    """half of the smallest step of the type, near zero"""
    return torch.finfo(t).smallest_normal * torch.finfo(t).eps / 2


def close(got, want, bound, what):
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    same = (got == want) | (torch.isnan(got) & torch.isnan(want))       # infinities, too
    off = torch.where(same, torch.zeros_like(want), (got - want).abs() - bound)
    bad = ~(off <= 0)
    if bad.any():
        at = tuple(int(i) for i in bad.nonzero()[0])
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} values are off, the first at {at}: got {got[at].item()}, want {want[at].item()}, "
                             f"bound {(bound if not torch.is_tensor(bound) else bound.expand_as(want)[at]).item() if torch.is_tensor(bound) else bound}")


# ---- layer norm ------------------------------------------------------------------------

def layernorm_fwd(x, w, b, res, eps):
    """{name: (value, bound)}"""
    t = x.dtype
    h = x if res is None else (x.double() + res.double()).to(t)
    f, wd = h.double(), w.double()
    bd = torch.zeros_like(wd) if b is None else b.double()
    C = f.shape[1]
    mean = f.mean(1, keepdim=True)
    var = ((f - mean) ** 2).mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(var + eps)
    y = (f - mean) * rstd * wd + bd
    # a lane adds up to 64 elements, then 6 + 16 partial sums: 100 additions with the products
    c = 100 * U
    e_mean = c * f.abs().mean(1, keepdim=True)
    e_var = c * var + 2 * e_mean * (f - mean).abs().mean(1, keepdim=True) + e_mean ** 2
    e_rstd = rstd * (e_var / (2 * (var + eps)) + 4 * U)
    e_y = wd.abs() * (rstd * (e_mean + U * (f.abs() + mean.abs())) + (f - mean).abs() * e_rstd) + 4 * U * (wd * (f - mean) * rstd).abs() + 2 * U * y.abs()
    return {"y": (y, half(t) * y.abs() + e_y * 1.01 + tiny(t)), "h": (f, 0.0), "mean": (mean[:, 0], e_mean[:, 0] + U * mean[:, 0].abs()), "rstd": (rstd[:, 0], e_rstd[:, 0])}


def layernorm_bwd(dy, h, w, mean, rstd, dh):
    t = h.dtype
    dyd, f, wd, r = dy.double(), h.double(), w.double(), rstd.double()[:, None]
    m = mean.double()[:, None]
    xh = (f - m) * r
    e_xh = 2 * U * xh.abs() + U * r * (f - m).abs()
    g = dyd * wd
    mg, mx = g.mean(1, keepdim=True), (g * xh).mean(1, keepdim=True)
    dx = r * (g - mg - xh * mx)
    if dh is not None:
        dx = dx + dh.double()
    c = 100 * U
    e_mg = c * g.abs().mean(1, keepdim=True)
    e_mx = c * (g * xh).abs().mean(1, keepdim=True) + (g.abs() * e_xh).mean(1, keepdim=True)
    e_dx = r * (4 * U * g.abs() + e_mg + 2 * U * mg.abs() + xh.abs() * e_mx + (e_xh + 4 * U * xh.abs()) * mx.abs()) + 4 * U * dx.abs()
    if dh is not None:
        e_dx = e_dx + 2 * U * dh.double().abs()
    # a lane adds every 2048th row or so, then 4 waves, a sixteenth of at most 1024 partial sums and 16 of those
    cr = (8 + h.shape[0] / 512 + 4 + 64 + 16) * U
    dw, db = (dyd * xh).sum(0), dyd.sum(0)
    e_dw = cr * (dyd * xh).abs().sum(0) + (dyd.abs() * e_xh).sum(0)
    return {"dx": (dx, half(t) * dx.abs() + e_dx + tiny(t)), "dw": (dw, half(t) * dw.abs() + 1.01 * e_dw + tiny(t)),
            "db": (db, half(t) * db.abs() + 1.01 * cr * dyd.abs().sum(0) + tiny(t))}


# ---- attention -------------------------------------------------------------------------

def sees(B, Sq, Sk, causal, q_lengths, kv_lengths, device):
    i, j = torch.arange(Sq, device=device).view(1, 1, Sq, 1), torch.arange(Sk, device=device).view(1, 1, 1, Sk)
    nq = torch.full((B,), Sq, device=device) if q_lengths is None else q_lengths.long().clamp(0, Sq)
    nk = torch.full((B,), Sk, device=device) if kv_lengths is None else kv_lengths.long().clamp(0, Sk)
    nq, nk = nq.view(B, 1, 1, 1), nk.view(B, 1, 1, 1)
    see = (i < nq) & (j < nk)
    return see & (j <= i + nk - nq) if causal else see


def _attention(q, k, v, causal, q_lengths, kv_lengths, scale):
    B, H, Sq, D = q.shape
    G = H // k.shape[1]
    Sk = k.shape[2]
    see = sees(B, Sq, Sk, causal, q_lengths, kv_lengths, q.device).expand(B, H, Sq, Sk)
    # what nobody may see does not count, whatever it holds
    keys = sees(B, 1, Sk, False, None, kv_lengths, q.device).view(B, 1, Sk, 1)
    rows = sees(B, Sq, 1, False, q_lengths, None, q.device).view(B, 1, Sq, 1)
    qd = torch.where(rows, q.double(), 0.0)
    kd, vd = (torch.where(keys, x.double(), 0.0).repeat_interleave(G, 1) for x in (k, v))
    z = torch.where(see, scale * (qd @ kd.transpose(2, 3)), -math.inf)
    lse = torch.logsumexp(z, 3)
    p = torch.exp(z - torch.where(torch.isinf(lse), 0.0, lse)[..., None])
    # the scores' error: D additions at most (in fact D / 16 steps), the scale's rounding, the exponent's argument
    a = scale * (qd.abs() @ kd.abs().transpose(2, 3))
    e_z = U * ((D / 4 + 4) * a + 4 * z.abs().nan_to_num(posinf=0))
    return qd, kd, vd, z, lse, p, torch.where(see, e_z, 0.0), rows


def attention_fwd(q, k, v, causal=False, q_lengths=None, kv_lengths=None, scale=None):
    t = q.dtype
    scale = q.shape[3] ** -0.5 if scale is None else scale
    qd, kd, vd, z, lse, p, e_z, _ = _attention(q, k, v, causal, q_lengths, kv_lengths, scale)
    o = p @ vd
    worst = e_z.amax(3, keepdim=True) if z.shape[3] else torch.zeros_like(z.sum(3, keepdim=True))
    n = z.shape[3]
    # numerator: p rounded once; both sums: a lane's share of the keys in turn, at most all of them / 2, and the rescalings
    c = half(t) + 4 * worst + (n / 16 + 64) * U
    return {"o": (o, half(t) * o.abs() + 1.01 * c * (p @ vd.abs()) + tiny(t) * (1 + n / 256)),
            "lse": (lse, torch.where(torch.isinf(lse), 0.0, worst[..., 0] + (n / 16 + 64) * U + 4 * U * lse.abs()))}


def attention_bwd(dout, q, k, v, causal=False, q_lengths=None, kv_lengths=None, scale=None):
    """from the exact o and lse, which the kernel gets rounded to the type and to float"""
    t = q.dtype
    B, H, Sq, D = q.shape
    K, Sk = k.shape[1], k.shape[2]
    scale = D ** -0.5 if scale is None else scale
    qd, kd, vd, z, lse, p, e_z, rows = _attention(q, k, v, causal, q_lengths, kv_lengths, scale)
    do = torch.where(rows, dout.double(), 0.0)
    o = p @ vd
    dp = do @ vd.transpose(2, 3)
    delta = (do * o).sum(3, keepdim=True)
    ds = p * (dp - delta)
    dq, dk, dv = scale * ds @ kd, scale * ds.transpose(2, 3) @ qd, p.transpose(2, 3) @ do
    e_p = half(t) + 2 * e_z + 4 * U * lse.abs().nan_to_num(posinf=0)[..., None] + 16 * U           # relative, of p as the products see it
    mag = do.abs() @ vd.abs().transpose(2, 3)
    e_delta = (half(t) + (D / 4) * U) * (do * o).abs().sum(3, keepdim=True)
    # ds: rounded once; its parts in 32 bits; the smallest step of the type relative to the largest |do| of the group's heads
    unit = do.abs().amax((2, 3)).view(B, K, H // K).amax(2).repeat_interleave(H // K, 1).view(B, H, 1, 1) if do.numel() else 0
    e_ds = e_p * ds.abs() + p * (e_delta + (D / 4 + 8) * U * (mag + delta.abs())) + tiny(t) * unit * (p > 0)
    n = Sq * (H // K)
    c = lambda m: (m / 16 + 64) * U         # additions of the sums over keys or rows

    def group(x):
        return x.reshape(B, K, H // K, Sk, D).sum(2)

    b_q = scale * (e_ds + c(Sk) * ds.abs()) @ kd.abs()
    b_k = scale * group((e_ds + c(n) * ds.abs()).transpose(2, 3) @ qd.abs())
    b_v = group(((e_p + c(n)) * p + tiny(t) * (p > 0) / (1024 if t == torch.float16 else 1)).transpose(2, 3) @ do.abs())
    dk, dv = group(dk), group(dv)
    return {"dq": (dq, half(t) * dq.abs() + 1.01 * b_q + tiny(t)), "dk": (dk, half(t) * dk.abs() + 1.01 * b_k + tiny(t)),
            "dv": (dv, half(t) * dv.abs() + 1.01 * b_v + tiny(t))}, o, lse


# ---- loss over a vocabulary ------------------------------------------------------------

def _vocab(x, w, targets, ignore_index, first):
    xd, wd = x.double(), w.double()
    z = xd @ wd.t()
    at = targets.long() - first
    live = targets != ignore_index
    here = live & (at >= 0) & (at < w.shape[0])
    D = x.shape[1]
    e_z = U * (D / 4 + 8) * (xd.abs() @ wd.abs().t())
    return xd, wd, z, at.clamp(0, w.shape[0] - 1), live, here, e_z


def vocab_loss_fwd(x, w, targets, ignore_index=-100, first=0):
    xd, wd, z, at, live, here, e_z = _vocab(x, w, targets, ignore_index, first)
    lse = torch.logsumexp(z, 1)
    zt = torch.where(here, z.gather(1, at[:, None])[:, 0], 0.0)
    worst = e_z.amax(1) + 4 * U * z.abs().amax(1)
    e = worst + (w.shape[0] / 1024 + 128) * U + 4 * U * lse.abs()
    loss = torch.where(live, torch.where(here, lse - zt, math.nan), 0.0)
    return {"loss": (loss, e + worst + U * loss.abs().nan_to_num()), "lse": (lse, e), "target_logit": (zt, worst)}


def vocab_loss_bwd(dloss, x, w, targets, lse, ignore_index=-100, first=0):
    """with the lse that the kernel is given"""
    t = x.dtype
    xd, wd, z, at, live, here, e_z = _vocab(x, w, targets, ignore_index, first)
    p = torch.exp(z - lse.double()[:, None])
    hot = torch.zeros_like(p).scatter_(1, at[:, None], here.double()[:, None])
    f = torch.where(live, dloss.double(), 0.0)[:, None]
    g = (p - hot) * f
    e_g = half(t) * g.abs() + f.abs() * p * (2 * e_z + 8 * U * (1 + z.abs() + lse.double().abs()[:, None])) + 4 * U * g.abs()
    if t == torch.float16:      # the smallest step of the type, relative to the largest |dloss|, times 2^12
        e_g = e_g + tiny(t) * dloss.abs().max().double() / 4096 * (f != 0) if dloss.numel() else e_g
    dx, dw = g @ wd, g.t() @ xd
    c = lambda m: (m / 8 + 64) * U
    return {"dx": (dx, half(t) * dx.abs() + 1.01 * (e_g + c(w.shape[0]) * g.abs()) @ wd.abs() + tiny(t)),
            "dw": (dw, half(t) * dw.abs() + 1.01 * (e_g + c(x.shape[0]) * g.abs()).t() @ xd.abs() + tiny(t))}
