"""What is measured of the operators that a decoder answers with: a paged cache of keys and values as it is written (held in 16, 8 or 4
bits) and read back, attention of new tokens over it, and the choice of the next token from its logits; cases over the range of sizes
that they serve, with the plain form of each (elementary torch operations in 32 bits, the choice in 64) and its definition in 64 bits.

A case's "op" names the operator; its other entries are sizes and options:
  cache_write, cache_read, attention
        batch sequences of up to kv_len positions in pages of `page` positions, kv_heads heads of dim elements; `held`: "same" (the type
        itself), "e4m3" (8 bits, a power of two for each row of a head) or "e2m1" (4 bits, a power of two for every 32 elements of it);
        `ragged`: each sequence has a length of its own, one of them none
  cache_write   new: positions written at the end of each sequence.  What is held in fewer bits is read back in the same pass
  attention     heads query heads and new queries for each sequence, the last of which sees all keys
  sample        rows x vocab logits; temperature, top_k, top_p, min_p; `each`: every row has parameters of its own around these
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}


def listed():
    def cache(name, op, dtype, held, batch, kv_heads, kv_len, dim, page, ragged=False, **more):
        return {"name": name, "op": op, "dtype": dtype, "held": held, "batch": batch, "kv_heads": kv_heads, "kv_len": kv_len, "dim": dim, "page": page, "ragged": ragged, **more}

    def sample(name, dtype, rows, vocab, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, each=False):
        return {"name": name, "op": "sample", "dtype": dtype, "rows": rows, "vocab": vocab, "temperature": temperature, "top_k": top_k, "top_p": top_p, "min_p": min_p, "each": each}

    return [
        # a step of 64 sequences: one position each, latency alone
        cache("write step", "cache_write", "bf16", "same", 64, 8, 256, 128, 16, new=1),
        # prompts of different lengths, held in 8 bits, and read for what follows them
        cache("write prompts e4m3", "cache_write", "bf16", "e4m3", 16, 8, 2048, 128, 64, ragged=True, new=2048),
        # an odd batch of the translation graph's 16 heads of 64, in 4 bits
        cache("write odd e2m1", "cache_write", "f16", "e2m1", 7, 16, 1003, 64, 32, ragged=True, new=501),
        # long sequences are laid out for a pass over all of their positions
        cache("read e4m3", "cache_read", "bf16", "e4m3", 8, 8, 16384, 128, 64, ragged=True),
        cache("read small", "cache_read", "f16", "same", 3, 16, 40, 64, 16, ragged=True),
        # the translation graph's decoder, 40 steps of 64 sentences, 16 heads of 64: latency
        cache("att step small", "attention", "bf16", "same", 64, 16, 40, 64, 16, ragged=True, heads=16, new=1),
        # one new token of each sequence over what came before it
        cache("att step", "attention", "bf16", "same", 8, 8, 16384, 128, 16, ragged=True, heads=32, new=1),
        # the same in 8 bits, more and longer sequences
        cache("att step e4m3", "attention", "bf16", "e4m3", 16, 8, 32768, 128, 64, ragged=True, heads=32, new=1),
        # four tokens to be checked at once, 4 bits
        cache("att four e2m1", "attention", "f16", "e2m1", 32, 4, 8191, 128, 32, ragged=True, heads=32, new=4),
        # one answer, all of the vocabulary: latency
        sample("sample one", "f32", 1, 32768, temperature=0.8),
        # a step of 64 sequences of the translation graph, every one with its own parameters
        sample("sample step", "bf16", 64, 32768, temperature=0.7, top_k=50, top_p=0.95, each=True),
        # many sequences and words, a wide nucleus
        sample("sample wide", "f32", 256, 131071, temperature=1.0, top_p=0.9, min_p=0.0005),
    ]


def _log_int(rng, lo, hi):
    """an integer spread over the logarithm of lo..hi; half of the time a multiple of eight where that fits"""
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    return max(lo, min(hi, n // 8 * 8 if n >= 16 and rng.random() < 0.5 else n))


def _cost(case):
    w = work(case)
    return max(w["bytes"] / 5e12, w["flops"] / 1e15)


def _draw(rng):
    op = rng.choice(["cache_write", "cache_read", "attention", "attention", "attention", "sample", "sample"])
    if op == "sample":
        return {"op": op, "dtype": rng.choice(["f32", "f16", "bf16"]), "rows": _log_int(rng, 1, 512), "vocab": _log_int(rng, 100, 200000), "temperature": rng.choice([0.0, 0.3, 0.7, 1.0, 1.0, 1.5]),
                "top_k": rng.choice([0, 0, 1, 20, 50, 1000]), "top_p": rng.choice([1.0, 1.0, 0.5, 0.9, 0.95]), "min_p": rng.choice([0.0, 0.0, 0.05, 0.001]), "each": rng.random() < 0.5}
    held = rng.choice(["same", "e4m3", "e2m1"])
    case = {"op": op, "dtype": rng.choice(["f16", "bf16", "bf16"]), "held": held, "batch": _log_int(rng, 1, 128), "kv_heads": rng.choice([1, 2, 4, 8, 16]), "kv_len": _log_int(rng, 1, 32768),
            "dim": rng.choice({"same": [32, 64, 64, 72, 128, 128], "e4m3": [32, 64, 80, 128, 128], "e2m1": [32, 64, 96, 128, 128]}[held]), "page": rng.choice([16, 16, 32, 64, 128, 256]), "ragged": rng.random() < 0.5}
    if op == "cache_write":
        case["new"] = rng.choice([1, case["kv_len"], _log_int(rng, 1, case["kv_len"])])
    if op == "attention":
        case["heads"] = case["kv_heads"] * rng.choice([1, 1, 2, 3, 4, 8, 16])
        case["new"] = rng.choice([1, 1, 1, 2, 5, 8])
    return case


def draw(rng):
    most = max(_cost(c) for c in listed())
    while True:
        case = _draw(rng)
        # the plain form holds all positions in 32 bits and every pair of them
        held = 0 if case["op"] == "sample" else case["batch"] * case["kv_heads"] * case["kv_len"] * case["dim"]
        pairs = case["batch"] * case["heads"] * case["new"] * case["kv_len"] if case["op"] == "attention" else 0
        if _cost(case) <= most and held <= 6e8 and pairs <= 3e8:
            return case


# ---- what a power of two and few bits stand for ----------------------------------------

def _block(held, dim):
    return dim if held == "e4m3" else 32


def _power(scale):
    """2^(scale - 127) of bytes; 255 is no number"""
    s = scale.int()
    f = torch.where(s == 0, 1 << 22, s << 23).view(torch.float32)
    return torch.where(s == 255, math.nan, f)


def _held(x, held):
    """(codes, scales) of rows x [..., dim]: every block's largest value at most 448 or 6 times its power of two.  A block with a value that is not finite has no power"""
    top, t = (448.0, x.dtype) if held == "e4m3" else (6.0, x.dtype)
    f = x.float().unflatten(-1, (-1, _block(held, x.shape[-1])))
    fine = torch.isfinite(f).all(-1, keepdim=True)
    f = torch.where(fine, f, 0.0)
    # the largest value that the codes can stand for within the type
    m = (1.875 if held == "e4m3" else 1.5) * 2.0 ** (15 if t is torch.float16 else 127)
    f = f.clamp(-m, m)
    fraction, e = torch.frexp(f.abs().amax(-1, keepdim=True))
    limit, place = (0.875, 9) if held == "e4m3" else (0.75, 3)
    scale = (e - place + (fraction > limit).int() + 127).clamp(0, 254)
    scale = torch.where(fraction == 0, 0, scale)
    # x / 2^(scale - 127), in 64 bits because a float's exponents do not reach that far
    r = (f.double() / _power(scale).double()).clamp(-top, top).float()
    if held == "e4m3":
        codes = r.flatten(-2).to(torch.float8_e4m3fn)
    else:
        a = r.abs()
        c = ((a > 0.25).int() + (a >= 0.75).int() + (a > 1.25).int() + (a >= 1.75).int() + (a > 2.5).int() + (a >= 3.5).int() + (a > 5).int() + 8 * torch.signbit(r).int()).flatten(-2).to(torch.uint8)
        codes = c[..., 0::2] | c[..., 1::2] << 4
    return codes, torch.where(fine, scale, 255).squeeze(-1).to(torch.uint8)


_E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0]


def _stands_for(pages, scales, t):
    """values in 32 bits of pages [..., page, dim] with scales [..., blocks, page], rounded to the type that they were written in"""
    if scales is None:
        return pages.float()
    if pages.dtype is torch.uint8:
        table = torch.tensor(_E2M1 + [-v for v in _E2M1], device=pages.device)
        f = table[torch.stack([pages & 15, pages >> 4], -1).flatten(-2).int()]
    else:
        f = pages.float()
    blocks = scales.shape[-2]
    power = _power(scales).transpose(-1, -2).unsqueeze(-1)
    return (f.unflatten(-1, (blocks, -1)) * power).flatten(-2).to(t).float()


# ---- inputs ----------------------------------------------------------------------------

def _lengths(gen, batch, most, ragged):
    """each sequence's own length, 0..most: one of them whole, one of them empty where there are three or more"""
    n = torch.full((batch,), most, device="cuda", dtype=torch.int32)
    if ragged:
        n = torch.randint(1, most + 1, (batch,), generator=gen, device="cuda", dtype=torch.int32)
        n[0] = most
        if batch >= 3:
            n[1] = 0
    return n


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    t = TYPES[case["dtype"]]
    s = {"op": case["op"], "dtype": t}
    if case["op"] == "sample":
        R, V = case["rows"], case["vocab"]
        # most words are far from the few that fit
        z = 2.5 * torch.randn(R, V, generator=gen, device="cuda")
        n = min(24, V)
        at = torch.randint(0, V, (R, n), generator=gen, device="cuda")
        z.scatter_add_(1, at, 6 + 6 * torch.rand(R, n, generator=gen, device="cuda"))
        s["logits"], s["u"] = z.to(t), torch.rand(R, generator=gen, device="cuda")
        for name in ("temperature", "top_k", "top_p", "min_p"):
            s[name] = case[name]
            if case["each"]:
                f = 0.5 + torch.rand(R, generator=gen, device="cuda")
                if name == "top_p":
                    s[name] = 1 - (1 - case[name]) * f
                elif name == "top_k":
                    s[name] = (case[name] * f).ceil().int()
                else:
                    s[name] = case[name] * f
                if name == "temperature" and R >= 4:
                    s[name][3] = 0.0        # one row wants its most likely word
        return s
    B, K, S, D, P, held = (case[n] for n in ("batch", "kv_heads", "kv_len", "dim", "page", "held"))
    per = -(-S // P)
    s["kv_len"] = S
    s["kv_lengths"] = _lengths(gen, B, S, case["ragged"])
    # a sequence's pages lie anywhere; entries that it does not use name none
    table = torch.randperm(B * per, generator=gen, device="cuda").int().view(B, per)
    used = torch.arange(per, device="cuda") * P < s["kv_lengths"][:, None]
    s["table"] = torch.where(used, table, -1)

    def pages():
        p = torch.randn(B * per, K, P, D, generator=gen, device="cuda").to(t)
        if held == "same":
            return p, None
        codes, scales = zip(*(_held(q, held) for q in p.split(max(1, (1 << 27) // (K * P * D)))))
        return torch.cat(codes), torch.cat(scales).transpose(-1, -2).contiguous()

    s["k_pages"], s["k_scales"] = pages()
    s["v_pages"], s["v_scales"] = pages()
    if case["op"] == "cache_write":
        n = case["new"]
        s["k"], s["v"] = (torch.randn(B, n, K, D, generator=gen, device="cuda").to(t).transpose(1, 2) for _ in range(2))
        s["lengths"] = s["kv_lengths"].clamp(max=n)
        s["start"] = s["kv_lengths"] - s["lengths"]
    elif case["op"] == "attention":
        s["q"] = (1.5 * torch.randn(B, case["new"], case["heads"], D, generator=gen, device="cuda")).to(t).transpose(1, 2)
        s["causal"] = case["new"] > 1
    return s


# ---- plain forms -----------------------------------------------------------------------

def _plain_write(s):
    k, v, table = s["k"], s["v"], s["table"].long()
    B, K, n, D = k.shape
    P = s["k_pages"].shape[2]
    i = torch.arange(n, device="cuda")
    b, i = (i < s["lengths"][:, None]).nonzero(as_tuple=True)
    at = s["start"].long()[b] + i
    page, at = table[b, at // P], at % P
    for x, pages, scales in ((k, s["k_pages"], s["k_scales"]), (v, s["v_pages"], s["v_scales"])):
        rows = x[b, :, i]
        if scales is None:
            pages[page, :, at] = rows
        else:
            codes, powers = _held(rows, "e2m1" if pages.dtype is torch.uint8 else "e4m3")
            pages.view(torch.uint8)[page, :, at] = codes.view(torch.uint8)
            scales[page, :, :, at] = powers


def _plain_read(s):
    """[batch, kv_heads, kv_len, dim] in 32 bits, zero beyond a sequence's length"""
    got = []
    S, table = s["kv_len"], s["table"].clamp_min(0).long()
    live = (torch.arange(S, device="cuda") < s["kv_lengths"][:, None])[:, None, :, None]
    for pages, scales in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])):
        x = pages.view(torch.uint8)[table].view(pages.dtype) if scales is not None else pages[table]
        x = _stands_for(x, None if scales is None else scales[table], s["dtype"])
        x = x.transpose(1, 2).flatten(2, 3)[:, :, :S]
        got.append(torch.where(live, x, 0.0))
    return got


def _plain_attention(s):
    q = s["q"].float()
    k, v = _plain_read(s)
    B, H, n, D = q.shape
    K, S = k.shape[1:3]
    i, j = torch.arange(n, device="cuda")[:, None], torch.arange(S, device="cuda")[None]
    length = s["kv_lengths"][:, None, None]
    see = j < (length - n + 1 + i if s["causal"] else length)
    z = torch.matmul(q.reshape(B, K, H // K * n, D), k.transpose(2, 3)).view(B, H, n, S) / math.sqrt(D)
    z = torch.where(see[:, None], z, -math.inf)
    top = z.amax(3, keepdim=True)
    z -= torch.where(torch.isinf(top), 0.0, top)
    p = z.exp_()
    total = p.sum(3, keepdim=True)
    lse = (torch.log(total) + top).squeeze(3)
    p /= torch.where(total == 0, 1.0, total)
    o = torch.matmul(p.view(B, K, H // K * n, S), v).view(B, H, n, D)
    return o.to(s["dtype"]), lse


def _plain_sample(s):
    """a word is kept or not by sums that lie next to a border, so all of it is in 64 bits"""
    z, u = s["logits"], s["u"].double()
    R, V = z.shape
    temperature, k, p, m = (torch.as_tensor(s[n], device="cuda").to(to).expand(R)[:, None] for n, to in (("temperature", torch.float32), ("top_k", torch.long), ("top_p", torch.float32), ("min_p", torch.float32)))
    z, word = torch.sort(z.float(), dim=1, descending=True, stable=True)     # equal ones in the words' order
    greedy = temperature == 0
    e = torch.exp((z.double() - z[:, :1].double()) / torch.where(greedy, 1.0, temperature).double())
    rank = torch.arange(V, device="cuda")
    keep = (rank < torch.where(k > 0, k, V)) & (~greedy | (rank < 1))
    e = torch.where(keep, e, 0.0)
    total = e.cumsum(1)
    keep &= (total - e < p.double() * total[:, -1:]) | (p >= 1) | (rank < 1)
    keep &= (e >= m.double()) | (rank < 1)
    e = torch.where(keep, e, 0.0)
    total = e.cumsum(1)
    n = torch.minimum((total <= u[:, None] * total[:, -1:]).sum(1), keep.sum(1) - 1)[:, None]
    return word.gather(1, n)[:, 0].int(), torch.log(e.gather(1, n) / total[:, -1:])[:, 0].float()


def run(s):
    op = s["op"]
    if own:
        from paper_1807_05358_amd import operators
        if op == "sample":
            return operators.sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"])
        cache, scales = (s["k_pages"], s["v_pages"], s["table"]), {"k_scales": s["k_scales"], "v_scales": s["v_scales"]}
        if op == "cache_write":
            operators.cache_write(s["k"], s["v"], *cache, s["start"], lengths=s["lengths"], **scales)
            if s["k_scales"] is None:
                return s["k_pages"], s["v_pages"]
        if op == "attention":
            return operators.attention_paged_fwd(s["q"], *cache, s["kv_lengths"], causal=s["causal"], **scales)
        return operators.cache_read(*cache, s["kv_lengths"], kv_len=s["kv_len"], dtype=s["dtype"], **scales)
    if op == "sample":
        return _plain_sample(s)
    if op == "attention":
        return _plain_attention(s)
    if op == "cache_write":
        _plain_write(s)
        if s["k_scales"] is None:
            return s["k_pages"], s["v_pages"]
    return tuple(x.to(s["dtype"]) for x in _plain_read(s))


def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "sample":
        R, V = case["rows"], case["vocab"]
        return {"bytes": R * V * e + 12 * R, "flops": (10 if case["temperature"] else 1) * R * V}
    B, K, S, D = (case[n] for n in ("batch", "kv_heads", "kv_len", "dim"))
    row = {"same": D * e, "e4m3": D + 1, "e2m1": D / 2 + D / 32}[case["held"]]
    some = 0.5 if case["ragged"] else 1.0       # ragged lengths are uniform, so on average half of the positions
    held = 2 * B * K * S * some
    if case["op"] == "cache_read":
        return {"bytes": held * row + 2 * B * K * S * D * e, "flops": held * D}
    if case["op"] == "cache_write":
        new = 2 * B * K * case["new"] * (some if case["new"] > 1 else 1.0)
        written = {"bytes": new * (D * e + row), "flops": 3 * new * D}
        if case["held"] == "same":
            return written
        return {"bytes": written["bytes"] + held * row + 2 * B * K * S * D * e, "flops": written["flops"] + held * D}
    H, n = case["heads"], case["new"]
    return {"bytes": held * row + 2 * B * H * n * D * e + 4 * B * H * n, "flops": 4 * B * H * n * S * some * D}


# ---- definitions in 64 bits ------------------------------------------------------------

def _exact_power(e):
    """2^e, which a power of a tensor is not to the last bit"""
    return (e.long() + 1023 << 52).view(torch.float64)


def _exact_value(code, held):
    """of one code: its bits taken apart"""
    if held == "e4m3":
        c = code.view(torch.uint8).long()
        sign, e, m = c >> 7, c >> 3 & 15, c & 7
        bias, bits = 7, 3
    else:
        c = torch.stack((code % 16, code // 16), -1).flatten(-2).long()
        sign, e, m = c >> 3, c >> 1 & 3, c & 1
        bias, bits = 1, 1
    f = torch.where(e > 0, 1 + m.double() / 2 ** bits, m.double() * 2.0 ** (1 - bits)) * _exact_power(e - bias)
    return torch.where(sign > 0, -f, f)


def _exact_hold(row, held):
    """what is read back of rows [..., dim] of finite values: the nearest of all codes' values, the even code of two as near"""
    x = row.double().unflatten(-1, (-1, _block(held, row.shape[-1])))
    top = 448.0 if held == "e4m3" else 6.0
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(amax > 0, amax, 1.0) / top))      # inputs are far from where the logarithm's rounding counts, but for whole powers:
    e = torch.where(amax / top <= _exact_power(e - 1), e - 1, e)
    e = torch.where(amax / top > _exact_power(e), e + 1, e).clamp_min(-127)
    if held == "e4m3":
        values = _exact_value(torch.arange(127, device=x.device, dtype=torch.uint8), held)
    else:
        values = _exact_value(torch.arange(8, device=x.device, dtype=torch.uint8), held)[0::2]
    a = (x / _exact_power(e)).abs().contiguous()
    hi = torch.searchsorted(values, a).clamp(1, len(values) - 1)
    lo = hi - 1
    far, near = values[hi] - a, a - values[lo]
    c = torch.where((far < near) | ((far == near) & (hi % 2 == 0)), hi, lo)
    return (torch.copysign(values[c], x) * _exact_power(e)).flatten(-2)


def _exact_sequences(case, s):
    """of each sequence its keys and values [kv_heads, length, dim] in 64 bits"""
    P = case["page"]
    for b, n in enumerate(s["kv_lengths"].tolist()):
        which = s["table"][b, :-(-n // P)].long()
        both = []
        for pages, scales in ((s["k_pages"], s["k_scales"]), (s["v_pages"], s["v_scales"])):
            x = pages.view(torch.uint8)[which].view(pages.dtype) if scales is not None else pages[which]
            if scales is None:
                x = x.double()
            else:
                power = scales[which].view(torch.float8_e8m0fnu).to(torch.float32).double().transpose(2, 3)
                x = _exact_value(x, case["held"])
                x = x * power.repeat_interleave(x.shape[-1] // power.shape[-1], -1)
            both.append(x.permute(1, 0, 2, 3).reshape(x.shape[1], -1, x.shape[-1])[:, :n])
        yield b, n, *both


def _exact_sample(s):
    """row after row: the words in the order of their logits, and where the sums pass what they are asked to"""
    words, logs = [], []
    R, V = s["logits"].shape
    of = {n: s[n].tolist() if torch.is_tensor(s[n]) else [s[n]] * R for n in ("temperature", "top_k", "top_p", "min_p")}
    single = lambda x: float(torch.tensor(x, dtype=torch.float32))  # noqa: E731
    for r in range(R):
        order = torch.argsort(s["logits"][r], dim=0, descending=True, stable=True)
        temperature, k, p, m = (of[n][r] for n in ("temperature", "top_k", "top_p", "min_p"))
        if temperature == 0:
            words.append(order[0])
            logs.append(torch.zeros((), dtype=torch.float64, device="cuda"))
            continue
        if k > 0:
            order = order[:k]
        z = s["logits"][r, order].double() / single(temperature)
        e = (z - z[0]).exp()
        if p < 1:
            n = int(torch.searchsorted(e.cumsum(0), single(p) * e.sum().reshape(1))) + 1
            e = e[:max(1, n)]
        e = e[:max(1, int((e >= single(m)).sum()))]
        total = e.cumsum(0)
        n = min(int(torch.searchsorted(total, s["u"][r].double().reshape(1) * total[-1], right=True)), len(e) - 1)
        words.append(order[n])
        logs.append(torch.log(e[n] / total[-1]))
    return torch.stack(words).int(), torch.stack(logs)


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        return _exact_sample(s)
    B, K, S, D = (case[n] for n in ("batch", "kv_heads", "kv_len", "dim"))
    if case["op"] == "attention":
        H, n = case["heads"], case["new"]
        o, lse = torch.zeros(B, H, n, D, device="cuda", dtype=torch.float64), torch.full((B, H, n), -math.inf, device="cuda", dtype=torch.float64)
        for b, length, k, v in _exact_sequences(case, s):
            if length:
                z = s["q"][b].double() @ k.repeat_interleave(H // K, 0).transpose(1, 2) * D ** -0.5
                if s["causal"]:
                    z.masked_fill_(torch.ones(n, length, device="cuda", dtype=torch.bool).triu(length - n + 1), -math.inf)
                lse[b] = torch.logsumexp(z, 2)
                o[b] = torch.softmax(z, 2).nan_to_num_(0.0) @ v.repeat_interleave(H // K, 0)
        return o, lse
    if case["op"] == "cache_write" and case["held"] == "same":
        both = s["k_pages"].double(), s["v_pages"].double()
        starts, lengths, table = (s[n].tolist() for n in ("start", "lengths", "table"))
        if sum(lengths) > 20000:
            return None         # one position after another
        for x, pages in zip((s["k"], s["v"]), both):
            for b in range(B):
                for i in range(lengths[b]):
                    at = starts[b] + i
                    pages[table[b][at // case["page"]], :, at % case["page"]] = x[b, :, i].double()
        return both
    k, v = (torch.zeros(B, K, S, D, device="cuda", dtype=torch.float64) for _ in range(2))
    starts = s["start"].tolist() if case["op"] == "cache_write" else None
    for b, n, *both in _exact_sequences(case, s):
        for to, x, new in zip((k, v), both, (s.get("k"), s.get("v"))):
            to[b, :, :n] = x
            if starts is not None and n:
                to[b, :, starts[b]:n] = _exact_hold(new[b, :, :n - starts[b]], case["held"])
    return k, v
