"""The key-value cache and the attention that reads it, as cases that can be timed.

Three kinds:
  cache   k and v of `tokens` new tokens are written into a paged cache that holds `bits` bits a value, and `context` tokens
          (the new ones among them) are read back as packed 16-bit k and v.
  decode  one new token for each of `requests` requests attends to its own tokens in the cache.
  prompt  packed prompts attend to themselves, causally, and to the tokens that came before them.

Lengths run from `shortest` to `longest` over the requests, the same ones for every seed, in an order that the seed gives.  Cache
layout: k and v [pages, kv_heads, page, head_dim] in 16 bits or as codes of 8 or 4 bits (two to a byte, the first in the low
half), scales [pages, kv_heads, page, 4] in bf16: k scale, k offset, v scale, v offset of a token; value = scale * code + offset.
Slot s of the cache is token s % page of page s // page.
"""
import math

import torch

own = False


def _cache(name, tokens, context, bits, kv_heads=8, head_dim=128, page=16, dtype="bf16"):
    c = {"kind": "cache", "tokens": tokens, "context": context, "bits": bits, "kv_heads": kv_heads, "head_dim": head_dim,
         "page": page, "dtype": dtype}
    return dict(c, name=name) if name else c


def _decode(name, requests, shortest, longest, bits, heads=32, kv_heads=8, head_dim=128, page=16, dtype="bf16"):
    c = {"kind": "decode", "requests": requests, "shortest": shortest, "longest": longest, "bits": bits, "heads": heads,
         "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype}
    return dict(c, name=name) if name else c


def _prompt(name, requests, shortest, longest, before=0, heads=32, kv_heads=8, head_dim=128, dtype="bf16"):
    c = {"kind": "prompt", "requests": requests, "shortest": shortest, "longest": longest, "before": before, "heads": heads,
         "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # the newest token of each of 16 requests is kept as it is: what one call of each costs
        _cache("cache_16_tokens_16bit", 16, 16, 16),
        # a prompt of odd length goes into an 8-bit cache and comes back for a check or a second pass
        _cache("cache_prompt_8bit", 2047, 2047, 8, page=64),
        # a chunk of a long prompt is added to a 4-bit cache, and the whole context is read for the prompt's attention
        _cache("cache_chunk_4bit_fp16", 1000, 32768, 4, dtype="f16", page=32),
        # many prompts at once into a 16-bit cache, and their contexts out of it
        _cache("cache_large_16bit", 16384, 65536, 16),
        # a chat of one user, a few hundred tokens in: latency
        _decode("decode_one_request", 1, 333, 333, 16),
        # one user over a long document: all of the chip works on one request
        _decode("decode_long_document_4bit", 1, 131071, 131071, 4, heads=64, page=64),
        # a served batch whose requests are anywhere between their first and their last token
        _decode("decode_ragged_batch_8bit", 32, 1, 4096, 8, page=16),
        # small heads, one KV head to each query head, fp16
        _decode("decode_own_kv_heads_fp16", 24, 100, 3000, 16, heads=16, kv_heads=16, head_dim=64, page=32, dtype="f16"),
        # a full batch in a 16-bit cache: the bandwidth case
        _decode("decode_full_batch", 64, 2048, 8192, 16, page=64),
        # a question of a few dozen tokens: latency
        _prompt("prompt_one_short", 1, 77, 77),
        # prompts of different lengths that arrived together, packed, most of them behind a longer or shorter context
        _prompt("prompt_packed", 12, 65, 2048, before=1024),
        # whole long prompts: the matrix cores' case
        _prompt("prompt_long", 2, 8192, 8192),
    ]


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("cache", "decode", "prompt"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    head_dim = rng.choice((128, 128, 64))
    bits, page = rng.choice((16, 8, 4)), rng.choice((16, 32, 64, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 8))
    if kind == "cache":
        context = _log_between(rng, 1, 65536)
        return _cache(None, min(context, _log_between(rng, 1, 16384)), context, bits, kv_heads, head_dim, page, dtype)
    if kind == "decode":
        requests = _log_between(rng, 1, 64)
        longest = _log_between(rng, 1, min(131072, 64 * 8192 // requests))
        return _decode(None, requests, _log_between(rng, 1, longest), longest, bits, kv_heads * rng.choice((1, 4, 4, 8)), kv_heads,
                       head_dim, page, dtype)
    longest = _log_between(rng, 1, 8192)
    requests = _log_between(rng, 1, max(1, min(16, (8192 // longest) ** 2)))
    heads = kv_heads * rng.choice([g for g in (1, 4, 4, 8) if g * kv_heads <= 32])
    return _prompt(None, requests, _log_between(rng, 1, longest), longest, rng.choice((0, 0, _log_between(rng, 1, 2048))) if longest <= 4096 else 0,
                   heads, kv_heads, head_dim, dtype)


def _lengths(case, shortest, longest):
    n = case["requests"]
    return [longest if n == 1 else round(shortest + (longest - shortest) * i / (n - 1)) for i in range(n)]


def _befores(case):
    """tokens in front of each prompt"""
    n = case["requests"]
    return [round(case["before"] * (i + 1) / n) for i in range(n)]


def _dtype(case):
    return torch.float16 if case["dtype"] == "f16" else torch.bfloat16


def _codes(shape, bits, g):
    """codes as values of a normal distribution get them: a range of about five deviations over all codes"""
    def some():
        return torch.randn(shape, generator=g, device="cuda", dtype=torch.float16).mul_((1 << bits) / 5.2).add_(((1 << bits) - 1) / 2).round_().clamp_(0, (1 << bits) - 1).to(torch.uint8)
    return some() if bits == 8 else some() | (some() << 4)


def _pages(case, pages, g):
    """a cache with something in every slot; k has about the spread that attention sees, v less"""
    hk, p, d, bits = case["kv_heads"], case["page"], case["head_dim"], case["bits"]
    if bits == 16:
        k = torch.randn((pages, hk, p, d), generator=g, device="cuda", dtype=_dtype(case))
        return k, torch.randn((pages, hk, p, d), generator=g, device="cuda", dtype=_dtype(case)).mul_(0.5), None
    k, v = (_codes((pages, hk, p, d * bits // 8), bits, g) for _ in range(2))
    step = 5.2 / ((1 << bits) - 1) * torch.rand((pages, hk, p, 2), generator=g, device="cuda").add_(0.5)
    step[..., 1] *= 0.5
    low = -step * (((1 << bits) - 1) / 2) * torch.rand((pages, hk, p, 2), generator=g, device="cuda").mul_(0.4).add_(0.8)
    scales = torch.stack((step[..., 0], low[..., 0], step[..., 1], low[..., 1]), -1)
    return k, v, scales.to(torch.bfloat16).contiguous()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt, d, hk = _dtype(case), case["head_dim"], case["kv_heads"]
    s = dict(case)

    def normal(*shape, by=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(by).to(dt)

    if case["kind"] == "cache":
        n, ctx, p = case["tokens"], case["context"], case["page"]
        pages = -(-ctx // p) + 3
        s["cache_k"], s["cache_v"], s["scales"] = _pages(case, pages, g)
        # the context's pages lie anywhere; its last tokens are the new ones
        order = torch.randperm(pages, generator=host)[: -(-ctx // p)]
        t = torch.arange(ctx)
        s["slots"] = (order[t // p] * p + t % p).cuda()
        s["new_slots"] = s["slots"][ctx - n:].contiguous()
        # k and v as the fused projection's output has them: one row a token
        row = normal(n, 2 * hk * d)
        s["k"], s["v"] = row[:, : hk * d].view(n, hk, d), row[:, hk * d:].view(n, hk, d)
        return s
    h = case["heads"]
    lengths = _lengths(case, case["shortest"], case["longest"])
    order = torch.randperm(len(lengths), generator=host).tolist()
    if case["kind"] == "decode":
        p = case["page"]
        lengths = [lengths[i] for i in order]
        need = [-(-n // p) for n in lengths]
        pages = sum(need) + 3
        s["cache_k"], s["cache_v"], s["scales"] = _pages(case, pages, g)
        ids = torch.randperm(pages, generator=host)
        table = torch.zeros((len(lengths), max(need)), dtype=torch.int32)
        at = 0
        for i, n in enumerate(need):
            table[i, :n] = ids[at:at + n]
            at += n
        s["page_table"], s["lengths"] = table.cuda(), torch.tensor(lengths, dtype=torch.int32, device="cuda")
        # q in the front of the fused projection's rows
        s["q"] = normal(len(lengths), (h + 2 * hk) * d, by=1.5)[:, : h * d].view(len(lengths), h, d)
        return s
    before = _befores(case)
    nq, nk = [lengths[i] for i in order], [lengths[i] + before[i] for i in order]
    s["q_starts"], s["k_starts"] = (torch.tensor([0] + n, dtype=torch.int32).cumsum(0).to(torch.int32).cuda() for n in (nq, nk))
    # (the longest is known where the plain form pads; the packed form takes what the starts say)
    s["longest_q"], s["longest_k"] = max(nq), max(nk)
    if not case["before"]:
        row = normal(sum(nq), (h + 2 * hk) * d)
        q, k, v = row[:, : h * d], row[:, h * d:(h + hk) * d], row[:, (h + hk) * d:]
        q.mul_(1.5)
    else:
        q, k, v = normal(sum(nq), h * d, by=1.5), normal(sum(nk), hk * d), normal(sum(nk), hk * d)
    s["q"], s["k"], s["v"] = q.view(-1, h, d), k.view(-1, hk, d), v.view(-1, hk, d)
    return s


# The plain forms

def _unpack(codes, bits):
    return codes if bits == 8 else torch.stack((codes & 15, codes >> 4), -1).flatten(-2)


def _values(codes, scales, bits, which):
    """what the codes stand for, in 32 bits"""
    if bits == 16:
        return codes.float()
    return _unpack(codes, bits).float() * scales[..., 2 * which, None].float() + scales[..., 2 * which + 1, None].float()


def _encode(x, bits):
    """codes, scale and offset of each last axis"""
    x, top = x.float(), torch.full((), float((1 << bits) - 1), device=x.device)
    low = x.amin(-1, keepdim=True)
    scale = ((x.amax(-1, keepdim=True) - low) / top).to(torch.bfloat16)
    scale = torch.where(scale == 0, torch.ones_like(scale), scale)
    offset = low.to(torch.bfloat16)
    code = torch.minimum(((x - offset.float()) / scale.float()).round().clamp_min(0), top).to(torch.uint8)
    return (code if bits == 8 else code[..., 0::2] | (code[..., 1::2] << 4)), torch.cat((scale, offset), -1)


def _plain_cache(s):
    p, bits = s["page"], s["bits"]
    page, at = s["new_slots"] // p, s["new_slots"] % p
    if bits == 16:
        s["cache_k"][page, :, at], s["cache_v"][page, :, at] = s["k"], s["v"]
    else:
        (ck, ak), (cv, av) = _encode(s["k"], bits), _encode(s["v"], bits)
        s["cache_k"][page, :, at], s["cache_v"][page, :, at], s["scales"][page, :, at] = ck, cv, torch.cat((ak, av), -1)
    page, at = s["slots"] // p, s["slots"] % p
    scales = None if bits == 16 else s["scales"][page, :, at]
    return tuple(_values(s[c][page, :, at], scales, bits, w).to(_dtype(s)) for w, c in enumerate(("cache_k", "cache_v")))


def _softmax(scores, seen):
    """rows of zeros where nothing is seen"""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    return e.div_(e.sum(-1, keepdim=True).clamp_min(1e-37))


def _plain_decode(s):
    hk, d, bits = s["kv_heads"], s["head_dim"], s["bits"]
    table = s["page_table"].long()
    n, tokens = table.shape[0], table.shape[1] * s["page"]
    scales = None if bits == 16 else s["scales"][table]
    k, v = (_values(s[c][table], scales, bits, w).transpose(1, 2).reshape(n * hk, tokens, d) for w, c in enumerate(("cache_k", "cache_v")))
    q = s["q"].float().reshape(n * hk, -1, d)
    seen = torch.arange(tokens, device="cuda") < s["lengths"][:, None, None, None]
    scores = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(n, hk, -1, tokens)
    weights = _softmax(scores, seen).view(n * hk, -1, tokens)
    return torch.bmm(weights, v).view(n, -1, d).to(_dtype(s))


def _plain_prompt(s):
    h, hk, d, n = s["heads"], s["kv_heads"], s["head_dim"], s["requests"]

    def padded(x, starts, longest):
        """[n, longest] places of packed rows, and which of them are rows"""
        at = starts[:-1, None].long() + torch.arange(longest, device="cuda")
        there = at < starts[1:, None]
        return x.float()[at.clamp_max(x.shape[0] - 1)].transpose(1, 2), at, there

    q, q_at, q_there = padded(s["q"], s["q_starts"], s["longest_q"])
    k, _, k_there = padded(s["k"], s["k_starts"], s["longest_k"])
    v, _, _ = padded(s["v"], s["k_starts"], s["longest_k"])
    lq, lk = (s[x][1:] - s[x][:-1] for x in ("q_starts", "k_starts"))
    # the heads that share a KV head stand under each other
    q = q.reshape(n * hk, h // hk * s["longest_q"], d)
    scores = torch.bmm(q, k.reshape(n * hk, -1, d).transpose(1, 2).contiguous()).mul_(d ** -0.5).view(n, hk, h // hk, s["longest_q"], s["longest_k"])
    i, j = torch.arange(s["longest_q"], device="cuda"), torch.arange(s["longest_k"], device="cuda")
    seen = (j <= i[:, None] + (lk - lq)[:, None, None]) & k_there[:, None, :]
    weights = _softmax(scores, seen[:, None, None]).view(n * hk, -1, s["longest_k"])
    o = torch.bmm(weights, v.reshape(n * hk, -1, d)).view(n, h, s["longest_q"], d).transpose(1, 2)
    out = torch.empty((s["q"].shape[0], h, d), dtype=_dtype(s), device="cuda")
    out[q_at[q_there]] = o[q_there].to(out.dtype)
    return out


def run(s):
    if not own:
        return {"cache": _plain_cache, "decode": _plain_decode, "prompt": _plain_prompt}[s["kind"]](s)
    import paper_2507_04610_amd as any4
    if s["kind"] == "cache":
        any4.any4_kv_write(s["k"], s["v"], s["new_slots"], s["cache_k"], s["cache_v"], s["scales"], bits=s["bits"])
        return any4.any4_kv_read(s["cache_k"], s["cache_v"], s["slots"], s["scales"], bits=s["bits"], dtype=s["k"].dtype)
    if s["kind"] == "decode":
        return any4.any4_attn_decode(s["q"], s["cache_k"], s["cache_v"], s["page_table"], s["lengths"], s["scales"], bits=s["bits"])
    return any4.any4_attn_prompt(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"])


def work(case):
    d, hk = case["head_dim"], case["kv_heads"]
    if case["kind"] == "prompt":
        h, lengths, before = case["heads"], _lengths(case, case["shortest"], case["longest"]), _befores(case)
        pairs = sum(n * b + n * (n + 1) // 2 for n, b in zip(lengths, before))
        nq, nk = sum(lengths), sum(lengths) + sum(before)
        return {"bytes": 4 * d * (nq * h + nk * hk) + 8 * (len(lengths) + 1), "flops": 4 * d * h * pairs}
    kept = hk * (d * case["bits"] // 4 + (8 if case["bits"] < 16 else 0))              # bytes of a token in the cache
    if case["kind"] == "cache":
        whole = hk * 4 * d
        return {"bytes": (case["tokens"] + case["context"]) * (whole + kept + 8), "flops": 6 * (case["tokens"] + case["context"]) * hk * d}
    h, lengths = case["heads"], _lengths(case, case["shortest"], case["longest"])
    return {"bytes": sum(lengths) * kept + 4 * sum(-(-n // case["page"]) for n in lengths) + 4 * len(lengths) * (h * d + 1),
            "flops": 4 * sum(lengths) * h * d}


# The definition in 64 bits, one request and head at a time

def _exact_values(codes, scales, bits, which):
    """[tokens, head_dim] of one KV head in 64 bits"""
    if bits == 16:
        return codes.double()
    c = codes.int()
    if bits == 4:
        wide = torch.empty((c.shape[0], 2 * c.shape[1]), dtype=torch.int32, device=c.device)
        wide[:, 0::2], wide[:, 1::2] = c % 16, c // 16
        c = wide
    return c.double() * scales[:, 2 * which:2 * which + 1].double() + scales[:, 2 * which + 1:2 * which + 2].double()


def _exact_attention(q, k, v, seen):
    """q [n, d], k and v [m, d], seen [n, m]"""
    s = (q @ k.T.contiguous()) / math.sqrt(q.shape[1])
    s[~seen] = -math.inf
    w = torch.softmax(s, -1)
    w[~seen.any(-1)] = 0
    return w @ v


def exact(case, seed):
    s = prepare(case, seed)
    d, hk = case["head_dim"], case["kv_heads"]
    if case["kind"] == "cache":
        bits, p = case["bits"], case["page"]
        out = []
        for w, (new, cache) in enumerate((("k", "cache_k"), ("v", "cache_v"))):
            got = torch.empty((case["context"], hk, d), dtype=torch.float64, device="cuda")
            for j in range(hk):
                held = s[cache][:, j].flatten(0, 1)[s["slots"]]
                got[:, j] = _exact_values(held, None if bits == 16 else s["scales"][:, j].flatten(0, 1)[s["slots"]], bits, w)
                x = s[new][:, j].double()
                if bits < 16:
                    low, high, top = x.min(1, keepdim=True).values, x.max(1, keepdim=True).values, 2 ** bits - 1
                    step, low = ((high - low) / top).to(torch.bfloat16).double(), low.to(torch.bfloat16).double()
                    step[step == 0] = 1
                    x = torch.clamp(torch.round((x - low) / step), 0, top) * step + low
                got[case["context"] - case["tokens"]:, j] = x
            out.append(got)
        return tuple(out)
    h = case["heads"]
    shared = h // hk
    if case["kind"] == "decode":
        out = torch.zeros((case["requests"], h, d), dtype=torch.float64, device="cuda")
        for i, n in enumerate(s["lengths"].tolist()):
            at = s["page_table"][i, :-(-n // case["page"])].long()
            for j in range(hk):
                sc = None if case["bits"] == 16 else s["scales"][at, j].flatten(0, 1)[:n]
                k, v = (_exact_values(s[c][at, j].flatten(0, 1)[:n], sc, case["bits"], w) for w, c in enumerate(("cache_k", "cache_v")))
                q = s["q"][i, j * shared:(j + 1) * shared].double()
                out[i, j * shared:(j + 1) * shared] = _exact_attention(q, k, v, torch.ones((shared, n), dtype=torch.bool, device="cuda"))
        return out
    out = torch.zeros((s["q"].shape[0], h, d), dtype=torch.float64, device="cuda")
    qs, ks = s["q_starts"].tolist(), s["k_starts"].tolist()
    for i in range(case["requests"]):
        nq, nk = qs[i + 1] - qs[i], ks[i + 1] - ks[i]
        seen = torch.ones((nq, nk), dtype=torch.bool, device="cuda").tril(nk - nq)
        for j in range(h):
            rows = slice(qs[i], qs[i + 1])
            keys = slice(ks[i], ks[i + 1])
            out[rows, j] = _exact_attention(s["q"][rows, j].double(), s["k"][keys, j // shared].double(), s["v"][keys, j // shared].double(), seen)
    return out
