"""What stands between a fused QKV projection and attention, and attention that sees part of a cache, as cases that can be timed.

Five kinds:
  rope     queries and keys of `tokens` tokens: each head is normalised (`norms`) and turned by its token's positions.
  append   the same on the way into a paged cache that holds `bits` bits a value, v beside k.
  chunk    several new tokens of each of `requests` requests attend to all of their request's tokens in the cache, causally.
  decode   one new token of each request attends to the last `window` tokens of its request and to the first `sinks`.
  prompt   packed prompts attend to themselves and to what came before them, each query to the last `window` keys up to its own
           and to the first `sinks`.

Lengths run from `shortest` to `longest` (new tokens from `fewest` to `most`) over the requests, the same ones for every seed, in an order
that the seed gives.  Cache layout: k and v [pages, kv_heads, page, head_dim] in 16 bits or as codes of 8 or 4 bits (two to a byte, the
first in the low half), scales [pages, kv_heads, page, 4] in bf16: k scale, k offset, v scale, v offset of a token; value = scale * code +
offset.  Slot s of the cache is token s % page of page s // page.
"""
import math

import torch

own = False

EPS = 1e-6


def _rope(name, tokens, heads=32, kv_heads=8, head_dim=128, rotary=128, axes=1, interleaved=False, norms=True, dtype="bf16"):
    c = {"kind": "rope", "tokens": tokens, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "rotary": rotary, "axes": axes,
         "interleaved": interleaved, "norms": norms, "dtype": dtype}
    return dict(c, name=name) if name else c


def _append(name, tokens, bits, page=16, longest=32768, heads=32, kv_heads=8, head_dim=128, rotary=128, axes=1, interleaved=False, norms=True,
            dtype="bf16"):
    c = {"kind": "append", "tokens": tokens, "bits": bits, "page": page, "longest": longest, "heads": heads, "kv_heads": kv_heads,
         "head_dim": head_dim, "rotary": rotary, "axes": axes, "interleaved": interleaved, "norms": norms, "dtype": dtype}
    return dict(c, name=name) if name else c


def _chunk(name, requests, fewest, most, shortest, longest, bits, window=0, sinks=0, heads=32, kv_heads=8, head_dim=128, page=16, dtype="bf16"):
    """shortest, longest: tokens in the cache in front of the new ones"""
    c = {"kind": "chunk", "requests": requests, "fewest": fewest, "most": most, "shortest": shortest, "longest": longest, "bits": bits,
         "window": window, "sinks": sinks, "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype}
    return dict(c, name=name) if name else c


def _decode(name, requests, shortest, longest, window, sinks, bits, heads=32, kv_heads=8, head_dim=128, page=16, dtype="bf16"):
    c = {"kind": "decode", "requests": requests, "shortest": shortest, "longest": longest, "window": window, "sinks": sinks, "bits": bits,
         "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "page": page, "dtype": dtype}
    return dict(c, name=name) if name else c


def _prompt(name, requests, shortest, longest, window, sinks, before=0, heads=32, kv_heads=8, head_dim=128, dtype="bf16"):
    c = {"kind": "prompt", "requests": requests, "shortest": shortest, "longest": longest, "window": window, "sinks": sinks, "before": before,
         "heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "dtype": dtype}
    return dict(c, name=name) if name else c


def listed():
    return [
        # an image between two texts: three positions for each token, neighbouring values turned together
        _rope("rope_image_fp16", 5001, axes=3, interleaved=True, dtype="f16"),
        # a question of a few dozen tokens, no norms, half of each head turned: latency
        _rope("rope_question", 45, heads=16, kv_heads=2, rotary=64, norms=False),
        # the newest token of each of 16 requests: what a call costs
        _append("append_16_tokens", 16, 16),
        # many prompts at once into an 8-bit cache
        _append("append_prompts_8bit", 16384, 8, page=64),
        # a chat's next message behind a few hundred tokens: latency
        _chunk("chunk_message", 1, 19, 19, 333, 333, 16),
        # up to eight drafted tokens for each request of a batch, to be checked in one pass: the cache's bandwidth
        _chunk("chunk_drafts_4bit", 16, 1, 8, 500, 16000, 4, page=64),
        # a served batch: requests in the middle of their prompts beside requests that get one token each
        _chunk("chunk_mixed_batch_8bit_fp16", 24, 1, 511, 0, 4000, 8, page=32, dtype="f16"),
        # a part of a long document: the matrix cores' case
        _chunk("chunk_long_document", 1, 2048, 2048, 30720, 30720, 16, page=64),
        # a batch whose requests have long left their first window behind, or are still in it
        _decode("window_batch", 48, 1, 32768, 4096, 4, 16, page=64),
        # one user far into a long document, small heads
        _decode("window_one_request_4bit_fp16", 1, 131071, 131071, 8191, 100, 4, heads=64, head_dim=64, page=32, dtype="f16"),
        # prompts of different lengths that arrived together, packed, behind contexts
        _prompt("window_prompts_packed_fp16", 6, 33, 2999, 777, 3, before=512, heads=16, kv_heads=2, head_dim=64, dtype="f16"),
        # one long prompt of odd length
        _prompt("window_prompt_long", 1, 12011, 12011, 2048, 16),
    ]


def _log_between(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    kind = rng.choice(("rope", "append", "chunk", "chunk", "decode", "prompt"))
    dtype = rng.choice(("bf16", "bf16", "f16"))
    head_dim = rng.choice((128, 128, 64))
    bits, page = rng.choice((16, 8, 4)), rng.choice((16, 32, 64, 128))
    kv_heads = rng.choice((1, 2, 4, 8, 8))
    heads = kv_heads * rng.choice([g for g in (1, 4, 4, 7) if g * kv_heads <= 32])
    window, sinks = _log_between(rng, 1, 8192), rng.choice((0, 1, 4, _log_between(rng, 1, 300)))
    if kind in ("rope", "append"):
        turn = {"heads": heads, "kv_heads": kv_heads, "head_dim": head_dim, "rotary": rng.choice((head_dim, head_dim, head_dim // 2, 16)),
                "axes": rng.choice((1, 1, 2, 3)), "interleaved": rng.random() < 0.3, "norms": rng.random() < 0.7, "dtype": dtype}
        if kind == "rope":
            return _rope(None, _log_between(rng, 1, 16384), **turn)
        # (a value between two codes of 4 bits moves by much if its last bit in 32 does: with fewer of them a case says more)
        return _append(None, _log_between(rng, 1, 16384 if bits > 4 else 1024), bits, page, rng.choice((4096, 131072, 1000000)), **turn)
    if kind == "chunk":
        longest = _log_between(rng, 1, 30720)
        most = _log_between(rng, 1, 2048)
        requests = _log_between(rng, 1, max(1, min(32, 2048 * 32768 // (most * (longest + most)))))
        where = {"window": window, "sinks": sinks} if rng.random() < 0.3 else {}
        return _chunk(None, requests, _log_between(rng, 1, most), most, rng.choice((0, _log_between(rng, 1, longest))), longest, bits, heads=heads,
                      kv_heads=kv_heads, head_dim=head_dim, page=page, dtype=dtype, **where)
    if kind == "decode":
        requests = _log_between(rng, 1, 64)
        longest = _log_between(rng, 1, min(131072, 64 * 16384 // requests))
        return _decode(None, requests, _log_between(rng, 1, longest), longest, window, sinks, bits, heads, kv_heads, head_dim, page, dtype)
    longest = _log_between(rng, 1, 8192)
    requests = _log_between(rng, 1, max(1, min(16, (8192 // longest) ** 2)))
    return _prompt(None, requests, _log_between(rng, 1, longest), longest, window, sinks, rng.choice((0, _log_between(rng, 1, 2048))) if longest <= 4096 else 0,
                   heads, kv_heads, head_dim, dtype)


def _spread(low, high, n):
    return [high if n == 1 else round(low + (high - low) * i / (n - 1)) for i in range(n)]


def _chunk_lengths(case):
    """(new tokens, tokens in front of them) of each request; long contexts with few and with many new tokens"""
    n = case["requests"]
    new, before = _spread(case["fewest"], case["most"], n), _spread(case["shortest"], case["longest"], n)
    return [(new[i], before[(7 * i + 3) % n] if n % 7 else before[n - 1 - i]) for i in range(n)]


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


def _table(lengths, page, host):
    """pages of requests of these lengths, anywhere in a cache with a few more: page table, pages"""
    need = [-(-n // page) for n in lengths]
    ids = torch.randperm(sum(need) + 3, generator=host)
    table = torch.zeros((len(need), max(1, max(need))), dtype=torch.int32)
    at = 0
    for i, n in enumerate(need):
        table[i, :n] = ids[at:at + n]
        at += n
    return table.cuda(), sum(need) + 3


def _starts(lengths):
    return torch.tensor([0] + lengths, dtype=torch.int32).cumsum(0).to(torch.int32).cuda()


def prepare(case, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    host = torch.Generator().manual_seed(seed)
    dt, d, h, hk = _dtype(case), case["head_dim"], case["heads"], case["kv_heads"]
    s = dict(case)

    def normal(*shape, by=1.0):
        return torch.randn(shape, generator=g, device="cuda").mul_(by).to(dt)

    if case["kind"] in ("rope", "append"):
        n, rotary = case["tokens"], case["rotary"]
        # q, k and v as the fused projection's output has them: one row a token
        row = normal(n, (h + 2 * hk) * d)
        s["q"], s["k"], s["v"] = (x.view(n, -1, d) for x in row.split((h * d, hk * d, hk * d), 1))
        s["q_norm"], s["k_norm"] = (normal(d, by=0.2).add_(1) for _ in range(2)) if case["norms"] else (None, None)
        s["freqs"] = 500000.0 ** (torch.arange(rotary // 2, dtype=torch.float64, device="cuda") * (-2.0 / rotary))
        longest = case.get("longest", 32768)
        if case["axes"] == 1:
            # requests' tokens one behind the other, from some place on in each
            s["positions"] = (torch.arange(n) % 1711 + int(torch.randint(max(1, longest - 1711), (1,), generator=host))).cuda()
            s["axis_of"] = None
        else:
            # time moves on, height and width go over an image 40 wide
            t, first = torch.arange(n), int(torch.randint(max(1, longest - n), (1,), generator=host))
            s["positions"] = torch.stack((first + t // 1000, first + t % 1000 // 40, first + t % 40)[:case["axes"]]).cuda()
            s["axis_of"] = (torch.arange(rotary // 2) % case["axes"]).to(torch.uint8).cuda()
        if case["kind"] == "append":
            p = case["page"]
            pages = -(-n // p) + 3
            s["cache_k"], s["cache_v"], s["scales"] = _pages(case, pages, g)
            order, t = torch.randperm(pages, generator=host), torch.arange(n)
            s["slots"] = (order[t // p] * p + t % p).cuda()
        return s
    n = case["requests"]
    order = torch.randperm(n, generator=host).tolist()
    if case["kind"] == "chunk":
        lengths = _chunk_lengths(case)
        lengths = [lengths[i] for i in order]
        nq, nk = [a for a, _ in lengths], [a + b for a, b in lengths]
    else:
        lengths = _spread(case["shortest"], case["longest"], n)
        lengths = [lengths[i] for i in order]
        if case["kind"] == "decode":
            nq, nk = [1] * n, lengths
        else:
            before = _befores(case)
            nq, nk = lengths, [lengths[at] + before[i] for at, i in enumerate(order)]
    if case["kind"] != "prompt":
        s["page_table"], pages = _table(nk, case["page"], host)
        s["cache_k"], s["cache_v"], s["scales"] = _pages(case, pages, g)
        s["lengths"] = torch.tensor(nk, dtype=torch.int32, device="cuda")
        # q in the front of the fused projection's rows
        s["q"] = normal(sum(nq), (h + 2 * hk) * d, by=1.5)[:, : h * d].view(sum(nq), h, d)
    elif not case["before"]:
        row = normal(sum(nq), (h + 2 * hk) * d)
        q, k, v = row.split((h * d, hk * d, hk * d), 1)
        q.mul_(1.5)
        s["q"], s["k"], s["v"] = (x.view(-1, y, d) for x, y in ((q, h), (k, hk), (v, hk)))
    else:
        s["q"], s["k"], s["v"] = normal(sum(nq), h, d, by=1.5), normal(sum(nk), hk, d), normal(sum(nk), hk, d)
    s["q_starts"] = _starts(nq)
    if case["kind"] == "prompt":
        s["k_starts"] = _starts(nk)
    # (the longest are known where the plain form pads; the packed form takes what the starts say)
    s["longest_q"], s["longest_k"] = max(nq), max(nk)
    return s


# The plain forms

def _turn(x, weight, s):
    """[tokens, heads, head_dim], normalised and turned, rounded once"""
    x = x.float()
    if weight is not None:
        x = x * (x.square().mean(-1, keepdim=True) + EPS).rsqrt() * weight.float()
    half = s["rotary"] // 2
    at = s["positions"][s["axis_of"].long()].T if s["axis_of"] is not None else s["positions"][:, None]
    angle = at.double() * s["freqs"]                                       # (in 32 bits a far position's is off by whole turns' parts)
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    even, odd = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if s["interleaved"] else (slice(0, half), slice(half, 2 * half))
    a, b = x[..., even], x[..., odd]
    y = x.clone()
    y[..., even], y[..., odd] = a * cos - b * sin, b * cos + a * sin
    return y.to(_dtype(s))


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


def _plain_append(s):
    """turned keys are rounded to 16 bits, then held as k and v are"""
    p, bits = s["page"], s["bits"]
    q, k = _turn(s["q"], s["q_norm"], s), _turn(s["k"], s["k_norm"], s)
    page, at = s["slots"] // p, s["slots"] % p
    if bits == 16:
        s["cache_k"][page, :, at], s["cache_v"][page, :, at] = k, s["v"]
        return q, s["cache_k"], s["cache_v"]
    (ck, ak), (cv, av) = _encode(k, bits), _encode(s["v"], bits)
    s["cache_k"][page, :, at], s["cache_v"][page, :, at], s["scales"][page, :, at] = ck, cv, torch.cat((ak, av), -1)
    scales = s["scales"][page, :, at]
    return (q, *(_values(s[c][page, :, at], scales, bits, w).to(_dtype(s)) for w, c in enumerate(("cache_k", "cache_v"))))


def _softmax(scores, seen):
    """rows of zeros where nothing is seen"""
    scores = scores.masked_fill_(~seen, -math.inf)
    top = scores.amax(-1, keepdim=True)
    e = scores.sub_(torch.where(top == -math.inf, torch.zeros_like(top), top)).exp_()
    return e.div_(e.sum(-1, keepdim=True).clamp_min(1e-37))


def _from_pages(s, token):
    """k and v [requests * kv_heads, tokens, head_dim] of these tokens [requests, tokens] of the requests"""
    p, bits, n = s["page"], s["bits"], token.shape[0]
    page, at = s["page_table"].long().gather(1, token // p), token % p
    scales = None if bits == 16 else s["scales"][page, :, at]
    return (_values(s[c][page, :, at], scales, bits, w).transpose(1, 2).reshape(n * s["kv_heads"], -1, s["head_dim"]) for w, c in enumerate(("cache_k", "cache_v")))


def _plain_decode(s):
    hk, d, n = s["kv_heads"], s["head_dim"], s["requests"]
    length = s["lengths"][:, None].long()
    # the first tokens, then the last ones that are none of the first
    j = torch.arange(min(s["sinks"] + s["window"], s["longest_k"]), device="cuda")
    token = torch.where(j < s["sinks"], j, (length - s["window"]).clamp_min(s["sinks"]) + j - s["sinks"])
    seen = token < length
    k, v = _from_pages(s, torch.where(seen, token, torch.zeros_like(token)))
    q = s["q"].float().reshape(n * hk, -1, d)
    scores = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(n, hk, -1, j.numel())
    weights = _softmax(scores, seen[:, None, None]).view(n * hk, -1, j.numel())
    return torch.bmm(weights, v).view(n, -1, d).to(_dtype(s))


def _padded(x, starts, longest):
    """[n, longest] places of packed rows, and which of them are rows"""
    at = starts[:-1, None].long() + torch.arange(longest, device="cuda")
    there = at < starts[1:, None]
    return x.float()[at.clamp_max(x.shape[0] - 1)].transpose(1, 2), at, there


def _plain_rows(s, k, v, lk):
    """k, v [requests * kv_heads, longest, head_dim] and how many of them are the requests'"""
    h, hk, d, n = s["heads"], s["kv_heads"], s["head_dim"], s["requests"]
    q, q_at, q_there = _padded(s["q"], s["q_starts"], s["longest_q"])
    lq = s["q_starts"][1:] - s["q_starts"][:-1]
    # the heads that share a KV head stand under each other
    q = q.reshape(n * hk, h // hk * s["longest_q"], d)
    scores = torch.bmm(q, k.transpose(1, 2).contiguous()).mul_(d ** -0.5).view(n, hk, h // hk, s["longest_q"], s["longest_k"])
    i, j = torch.arange(s["longest_q"], device="cuda")[:, None] + (lk - lq)[:, None, None], torch.arange(s["longest_k"], device="cuda")
    seen = (j <= i) & (j < lk[:, None, None])
    if s["window"]:
        seen &= (j > i - s["window"]) | (j < s["sinks"])
    weights = _softmax(scores, seen[:, None, None]).view(n * hk, -1, s["longest_k"])
    o = torch.bmm(weights, v).view(n, h, s["longest_q"], d).transpose(1, 2)
    out = torch.empty((s["q"].shape[0], h, d), dtype=_dtype(s), device="cuda")
    out[q_at[q_there]] = o[q_there].to(out.dtype)
    return out


def _plain_chunk(s):
    token = torch.arange(s["longest_k"], device="cuda").expand(s["requests"], -1)
    there = token < s["lengths"][:, None]
    k, v = _from_pages(s, torch.where(there, token, torch.zeros_like(token)))
    return _plain_rows(s, k, v, s["lengths"])


def _plain_prompt(s):
    k, v = (_padded(s[x], s["k_starts"], s["longest_k"])[0].reshape(s["requests"] * s["kv_heads"], -1, s["head_dim"]) for x in "kv")
    return _plain_rows(s, k, v, s["k_starts"][1:] - s["k_starts"][:-1])


def run(s):
    if not own:
        if s["kind"] == "rope":
            return _turn(s["q"], s["q_norm"], s), _turn(s["k"], s["k_norm"], s)
        return {"append": _plain_append, "chunk": _plain_chunk, "decode": _plain_decode, "prompt": _plain_prompt}[s["kind"]](s)
    import paper_2507_04610_amd as any4
    if s["kind"] in ("rope", "append"):
        turn = {"q_norm": s["q_norm"], "k_norm": s["k_norm"], "eps": EPS, "interleaved": s["interleaved"], "axis_of": s["axis_of"]}
        if s["kind"] == "rope":
            return any4.any4_rope(s["q"], s["k"], s["positions"], s["freqs"], **turn)
        q = any4.any4_rope_kv_write(s["q"], s["k"], s["v"], s["positions"], s["freqs"], s["slots"], s["cache_k"], s["cache_v"], s["scales"], bits=s["bits"], **turn)
        if s["bits"] == 16:
            return q, s["cache_k"], s["cache_v"]
        return (q, *any4.any4_kv_read(s["cache_k"], s["cache_v"], s["slots"], s["scales"], bits=s["bits"], dtype=q.dtype))
    # (no window is None)
    part = {"window": s["window"] or None, "sinks": s["sinks"]}
    if s["kind"] == "prompt":
        return any4.any4_attn_prompt(s["q"], s["k"], s["v"], s["q_starts"], s["k_starts"], **part)
    if s["kind"] == "decode":
        return any4.any4_attn_decode(s["q"], s["cache_k"], s["cache_v"], s["page_table"], s["lengths"], s["scales"], bits=s["bits"], **part)
    return any4.any4_attn_chunk(s["q"], s["cache_k"], s["cache_v"], s["page_table"], s["q_starts"], s["lengths"], s["scales"], bits=s["bits"], **part)


def _pairs(nq, nk, window, sinks):
    """(keys that the nq last of nk tokens see, added up; keys that some of them sees)"""
    if nq == 0:
        return 0, 0
    first = nk - nq
    if not window:
        return nq * first + nq * (nq + 1) // 2, nk
    seen = sum(min(p + 1, window) + min(sinks, max(0, p + 1 - window)) for p in range(first, nk))
    start = max(0, first + 1 - window)
    return seen, nk - start + min(sinks, start)


def work(case):
    d, h, hk = case["head_dim"], case["heads"], case["kv_heads"]
    if case["kind"] == "rope":
        return {"bytes": case["tokens"] * (4 * d * (h + hk) + 8 * case["axes"]) + 4 * case["rotary"], "flops": 8 * case["tokens"] * (h + hk) * d}
    if case["kind"] == "prompt":
        lengths = _spread(case["shortest"], case["longest"], case["requests"])
        nk = [n + b for n, b in zip(lengths, _befores(case))]
        pairs = [_pairs(n, m, case["window"], case["sinks"]) for n, m in zip(lengths, nk)]
        return {"bytes": 4 * d * (sum(lengths) * h + sum(n for _, n in pairs) * hk) + 8 * (len(lengths) + 1), "flops": 4 * d * h * sum(n for n, _ in pairs)}
    kept = hk * (d * case["bits"] // 4 + (8 if case["bits"] < 16 else 0))              # bytes of a token in the cache
    if case["kind"] == "append":
        back = 0 if case["bits"] == 16 else kept + hk * 4 * d + 8                     # (codes are read back as values)
        return {"bytes": case["tokens"] * (4 * d * h + 4 * d * hk + kept + 8 * case["axes"] + 8 + back) + 4 * case["rotary"],
                "flops": 8 * case["tokens"] * (h + 2 * hk) * d}
    lengths = _chunk_lengths(case) if case["kind"] == "chunk" else [(1, n - 1) for n in _spread(case["shortest"], case["longest"], case["requests"])]
    pairs = [_pairs(a, a + b, case["window"], case["sinks"]) for a, b in lengths]
    read = sum(n for _, n in pairs)
    return {"bytes": read * kept + 4 * sum(-(-n // case["page"]) for _, n in pairs) + sum(a for a, _ in lengths) * 4 * h * d + 8 * len(lengths),
            "flops": 4 * d * h * sum(n for n, _ in pairs)}


# The definitions in 64 bits

def _exact_turn(x, weight, s):
    """one head at a time, as complex numbers"""
    out = torch.empty(x.shape, dtype=torch.float64, device=x.device)
    half = s["rotary"] // 2
    position = s["positions"].reshape(-1, x.shape[0]).double()
    angle = torch.stack([position[0 if s["axis_of"] is None else int(s["axis_of"][i])] * s["freqs"][i] for i in range(half)], 1)
    turn = torch.polar(torch.ones_like(angle), angle)
    first = torch.arange(half, device=x.device) * (2 if s["interleaved"] else 1)
    second = first + (1 if s["interleaved"] else half)
    for j in range(x.shape[1]):
        y = x[:, j].double()
        if weight is not None:
            y = y / torch.sqrt((y * y).sum(1, keepdim=True) / y.shape[1] + EPS) * weight.double()
        z = torch.complex(y[:, first], y[:, second]) * turn
        out[:, j] = y
        out[:, j, first], out[:, j, second] = z.real, z.imag
    return out


def _exact_held(x, bits):
    """what a cache of 8 or 4 bits makes of x [tokens, heads, head_dim] in 64 bits"""
    low, high, top = x.min(-1, keepdim=True).values, x.max(-1, keepdim=True).values, 2 ** bits - 1
    step, low = ((high - low) / top).to(torch.bfloat16).double(), low.to(torch.bfloat16).double()
    step[step == 0] = 1
    return torch.clamp(torch.round((x - low) / step), 0, top) * step + low


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


def _exact_attention(q, k, v, window, sinks):
    """the n queries [n, d] of the last of m tokens, k and v [m, d]; as many at a time as leave the scores small"""
    n, m = q.shape[0], k.shape[0]
    out = torch.zeros_like(q)
    if m == 0:
        return out
    for a in range(0, n, 2048):
        p = torch.arange(a, min(n, a + 2048), device=q.device)[:, None] + (m - n)
        t = torch.arange(m, device=q.device)[None]
        hidden = (t > p) | ((t <= p - window) & (t >= sinks)) if window else t > p
        s = (q[a:a + 2048] @ k.T.contiguous()) / math.sqrt(q.shape[1])
        s[hidden] = -math.inf
        w = torch.softmax(s, -1)
        w[hidden.all(-1)] = 0
        out[a:a + 2048] = w @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    h, hk = case["heads"], case["kv_heads"]
    if case["kind"] in ("rope", "append"):
        q, k = _exact_turn(s["q"], s["q_norm"], s), _exact_turn(s["k"], s["k_norm"], s)
        if case["kind"] == "rope":
            return q, k
        if case["bits"] < 16:
            return q, _exact_held(k.to(s["k"].dtype).double(), case["bits"]), _exact_held(s["v"].double(), case["bits"])
        cache = [s["cache_k"].double(), s["cache_v"].double()]
        for c, x in zip(cache, (k, s["v"].double())):
            for j in range(hk):
                flat = c[:, j].reshape(-1, case["head_dim"])
                flat[s["slots"]] = x[:, j]
                c[:, j] = flat.view(c.shape[0], case["page"], case["head_dim"])
        return (q, *cache)
    shared = h // hk
    out = torch.zeros((s["q"].shape[0], h, case["head_dim"]), dtype=torch.float64, device="cuda")
    qs = s["q_starts"].tolist()
    ks = s["k_starts"].tolist() if case["kind"] == "prompt" else None
    lengths = None if case["kind"] == "prompt" else s["lengths"].tolist()
    for i in range(case["requests"]):
        rows = slice(qs[i], qs[i + 1])
        for j in range(hk):
            if case["kind"] == "prompt":
                k, v = (s[x][ks[i]:ks[i + 1], j].double() for x in "kv")
            else:
                n = lengths[i]
                at = s["page_table"][i, :-(-n // case["page"])].long()
                sc = None if case["bits"] == 16 else s["scales"][at, j].flatten(0, 1)[:n]
                k, v = (_exact_values(s[c][at, j].flatten(0, 1)[:n], sc, case["bits"], w) for w, c in enumerate(("cache_k", "cache_v")))
            for x in range(j * shared, (j + 1) * shared):
                out[rows, x] = _exact_attention(s["q"][rows, x].double(), k, v, case["window"], case["sinks"])
    return out
