"""any4_attn_prompt against attention in 64 bits (attention_reference.py has the bound)."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2507_04610_amd as any4

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def starts(lengths, first=0):
    return torch.tensor(np.cumsum([first] + list(lengths)), dtype=torch.int32).cuda()


def tensors(nq, nk, heads, kv_heads, dim, dtype, seed, fused, q_by=1.0):
    g = torch.Generator().manual_seed(seed)
    if fused and nq == nk:
        row = torch.randn(nq, (heads + 2 * kv_heads) * dim, generator=g).to(dtype).cuda()
        row[:, :heads * dim] *= q_by
        q, k, v = row.split((heads * dim, kv_heads * dim, kv_heads * dim), 1)
        return q.view(nq, heads, dim), k.view(nk, kv_heads, dim), v.view(nk, kv_heads, dim)
    q = (torch.randn(nq, heads, dim, generator=g) * q_by).to(dtype).cuda()
    k, v = (torch.randn(kv_heads, nk, dim, generator=g).to(dtype).cuda().transpose(0, 1) for _ in range(2))
    return q, k, v


def check(out, q, k, v, nq, nk, causal, scale=None, first_q=0, first_k=0):
    heads, kv_heads, dim = q.shape[1], k.shape[1], q.shape[2]
    out, qd, kd, vd = (t.double().cpu().numpy() for t in (out, q, k, v))
    aq, ak = first_q, first_k
    for n, m in zip(nq, nk):
        seen = np.tril(np.ones((n, m), bool), m - n) if causal else np.ones((n, m), bool)
        for h in range(heads):
            j = h // (heads // kv_heads)
            o, allowed = ref.bound(qd[aq:aq + n, h], kd[ak:ak + m, j], vd[ak:ak + m, j], seen, scale or dim ** -0.5, q.dtype)
            got = out[aq:aq + n, h]
            assert (np.abs(got - o) <= allowed).all(), (n, m, h, np.max(np.abs(got - o) / allowed))
        aq, ak = aq + n, ak + m


LENGTHS = [1, 0, 2, 31, 32, 33, 0, 63, 64, 65, 100, 127, 128, 129, 0, 191, 193, 255, 257, 300]


@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("heads,kv_heads,fused", [(4, 2, True), (3, 3, False)])
def test_packed_lengths_around_every_edge(causal, dtype, dim, heads, kv_heads, fused):
    n = sum(LENGTHS)
    q, k, v = tensors(n, n, heads, kv_heads, dim, dtype, 1, fused)
    check(any4.any4_attn_prompt(q, k, v, starts(LENGTHS), causal=causal), q, k, v, LENGTHS, LENGTHS, causal)


@pytest.mark.parametrize("causal", (True, False))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
def test_contexts_and_queries_without_keys(causal, dtype, dim):
    """keys before the prompt, more and fewer keys than queries, none at all"""
    nq = [1, 1, 5, 40, 130, 200, 64, 3, 70, 0]
    nk = [1, 700, 64, 0, 131, 100, 500, 2, 333, 9]
    q, k, v = tensors(sum(nq), sum(nk), 4, 1, dim, dtype, 2, False)
    out = any4.any4_attn_prompt(q, k, v, starts(nq), starts(nk), causal=causal)
    check(out, q, k, v, nq, nk, causal)
    a = sum(nq[:3])
    assert not out[a:a + 40].any()
    if causal:
        a = sum(nq[:5])
        assert not out[a:a + 100].any() and out[a + 100:a + 200].any()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (32, 8), (5, 1), (18, 3)])
def test_heads(heads, kv_heads):
    nq = [150, 20]
    q, k, v = tensors(170, 170, heads, kv_heads, 128, BF16, 3, True)
    check(any4.any4_attn_prompt(q, k, v, starts(nq)), q, k, v, nq, nq, True)


@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("dtype", (BF16, F16))
def test_one_long_prompt(dim, dtype):
    q, k, v = tensors(1537, 1537, 2, 1, dim, dtype, 4, True, q_by=3.0)
    check(any4.any4_attn_prompt(q, k, v, starts([1537])), q, k, v, [1537], [1537], True)


def test_many_short_requests():
    """more requests than a wavefront has lanes"""
    nq = [(7 * i) % 11 for i in range(300)]
    q, k, v = tensors(sum(nq), sum(nq), 2, 2, 64, BF16, 5, True)
    check(any4.any4_attn_prompt(q, k, v, starts(nq)), q, k, v, nq, nq, True)


@pytest.mark.parametrize("q_by,scale", [(100.0, None), (1e-3, None), (1.0, 5.0), (1.0, 1e-3)])
@pytest.mark.parametrize("dtype", (BF16, F16))
def test_sizes_of_scores(q_by, scale, dtype):
    nq = [400, 77]
    q, k, v = tensors(477, 477, 4, 2, 128, dtype, 6, True, q_by=q_by)
    check(any4.any4_attn_prompt(q, k, v, starts(nq), softmax_scale=scale), q, k, v, nq, nq, True, scale)


def test_maximum_that_rises_with_every_key():
    n = 900
    q, k, v = tensors(n, n, 2, 1, 64, BF16, 7, False)
    q.fill_(0.25)
    k.copy_((torch.linspace(-40, 40, n)[:, None, None] * torch.ones(1, 1, 64)).to(BF16))
    for keys in (k, k.flip(0).contiguous()):
        check(any4.any4_attn_prompt(q, keys, v, starts([n])), q, keys, v, [n], [n], True)


@pytest.mark.parametrize("what", (float("nan"), float("inf"), -float("inf")))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("of", ("k", "v", "kv"))
def test_a_key_has_no_influence_on_queries_that_do_not_see_it(what, dtype, dim, of):
    """keys 70, 71, 130, 199 of 200 hold what is not finite; so do all keys of the request in between, and its queries"""
    nq = [200, 90, 150]
    q, k, v = tensors(440, 440, 4, 2, dim, dtype, 8, False)
    want = any4.any4_attn_prompt(q, k, v, starts(nq))
    odd, whole = [70, 71, 130, 199] + list(range(200, 290)), v.clone()
    if "k" in of:
        k[odd, 0, ::3] = what
        q[200:290] = float("nan")
    if "v" in of:
        v[odd, 0, 5:40] = what
    out = any4.any4_attn_prompt(q, k, v, starts(nq))
    assert torch.equal(out[:70], want[:70]) and torch.equal(out[290:], want[290:])
    assert torch.equal(out[:200, 2:], want[:200, 2:])                     # the other KV head's queries
    if of == "v":
        seen = np.tril(np.ones((200, 200), bool))                         # places that hold nothing odd
        for h in range(2):
            o, allowed = ref.bound(*(x.double().cpu().numpy() for x in (q[:200, h], k[:200, 0], whole[:200, 0])), seen, dim ** -0.5, dtype)
            assert (np.abs(out[:200, h].double().cpu().numpy() - o) <= allowed)[:, 40:].all()
        inside = out[70:199, :2, 5:40].float()
        assert not inside.isfinite().any() and (inside.isnan().all() if what != what else (inside.isnan() | (inside == what)).all())


def test_infinite_values_give_what_the_sum_gives():
    """+inf of weights above 0 is +inf, both signs together NaN"""
    n = 100
    q, k, v = tensors(n, n, 2, 1, 128, BF16, 9, False, q_by=0.1)
    v[60, 0, 0], v[80, 0, 0], v[70, 0, 1], v[90, 0, 1] = float("inf"), float("inf"), float("inf"), -float("inf")
    out = any4.any4_attn_prompt(q, k, v, starts([n])).float()
    assert out[:60, :, 0].isfinite().all() and (out[60:, :, 0] == float("inf")).all()
    assert out[:70, :, 1].isfinite().all() and (out[70:90, :, 1] == float("inf")).all() and out[90:, :, 1].isnan().all()
    assert out[:, :, 2:].isfinite().all()


def test_rows_outside_the_requests_are_left_alone():
    nq = [40, 30]
    q, k, v = tensors(100, 100, 2, 1, 128, BF16, 10, True)
    out = torch.full((100, 2, 128), 7.0, dtype=BF16, device="cuda")
    assert any4.any4_attn_prompt(q, k, v, starts(nq, 20), out=out) is out
    assert (out[:20] == 7).all() and (out[90:] == 7).all()
    check(out, q, k, v, nq, nq, True, first_q=20, first_k=20)
    # starts past the rows are taken as their number, descending ones as nothing
    wild = torch.tensor([0, 60, 1 << 30, 50, 40], dtype=torch.int32, device="cuda")
    out = any4.any4_attn_prompt(q, k, v, wild)
    check(out, q, k, v, [60, 40], [60, 40], True)


def test_guard_words():
    """nothing outside of out is written"""
    nq = [77, 130]
    q, k, v = tensors(207, 207, 4, 4, 64, F16, 11, True)
    room = torch.full((207 + 64, 4, 64), 5.0, dtype=F16, device="cuda")
    any4.any4_attn_prompt(q, k, v, starts(nq), out=room[32:239])
    check(room[32:239], q, k, v, nq, nq, True)
    assert (room[:32] == 5).all() and (room[239:] == 5).all()


def test_graph_on_another_stream_and_the_same_bits_every_time():
    nq, nk = torch.tensor([0, 100, 300], dtype=torch.int32).cuda(), torch.tensor([0, 400, 600], dtype=torch.int32).cuda()
    q, k, v = tensors(300, 600, 8, 2, 128, BF16, 12, False)
    out = any4.any4_attn_prompt(q, k, v, nq, nk)
    held = torch.empty_like(out)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        any4.any4_attn_prompt(q, k, v, nq, nk, out=held)
    for a, b in ((100, 400), (250, 260), (0, 600), (300, 1)):
        nq[1], nk[1] = a, b
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(held.view(torch.int16), any4.any4_attn_prompt(q, k, v, nq, nk).view(torch.int16))
        check(held, q, k, v, [a, 300 - a], [b, 600 - b], True)


def test_strides_past_32_bits():
    """rows of k and v more than 4 GB apart in all"""
    n, step = 700, (1 << 23) - 8
    big = torch.empty(n * step // 2, dtype=BF16, device="cuda")            # 5.9 GB
    q, k, v = tensors(n // 2, n // 2, 2, 1, 128, BF16, 13, False)
    kk = big[:n // 2 * step].view(n // 2, step)[:, :128].view(n // 2, 1, 128)
    vv = big[:n // 2 * step].view(n // 2, step)[:, 4096:4224].view(n // 2, 1, 128)
    kk.copy_(k)
    vv.copy_(v)
    s = starts([n // 2])
    assert torch.equal(any4.any4_attn_prompt(q, kk, vv, s), any4.any4_attn_prompt(q, k, v, s))


def test_refusals_name_the_mistake():
    q, k, v = tensors(50, 50, 4, 2, 128, BF16, 14, True)
    s = starts([50])
    for args, words in (((q, k.half(), v, s), "k must have dtype"), ((q, k, v[:, :1], s), "v must have shape"), ((q[:, :3], k, v, s), "no multiple"),
                        ((q, k, v, s.long()), "q_starts must have dtype"), ((q, k[:40], v[:40], s), "without k_starts"),
                        ((q, k, v, s, starts([20, 30])), "k_starts must have shape"), ((q[:, :, :64], k, v, s), "k must have shape"),
                        ((q, k, v[:, :, ::2], s), "v must have shape"), ((q.float(), k, v, s), "bf16 or fp16"), ((q[0], k, v, s), "3 dimensions")):
        with pytest.raises(any4.Any4Error, match=words):
            any4.any4_attn_prompt(*args)
    with pytest.raises(any4.Any4Error, match="bad shape"):
        any4.any4_attn_prompt(q[:, :, :96].contiguous(), k[:, :, :96].contiguous(), v[:, :, :96].contiguous(), s)
    with pytest.raises(any4.Any4Error, match="bad shape"):
        any4.any4_attn_prompt(q, k, v, s, softmax_scale=-1.0)
    assert any4.any4_attn_prompt(q[:0], k[:0], v[:0], starts([0])).shape == (0, 4, 128)
