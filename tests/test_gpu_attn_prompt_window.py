"""any4_attn_prompt with a window and first keys that stay visible, against attention in 64 bits (attention_reference.py has the bound)."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2507_04610_amd as any4
from test_gpu_attn_prompt import starts, tensors

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def seen(n, m, window, sinks):
    p, t = np.arange(n)[:, None] + m - n, np.arange(m)[None]
    return (t <= p) & ((t > p - window) | (t < sinks))


def check(out, q, k, v, nq, nk, window, sinks, scale=None):
    heads, kv_heads, dim = q.shape[1], k.shape[1], q.shape[2]
    out, qd, kd, vd = (t.double().cpu().numpy() for t in (out, q, k, v))
    aq = ak = 0
    for n, m in zip(nq, nk):
        for h in range(heads):
            j = h // (heads // kv_heads)
            o, allowed = ref.bound(qd[aq:aq + n, h], kd[ak:ak + m, j], vd[ak:ak + m, j], seen(n, m, window, sinks), scale or dim ** -0.5, q.dtype)
            off = np.abs(out[aq:aq + n, h] - o)
            assert (off <= allowed).all(), (n, m, h, np.max(off / allowed))
        aq, ak = aq + n, ak + m


LENGTHS = [1, 0, 2, 31, 32, 33, 0, 63, 64, 65, 100, 127, 128, 129, 0, 193, 300]


@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (64, 64), (65, 0), (100, 130), (1 << 40, 7)])
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("heads,kv_heads,fused", [(4, 2, True), (3, 3, False)])
def test_packed_lengths_around_every_edge(window, sinks, dtype, dim, heads, kv_heads, fused):
    n = sum(LENGTHS)
    q, k, v = tensors(n, n, heads, kv_heads, dim, dtype, 1, fused)
    check(any4.any4_attn_prompt(q, k, v, starts(LENGTHS), window=window, sinks=sinks), q, k, v, LENGTHS, LENGTHS, window, sinks)


@pytest.mark.parametrize("window,sinks", [(40, 3), (300, 0), (5000, 0)])
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
def test_contexts_and_queries_without_keys(window, sinks, dtype, dim):
    nq = [1, 1, 5, 40, 130, 200, 64, 3, 70, 0]
    nk = [1, 700, 64, 0, 131, 100, 500, 2, 333, 9]
    q, k, v = tensors(sum(nq), sum(nk), 4, 1, dim, dtype, 2, False)
    out = any4.any4_attn_prompt(q, k, v, starts(nq), starts(nk), window=window, sinks=sinks)
    check(out, q, k, v, nq, nk, window, sinks)
    a = sum(nq[:5])
    assert not out[sum(nq[:3]):sum(nq[:4])].any() and not out[a:a + 100].any() and out[a + 100:a + 200].any()


@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (8, 8), (32, 8), (5, 1), (18, 3), (200, 1)])
def test_heads(heads, kv_heads):
    nq = [150, 20]
    q, k, v = tensors(170, 170, heads, kv_heads, 128, BF16, 3, True)
    check(any4.any4_attn_prompt(q, k, v, starts(nq), window=50, sinks=2), q, k, v, nq, nq, 50, 2)


@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("dtype", (BF16, F16))
def test_a_long_prompt_and_a_wide_window_is_none(dim, dtype):
    q, k, v = tensors(1537, 1537, 2, 1, dim, dtype, 4, True, q_by=3.0)
    check(any4.any4_attn_prompt(q, k, v, starts([1537]), window=700, sinks=70), q, k, v, [1537], [1537], 700, 70)
    check(any4.any4_attn_prompt(q, k, v, starts([1537]), window=1537), q, k, v, [1537], [1537], 1537, 0)


def test_many_short_requests():
    nq = [(7 * i) % 11 for i in range(300)]
    q, k, v = tensors(sum(nq), sum(nq), 2, 2, 64, BF16, 5, True)
    check(any4.any4_attn_prompt(q, k, v, starts(nq), window=4, sinks=1), q, k, v, nq, nq, 4, 1)


@pytest.mark.parametrize("what", (float("nan"), float("inf"), -float("inf")))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("of", ("k", "v", "kv"))
def test_a_key_has_no_influence_on_queries_that_do_not_see_it(what, dtype, dim, of):
    nq, window, sinks = [200, 90, 150], 60, 3
    q, k, v = tensors(440, 440, 4, 2, dim, dtype, 8, False)
    want = any4.any4_attn_prompt(q, k, v, starts(nq), window=window, sinks=sinks)
    bad = [2, 70, 71, 130, 199]
    for t in [x for x, name in ((k, "k"), (v, "v")) if name in of]:
        t[bad] = what
        t[200:290] = what
    got = any4.any4_attn_prompt(q, k, v, starts(nq), window=window, sinks=sinks)
    touched = torch.from_numpy(seen(200, 200, window, sinks)[:, bad].any(1))
    assert torch.equal(got[:200].cpu()[~touched].view(torch.int16), want[:200].cpu()[~touched].view(torch.int16))
    assert torch.equal(got[290:].view(torch.int16), want[290:].view(torch.int16))
    assert not got[:200].cpu()[touched].isfinite().flatten(1).all(1).any()


def test_maximum_that_rises_with_every_key():
    n = 900
    q, k, v = tensors(n, n, 2, 1, 64, BF16, 7, False)
    q.fill_(0.25)
    k.copy_((torch.linspace(-40, 40, n)[:, None, None] * torch.ones(1, 1, 64)).to(BF16))
    for keys in (k, k.flip(0).contiguous()):
        check(any4.any4_attn_prompt(q, keys, v, starts([n]), window=200, sinks=5), q, keys, v, [n], [n], 200, 5)


def test_rows_of_no_request_graphs_and_the_checked_call(monkeypatch):
    from paper_2507_04610_amd import binding
    nq = [70, 200]
    q, k, v = tensors(300, 300, 4, 2, 128, BF16, 9, True)
    at, out = starts(nq, 10), torch.full((300, 4, 128), 5.0, dtype=BF16, device="cuda")
    any4.any4_attn_prompt(q, k, v, at, window=33, sinks=2, out=out)
    assert (out[:10] == 5).all() and (out[280:] == 5).all()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        any4.any4_attn_prompt(q, k, v, at, window=33, sinks=2, out=out)
    for i in range(3):
        q.mul_(1.1)
        at.copy_(starts([70 - 3 * i, 200 + i], 10))
        graph.replay()
        torch.cuda.synchronize()
        again = out.clone()
        any4.any4_attn_prompt(q, k, v, at, window=33, sinks=2, out=out)
        assert torch.equal(again, out)
    monkeypatch.setattr(binding, "_native_calls", binding._NoNativeCalls)
    any4.any4_attn_prompt(q, k, v, at, window=33, sinks=2, out=out)
    assert torch.equal(again, out)


def test_a_window_is_of_causal_attention():
    q = torch.zeros(3, 2, 64, dtype=BF16, device="cuda")
    with pytest.raises(any4.Any4Error, match="causal"):
        any4.any4_attn_prompt(q, q, q, starts([3]), causal=False, window=4)
