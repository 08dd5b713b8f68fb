"""any4_attn_decode with a window and first tokens that stay visible, against attention in 64 bits over the tokens that are seen."""
import numpy as np
import pytest
import torch

import attention_reference as ref
import paper_2507_04610_amd as any4
from test_gpu_attn_decode import Problem

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def seen(n, window, sinks):
    t = np.arange(n)
    return (t >= n - window) | (t < sinks)


def check(p, out, window, sinks, requests=None, scale=None):
    assert out.shape == (len(p.lengths), p.heads, p.dim) and out.dtype == p.dtype
    out, q = out.double().cpu().numpy(), p.q.double().cpu().numpy()
    shared = p.heads // p.kv_heads
    for i in requests if requests is not None else range(len(p.lengths)):
        keep = seen(p.lengths[i], window, sinks)
        for j in range(p.kv_heads):
            k, v, *codes = p.held(i, j)
            k, v, *codes = (x if x is None else x[keep] for x in (k, v, *codes))
            rows = slice(j * shared, (j + 1) * shared)
            o, allowed = ref.bound(q[i, rows], k, v, np.ones((shared, len(k)), bool), scale or p.dim ** -0.5, p.dtype, p.bits, *codes)
            assert (np.abs(out[i, rows] - o) <= allowed).all(), (i, j, window, sinks, np.max(np.abs(out[i, rows] - o) / allowed))


def spoil(p, window, sinks, pages=True):
    """the tokens that are not seen are no numbers, pages without a seen token no pages"""
    for i, n in enumerate(p.lengths):
        keep = seen(n, window, sinks)
        for t in np.nonzero(~keep)[0]:
            page, at = p.pages_of[i][t // p.page], t % p.page
            if p.bits == 16:
                p.ck[page, :, at] = p.cv[page, :, at] = float("nan")
            else:
                p.sc[page, :, at] = float("nan")
        if pages:
            for x in range(-(-n // p.page)):
                if not keep[x * p.page:(x + 1) * p.page].any():
                    p.table[i, x] = -7 if x % 2 else 1 << 30


LENGTHS = [0, 1, 2, 31, 32, 33, 64, 65, 100, 128, 129, 160, 255, 256, 257, 300, 511, 700]


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (32, 32), (33, 33), (100, 0), (128, 40), (257, 300), (5000, 3)])
def test_windows_around_every_edge(bits, dtype, dim, window, sinks):
    p = Problem(LENGTHS, bits, dtype, dim, 4, 2, 16, seed=bits)
    out = p.run(window=window, sinks=sinks)
    assert not out[0].any()
    check(p, out, window, sinks)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("page", (16, 64))
@pytest.mark.parametrize("window,sinks", [(1, 0), (40, 5), (100, 0), (130, 70)])
def test_what_is_not_seen_may_be_anything(bits, page, window, sinks):
    p = Problem([700, 33, 0, 257, 96, 512], bits, BF16, 128, 8, 2, page, seed=2)
    want = p.run(window=window, sinks=sinks)
    check(p, want, window, sinks)
    spoil(p, window, sinks)
    got = p.run(window=window, sinks=sinks)
    assert torch.equal(got.view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("window,sinks", [(20000, 0), (20000, 1000), (1 << 40, 0), (40000, 1 << 40)])
def test_long_requests_are_cut_and_joined(bits, dim, window, sinks):
    p = Problem([30001, 0, 5, 9000, 20001], bits, BF16, dim, 4, 1, 128, seed=1)
    out = p.run(window=window, sinks=sinks)
    check(p, out, window, sinks)
    for _ in range(3):
        assert torch.equal(p.run(window=window, sinks=sinks).view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("requests", (65, 300, 2100))
def test_many_requests(requests):
    p = Problem([(37 * i) % 300 for i in range(requests)], 8, BF16, 64, 4, 2, 16, seed=3)
    out = p.run(window=70, sinks=9)
    check(p, out, 70, 9, requests=range(0, requests, 7))
    assert not out[0].any()


@pytest.mark.parametrize("bits", (16, 4))
def test_heads(bits):
    p = Problem([5, 1100, 400], bits, BF16, 128, 40, 1, 32, seed=4)
    check(p, p.run(window=300, sinks=17), 300, 17)


def test_requests_whose_seen_pages_do_not_exist():
    p = Problem([600, 600], 8, BF16, 128, 4, 2, 16)
    p.table[0, 20:] = -1                                                    # the window's pages
    out = p.run(window=200, sinks=0)
    assert not out[0].any()
    check(p, out, 200, 0, requests=[1])


def test_the_native_and_the_checked_call_are_one(monkeypatch):
    from paper_2507_04610_amd import binding
    p = Problem([600, 3000], 8, BF16, 128, 4, 2, 16)
    want = p.run(window=333, sinks=4)
    monkeypatch.setattr(binding, "_native_calls", binding._NoNativeCalls)
    assert torch.equal(p.run(window=333, sinks=4), want)


def test_a_graph_follows_the_lengths():
    p = Problem([600, 3000, 40], 8, BF16, 128, 8, 2, 16)
    need = any4.any4_attn_decode_workspace_bytes(3, 8, 2, 128, p.width * 16)
    ws, out = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), torch.empty(3, 8, 128, dtype=BF16, device="cuda")
    p.run(window=500, sinks=4, out=out, workspace=ws)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        p.run(window=500, sinks=4, out=out, workspace=ws)
    for lengths in ([600, 3000, 40], [1, 2999, 0], [599, 4, 33], [600, 3000, 40]):
        p.len.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = out.clone()
        assert torch.equal(got, p.run(window=500, sinks=4))
