"""any4_attn_chunk against attention in 64 bits over what the cache holds (attention_reference.py has the bound)."""
import numpy as np
import pytest
import torch

import attention_close as close
import attention_reference as ref
import paper_2507_04610_amd as any4
from test_gpu_attn_decode import Problem

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


class Chunks(Problem):
    """requests of (new tokens, tokens in front of them)"""

    def __init__(self, parts, bits, dtype, dim, heads, kv_heads, page=16, seed=0, q_by=1.0, first=0, behind=0, **kw):
        super().__init__([a + b for a, b in parts], bits, dtype, dim, heads, kv_heads, page, seed, **kw)
        self.new = [a for a, _ in parts]
        self.starts = torch.tensor(np.cumsum([first] + self.new), dtype=torch.int32).cuda()
        n = first + sum(self.new) + behind
        g = torch.Generator().manual_seed(seed + 100)
        row = (torch.randn(n, (heads + 3) * dim, generator=g) * q_by).to(dtype).cuda()
        self.q = row[:, dim:(heads + 1) * dim].view(n, heads, dim)

    def run(self, **kw):
        return any4.any4_attn_chunk(self.q, self.ck, self.cv, self.table, self.starts, self.len, self.sc, bits=self.bits, **kw)

    def write(self, i, k, v):
        """other keys and values of a request's tokens"""
        t = torch.arange(self.lengths[i])
        slots = (torch.tensor(self.pages_of[i])[t // self.page] * self.page + t % self.page).cuda()
        any4.any4_kv_write(k.to(self.dtype).cuda(), v.to(self.dtype).cuda(), slots, self.ck, self.cv, self.sc, bits=self.bits)

    def seen(self, i, window=None, sinks=0):
        n, nq = self.lengths[i], self.new[i]
        p, t = np.arange(nq)[:, None] + n - nq, np.arange(n)[None]
        return (t <= p) & ((t > p - window) | (t < sinks)) if window else t <= p

    def check(self, out, scale=None, requests=None, window=None, sinks=0):
        assert out.shape == self.q.shape and out.dtype == self.dtype
        out, q, starts = out.double().cpu().numpy(), self.q.double().cpu().numpy(), self.starts.tolist()
        shared = self.heads // self.kv_heads
        for i in requests if requests is not None else range(len(self.lengths)):
            rows, seen = slice(starts[i], starts[i + 1]), self.seen(i, window, sinks)
            some = seen.any(0)
            for j in range(self.kv_heads):
                k, v, *codes = self.held(i, j)
                k, v, *codes = (x if x is None else x[some] for x in (k, v, *codes))
                for h in range(j * shared, (j + 1) * shared):
                    o, allowed = ref.bound(q[rows, h], k, v, seen[:, some], scale or self.dim ** -0.5, self.dtype, self.bits, *codes)
                    # (the bound's rounding of the result is relative; below 2^-14 fp16 values lie 2^-24 apart, and half of that is the rounding)
                    allowed = allowed + (2.0 ** -25 if self.dtype == F16 else 0.0)
                    off = np.abs(out[rows, h] - o)
                    assert (off <= allowed).all(), (i, h, np.max(off / allowed))


EDGES = [(1, 0), (0, 5), (2, 0), (31, 1), (32, 32), (33, 30), (64, 0), (65, 63), (1, 63), (1, 64), (3, 61), (0, 0), (100, 27), (128, 1), (129, 300), (5, 191), (16, 48), (300, 0)]


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("heads,kv_heads,page", [(8, 2, 16), (3, 3, 64)])
def test_lengths_around_every_edge(bits, dtype, dim, heads, kv_heads, page):
    p = Chunks(EDGES, bits, dtype, dim, heads, kv_heads, page, seed=bits)
    p.check(p.run())


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (31, 4), (64, 64), (65, 65), (100, 0), (128, 40), (257, 300), (5000, 3)])
def test_windows(bits, dtype, window, sinks):
    dim = 128 if window % 2 else 64
    p = Chunks(EDGES + [(70, 600), (1, 900)], bits, dtype, dim, 4, 2, 16, seed=bits)
    p.check(p.run(window=window, sinks=sinks), window=window, sinks=sinks)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (16, 1), (17, 1), (40, 1), (48, 2), (7, 7), (64, 8), (200, 1)])
def test_heads(bits, heads, kv_heads):
    """rows are queries times the heads that share a KV head: tiles begin and end in the middle of a query's heads"""
    p = Chunks([(5, 0), (9, 500), (40, 33), (1, 700)], bits, BF16, 128, heads, kv_heads, 32, seed=heads)
    p.check(p.run())


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("where", ({}, {"window": 12000, "sinks": 100}))
def test_long_contexts_are_cut_and_joined(bits, dim, where):
    p = Chunks([(19, 30001), (0, 40), (1, 9000), (200, 5000), (7, 0)], bits, BF16, dim, 8, 2, 128, seed=1)
    need = any4.any4_attn_chunk_workspace_bytes(5, len(p.q), 8, 2, dim, p.width * 128)
    assert need > 0
    out = p.run(**where)
    p.check(out, **where)
    # the same bits again, and in a workspace that held something else
    ws = torch.randint(0, 256, (need,), dtype=torch.uint8, device="cuda")
    for _ in range(3):
        assert torch.equal(p.run(workspace=ws, **where).view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
def test_outputs_lie_as_near_as_their_roundings_say(bits, dtype, dim):
    """the last query of a request sees all of its tokens: within what independent roundings add up to, which zeros, even weights and a missing
    piece exceed"""
    p = Chunks([(3, 20000), (40, 700), (1, 33)], bits, dtype, dim, 8, 2, 64, seed=7)
    out = p.run().double().cpu().numpy()
    for i, last in enumerate(p.starts.tolist()[1:]):
        for j in range(2):
            held = close.Held.__new__(close.Held)                               # (from the cache, not from what was written)
            held.bits, held.dtype = bits, dtype
            held.k, held.v, ks, vs, vo = p.held(i, j)
            if bits != 16:
                held.k_scale, held.v_scale, held.v_offset = ks[:, None], vs[:, None], vo[:, None]
                held.codes = np.rint((held.v - held.v_offset) / held.v_scale)
            q = p.q[last - 1, 4 * j:4 * j + 4].double().cpu().numpy()
            most, mean = close.fits(out[last - 1, 4 * j:4 * j + 4], q, held, dim ** -0.5)
            assert most <= 1 and mean <= 1, (i, j, most, mean)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("requests", (65, 300, 2100))
def test_many_requests(bits, requests):
    """decoding requests beside such in the middle of their prompts, more than a wavefront has lanes"""
    p = Chunks([(1 if i % 3 else (11 * i) % 40, (37 * i) % 300) for i in range(requests)], bits, BF16, 64, 4, 2, 16, seed=3)
    p.check(p.run(), requests=range(0, requests, 7 if requests < 1000 else 53))


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("requests", (64, 65, 200))
def test_long_contexts_among_many_requests(bits, requests):
    """what is cut and joined where blocks look for their work themselves, and where a first launch has found it"""
    parts = [((5 * i) % 7, (29 * i) % 90) for i in range(requests)]
    parts[3], parts[40], parts[-1] = (3, 15000), (150, 4000), (30, 9000)
    p = Chunks(parts, bits, BF16, 128, 8, 2, 64, seed=13)
    out = p.run()
    p.check(out, requests=[0, 2, 3, 4, 39, 40, 41, 63, requests - 2, requests - 1])
    p.check(p.run(window=3000, sinks=70), requests=[3, 40, requests - 1], window=3000, sinks=70)
    for _ in range(2):
        assert torch.equal(p.run().view(torch.int16), out.view(torch.int16))


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("k_by,v_by,q_by,scale", [(5.0, 1.0, 1.0, None), (0.5, 300.0, 1.0, None), (1.0, 1e-4, 1.0, None), (1.0, 0.5, 100.0, None), (1.0, 0.5, 1e-3, None),
                                                  (1.0, 0.5, 1.0, 5.0), (1.0, 0.5, 1.0, 1e-3)])
@pytest.mark.parametrize("dtype", (BF16, F16))
def test_sizes_of_values(bits, dtype, k_by, v_by, q_by, scale):
    p = Chunks([(70, 300), (1, 700), (130, 0)], bits, dtype, 128, 8, 2, 64, seed=4, k_by=k_by, v_by=v_by, q_by=q_by)
    p.check(p.run(softmax_scale=scale), scale=scale)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("q_by,k_by,v_by", [(1e-15, 1e15, 1e25), (1e12, 1e-12, 1e-25), (1.0, 1.0, 1e32)])
def test_values_far_from_fp16(bits, q_by, k_by, v_by):
    """bf16 reaches further than the fp16 that codes pass through"""
    p = Chunks([(40, 300), (1, 100)], bits, BF16, 128, 4, 2, 64, seed=5, k_by=k_by, v_by=v_by, q_by=q_by)
    p.check(p.run())


@pytest.mark.parametrize("bits", (8, 4))
def test_tokens_of_very_different_sizes(bits):
    """v's scales grow and shrink by powers of ten from tile to tile"""
    p = Chunks([(70, 900)], bits, BF16, 128, 4, 2, 64, seed=6)
    by = torch.tensor([1e-20, 1.0, 1e20, 1e-5, 1e25, 1.0, 1e-30, 1e10])
    at = torch.arange(970)
    g = torch.Generator().manual_seed(1)
    p.write(0, torch.randn(970, 2, 128, generator=g), torch.randn(970, 2, 128, generator=g) * by[at // 128][:, None, None])
    p.check(p.run())


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("what", (float("nan"), float("inf")))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("where", ({}, {"window": 100, "sinks": 30}))
def test_a_token_has_no_influence_on_queries_that_do_not_see_it(bits, what, dim, where):
    p = Chunks([(200, 150), (90, 0), (3, 300)], bits, BF16, dim, 4, 2, 16, seed=8)
    want = p.run(**where)
    spoilt = {0: (200, 201, 260, 349), 1: (50, 64), 2: (302,)}
    for i, tokens in spoilt.items():
        for t in tokens:
            page, at = p.pages_of[i][t // 16], t % 16
            if bits == 16:
                (p.ck if t % 2 else p.cv)[page, :, at, 3] = what
            else:
                p.sc[page, :, at, (0 if t % 2 else 2)] = what
    got = p.run(**where)
    starts = p.starts.tolist()
    for i, tokens in spoilt.items():
        touched = p.seen(i, **where)[:, list(tokens)].any(1)
        a, b = got[starts[i]:starts[i + 1]].cpu(), want[starts[i]:starts[i + 1]].cpu()
        keep = torch.from_numpy(~touched)
        assert torch.equal(a[keep].view(torch.int16), b[keep].view(torch.int16))
        assert (~a[~keep].isfinite()).flatten(1).any(1).all()


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("page", (16, 64))
def test_what_no_query_sees_may_be_anything(bits, page):
    window, sinks = 90, 20
    p = Chunks([(40, 700), (1, 33), (70, 200)], bits, BF16, 128, 8, 2, page, seed=2)
    want = p.run(window=window, sinks=sinks)
    for i in range(3):
        some = p.seen(i, window, sinks).any(0)
        for t in np.nonzero(~some)[0]:
            for c in (p.ck, p.cv) if bits == 16 else (p.sc,):
                c[p.pages_of[i][t // page], :, t % page] = float("nan")
        for x in range(-(-p.lengths[i] // page)):
            if not some[x * page:(x + 1) * page].any():
                p.table[i, x] = -7 if x % 2 else 1 << 30
    assert torch.equal(p.run(window=window, sinks=sinks).view(torch.int16), want.view(torch.int16))


@pytest.mark.parametrize("bits", (16, 8))
def test_pages_that_do_not_exist_have_no_tokens(bits):
    p = Chunks([(50, 200), (50, 200)], bits, BF16, 128, 4, 2, 16, seed=9)
    p.table[0, 3], p.table[0, 14], p.table[1, :] = -1, 1 << 30, -1
    out = p.run()
    assert not out[50:].any()
    keep = [t for t in range(250) if t // 16 not in (3, 14)]
    seen = p.seen(0)[:, keep]
    for j in range(2):
        k, v, *codes = p.held(0, j)
        k, v, *codes = (x if x is None else x[keep] for x in (k, v, *codes))
        for h in (2 * j, 2 * j + 1):
            o, allowed = ref.bound(p.q[:50, h].double().cpu().numpy(), k, v, seen, 128 ** -0.5, BF16, bits, *codes)
            assert (np.abs(out[:50, h].double().cpu().numpy() - o) <= allowed).all()


@pytest.mark.parametrize("bits", (16, 4))
def test_queries_without_tokens_and_rows_of_no_request(bits):
    p = Chunks([(30, 0), (20, 100)], bits, BF16, 128, 4, 2, 16, first=5, behind=7)
    want = p.run()
    p.len.copy_(torch.tensor([12, 0], dtype=torch.int32))
    out = torch.full_like(p.q, 3.0)
    out = out.contiguous()
    assert p.run(out=out) is out
    assert (out[:5] == 3).all() and (out[55:] == 3).all()
    assert not out[5:23].any() and not out[35:55].any() and out[23:35].any(2).all()
    # starts that do not ascend, and such outside of q: rows of nobody, and no others
    p.len.copy_(torch.tensor(p.lengths, dtype=torch.int32))
    for starts, same in (([5, 35, 10], slice(5, 35)), ([-9, 0, 1 << 30], slice(0, 0)), ([70, 60, 50], slice(0, 0))):
        p.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        assert torch.equal(p.run(out=out)[same], want[same])


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("requests", (3, 41, 80))
def test_starts_that_go_back_behind_long_contexts(bits, requests):
    """rows of one request alone are its own, and all stays within the rows that some request names, whatever the workspace holds"""
    p = Chunks([(64, 6000)] + [(0, 6064)] * (requests - 1), bits, BF16, 128, 8, 2, 64, behind=6)
    need = any4.any4_attn_chunk_workspace_bytes(requests, len(p.q), 8, 2, 128, p.width * 64)
    ws = torch.empty(need + 4096, dtype=torch.uint8, device="cuda").fill_(0xA5)
    p.check(p.run(workspace=ws[:need]))                          # (leaves what it cut in the workspace)
    out = torch.full(p.q.shape, 3.0, dtype=BF16, device="cuda")
    starts = [0, 40, 10, 60] + [60] * (requests - 3)
    p.starts.copy_(torch.tensor(starts, dtype=torch.int32))
    p.run(out=out, workspace=ws[:need])
    assert (out[60:] == 3).all() and (ws[need:] == 0xA5).all()
    for i, alone, at in ((0, range(0, 10), 0), (2, range(40, 60), 10)):
        p.new[i] = starts[i + 1] - starts[i]
        seen = p.seen(i)
        for h in range(8):
            k, v, *codes = p.held(i, h // 4)
            rows = slice(alone.start, alone.stop)
            o, allowed = ref.bound(p.q[rows, h].double().cpu().numpy(), k, v, seen[alone.start - at:alone.stop - at], 128 ** -0.5, BF16, bits, *codes)
            assert (np.abs(out[rows, h].double().cpu().numpy() - o) <= allowed).all()
    p.starts.copy_(torch.tensor(([0, 64] * requests)[:requests + 1], dtype=torch.int32))      # more rows together than the call has
    p.run(out=out, workspace=ws[:need])
    assert (out[64:] == 3).all() and (ws[need:] == 0xA5).all() and out.isfinite().all()


@pytest.mark.parametrize("dtype,by", [(F16, 2.0 ** 13), (BF16, 2.0 ** 14), (BF16, 2.0 ** 17)])
@pytest.mark.parametrize("bits", (16, 8))
def test_far_scores(dtype, by, bits):
    """scores of 2^26 and more: the one largest key has all the weight"""
    p = Chunks([(5, 200), (130, 10)], bits, dtype, 128, 4, 2, 16, seed=11)
    g = torch.Generator().manual_seed(12)
    p.q.mul_(by)
    for i, n in enumerate(p.lengths):
        p.write(i, torch.randn(n, 2, 128, generator=g) * (by), torch.randn(n, 2, 128, generator=g) * 0.5)
    out, starts = p.run().double().cpu().numpy(), p.starts.tolist()
    for i in range(2):
        for h in range(4):
            kk, v, *_ = p.held(i, h // 2)
            s = np.where(p.seen(i), p.q[starts[i]:starts[i + 1], h].double().cpu().numpy() @ kk.T, -np.inf)
            two = np.sort(s, 1)[:, -2:]
            clear = (two[:, 1] - two[:, 0]) * 128 ** -0.5 > 2.0 ** -18 * np.abs(two[:, 1]) * 128 ** -0.5 + 40      # (fp32 sums tell them apart)
            assert clear.sum() > len(clear) // 2
            want = v[s.argmax(1)][clear]
            assert (np.abs(out[starts[i]:starts[i + 1], h][clear] - want) <= 2.0 ** -7 * np.abs(want) + 1e-3 * np.abs(v).max() * (bits < 16)).all()


def test_the_native_and_the_checked_call_are_one(monkeypatch):
    from paper_2507_04610_amd import binding
    p = Chunks([(19, 600), (1, 3000)], 8, BF16, 128, 4, 2, 16)
    want = p.run(), p.run(window=333, sinks=4)
    monkeypatch.setattr(binding, "_native_calls", binding._NoNativeCalls)
    assert torch.equal(p.run(), want[0]) and torch.equal(p.run(window=333, sinks=4), want[1])


@pytest.mark.parametrize("bits", (16, 4))
def test_a_graph_follows_starts_and_lengths(bits):
    p = Chunks([(60, 600), (1, 3000), (4, 40)], bits, BF16, 128, 8, 2, 16)
    need = any4.any4_attn_chunk_workspace_bytes(3, 65, 8, 2, 128, p.width * 16)
    ws, out = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), torch.zeros(65, 8, 128, dtype=BF16, device="cuda")
    p.run(out=out, workspace=ws)
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        p.run(out=out, workspace=ws)
    for starts, lengths in (([0, 60, 61, 65], [660, 3001, 44]), ([0, 1, 2, 65], [1, 2999, 33]), ([0, 30, 65, 65], [660, 35, 0]), ([0, 60, 61, 65], [660, 3001, 44])):
        p.starts.copy_(torch.tensor(starts, dtype=torch.int32))
        p.len.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out, p.run())


def test_no_requests_and_no_tokens():
    p = Chunks([(0, 5), (0, 0)], 16, BF16, 128, 4, 2)
    assert p.run().shape == (0, 4, 128)
    i32 = torch.zeros(1, dtype=torch.int32, device="cuda")
    q = torch.zeros(3, 4, 128, dtype=BF16, device="cuda")
    out = torch.full_like(q, 2.0)
    any4.any4_attn_chunk(q, p.ck, p.cv, torch.zeros(0, 2, dtype=torch.int32, device="cuda"), i32, i32[:0], out=out)
    assert (out == 2).all()
