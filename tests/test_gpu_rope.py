"""any4_rope and any4_rope_kv_write against norm and rotation in 64 bits (rope_reference.py has the bound), and against each other."""
import numpy as np
import pytest
import torch

import paper_2507_04610_amd as any4
import rope_reference as ref

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


class Problem:
    """rows of a fused projection, [tokens, (heads + 2 kv_heads) * dim]"""

    def __init__(self, tokens, dtype=BF16, dim=128, heads=6, kv_heads=2, rotary=None, axes=1, interleaved=False, norms=True, seed=0, far=70000):
        g = torch.Generator().manual_seed(seed)
        self.dtype, self.dim, self.heads, self.kv_heads, self.interleaved, self.tokens = dtype, dim, heads, kv_heads, interleaved, tokens
        rotary = dim if rotary is None else rotary
        self.row = torch.randn(tokens, (heads + 2 * kv_heads) * dim, generator=g).to(dtype).cuda()
        self.q, self.k, self.v = (self.row[:, a * dim:b * dim].view(tokens, b - a, dim)
                                  for a, b in ((0, heads), (heads, heads + kv_heads), (heads + kv_heads, heads + 2 * kv_heads)))
        self.freqs = 10000.0 ** (-torch.arange(rotary // 2, dtype=torch.float64) * 2 / rotary)
        self.positions = torch.randint(-far, far, (axes, tokens), generator=g)
        self.axis_of = torch.randint(0, axes, (rotary // 2,), generator=g).to(torch.uint8) if axes > 1 else None
        self.norms = [(torch.randn(dim, generator=g) * 0.3 + 1).to(dtype).cuda() if norms else None for _ in range(2)]

    def kw(self, eps=1e-6):
        return dict(q_norm=self.norms[0], k_norm=self.norms[1], eps=eps, interleaved=self.interleaved,
                    axis_of=None if self.axis_of is None else self.axis_of.cuda())

    def where(self):
        return self.positions.squeeze(0).cuda() if len(self.positions) == 1 else self.positions.cuda()

    def run(self, eps=1e-6, **kw):
        return any4.any4_rope(self.q, self.k, self.where(), self.freqs.cuda(), **self.kw(eps), **kw)

    def expected(self, x, norm, eps=1e-6):
        w = None if norm is None else norm.double().cpu().numpy()
        return ref.turn(x.double().cpu().numpy(), w, self.positions.numpy(), self.freqs.numpy(),
                        None if self.axis_of is None else self.axis_of.numpy().astype(int), self.interleaved, eps)

    def check(self, got, eps=1e-6):
        for y, x, norm in zip(got, (self.q, self.k), self.norms):
            assert y.shape == x.shape and y.dtype == self.dtype
            want, size = self.expected(x, norm, eps)
            off = np.abs(y.double().cpu().numpy() - want)
            limit = ref.allowed(want, size, self.dtype)
            assert (off <= limit).all(), np.max(off / limit)


@pytest.mark.parametrize("norms", (True, False))
@pytest.mark.parametrize("interleaved", (False, True))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim,rotary", [(128, 128), (128, 64), (128, 8), (128, 96), (64, 64), (64, 40), (64, 16)])
def test_shares_of_a_head_that_are_turned(dim, rotary, dtype, interleaved, norms):
    p = Problem(37, dtype, dim, rotary=rotary, interleaved=interleaved, norms=norms, seed=rotary)
    p.check(p.run())


@pytest.mark.parametrize("tokens", (1, 2, 3, 4, 5, 8, 500))
@pytest.mark.parametrize("heads,kv_heads,dim", [(1, 1, 128), (5, 3, 64), (32, 8, 128), (7, 1, 64)])
def test_tokens_and_heads(tokens, heads, kv_heads, dim):
    p = Problem(tokens, heads=heads, kv_heads=kv_heads, dim=dim, seed=tokens)
    p.check(p.run())


@pytest.mark.parametrize("axes", (2, 3, 4))
@pytest.mark.parametrize("interleaved", (False, True))
def test_axes(axes, interleaved):
    p = Problem(70, axes=axes, interleaved=interleaved, rotary=96)
    got = p.run()
    p.check(got)
    # an axis that does not exist is the last one
    p.axis_of = torch.where(p.axis_of == axes - 1, 200, p.axis_of).to(torch.uint8)
    assert all(torch.equal(a, b) for a, b in zip(p.run(), got))


@pytest.mark.parametrize("far", (10, 1 << 20, 1 << 40))
def test_far_positions(far):
    """in fp64 a position of 2^40 leaves 2^-12 of a radian"""
    p = Problem(64, far=far, dtype=BF16)
    if far > 1 << 30:
        p.freqs = p.freqs.clamp_max(1e-3)
    p.check(p.run())


def test_sizes_of_values():
    """tiny, large and zero heads, and an eps that matters"""
    for by in (1e-4, 1.0, 1e4):
        p = Problem(40, by and BF16, seed=3)
        p.row.mul_(by)
        p.check(p.run())
        p.check(p.run(eps=0.5), eps=0.5)
    p.q[:, 1] = 0
    y = p.run()[0]
    assert not y[:, 1].any() and y[:, 0].isfinite().all()


@pytest.mark.parametrize("interleaved", (False, True))
def test_in_place_and_into_strided_rows(interleaved):
    p = Problem(50, interleaved=interleaved, rotary=64)
    want = p.run()
    rows = torch.full((50, 3, 6, 136), 7.0, dtype=BF16, device="cuda")
    out = rows[:, 1, :, :128], torch.zeros(2, 50, 128, dtype=BF16, device="cuda").transpose(0, 1)
    got = p.run(out=out)
    assert got[0] is out[0] and got[1] is out[1] and all(torch.equal(a, b) for a, b in zip(got, want))
    assert (rows[:, 0] == 7).all() and (rows[:, 2] == 7).all() and (rows[:, 1, :, 128:] == 7).all()
    v = p.v.clone()
    got = p.run(out=(p.q, p.k))
    assert all(torch.equal(a, b) for a, b in zip(got, want)) and torch.equal(p.v, v)


def test_a_head_that_is_not_finite_stays_alone():
    p = Problem(20)
    want = p.run()
    p.q[3, 2, 5], p.k[7, 1, 100] = float("nan"), float("inf")
    got = p.run()
    bad = [torch.zeros(t.shape[:2], dtype=torch.bool) for t in got]
    bad[0][3, 2] = bad[1][7, 1] = True
    for y, w, b in zip(got, want, bad):
        assert torch.equal(y.cpu()[~b], w.cpu()[~b])
    # (the definition: a square that is not a number leaves none, an infinite one zeros beside infinity over infinity and what that is turned with)
    assert not got[0][3, 2].isfinite().any()
    at = torch.tensor([36, 100])
    assert got[1][7, 1, at].isnan().all() and not got[1][7, 1, [i for i in range(128) if i not in (36, 100)]].any()


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("dim", (128, 64))
@pytest.mark.parametrize("interleaved,rotary,norms", [(False, 64, True), (True, 48, False), (False, 16, True)])
def test_the_cache_holds_what_the_two_calls_would_put_there(bits, dtype, dim, interleaved, rotary, norms):
    p = Problem(101, dtype, dim, heads=5, kv_heads=3, rotary=rotary, interleaved=interleaved, norms=norms)
    page, pages = 32, 5
    slots = torch.randperm(page * pages, generator=torch.Generator().manual_seed(bits))[:101]
    slots[17], slots[50], slots[99] = -1, page * pages, -(1 << 40)              # left out
    slots = slots.cuda()
    p.row[3, 5 * dim + 2 * dim + 9] = float("inf")                                # a key that codes cannot hold
    caches = [any4.any4_kv_cache(pages, 3, dim, page, bits, dtype) for _ in range(2)]
    for cache in caches:
        for t in cache:
            if t is not None:
                t.view(torch.uint8).fill_(0x5A)
    q, k = p.run()
    any4.any4_kv_write(k, p.v, slots, *caches[0], bits=bits)
    k_out = torch.empty_like(k)
    got = any4.any4_rope_kv_write(p.q, p.k, p.v, p.where(), p.freqs.cuda(), slots, *caches[1], bits=bits, k_out=k_out, **p.kw())
    assert torch.equal(got.view(torch.int16), q.view(torch.int16)) and torch.equal(k_out.view(torch.int16), k.view(torch.int16))
    for a, b in zip(*caches):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))
    # without rows for the keys, and q in place
    for t in caches[1]:
        if t is not None:
            t.view(torch.uint8).fill_(0x5A)
    any4.any4_rope_kv_write(p.q, p.k, p.v, p.where(), p.freqs.cuda(), slots, *caches[1], bits=bits, out=p.q, **p.kw())
    assert torch.equal(p.q.view(torch.int16), q.view(torch.int16))
    for a, b in zip(*caches):
        assert a is None or torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def test_the_native_and_the_checked_call_are_one(monkeypatch):
    from paper_2507_04610_amd import binding
    p = Problem(33, axes=3)
    slots = torch.arange(33).cuda()
    results = []
    for calls in (binding._calls(), binding._NoNativeCalls):
        monkeypatch.setattr(binding, "_native_calls", calls)
        cache = any4.any4_kv_cache(4, 2, 128, 16, 8)
        results.append([*p.run(), any4.any4_rope_kv_write(p.q, p.k, p.v, p.where(), p.freqs.cuda(), slots, *cache, bits=8, **p.kw()), *cache])
    assert all(torch.equal(a, b) for a, b in zip(*results))


def test_empty_calls_another_stream_and_a_graph():
    p = Problem(0)
    assert [t.shape[0] for t in p.run()] == [0, 0]
    p = Problem(64, seed=5)
    cache = any4.any4_kv_cache(5, 2, 128, 16, 8)
    slots, freqs, where, kw = torch.arange(64).cuda(), p.freqs.cuda(), p.where(), p.kw()
    out = torch.empty_like(p.q)

    def call():
        any4.any4_rope_kv_write(p.q, p.k, p.v, where, freqs, slots, *cache, bits=8, out=out, **kw)
    call()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    for i in range(3):
        p.row.copy_(torch.randn(p.row.shape, generator=torch.Generator().manual_seed(i)).to(BF16))
        where.add_(i)
        graph.replay()
        torch.cuda.synchronize()
        got = [out.clone(), *(t.clone() for t in cache)]
        call()
        assert all(torch.equal(a, b) for a, b in zip(got, [out, *cache]))
