"""Captured calls of any4_attn_chunk, and of attention with a window, replayed with starts and lengths other than those of the capture: each replay against 64 bits.
(The host plans a call by its sizes alone; the requests that a replay finds may have nothing to do with them.)"""
import numpy as np
import pytest
import torch

import paper_2507_04610_amd as any4
import test_gpu_attn_decode_window as decode_window
import test_gpu_attn_prompt_window as prompt_window
from test_gpu_attn_chunk import Chunks
from test_gpu_attn_decode import Problem
from test_gpu_attn_prompt import starts, tensors

pytestmark = pytest.mark.gpu

BF16, F16 = torch.bfloat16, torch.float16


def captured(call):
    """a graph of the call, made behind a first run of it"""
    call()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call()
    return graph


def check_first(p, out, rows):
    """the rows that requests name"""
    q = p.q
    p.q = q[:rows]
    p.check(out[:rows])
    p.q = q


# (starts, lengths): as captured, one token each beside all rows in the last, rows of one alone, a request without rows or tokens, as captured
FEW = [([0, 60, 61, 65], [660, 3001, 44]), ([0, 1, 2, 65], [1, 2999, 33]), ([0, 0, 65, 65], [660, 3001, 44]), ([0, 30, 65, 65], [660, 35, 0]), ([0, 3, 40, 65], [9, 3001, 20]),
       ([0, 60, 61, 65], [660, 3001, 44])]


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
@pytest.mark.parametrize("where", ({}, {"window": 900, "sinks": 70}))
def test_chunks(bits, dtype, where):
    p = Chunks([(60, 600), (1, 3000), (4, 40)], bits, dtype, 128, 8, 2, 16, seed=41)
    need = any4.any4_attn_chunk_workspace_bytes(3, 65, 8, 2, 128, p.width * 16)
    assert need > 0
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(65, 8, 128, dtype=dtype, device="cuda")
    graph = captured(lambda: p.run(out=out, workspace=ws, **where))
    for first, lengths in FEW:
        p.starts.copy_(torch.tensor(first, dtype=torch.int32))
        p.len.copy_(torch.tensor(lengths, dtype=torch.int32))
        ws.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        p.new, p.lengths = np.diff(first).tolist(), lengths
        p.check(out, **where)
        assert torch.equal(out, p.run(**where))


@pytest.mark.parametrize("bits", (16, 8, 4))
def test_chunks_of_many_requests(bits):
    """a launch of its own finds the work"""
    n = 90
    p = Chunks([(3 + i % 2, 40 + 17 * i) for i in range(n)], bits, BF16, 64, 4, 2, 64, seed=42)
    rows, full = len(p.q), list(p.lengths)
    need = any4.any4_attn_chunk_workspace_bytes(n, rows, 4, 2, 64, p.width * 64)
    ws, out = torch.empty(need, dtype=torch.uint8, device="cuda"), torch.zeros(rows, 4, 64, dtype=BF16, device="cuda")
    graph = captured(lambda: p.run(out=out, workspace=ws))
    as_captured = p.starts.tolist()
    for first, lengths in ((as_captured, full), ([0] * 40 + [rows] * (n - 39), full), ([min(i, rows) for i in range(n)] + [rows], [0 if i % 3 == 1 else full[i] for i in range(n)]),
                           ([min(4 * i, rows) for i in range(n + 1)], [min(x, 1 + 7 * i) for i, x in enumerate(full)]), (as_captured, full)):
        p.starts.copy_(torch.tensor(first, dtype=torch.int32))
        p.len.copy_(torch.tensor(lengths, dtype=torch.int32))
        ws.fill_(0xA5)
        graph.replay()
        torch.cuda.synchronize()
        p.new, p.lengths = np.diff(first).tolist(), lengths
        check_first(p, out, first[-1])
        assert torch.equal(out[:first[-1]], p.run()[:first[-1]])


@pytest.mark.parametrize("dtype,dim", [(BF16, 128), (F16, 64)])
def test_prompts_with_a_window(dtype, dim):
    q, k, v = tensors(300, 300, 4, 2, dim, dtype, 43, True)
    at, out = starts([70, 200, 30]), torch.zeros(300, 4, dim, dtype=dtype, device="cuda")
    graph = captured(lambda: any4.any4_attn_prompt(q, k, v, at, window=33, sinks=2, out=out))
    for nq in ([70, 200, 30], [1, 1, 298], [300, 0, 0], [0, 299, 1], [129, 128, 43]):
        at.copy_(starts(nq))
        graph.replay()
        torch.cuda.synchronize()
        prompt_window.check(out, q, k, v, nq, nq, 33, 2)


@pytest.mark.parametrize("bits", (16, 8, 4))
@pytest.mark.parametrize("dtype", (BF16, F16))
def test_single_tokens_with_a_window(bits, dtype):
    p = Problem([600, 3000, 40], bits, dtype, 128, 8, 2, 16, seed=44)
    need = any4.any4_attn_decode_workspace_bytes(3, 8, 2, 128, p.width * 16)
    ws, out = torch.empty(max(need, 1), dtype=torch.uint8, device="cuda"), torch.empty(3, 8, 128, dtype=dtype, device="cuda")
    graph = captured(lambda: p.run(window=500, sinks=4, out=out, workspace=ws))
    for lengths in ([600, 3000, 40], [1, 2999, 0], [599, 4, 33], [0, 504, 40], [600, 3000, 40]):
        p.len.copy_(torch.tensor(lengths, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        p.lengths = lengths
        some = [i for i in range(3) if lengths[i] > 0]
        decode_window.check(p, out, 500, 4, requests=some)
        assert not any(out[i].any() for i in range(3) if lengths[i] == 0)
