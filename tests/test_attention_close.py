"""attention_close.py says no to what it is there to find: nothing, even weights, a piece of the tokens left out - for every case that the
GPU tests run."""
import numpy as np
import pytest
import torch

import attention_close as close


@pytest.mark.parametrize("name", close.CASES)
def test_wrong_outputs_lie_outside(name):
    p = close.Requests(*close.CASES[name][0])
    for i, _, q, held in p.each(requests=(0, 3, 5, 40)):
        o, allowed, _ = close.expected(q, held, p.scale)
        assert np.isfinite(allowed).all() and (allowed > 0).all()

        def rejected(got):
            return max(close.fits(got, q, held, p.scale)) > 1
        n = p.lengths[i]
        assert rejected(0 * o)
        if n < 2:
            continue
        assert rejected(close.weigh(q, held, p.scale, even=True)[0] @ held.v)
        # a piece of a request that is cut for all of the chip's blocks (128 tokens at least), its first, a middle and its last one
        piece = max(n // 256, 128) if n > 256 else n // 2
        for at in (0, n // 2, n - piece):
            keep = np.ones(n, bool)
            keep[at:at + piece] = False
            assert rejected(close.weigh(q, held, p.scale, keep=keep)[0] @ held.v), (i, at, piece)


@pytest.mark.parametrize("name", close.CASES)
def test_right_outputs_lie_inside(name):
    """64 bits, rounded once to the output's type"""
    p = close.Requests(*close.CASES[name][0])
    for _, _, q, held in p.each(requests=(0, 2, 3, 5, 40)):
        o, _, _ = close.expected(q, held, p.scale)
        assert max(close.fits(torch.from_numpy(o).to(p.dtype).double().numpy(), q, held, p.scale)) < 1


def test_a_bias_that_does_not_go_away_lies_outside():
    """the sum of weights times codes with their bias in fp32, the bias taken off at the end, lies outside at 32768
    tokens; the same with the bias taken off in front of every 32 tokens' sum inside"""
    p = close.Requests([32768], 4, close.F16, 64, 2, 1, 7)
    for _, _, q, held in p.each():
        w, _, _ = close.weigh(q, held, p.scale)
        w = w / w.max(1, keepdims=True)
        unit = 2.0 ** -np.floor(np.log2(held.v_scale.max()))
        rounded = (w * (held.v_scale[:, 0] * unit)).astype(np.float16).astype(np.float64)
        rest = w @ (held.v_offset + 8 * held.v_scale)
        for stepwise, most in ((False, np.inf), (True, 1)):
            sums, ones = np.zeros((2, 64), np.float32), np.zeros((2, 1), np.float32)
            for t in range(0, 32768, 32):
                r, c = rounded[:, t:t + 32], held.codes[t:t + 32]
                if stepwise:
                    sums = (sums - 1032 * r.sum(1, keepdims=True)).astype(np.float32)
                else:
                    ones = (ones + r.sum(1, keepdims=True)).astype(np.float32)
                sums = (sums + r @ (c + 1024)).astype(np.float32)
            got = ((sums - 1032.0 * ones) / unit + rest) / w.sum(1, keepdims=True)
            worst, mean = close.fits(got.astype(np.float16).astype(np.float64), q, held, p.scale)
            assert max(worst, mean) <= most and (stepwise or max(worst, mean) > 1)
