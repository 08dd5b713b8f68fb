"""any4_kv_read's out: anything but a pair is named as the mistake"""
import pytest
import torch

import paper_2507_04610_amd as any4


@pytest.mark.parametrize("make", [lambda t: t, lambda t: (t,), lambda t: (t, t, t), lambda t: 5, lambda t: iter((t,))])
def test_out_that_is_no_pair_is_refused(make):
    ck, cv, _ = any4.any4_kv_cache(2, 2, 128, 16, device="cpu")
    out = make(torch.empty(3, 2, 128, dtype=torch.bfloat16))
    with pytest.raises(any4.Any4Error, match="pair"):
        any4.any4_kv_read(ck, cv, torch.arange(3), out=out)


@pytest.mark.gpu
@pytest.mark.parametrize("make", [tuple, list, torch.stack])
def test_pairs(make):
    ck, cv, _ = any4.any4_kv_cache(2, 2, 128, 16)
    ck.normal_()
    cv.normal_()
    slots = torch.tensor([3, 17, 0], device="cuda")
    want = any4.any4_kv_read(ck, cv, slots)
    out = make([torch.empty(3, 2, 128, dtype=torch.bfloat16, device="cuda") for _ in range(2)])
    got = any4.any4_kv_read(ck, cv, slots, out=out)
    assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(got, want, out))
