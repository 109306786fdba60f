"""What the exact 4-bit products see, on the CPU: mistakes planted in the reference."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import ops_exact as X  # noqa: E402
import ops_reference as R  # noqa: E402

BF, F32 = torch.bfloat16, torch.float32


@pytest.mark.parametrize("M,R_,K,group", [(1, 300, 7168, 128), (9, 40, 4224, 128), (30, 20, 7296, 128),
                                          (3, 60, 16544, 32), (5, 33, 9088, 64), (64, 20, 96, 32)])
@pytest.mark.parametrize("scale", [F32, BF])
def test_mistakes_change_the_output(M, R_, K, group, scale):
    g = torch.Generator().manual_seed(K + M)
    x, (codes, s) = X.rows(g, M, K, "cpu"), X.matrix(g, R_, K=K, group=group, scale=scale, device="cpu")
    y = X.product(x, codes, s, group)
    assert torch.equal(y, R.w4_product(x, codes, s, group)[0])
    # fp32 sums in another order are the same
    w = R.w4_matrix(codes, s, group).float()
    assert torch.equal(x.float().flip(1) @ w.flip(1).T, y.float())
    out = y.float().to(BF)

    def seen(x, codes, s):
        return not torch.equal(X.product(x, codes, s, group).float().to(BF), out)

    for col in (0, K // 2 + 1, K - 1):   # a column lost
        cut = x.clone()
        cut[:, col] = 0
        assert seen(cut, codes, s), col
    cut = x.clone()
    cut[:, -32:] = 0
    assert seen(cut, codes, s)           # a step past a panel's end
    assert seen(x, codes, s.roll(1, 1))  # the neighbour's scale
    assert seen(x, codes, s.roll(1, 0))
    assert seen(x, (codes >> 4) | (codes << 4), s)
    if scale is F32:                     # weights or scales rounded to bf16
        assert seen(x, codes, s.to(BF).float())
        assert not torch.equal((x.double() @ w.to(BF).double().T).float().to(BF), out)


def test_gate_sums_take_silu_to_its_ends():
    g = torch.Generator().manual_seed(1)
    x, (codes, s) = X.rows(g, 4, 512, "cpu"), X.matrix(g, 60, K=512, group=64, scale=F32, device="cpu", unit=X.GATE_UNIT)
    v = X.product(x, codes, s, 64, X.GATE_UNIT).float()
    assert bool(((v == 0) | (v.abs() >= X.GATE_UNIT)).all())
    assert torch.equal(v / (1 + torch.exp(-v)), v.clamp(min=0))
