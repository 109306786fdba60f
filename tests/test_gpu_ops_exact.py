"""4-bit products on the GPU with sums that fp32 holds exactly: outputs equal bit for bit, at the widths
that take several panels, wide ones, K parts and the tiled kernel, for one matrix and for experts."""
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import ops_exact as X  # noqa: E402
from gpu_util import say  # noqa: E402
from paper_2608_14385_amd import deamoe as D  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32


def matrices(g, *lead, K, group, scale):
    """A matrix for the linear product, and gate and up for the other."""
    return [X.matrix(g, *lead, K=K, group=group, scale=scale, device="cuda", unit=u) for u in (1, X.GATE_UNIT, 1)]


def wanted(x, mats, group):
    y, gate, up = (X.product(x, *m, group, u) for m, u in zip(mats, (1, X.GATE_UNIT, 1)))
    return y.float().to(BF), X.swiglu(gate, up)


@pytest.mark.parametrize("scale", [F32, BF])
@pytest.mark.parametrize("M,R,K,group", [
    (1, 1, 32, 32), (2, 17, 96, 32), (1, 2000, 7168, 128), (7, 300, 4224, 128), (16, 8300, 1056, 32),
    (12, 10000, 192, 64), (9, 12001, 4224, 128),                                        # K parts
    (16, 700, 7200, 32), (9, 300, 4288, 64), (30, 500, 7296, 128), (3, 260, 16544, 32), (5, 33, 9088, 64),   # wide panels
    (61, 2815, 2048, 64), (160, 700, 2112, 64), (161, 1500, 4128, 32), (250, 2100, 1152, 128),
    (2048, 2050, 1152, 128), (1100, 4000, 320, 64), (1030, 4097, 2080, 32),             # 64-row tiles
])
def test_one_matrix(M, R, K, group, scale):
    say(f"[gpu] exact w4 M={M} R={R} K={K} group={group} {scale}")
    g = torch.Generator(device="cuda").manual_seed(M + R)
    x, mats = X.rows(g, M, K, "cuda"), matrices(g, R, K=K, group=group, scale=scale)
    y, z = (torch.full((M, R), 9.0, dtype=BF, device="cuda") for _ in range(2))
    D.deamoe_w4_linear(x, *mats[0], y)
    D.deamoe_w4_swiglu(x, *mats[1], *mats[2], z)
    want = wanted(x, mats, group)
    assert torch.equal(y, want[0]) and torch.equal(z, want[1])


@pytest.mark.parametrize("scale", [F32, BF])
@pytest.mark.parametrize("rows,R,K,group", [
    ((3, 0, 9, 1), 70, 2144, 32), ((1,) * 8, 2048, 7168, 128), ((17, 0, 0, 5, 33), 300, 4224, 128),
    ((5,) * 30, 10900, 160, 32),                       # four weight tiles per wave
    ((30, 90, 64, 0, 129), 260, 2080, 32), ((400, 3), 200, 4288, 64),   # 64-row tiles
])
def test_experts(rows, R, K, group, scale):
    say(f"[gpu] exact w4 experts of {rows} R={R} K={K} group={group} {scale}")
    g, n, M = torch.Generator(device="cuda").manual_seed(R), len(rows), sum(rows)
    offset = torch.tensor([0, *rows]).cumsum(0)
    x, mats = X.rows(g, M, K, "cuda"), matrices(g, n, R, K=K, group=group, scale=scale)
    y, z = (torch.full((M, R), 9.0, dtype=BF, device="cuda") for _ in range(2))
    D.deamoe_w4_linear(x, *mats[0], y, offset=offset.to(I32).cuda())
    D.deamoe_w4_swiglu(x, *mats[1], *mats[2], z, offset=offset.to(I32).cuda())
    for e in range(n):
        at = slice(int(offset[e]), int(offset[e + 1]))
        want = wanted(x[at], [(c[e], s[e]) for c, s in mats], group)
        assert torch.equal(y[at], want[0]) and torch.equal(z[at], want[1]), e


@pytest.mark.parametrize("M,R,K,group", [(384, 5000, 192, 64), (385, 5000, 192, 64),     # 120 and 140 workgroups
                                         (64, 16000, 160, 32), (65, 16000, 160, 32)])    # two matrices: 126 and 252
def test_either_side_of_the_tiled_kernel(M, R, K, group):
    test_one_matrix(M, R, K, group, F32)


@pytest.mark.parametrize("each", [14, 15, 20, 21])   # the last streamed and the first tiled, one matrix and two
def test_either_side_of_the_tiled_kernel_for_experts(each):
    test_experts((each,) * 9, 150, 1120, 32, F32)
    test_experts((1, 2 * each, 0, 2 * each, each - 1), 150, 1120, 32, F32)   # the same mean, unevenly
