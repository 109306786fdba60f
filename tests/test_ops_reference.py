"""The 64-bit references of the operator tests, on the CPU: gradients against differences, lists
against their definition, and that a planted mistake is seen."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import ops_reference as R  # noqa: E402


def _difference(fn, inputs, cot, i, step=1e-5):
    """Directional derivative of sum(cot * fn) along a random direction of input i."""
    g = torch.Generator().manual_seed(i)
    d = torch.randn(inputs[i].shape, generator=g, dtype=torch.float64)
    val = []
    for s in (step, -step):
        moved = [t + s * d if j == i else t for j, t in enumerate(inputs)]
        val.append(sum((o * c).sum() for o, c in zip(fn(*moved), cot)))
    return (val[0] - val[1]) / (2 * step), d


@pytest.mark.parametrize("h", [1, 7, 64])
@pytest.mark.parametrize("shared", [True, False])
def test_norm_gradients_match_differences(h, shared):
    g = torch.Generator().manual_seed(h)
    T, a, eps = 3, 0.5, 1e-6

    def n(*s):
        return torch.randn(*s, generator=g, dtype=torch.float64)

    def fn(x, y, w, gate, w_next):
        z = R.postnorm(x, y, w, gate, a, eps)
        return z, R.rms(z, eps) * w_next

    inputs = [n(T, h), n(T, h), n(h), n(h) if shared else n(T, h), n(h)]
    cot = [n(T, h), n(T, h)]
    got = R.grads(fn, inputs, cot)
    for i in range(len(inputs)):
        slope, d = _difference(fn, inputs, cot, i)
        along = (got[i] * d).sum()
        # central differences of functions of order one: step^2 and 2^-52 / step
        assert abs(slope - along) <= 1e-5 * (1 + got[i].abs().sum()), i


def test_norm_gradients_by_formula():
    """The gradient that the kernels evaluate, against the differentiated forward."""
    g = torch.Generator().manual_seed(5)
    T, h, eps = 4, 33, 1e-6
    x, w, du = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((T, h), (h,), (T, h)))
    r = 1 / torch.sqrt((x * x).mean(-1, keepdim=True) + eps)
    hat, q = x * r, du * w
    dx, dw = R.grads(lambda x, w: (R.rms(x, eps) * w,), (x, w), (du,))
    assert torch.allclose(dx, r * (q - hat * (q * hat).mean(-1, keepdim=True)), rtol=1e-10, atol=1e-12)
    assert torch.allclose(dw, (du * hat).sum(0), rtol=1e-12, atol=1e-12)


def test_combine_gradients_match_differences():
    g = torch.Generator().manual_seed(1)
    ids = np.array([[0, 2], [2, -1], [1, 1], [-1, 9]], np.int32)
    offset, pair, row = (torch.from_numpy(a) for a in R.lists(ids, 3))
    w, ys, dy = (torch.randn(*s, generator=g, dtype=torch.float64) for s in ((4, 2), (8, 5), (4, 5)))
    dys, written, dw, _ = R.combine_backward(row, w, ys, dy)
    assert int(written.sum()) == int(offset[-1]) == 5
    for v, grad in ((w, dw), (ys, dys)):
        d = torch.randn(v.shape, generator=g, dtype=torch.float64)
        moved = [R.combine(row, w + s * d if v is w else w, ys + s * d if v is ys else ys)[0]
                 for s in (0.5, -0.5)]   # linear in either
        assert abs(((moved[0] - moved[1]) * dy).sum() - (grad * d).sum()) < 1e-12


def test_lists_by_definition():
    rng = np.random.default_rng(3)
    ids = rng.integers(-2, 9, (11, 3)).astype(np.int32)
    n, flat = 7, ids.reshape(-1)
    offset, pair, row = R.lists(ids, n)
    key = np.where((flat >= 0) & (flat < n), flat, n)
    for p in range(flat.size):
        want = int((key < key[p]).sum() + (key[:p] == key[p]).sum()) if key[p] < n else -1
        assert row.reshape(-1)[p] == want
        assert key[p] == n or pair[want] == p
    assert [int((key < e).sum()) for e in range(n + 1)] == offset.tolist()
    assert (pair[offset[n]:] == -1).all()


def test_w4_bound_sees_a_wrong_code():
    """One code off by one, a column in the wrong half of its byte, a scale of the next group."""
    g = torch.Generator().manual_seed(2)
    codes = torch.randint(0, 256, (8, 128), dtype=torch.uint8, generator=g)
    scale = torch.rand(8, 4, generator=g) + 0.5
    x = torch.randn(3, 256, generator=g).to(torch.bfloat16)
    want, bound = R.w4_product(x, codes, scale, 64)
    bound = bound + R.half_step(torch.bfloat16) * want.abs()
    swapped = (codes >> 4) | (codes << 4)
    assert ((R.w4_product(x, swapped, scale, 64)[0] - want).abs() > bound).float().mean() > 0.9
    assert ((R.w4_product(x, codes, scale.roll(1, 1), 64)[0] - want).abs() > bound).float().mean() > 0.9
    one = torch.zeros(1, 256, dtype=torch.bfloat16)
    one[0, 77] = 1.0
    assert torch.equal(R.w4_product(one, codes, scale, 64)[0][0],
                       (((codes[:, 38] >> 4).double() - 8) * scale[:, 1].double()))
