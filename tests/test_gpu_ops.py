"""The operators beside the layer on the GPU, against 64-bit references, at the sizes and values
where they can go wrong.  Tolerances follow from the roundings (ops_reference)."""
import os
import sys

import numpy as np
import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
import ops_reference as R  # noqa: E402
from gpu_util import say  # noqa: E402
from paper_2608_14385_amd import deamoe as D  # noqa: E402
from paper_2608_14385_amd import workloads as W  # noqa: E402

pytestmark = pytest.mark.gpu

BF, F32, I32 = torch.bfloat16, torch.float32, torch.int32
TYPES = {"bf16": BF, "f32": F32}


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def normal(g, *shape, dtype=F32, scale=1.0):
    return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)


def close(got, want, bound, dtype, what):
    """|got - want| within the bound plus the rounding of the output."""
    off = (got.double() - want).abs()
    most = bound + R.half_step(dtype) * want.abs() + torch.finfo(dtype).tiny
    bad = off > most
    assert not bool(bad.any()), (what, int(bad.sum()), float((off / most).max()))
    assert bool(torch.isfinite(got).all()), what


def same_bits(a, b):
    return torch.equal(a.contiguous().view(torch.uint8), b.contiguous().view(torch.uint8))


# ------------------------------------------------------------- sorted tokens


class Sorted:
    """One dispatch: its outputs, the unused parts filled beforehand."""

    def __init__(self, ids, n, x=None, ws=None, stream=None):
        T, k = ids.shape
        self.offset = torch.full((n + 1,), -7, dtype=I32, device="cuda")
        self.pair = torch.full((T * k,), -7, dtype=I32, device="cuda")
        self.row = torch.full((T, k), -7, dtype=I32, device="cuda")
        self.xs = torch.full((T * k, x.shape[1]), 3.0, dtype=x.dtype, device="cuda") if x is not None else None
        if stream is not None:
            torch.cuda.synchronize()   # the fills above ran on another stream
        D.deamoe_dispatch(ids, x, self.offset, self.pair, self.row, self.xs, ws=ws, stream=stream)

    def check(self, ids, n, x=None):
        k = ids.shape[1]
        for got, want in zip((self.offset, self.pair, self.row), R.lists(ids.cpu().numpy(), n)):
            assert np.array_equal(got.cpu().numpy(), want)
        if x is not None:
            used = int(self.offset[-1])
            assert torch.equal(self.xs[:used], x[self.pair[:used].long() // k])
            assert bool((self.xs[used:] == 3.0).all())


def ids_of(g, T, k, n, kind):
    if kind == "topk":        # distinct experts
        return torch.rand(T, n, device="cuda", generator=g).topk(k, 1).indices.to(I32)
    lo, hi = {"any": (0, n), "stray": (-3, n + 3), "none": (-5, 0), "one": (n - 1, n)}[kind]
    return torch.randint(lo, hi, (T, k), device="cuda", generator=g).to(I32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,n,h,kind", [
    (1, 1, 1, 1, "any"), (1, 8, 256, 7168, "topk"), (3, 2, 5, 7, "stray"), (5, 32, 2048, 33, "any"),
    (17, 10, 672, 1000, "topk"), (64, 8, 256, 2049, "stray"), (9, 4, 8, 64, "none"),
    (33, 3, 4, 40, "one"),
    # either side of the one-launch sort and of a chunk of the large one
    (512, 8, 64, 24, "topk"), (4097, 1, 3, 9, "stray"), (2048, 3, 1, 8, "any"),
    (1000, 6, 2047, 16, "any"), (683, 9, 1280, 130, "topk"), (8193, 2, 2048, 5, "stray"),
    (4100, 4, 7, 11, "none"), (6000, 5, 6, 8, "one"),
])
def test_dispatch(T, k, n, h, kind, dtype):
    say(f"[gpu] dispatch T={T} k={k} n={n} h={h} {kind} {dtype}")
    g = gen(T * 31 + k)
    ids, x = ids_of(g, T, k, n, kind), normal(g, T, h, dtype=TYPES[dtype])
    Sorted(ids, n, x).check(ids, n, x)
    Sorted(ids, n).check(ids, n)   # the lists alone


def test_dispatch_takes_routing_of_the_layer():
    """deamoe_route's experts and its padded departments; the lists agree with its own."""
    cfg = W.PRESETS["tiny_f32"].layer.replace(top_k=4)
    T = 40
    c = D.make_config(cfg, T)
    w, x = W.make_weights(cfg, 3, device="cuda"), W.make_tokens(cfg, T, 3, device="cuda")
    rt = D.Routing.alloc(cfg, T)
    D.deamoe_route(c, x, w["router"], rt, D.alloc_workspace(c))
    t = rt.tensors
    for ids, n, offset, tokens in ((t["topk_ids"], cfg.n_experts, "exp_offset", "exp_tokens"),
                                   (t["tok_depts"], cfg.n_depts, "dept_offset", "dept_tokens")):
        s = Sorted(ids, n, x)
        s.check(ids, n, x)
        used = int(s.offset[-1])
        assert torch.equal(s.offset, t[offset])
        assert torch.equal(s.pair[:used] // 4, t[tokens][:used])


def test_dispatch_rows_past_four_gigabytes():
    T, k, n, h = 40000, 8, 64, 7168
    g = gen(1)
    ids, x = ids_of(g, T, k, n, "topk"), normal(g, T, h, dtype=BF)
    say(f"[gpu] dispatch of {T * k * h * 2 / 2**30:.1f} GiB")
    s = Sorted(ids, n, x)
    tok = s.pair.long() // k
    for lo in range(0, T * k, 40000):
        assert torch.equal(s.xs[lo:lo + 40000], x[tok[lo:lo + 40000]])
    w = torch.rand(T, k, device="cuda", generator=g)
    y = torch.empty_like(x)
    D.deamoe_combine(s.row, w, s.xs, y)
    # every row of a token is x itself
    want = x[-500:].double() * w[-500:].double().sum(1, keepdim=True)
    close(y[-500:], want, 9 * R.U * want.abs(), BF, "combine")


def test_dispatch_of_the_most_pairs():
    T, k, n = 1 << 23, 8, 64
    say(f"[gpu] dispatch of {T * k} pairs")
    g = gen(2)
    ids, x = ids_of(g, T, k, n, "any"), normal(g, T, 1, dtype=BF)
    s = Sorted(ids, n, x)
    key, pair = torch.sort(ids.flatten(), stable=True)
    assert torch.equal(s.pair, pair.to(I32))
    assert torch.equal(s.row.flatten()[pair], torch.arange(T * k, dtype=I32, device="cuda"))
    assert torch.equal(s.offset, torch.searchsorted(key, torch.arange(n + 1, dtype=I32, device="cuda")).to(I32))
    assert torch.equal(s.xs, x[pair // k])
    dx = torch.empty_like(x)
    D.deamoe_dispatch_backward(s.row, s.xs, dx)
    assert torch.equal(dx, 8 * x)   # eight times the same, exactly


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,k,n,h,kind", [
    (1, 1, 1, 1, "any"), (1, 10, 672, 1024, "topk"), (7, 32, 64, 7, "stray"), (61, 8, 256, 7168, "topk"),
    (64, 3, 8, 2055, "stray"), (5, 4, 4, 65536, "any"), (12, 9, 6, 513, "none"), (3000, 6, 64, 96, "stray"),
])
def test_combine_and_gradients(T, k, n, h, kind, dtype):
    say(f"[gpu] combine T={T} k={k} n={n} h={h} {kind} {dtype}")
    g, t = gen(T + k), TYPES[dtype]
    row = Sorted(ids_of(g, T, k, n, kind), n).row
    used = int((row >= 0).sum())
    w, ys, dy = torch.randn(T, k, device="cuda", generator=g), normal(g, T * k, h, dtype=t), normal(g, T, h, dtype=t)
    # what no pair has is never read
    w[row < 0] = float("nan")
    ys[used:] = float("nan")
    y, dx = torch.full_like(dy, 9.0), torch.full_like(dy, 9.0)
    D.deamoe_combine(row, w, ys, y)
    clean = torch.where(row < 0, torch.zeros_like(w), w)
    want, bound = R.combine(row, clean, ys.nan_to_num())
    close(y, want, bound, t, "y")
    D.deamoe_dispatch_backward(row, ys, dx)
    want, bound = R.combine(row, torch.ones_like(w), ys.nan_to_num())
    close(dx, want, bound, t, "dx")
    dys, dw = torch.full_like(ys, 5.0), torch.full_like(w, 5.0)
    D.deamoe_combine_backward(row, w, ys, dy, dys, dw)
    wdys, written, wdw, dw_bound = R.combine_backward(row, clean, ys.nan_to_num(), dy)
    close(dys[written], wdys[written], R.U * wdys[written].abs(), t, "dys")
    assert bool((dys[~written] == 5.0).all())
    close(dw, wdw, dw_bound, F32, "dw")
    # either alone gives the same bits
    only_dys, only_dw = torch.full_like(ys, 5.0), torch.full_like(w, 5.0)
    D.deamoe_combine_backward(row, w, None, dy, only_dys, None)
    D.deamoe_combine_backward(row, None, ys, dy, None, only_dw)
    assert same_bits(only_dys, dys) and same_bits(only_dw, dw)


def test_combine_keeps_infinities_to_their_token():
    g = gen(4)
    row = Sorted(ids_of(g, 6, 2, 4, "any"), 4).row
    ys, w = normal(g, 12, 40, dtype=BF), torch.rand(6, 2, device="cuda", generator=g) + 0.5
    ys[row[2, 1].long()] = float("inf")
    y = torch.empty(6, 40, dtype=BF, device="cuda")
    D.deamoe_combine(row, w, ys, y)
    assert bool(torch.isinf(y[2]).all()) and bool(torch.isfinite(y[[0, 1, 3, 4, 5]]).all())


# ------------------------------------------------------------ 4-bit products


def matrix(g, *lead, K, group, scale=F32):
    codes = torch.randint(0, 256, (*lead, K // 2), dtype=torch.uint8, device="cuda", generator=g)
    s = (torch.rand(*lead, K // group, device="cuda", generator=g) + 0.5) / K ** 0.5
    s[..., 0] *= -1.0   # scales of either sign
    return codes, s.to(scale)


@pytest.mark.parametrize("scale", [F32, BF])
@pytest.mark.parametrize("M,R_,K,group", [
    (1, 1, 32, 32), (1, 7168, 7168, 128), (2, 17, 96, 32), (15, 33, 64, 64), (16, 16, 128, 128),
    (17, 100, 320, 64), (33, 65, 2048, 128), (61, 2815, 2048, 64), (64, 130, 1408, 128),
    (65, 64, 4128, 32), (129, 257, 1152, 128), (300, 511, 640, 64), (1024, 384, 1536, 128),
])
def test_w4_linear(M, R_, K, group, scale):
    say(f"[gpu] w4_linear M={M} R={R_} K={K} group={group} {scale}")
    g = gen(M + R_)
    codes, s = matrix(g, R_, K=K, group=group, scale=scale)
    x, y = normal(g, M, K, dtype=BF), torch.full((M, R_), 9.0, dtype=BF, device="cuda")
    D.deamoe_w4_linear(x, codes, s, y)
    want, bound = R.w4_product(x, codes, s, group)
    close(y, want, bound, BF, "y")
    up, us = matrix(g, R_, K=K, group=group, scale=scale)
    D.deamoe_w4_swiglu(x, codes, s, up, us, y)
    want, bound = R.swiglu(want, bound, *R.w4_product(x, up, us, group))
    close(y, want, bound, BF, "swiglu")


@pytest.mark.parametrize("M", [1, 7, 40, 200])
def test_w4_every_weight_by_itself(M):
    """Rows of x with a single one pick single weights, exactly; so every column, row and scale is in
    its place, for every code."""
    g = gen(M)
    R_, K, group = 50, 384, 32
    codes, s = matrix(g, R_, K=K, group=group)
    w = R.w4_matrix(codes, s, group)
    for lo in range(0, K, M):
        cols = torch.arange(lo, lo + M, device="cuda") % K
        x = torch.zeros(M, K, dtype=BF, device="cuda")
        x[torch.arange(M, device="cuda"), cols] = 1.0
        y = torch.empty(M, R_, dtype=BF, device="cuda")
        D.deamoe_w4_linear(x, codes, s, y)
        assert torch.equal(y, w[:, cols].T.float().to(BF)), lo


@pytest.mark.parametrize("T,k,n,R_,K,group,kind", [
    (1, 8, 256, 64, 128, 128, "topk"), (4, 2, 16, 100, 256, 64, "stray"), (16, 8, 128, 1536, 1024, 128, "topk"),
    (61, 6, 64, 77, 320, 32, "any"), (300, 4, 8, 129, 256, 64, "topk"), (40, 4, 2048, 32, 64, 32, "any"),
    (700, 3, 5, 200, 512, 128, "one"), (50, 2, 9, 40, 64, 32, "none"),
])
def test_w4_experts(T, k, n, R_, K, group, kind):
    say(f"[gpu] w4 experts T={T} k={k} n={n} R={R_} K={K} {kind}")
    g = gen(T)
    offset = Sorted(ids_of(g, T, k, n, kind), n).offset
    (codes, s), (up, us) = (matrix(g, n, R_, K=K, group=group) for _ in range(2))
    x = normal(g, T * k, K, dtype=BF)
    y, z = (torch.full((T * k, R_), 9.0, dtype=BF, device="cuda") for _ in range(2))
    used = int(offset[-1])
    x[used:] = float("nan")   # rows of no expert
    D.deamoe_w4_linear(x, codes, s, y, offset=offset)
    D.deamoe_w4_swiglu(x, codes, s, up, us, z, offset=offset)
    assert bool((y[used:] == 9.0).all()) and bool((z[used:] == 9.0).all())
    o = offset.tolist()
    for e in range(n):
        if o[e] < o[e + 1]:
            at = slice(o[e], o[e + 1])
            want, bound = R.w4_product(x[at], codes[e], s[e], group)
            close(y[at], want, bound, BF, f"expert {e}")
            want, bound = R.swiglu(want, bound, *R.w4_product(x[at], up[e], us[e], group))
            close(z[at], want, bound, BF, f"swiglu of expert {e}")


@pytest.mark.parametrize("scale", [F32, BF])
@pytest.mark.parametrize("M,R_,K,group", [
    (2048, 2050, 1152, 128), (1100, 4000, 320, 64), (1030, 4097, 2080, 32),   # 64-row tiles
    (160, 700, 2112, 64), (161, 1500, 4128, 32), (250, 2100, 1152, 128),      # one and two token tiles
    (16, 8300, 1056, 32), (12, 10000, 192, 64), (9, 12001, 4224, 128),        # K over four, two waves, one
    (16, 700, 7200, 32), (9, 300, 4288, 64), (30, 500, 7296, 128), (3, 260, 16544, 32), (5, 33, 9088, 64),   # wide panels
])
def test_w4_linear_by_kernel(M, R_, K, group, scale):
    """Sizes on either side of what chooses the kernel and its split, with a K that ends inside a step
    and, for small groups, more scales than stand in LDS at once."""
    say(f"[gpu] w4 choice M={M} R={R_} K={K} group={group} {scale}")
    test_w4_linear(M, R_, K, group, scale)


def sampled_experts(offset, M, n, R_, K, group, g, scale=F32, mats=2):
    """One call over given offsets, checked on the rows around every few matrices' ends."""
    mat = [matrix(g, n, R_, K=K, group=group, scale=scale) for _ in range(mats)]
    x, y = normal(g, M, K, dtype=BF), torch.full((M, R_), 9.0, dtype=BF, device="cuda")
    if mats == 2:
        D.deamoe_w4_swiglu(x, *mat[0], *mat[1], y, offset=offset)
    else:
        D.deamoe_w4_linear(x, *mat[0], y, offset=offset)
    o = offset.tolist()
    assert bool((y[o[-1]:] == 9.0).all()) and bool((y[:o[0]] == 9.0).all())
    held = [e for e in range(n) if o[e] < o[e + 1]]
    for e in sorted({held[0], held[-1], *held[::max(len(held) // 6, 1)]}):
        rows = torch.unique(torch.cat([torch.arange(o[e], min(o[e] + 40, o[e + 1])),
                                       torch.arange(max(o[e + 1] - 40, o[e]), o[e + 1])])).cuda()
        want, bound = R.w4_product(x[rows], mat[0][0][e], mat[0][1][e], group)
        if mats == 2:
            want, bound = R.swiglu(want, bound, *R.w4_product(x[rows], mat[1][0][e], mat[1][1][e], group))
        close(y[rows], want, bound, BF, f"matrix {e}")


@pytest.mark.parametrize("scale", [F32, BF])
@pytest.mark.parametrize("mats", [1, 2])
@pytest.mark.parametrize("T,k,n,R_,K,group,kind", [
    (60, 5, 64, 4100, 160, 32, "topk"), (60, 5, 64, 4100, 1152, 128, "topk"), (60, 5, 64, 4100, 320, 64, "stray"),
    (20, 2, 4, 70, 2144, 32, "any"),                                      # few workgroups
    (900, 4, 2047, 65, 1056, 32, "any"), (4000, 8, 100, 260, 2080, 32, "topk"),
    (2000, 2, 64, 130, 192, 64, "stray"), (500, 2, 16, 300, 4224, 128, "any"), (1300, 1, 1, 100, 128, 64, "any"),
])
def test_w4_experts_by_kernel(T, k, n, R_, K, group, kind, mats, scale):
    say(f"[gpu] w4 experts choice T={T} k={k} n={n} R={R_} K={K} group={group} {kind} {mats} {scale}")
    g = gen(T + n)
    offset = Sorted(ids_of(g, T, k, n, kind), n).offset
    sampled_experts(offset, T * k, n, R_, K, group, g, scale, mats)


def test_w4_uneven_experts():
    """Routing that the mean number of rows says nothing about: one matrix with nearly all rows, and
    rows before the first matrix and behind the last."""
    g = gen(3)
    for n, M, mats in ((200, 2500, 2), (200, 2500, 1), (6, 2500, 2)):
        o = torch.full((n + 1,), 2400, dtype=I32, device="cuda")
        o[:4] = torch.tensor([5, 5, 6, 23], dtype=I32)
        o[-2:] = torch.tensor([2400, 2431], dtype=I32)
        say(f"[gpu] w4 uneven n={n} M={M} {mats}")
        sampled_experts(o, M, n, 150, 256, 64, g, mats=mats)


def test_w4_more_items_than_workgroups():
    """Grids end at 2^20 workgroups, which walk over the rest."""
    g = gen(5)
    n, M, R_, K = 2048, 3000, 65536, 32
    say(f"[gpu] w4 swiglu of {n} x {R_} x {K}")
    offset = Sorted(ids_of(g, M, 1, n, "any"), n).offset
    sampled_experts(offset, M, n, R_, K, 32, g)


def test_w4_rows_past_four_gigabytes():
    g, n, M, K = gen(6), 3, 1 << 26, 64
    say(f"[gpu] w4 of {M * K * 2 / 2**30:.0f} GiB of rows")
    codes, s = matrix(g, n, 1, K=K, group=32)
    x = normal(g, 1 << 16, K, dtype=BF).repeat(M >> 16, 1)
    offset = torch.tensor([0, 33, (1 << 25) + 7, M], dtype=I32, device="cuda")
    y = torch.empty(M, 1, dtype=BF, device="cuda")
    D.deamoe_w4_linear(x, codes, s, y, offset=offset)
    for e, (lo, hi) in enumerate(((0, 33), (33, (1 << 25) + 7), ((1 << 25) + 7, M))):
        for at in (slice(lo, min(lo + 100, hi)), slice(max(hi - 100, lo), hi)):
            want, bound = R.w4_product(x[at], codes[e], s[e], 32)
            close(y[at], want, bound, BF, f"matrix {e}")


def test_w4_offsets_outside_the_rows():
    """Offsets past the rows are taken as their end, rows before the first stay as they were."""
    g = gen(8)
    codes, s = matrix(g, 3, 20, K=64, group=32)
    x, y = normal(g, 10, 64, dtype=BF), torch.full((10, 20), 9.0, dtype=BF, device="cuda")
    offset = torch.tensor([2, 5, 5, 99], dtype=I32, device="cuda")
    D.deamoe_w4_linear(x, codes, s, y, offset=offset)
    assert bool((y[:2] == 9.0).all())
    for lo, hi, e in ((2, 5, 0), (5, 10, 2)):
        want, bound = R.w4_product(x[lo:hi], codes[e], s[e], 32)
        close(y[lo:hi], want, bound, BF, "y")
    D.deamoe_w4_linear(x, codes, s, y, offset=torch.tensor([-4, -1, 0, 10], dtype=I32, device="cuda"))
    want, bound = R.w4_product(x, codes[2], s[2], 32)
    close(y, want, bound, BF, "y")


@pytest.mark.parametrize("M", [3, 20, 150])
def test_w4_keeps_bad_rows_to_themselves(M):
    g = gen(M)
    codes, s = matrix(g, 40, K=256, group=64)
    x, y, clean = normal(g, M, 256, dtype=BF), *(torch.empty(M, 40, dtype=BF, device="cuda") for _ in range(2))
    D.deamoe_w4_linear(x, codes, s, clean)
    x[1, 3], x[2, 255] = float("inf"), float("nan")
    D.deamoe_w4_linear(x, codes, s, y)
    assert bool(torch.isnan(y[1:3]).all())
    rest = torch.arange(M, device="cuda") % M != 1
    rest[2] = False
    assert same_bits(y[rest], clean[rest])


# -------------------------------------------------------------------- norms

EPS = 1e-6
NORM_SHAPES = [(1, 1), (3, 7), (16, 7168), (5, 64), (130, 1000), (64, 4096), (33, 2047), (9, 8200),
               (6, 16384), (3, 16392), (2, 65536), (1500, 256), (1100, 129)]
# several rows per workgroup for every split of a row over threads
LONG_SHAPES = [(70001, 24), (2100, 1030), (1030, 2050), (600, 5001), (520, 9000), (515, 17001)]
STAT = 60 * R.U   # r: a chain of at most 64 squares per thread and 10 joins, halved by the root; few roundings more


def norm_bounds(v, w):
    """Bound of v^ * w before its rounding."""
    return (STAT + 3 * R.U) * (v * w).abs()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,h", NORM_SHAPES)
def test_prenorm_and_gradient(T, h, dtype):
    say(f"[gpu] prenorm T={T} h={h} {dtype}")
    g, t = gen(T + h), TYPES[dtype]
    x, w, du, dres = normal(g, T, h, dtype=t), normal(g, h, dtype=t), normal(g, T, h, dtype=t), normal(g, T, h, dtype=t)
    x[T // 2] = 0   # a row of zeros
    u = torch.full_like(x, 9.0)
    D.deamoe_prenorm(x, w, u, eps=EPS)
    hat = R.rms(x.double(), EPS)
    close(u, hat * w.double(), norm_bounds(hat, w.double()), t, "u")
    rows = torch.arange(T, device="cuda") != T // 2
    for res in (None, dres):
        dx, dw = torch.full_like(x, 9.0), torch.full((h,), 9.0, device="cuda")
        D.deamoe_prenorm_backward(x, w, du, dx, dw, dres=res, eps=EPS)
        wx, ww = R.grads(lambda x, w: (R.rms(x, EPS) * w,), (x, w), (du,))
        r = 1 / torch.sqrt(x.double().pow(2).mean(-1, keepdim=True) + EPS)
        q = (du.double() * w.double()).abs()
        bound = 2 * STAT * r * (q + hat.abs() * (q * hat.abs()).mean(-1, keepdim=True))
        if res is not None:
            wx, bound = wx + res.double(), bound + R.U * (res.double().abs() + wx.abs())
        close(dx, wx, bound, t, "dx")
        terms = (du.double() * hat).abs().sum(0)
        close(dw, ww, (T / 100 + 300) * R.U * terms, F32, "dw")
    # in place: dres is dx, u is x
    D.deamoe_prenorm_backward(x, w, du, dres, dw, dres=dres, eps=EPS)
    assert same_bits(dres, dx)
    D.deamoe_prenorm(x, w, x, eps=EPS)
    assert same_bits(x, u) and bool((u[~rows] == 0).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("gate", ["none", "shared", "full"])
@pytest.mark.parametrize("following", [False, True])
@pytest.mark.parametrize("T,h", NORM_SHAPES)
def test_postnorm_and_gradient(T, h, following, gate, dtype):
    say(f"[gpu] postnorm T={T} h={h} {gate} {following} {dtype}")
    g, t, a = gen(T * 3 + h), TYPES[dtype], 0.5
    x, y, dz, du = (normal(g, T, h, dtype=t) for _ in range(4))
    w, wn = normal(g, h, dtype=t), normal(g, h, dtype=t)
    gt = {"none": None, "shared": normal(g, h, dtype=t), "full": normal(g, T, h, dtype=t)}[gate]
    y[0] = 0
    z, u = torch.full_like(x, 9.0), torch.full_like(x, 9.0) if following else None
    D.deamoe_postnorm(x, y, w, z, gate=gt, res_scale=a, w_next=wn if following else None, u=u, eps=EPS)
    gd = torch.ones((), dtype=torch.float64, device="cuda") if gt is None else gt.double()
    n = gd * (R.rms(y.double(), EPS) * w.double())
    close(z, a * x.double() + n, STAT * n.abs() + 5 * R.U * (n.abs() + (a * x.double()).abs()), t, "z")
    if following:
        again = torch.empty_like(u)
        D.deamoe_prenorm(z, wn, again, eps=EPS)
        assert same_bits(again, u)

    dx, dy, dw = torch.full_like(x, 9.0), torch.full_like(x, 9.0), torch.full((h,), 9.0, device="cuda")
    dgate = None if gt is None else torch.full_like(gt, 9.0, dtype=F32 if gate == "shared" else t)
    dwn = torch.full((h,), 9.0, device="cuda") if following else None
    kw = dict(gate=gt, dgate=dgate, res_scale=a, eps=EPS)
    if following:
        kw |= dict(z=z, w_next=wn, du=du, dw_next=dwn)
    D.deamoe_postnorm_backward(y, w, dz, dx, dy, dw, **kw)
    d, size = dz.double(), dz.double().abs()   # the gradient that reaches z, and a bound of its parts
    if following:
        more, wwn = R.grads(lambda z, w: (R.rms(z, EPS) * w,), (z, wn), (du,))
        zhat = R.rms(z.double(), EPS)
        r = 1 / torch.sqrt(z.double().pow(2).mean(-1, keepdim=True) + EPS)
        q = (du.double() * wn.double()).abs()
        d, size = d + more, size + r * (q + zhat.abs() * (q * zhat.abs()).mean(-1, keepdim=True))
        close(dwn, wwn, (T / 100 + 300) * R.U * (du.double() * zhat).abs().sum(0), F32, "dw_next")
    close(dx, a * d, 2 * STAT * a * size, t, "dx")
    ins = (y, w) if gt is None else (y, w, gt)
    want = R.grads(lambda y, w, g=1.0: (g * (R.rms(y, EPS) * w),), ins, (d,))
    yhat = R.rms(y.double(), EPS)
    ry = 1 / torch.sqrt(y.double().pow(2).mean(-1, keepdim=True) + EPS)
    q = size * gd.abs() * w.double().abs()
    close(dy, want[0], 4 * STAT * ry * (q + yhat.abs() * (q * yhat.abs()).mean(-1, keepdim=True)), t, "dy")
    long = (T / 100 + 400) * R.U
    close(dw, want[1], long * (size * gd.abs() * yhat.abs()).sum(0), F32, "dw")
    if gate == "shared":
        close(dgate, want[2], long * (size * (yhat * w.double()).abs()).sum(0), F32, "dgate")
    elif gate == "full":
        close(dgate, want[2], 4 * STAT * size * (yhat * w.double()).abs(), t, "dgate")
    # in place: dx is dz, z is x
    dz2 = dz.clone()
    D.deamoe_postnorm_backward(y, w, dz2, dz2, dy, dw, **kw)
    assert same_bits(dz2, dx)
    D.deamoe_postnorm(x, y, w, x, gate=gt, res_scale=a, eps=EPS)
    assert same_bits(x, z)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,h", LONG_SHAPES)
def test_norms_of_many_rows(T, h, dtype):
    test_prenorm_and_gradient(T, h, dtype)
    for gate, following in (("shared", True), ("full", False)):
        test_postnorm_and_gradient(T, h, following, gate, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T,h", [(7, 129), (3, 7168), (2, 16392), (2, 65536)])
def test_postnorm_in_place_with_the_next_norm(T, h, dtype):
    g, t = gen(h), TYPES[dtype]
    x, y, gate = (normal(g, T, h, dtype=t) for _ in range(3))
    w, wn = normal(g, h, dtype=t), normal(g, h, dtype=t)
    z, u, v = (torch.empty_like(x) for _ in range(3))
    D.deamoe_postnorm(x, y, w, z, gate=gate, w_next=wn, u=u)
    D.deamoe_postnorm(x, y, w, x, gate=gate, w_next=wn, u=v)
    assert same_bits(x, z) and same_bits(u, v)


def test_sums_over_no_tokens_are_zero():
    def full(*s, dtype=F32):
        return torch.full(s, 9.0, dtype=dtype, device="cuda")
    e, dw, dwn, dg = torch.empty(0, 40, device="cuda"), full(40), full(40), full(40)
    D.deamoe_prenorm_backward(e, full(40), e, e, dw)
    assert bool((dw == 0).all())
    dw = full(40)
    D.deamoe_postnorm_backward(e, full(40), e, e, e, dw, gate=full(40), dgate=dg, z=e, w_next=full(40), du=e,
                               dw_next=dwn)
    assert all(bool((t == 0).all()) for t in (dw, dwn, dg))
    offset = torch.full((6,), 9, dtype=I32, device="cuda")
    none = torch.empty(0, 3, dtype=I32, device="cuda")
    D.deamoe_dispatch(none, e, offset, none.flatten(), none, e)
    assert bool((offset == 0).all())
    D.deamoe_combine(none, torch.empty(0, 3, device="cuda"), e, e)
    x0 = torch.empty(0, 64, dtype=BF, device="cuda")
    codes, s = matrix(gen(0), 5, K=64, group=32)
    D.deamoe_w4_linear(x0, codes, s, torch.empty(0, 5, dtype=BF, device="cuda"))
    u0 = torch.empty(0, 40, device="cuda")
    D.deamoe_prenorm(u0, full(40), u0)


# ----------------------------------------------------- together, streams, graphs


def experts(g, n, h, d, group=32):
    gate, up = (matrix(g, n, d, K=h, group=group) for _ in range(2))
    return D.W4Experts(gate, up, matrix(g, n, h, K=d, group=group))


def experts_reference(ex, x, ids, w):
    """Expert by expert in 64 bits, with the roundings of the activation between (bf16) as a bound."""
    y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
    bound = torch.zeros_like(y)
    for e in range(ex.n):
        t, slot = (ids == e).nonzero(as_tuple=True)
        if not len(t):
            continue
        grp = ex.h // ex.gate[1].shape[-1]
        a, ea = R.swiglu(*R.w4_product(x[t], ex.gate[0][e], ex.gate[1][e], grp),
                         *R.w4_product(x[t], ex.up[0][e], ex.up[1][e], grp))
        ea = ea + R.half_step(BF) * a.abs()
        grp = ex.d // ex.down[1].shape[-1]
        m = R.w4_matrix(ex.down[0][e], ex.down[1][e], grp)
        o, eo = a @ m.T, R.w4_product(a, ex.down[0][e], ex.down[1][e], grp)[1] + ea @ m.abs().T
        eo = eo + R.half_step(BF) * (o.abs() + eo)
        p = w[t, slot].double()[:, None]
        y.index_add_(0, t, p * o)
        bound.index_add_(0, t, (p * eo).abs() + 2 * ids.shape[1] * R.U * (p * o).abs())
    return y, bound


@pytest.mark.parametrize("T", [1, 16, 200, 700])
def test_experts_together(T):
    """The operators as they are used: sorted tokens through 4-bit experts and back."""
    g = gen(T)
    ex = experts(g, 12, 256, 160)
    x, ids = normal(g, T, 256, dtype=BF), ids_of(g, T, 3, 12, "topk")
    w = torch.rand(T, 3, device="cuda", generator=g)
    if T > 1:
        ids[-T // 4:] = -1   # a padded batch
    y = ex(x, ids, w)
    want, bound = experts_reference(ex, x, ids, w)
    close(y, want, bound, BF, "y")
    if T > 1:
        assert bool((y[-T // 4:] == 0).all())


def test_experts_follow_the_layers_router():
    """A decode step: deamoe_route's experts and weights through 4-bit experts."""
    cfg = W.PRESETS["tiny_f32"].layer.replace(w_dtype="bf16", act_dtype="bf16", d_private=128)
    T, c = 7, D.make_config(W.PRESETS["tiny_f32"].layer.replace(w_dtype="bf16", act_dtype="bf16", d_private=128), 8)
    w, x = W.make_weights(cfg, 5, device="cuda"), W.make_tokens(cfg, T, 5, device="cuda")
    rt = D.Routing.alloc(cfg, T)
    D.deamoe_route(c, x, w["router"], rt, D.alloc_workspace(c))
    ex = experts(gen(5), cfg.n_experts, cfg.hidden, 96)
    ids, p = rt.tensors["topk_ids"], rt.tensors["topk_w"]
    want, bound = experts_reference(ex, x, ids, p)
    close(ex(x, ids, p), want, bound, BF, "y")


def test_block_around_a_layer():
    """Two blocks of the layer between their norms, the second taking the first's next norm."""
    cfg = W.PRESETS["tiny_f32"].layer
    T, h, g = 4, cfg.hidden, gen(2)
    layer = D.Layer(cfg, W.make_weights(cfg, 2, device="cuda"), T)
    x = normal(g, T, h)
    w1, w2, w3, gate = (normal(g, h) for _ in range(4))
    one = D.Block(layer, w1, w2, gate=gate, res_scale=0.5, w_next=w3)
    two = D.Block(layer, w3, w2)
    z, u = one(x)
    out = two(z, u)
    assert same_bits(out, two(z))   # the passed norm is the one it would make
    a = torch.empty_like(x)
    D.deamoe_prenorm(x, w1, a)
    want = 0.5 * x.double() + gate.double() * (R.rms(layer(a).double(), EPS) * w2.double())
    close(z, want, 2 * STAT * (want.abs() + (0.5 * x.double()).abs() * 2 + 1e-30), F32, "z")


def test_experts_and_blocks_on_a_given_stream():
    """Everything that the classes launch runs on the stream given, and no token at all is a batch."""
    g, s = gen(11), torch.cuda.Stream()
    ex = experts(g, 12, 256, 160)
    T = 400
    x, ids, w = normal(g, T, 256, dtype=BF), ids_of(g, T, 3, 12, "topk"), torch.rand(T, 3, device="cuda", generator=g)
    block = D.Block(lambda u, stream=None: ex(u, ids, w, stream=stream), *(normal(g, 256, dtype=BF) for _ in range(2)))
    want, zwant = ex(x, ids, w), block(x)
    late, y = torch.empty_like(x), torch.empty_like(x)
    big = torch.randn(4096, 4096, device="cuda")
    torch.cuda.synchronize()
    for _ in range(3):
        late.zero_()
        torch.cuda.synchronize()
        with torch.cuda.stream(s):
            for _ in range(5):
                big @ big            # x arrives late on this stream
            late.copy_(x)
        got = ex(late, ids, w, y=y, stream=s)
        z = block(late, stream=s)
        s.synchronize()
        assert got is y and same_bits(got, want) and same_bits(z, zwant)
    assert ex(x[:0], ids[:0], w[:0]).shape == (0, 256)


def test_streams_and_repeats():
    """Two calls at once on streams of their own, and again: the same bits every time."""
    g = gen(6)
    T, k, n, h = 3000, 4, 64, 512
    sets = [(ids_of(g, T, k, n, "stray"), normal(g, T, h, dtype=BF)) for _ in range(2)]
    first = [Sorted(ids, n, x) for ids, x in sets]
    du, w = normal(g, T, h, dtype=BF), normal(g, h, dtype=BF)

    def grads_of(x, stream=None):
        dx, dw = torch.empty_like(x), torch.empty(h, device="cuda")
        D.deamoe_prenorm_backward(x, w, du, dx, dw, stream=stream)
        return dx, dw
    norms = [grads_of(x) for _, x in sets]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in sets]
    for _ in range(3):
        more = [grads_of(x, s) for (_, x), s in zip(sets, streams)]
        again = [Sorted(ids, n, x, stream=s) for (ids, x), s in zip(sets, streams)]
        torch.cuda.synchronize()
        for a, b in zip(first, again):
            assert all(same_bits(getattr(a, f), getattr(b, f)) for f in ("offset", "pair", "row"))
        for a, b in zip(norms, more):
            assert all(same_bits(p, q) for p, q in zip(a, b))


@pytest.mark.parametrize("T", [8, 1500])
def test_captured_and_replayed(T):
    """The experts, the norms and the gradients in one graph, replayed on new inputs with eager
    work between the replays."""
    g = gen(T)
    k, n, h, d = 3, 10, 256, 96
    ex = experts(g, n, h, d)
    x, ids, w = normal(g, T, h, dtype=BF), ids_of(g, T, k, n, "stray"), torch.rand(T, k, device="cuda", generator=g)
    wp, wq, gate = (normal(g, h, dtype=BF) for _ in range(3))

    def step(x, ids, w):
        u, z, v = (torch.empty_like(x) for _ in range(3))
        D.deamoe_prenorm(x, wp, u)
        y = ex(u, ids, w)
        D.deamoe_postnorm(x, y, wq, z, gate=gate, w_next=wp, u=v)
        dx, dy, dw, dg, dwn = torch.empty_like(x), torch.empty_like(x), *(torch.empty(h, device="cuda") for _ in range(3))
        D.deamoe_postnorm_backward(y, wq, z, dx, dy, dw, gate=gate, dgate=dg, z=z, w_next=wp, du=v, dw_next=dwn)
        offset, pair = torch.empty(n + 1, dtype=I32, device="cuda"), torch.empty(T * k, dtype=I32, device="cuda")
        row, ys = torch.empty(T, k, dtype=I32, device="cuda"), torch.zeros(T * k, h, dtype=BF, device="cuda")
        D.deamoe_dispatch(ids, x, offset, pair, row, ys)
        dys, dwt = torch.zeros_like(ys), torch.empty_like(w)
        D.deamoe_combine_backward(row, w, ys, dy, dys, dwt)
        return y, z, v, dx, dy, dw, dg, dwn, dys, dwt

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step(x, ids, w)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = step(x, ids, w)
    for i in range(4):
        x.copy_(normal(g, T, h, dtype=BF))
        ids.copy_(ids_of(g, T, k, n, "stray"))
        want = [t.clone() for t in step(x, ids, w)]
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        for a, b in zip(out, want):
            assert same_bits(a, b), i
