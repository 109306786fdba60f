"""The operators beside the layer on the host: what they refuse, before any launch, and what they
do for empty batches.  No call here reaches a kernel launch, so the tests run without a GPU."""
import ctypes as C
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2608_14385_amd import deamoe as D  # noqa: E402

FAKE = 0x7f0000000000   # never dereferenced: validation rejects first
BIG = 1 << 40


@pytest.fixture(scope="module", autouse=True)
def built():
    if not os.path.exists(D.LIB_PATH):
        from paper_2608_14385_amd import build
        build.build()


def dispatch(T=4, k=2, n=8, h=64, act=D.BF16, ids=FAKE, x=FAKE, offset=FAKE, pair=FAKE, row=FAKE,
             xs=FAKE, ws=FAKE, ws_bytes=BIG):
    return D.lib().deamoe_dispatch(T, k, n, h, act, ids, x, offset, pair, row, xs, ws, ws_bytes, None)


@pytest.mark.parametrize("kw,expect", [
    (dict(T=-1), D.ERR_INVALID), (dict(k=0), D.ERR_INVALID), (dict(k=33), D.ERR_UNSUPPORTED),
    (dict(n=0), D.ERR_INVALID), (dict(n=2049), D.ERR_UNSUPPORTED), (dict(h=0), D.ERR_INVALID),
    (dict(h=65537), D.ERR_UNSUPPORTED), (dict(act=2), D.ERR_INVALID),
    (dict(T=(1 << 23) + 1), D.ERR_UNSUPPORTED), (dict(T=1 << 22, k=17), D.ERR_UNSUPPORTED),
    (dict(ids=None), D.ERR_INVALID), (dict(ids=FAKE + 2), D.ERR_INVALID), (dict(x=None), D.ERR_INVALID),
    (dict(x=FAKE + 1), D.ERR_INVALID), (dict(x=FAKE + 2, act=D.F32), D.ERR_INVALID),
    (dict(offset=None), D.ERR_INVALID), (dict(T=0, offset=None), D.ERR_INVALID),
    (dict(pair=None), D.ERR_INVALID), (dict(row=None), D.ERR_INVALID),
    # only sorts of more than 4096 pairs take a workspace
    (dict(T=4096, ws=None), D.ERR_WORKSPACE), (dict(T=4096, ws_bytes=16), D.ERR_WORKSPACE),
    (dict(T=4096, ws=FAKE + 4), D.ERR_WORKSPACE),
])
def test_dispatch_refusals(kw, expect):
    assert dispatch(**kw) == expect


def test_dispatch_workspace():
    assert D.deamoe_dispatch_workspace_bytes(0, 8, 256) == 0
    small, large = (D.deamoe_dispatch_workspace_bytes(T, 8, 256) for T in (512, 8192))
    assert small == 0 and 256 * 4 < large < 1 << 20
    for bad in ((-1, 8, 4), (4, 0, 4), (4, 8, 0)):
        with pytest.raises(D.DeamoeError) as e:
            D.deamoe_dispatch_workspace_bytes(*bad)
        assert e.value.status == D.ERR_INVALID
    assert D.lib().deamoe_dispatch_workspace_bytes(4, 2, 8, None) == D.ERR_INVALID


def test_combine_refusals():
    L = D.lib()

    def back(T=4, k=2, h=8, act=D.BF16, row=FAKE, dxs=FAKE, dx=FAKE):
        return L.deamoe_dispatch_backward(T, k, h, act, row, dxs, dx, None)

    def comb(T=4, k=2, h=8, act=D.BF16, row=FAKE, w=FAKE, ys=FAKE, y=FAKE):
        return L.deamoe_combine(T, k, h, act, row, w, ys, y, None)

    def comb_back(T=4, k=2, h=8, act=D.BF16, row=FAKE, w=FAKE, ys=FAKE, dy=FAKE, dys=FAKE, dw=FAKE):
        return L.deamoe_combine_backward(T, k, h, act, row, w, ys, dy, dys, dw, None)

    for f in (back, comb, comb_back):
        for kw in (dict(T=-1), dict(k=0), dict(h=0), dict(act=7), dict(row=None), dict(row=FAKE + 1)):
            assert f(**kw) == D.ERR_INVALID, (f, kw)
        for kw in (dict(k=33), dict(h=1 << 17), dict(T=1 << 24), dict(T=1 << 23, k=16)):
            assert f(**kw) == D.ERR_UNSUPPORTED, (f, kw)
        assert f(T=0, row=None) == D.OK
    for kw in (dict(dxs=None), dict(dx=None), dict(dx=FAKE + 1), dict(dx=FAKE + 2, act=D.F32)):
        assert back(**kw) == D.ERR_INVALID
    for kw in (dict(w=None), dict(ys=None), dict(y=None), dict(w=FAKE + 2), dict(y=FAKE + 1)):
        assert comb(**kw) == D.ERR_INVALID
    for kw in (dict(w=None), dict(ys=None), dict(dy=None), dict(dys=FAKE + 1), dict(dw=FAKE + 2)):
        assert comb_back(**kw) == D.ERR_INVALID
    assert comb_back(dys=None, dw=None, w=None, ys=None) == D.OK   # nothing asked for


def w4cfg(**kw):
    return D.deamoe_w4_config(**(dict(R=64, K=256, n=4, group=64, scale_dtype=D.F32) | kw))


@pytest.mark.parametrize("kw,expect", [
    (dict(R=0), D.ERR_INVALID), (dict(K=0), D.ERR_INVALID), (dict(n=0), D.ERR_INVALID),
    (dict(group=16), D.ERR_INVALID), (dict(group=256), D.ERR_INVALID), (dict(K=96), D.ERR_INVALID),
    (dict(K=96, group=32, n=2049), D.ERR_UNSUPPORTED), (dict(scale_dtype=2), D.ERR_INVALID),
    (dict(K=65536 + 128), D.ERR_UNSUPPORTED), (dict(R=65537), D.ERR_UNSUPPORTED),
])
def test_w4_config_refusals(kw, expect):
    L, c = D.lib(), w4cfg(**kw)
    for M in (0, 4):
        assert L.deamoe_w4_linear(C.byref(c), M, FAKE, FAKE, FAKE, FAKE, FAKE, None) == expect
        assert L.deamoe_w4_swiglu(C.byref(c), M, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, FAKE, None) == expect


def test_w4_refusals():
    L, c = D.lib(), w4cfg()

    def lin(c=c, M=4, x=FAKE, offset=FAKE, codes=FAKE, scale=FAKE, y=FAKE):
        return L.deamoe_w4_linear(C.byref(c), M, x, offset, codes, scale, y, None)

    def swi(c=c, M=4, x=FAKE, offset=FAKE, gc=FAKE, gs=FAKE, uc=FAKE, us=FAKE, y=FAKE):
        return L.deamoe_w4_swiglu(C.byref(c), M, x, offset, gc, gs, uc, us, y, None)

    for f in (lin, swi):
        for kw in (dict(M=-1), dict(x=None), dict(x=FAKE + 8), dict(y=None), dict(y=FAKE + 1),
                   dict(offset=None), dict(offset=FAKE + 2)):
            assert f(**kw) == D.ERR_INVALID, kw
        assert f(M=(1 << 26) + 1) == D.ERR_UNSUPPORTED
        assert f(M=0, x=None, offset=None) == D.OK
    for kw in (dict(codes=None), dict(codes=FAKE + 8), dict(scale=None), dict(scale=FAKE + 2)):
        assert lin(**kw) == D.ERR_INVALID
    for kw in (dict(gc=None), dict(uc=FAKE + 4), dict(gs=None), dict(us=None), dict(us=FAKE + 2)):
        assert swi(**kw) == D.ERR_INVALID
    assert L.deamoe_w4_linear(None, 4, FAKE, None, FAKE, FAKE, FAKE, None) == D.ERR_INVALID


def test_norm_refusals():
    L = D.lib()

    def pre(T=4, h=8, act=D.BF16, eps=1e-6, x=FAKE, w=FAKE, u=FAKE):
        return L.deamoe_prenorm(T, h, act, eps, x, w, u, None)

    def pre_back(T=4, h=8, act=D.BF16, eps=1e-6, x=FAKE, w=FAKE, du=FAKE, dres=None, dx=FAKE, dw=FAKE,
                 ws=FAKE, ws_bytes=BIG):
        return L.deamoe_prenorm_backward(T, h, act, eps, x, w, du, dres, dx, dw, ws, ws_bytes, None)

    def post(T=4, h=8, act=D.BF16, eps=1e-6, a=1.0, mode=0, x=FAKE, y=FAKE, w=FAKE, gate=None,
             w_next=None, z=FAKE, u=None):
        return L.deamoe_postnorm(T, h, act, eps, a, mode, x, y, w, gate, w_next, z, u, None)

    def post_back(T=4, h=8, act=D.BF16, eps=1e-6, a=1.0, mode=0, y=FAKE, w=FAKE, gate=None, z=None,
                  w_next=None, dz=FAKE, du=None, dx=FAKE, dy=FAKE, dw=FAKE, dgate=None, dw_next=None,
                  ws=FAKE, ws_bytes=BIG):
        return L.deamoe_postnorm_backward(T, h, act, eps, a, mode, y, w, gate, z, w_next, dz, du, dx, dy,
                                          dw, dgate, dw_next, ws, ws_bytes, None)

    for f in (pre, pre_back, post, post_back):
        for kw in (dict(T=-1), dict(h=0), dict(act=2), dict(eps=0.0), dict(eps=-1.0),
                   dict(eps=float("nan")), dict(eps=float("inf")), dict(w=None), dict(w=FAKE + 1),
                   dict(w=FAKE + 2, act=D.F32)):
            assert f(**kw) == D.ERR_INVALID, (f, kw)
        for kw in (dict(T=1 << 24), dict(h=65537)):
            assert f(**kw) == D.ERR_UNSUPPORTED, (f, kw)
    assert pre(T=0, x=None, w=None, u=None) == D.OK
    assert post(T=0, x=None, y=None, w=None, z=None) == D.OK
    for f in (post, post_back):
        for kw in (dict(a=float("nan")), dict(a=float("inf")), dict(mode=3), dict(mode=-1), dict(mode=1),
                   dict(mode=2), dict(gate=FAKE), dict(w_next=FAKE), dict(y=None)):
            assert f(**kw) == D.ERR_INVALID, (f, kw)
    for kw in (dict(x=None), dict(u=None)):
        assert pre(**kw) == D.ERR_INVALID
    for kw in (dict(u=FAKE), dict(z=None), dict(x=None)):
        assert post(**kw) == D.ERR_INVALID
    for kw in (dict(du=None), dict(x=None), dict(dx=None), dict(dw=None), dict(dres=FAKE + 1),
               dict(T=0, dw=None)):
        assert pre_back(**kw) == D.ERR_INVALID
    for kw in (dict(dz=None), dict(dx=None), dict(dy=None), dict(dw=None), dict(du=FAKE), dict(z=FAKE),
               dict(dw_next=FAKE), dict(dgate=FAKE), dict(mode=1, gate=FAKE), dict(mode=2, gate=FAKE),
               dict(du=FAKE, z=FAKE, w_next=FAKE), dict(T=0, dw=None), dict(T=0, mode=1, gate=FAKE)):
        assert post_back(**kw) == D.ERR_INVALID, kw
    for f in (pre_back, post_back):
        for kw in (dict(ws=None), dict(ws_bytes=16), dict(ws=FAKE + 4)):
            assert f(**kw) == D.ERR_WORKSPACE, (f, kw)
    assert D.deamoe_norm_workspace_bytes(4, 8) > 0
    assert L.deamoe_norm_workspace_bytes(-1, 8, C.byref(C.c_size_t())) == D.ERR_INVALID
    assert L.deamoe_norm_workspace_bytes(4, 8, None) == D.ERR_INVALID


def _refused(f, *a, **kw):
    with pytest.raises(D.DeamoeError) as e:
        f(*a, **kw)
    assert e.value.status == D.ERR_INVALID, str(e.value)


def test_binding_refuses_what_does_not_fit():
    """Shapes, types, strides and devices are refused before the library is called."""
    i32, bf, f32 = torch.int32, torch.bfloat16, torch.float32
    ids, x = torch.zeros(4, 2, dtype=i32), torch.zeros(4, 8, dtype=bf)
    off, pair, row = torch.zeros(9, dtype=i32), torch.zeros(8, dtype=i32), torch.zeros(4, 2, dtype=i32)
    xs, w = torch.zeros(8, 8, dtype=bf), torch.zeros(4, 2)
    for bad in ((ids.long(), x, off, pair, row, xs), (ids, x, off, pair[:7], row, xs),
                (ids, x, off, pair, row, xs[:7]), (ids, x, off, pair, row, xs.float()),
                (ids, x[:3], off, pair, row, xs), (ids, x.half(), off, pair, row, xs.half()),
                (ids.T.contiguous().T, x, off, pair, row, xs), (ids[0], x, off, pair, row, xs),
                (ids, x, off, pair, row, xs)):          # the last: right, but not on a GPU
        _refused(D.deamoe_dispatch, *bad)
    dy, dw = torch.zeros(4, 8, dtype=bf), torch.zeros(4, 2)
    _refused(D.deamoe_dispatch_backward, row, xs, dy[:, :7])
    _refused(D.deamoe_dispatch_backward, row, xs.float(), dy)
    _refused(D.deamoe_combine, row, w.to(bf), xs, dy)
    _refused(D.deamoe_combine, row, w, xs[:6], dy)
    _refused(D.deamoe_combine_backward, row, w, xs, dy, xs, dw[:3])
    _refused(D.deamoe_combine_backward, row, w, xs, dy, xs.T.contiguous().T, dw)
    codes, scale = torch.zeros(3, 5, 64, dtype=torch.uint8), torch.zeros(3, 5, 1)
    x4, y4, off4 = torch.zeros(6, 128, dtype=bf), torch.zeros(6, 5, dtype=bf), torch.zeros(4, dtype=i32)
    for bad in ((x4[:, :64], codes, scale, y4, off4), (x4, codes, scale.half(), y4, off4),
                (x4, codes, scale[0], y4, off4), (x4, codes.int(), scale, y4, off4),
                (x4, codes, scale, y4[:5], off4), (x4, codes, scale, y4, off4[:3]),
                (x4.float(), codes, scale, y4, off4), (x4, codes, torch.zeros(3, 5, 0), y4, off4),
                (x4, codes[0, 0], scale, y4, off4), (x4, codes, torch.zeros(3, 5, 3), y4, off4)):
        _refused(D.deamoe_w4_linear, *bad[:4], offset=bad[4])
        _refused(D.deamoe_w4_swiglu, *bad[:3], codes, scale, bad[3], offset=bad[4])
    _refused(D.deamoe_w4_swiglu, x4, codes, scale, codes[:2], scale[:2], y4, offset=off4)
    v = torch.zeros(8, dtype=bf)
    _refused(D.deamoe_prenorm, x, v[:7], x)
    _refused(D.deamoe_prenorm, x, v.float(), x)
    _refused(D.deamoe_prenorm_backward, x, v, x, x, v)                     # dw is fp32
    _refused(D.deamoe_postnorm, x, x, v, x, gate=v[:5])
    _refused(D.deamoe_postnorm, x, x[:, ::2], v, x)
    _refused(D.deamoe_postnorm_backward, x, v, x, x, x, v.float(), gate=v)   # no dgate
    _refused(D.deamoe_postnorm_backward, x, v, x, x, x, v.float(), du=x)     # du alone
    _refused(D.deamoe_postnorm_backward, x, v, x, x, x, v.float(), gate=v, dgate=v)   # dgate is fp32


def test_binding_refuses_missing_tensors():
    i32, bf = torch.int32, torch.bfloat16
    ids, x, off, pair = torch.zeros(4, 2, dtype=i32), torch.zeros(4, 8, dtype=bf), torch.zeros(9, dtype=i32), torch.zeros(8, dtype=i32)
    xs, w, v = torch.zeros(8, 8, dtype=bf), torch.zeros(4, 2), torch.zeros(8, dtype=bf)
    _refused(D.deamoe_dispatch, ids, None, off, pair, ids, xs)
    _refused(D.deamoe_dispatch, ids, x, off, None, ids, xs)
    _refused(D.deamoe_combine, ids, None, xs, x)
    _refused(D.deamoe_combine_backward, ids, None, xs, x, xs, w)   # dys needs w
    _refused(D.deamoe_combine_backward, ids, w, None, x, xs, w)    # dw needs ys
    _refused(D.deamoe_prenorm, x, None, x)
    _refused(D.deamoe_postnorm, x, None, v, x)
    _refused(D.deamoe_postnorm_backward, x, v, None, x, x, v.float())


def test_empty_batches_write_nothing_but_sums():
    """T = 0 with sums to clear is the only empty call that launches; the others return."""
    L = D.lib()
    assert L.deamoe_combine(0, 2, 8, D.BF16, None, None, None, None, None) == D.OK
    assert L.deamoe_combine_backward(0, 2, 8, D.BF16, None, None, None, None, None, None, None) == D.OK
