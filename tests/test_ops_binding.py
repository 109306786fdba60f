"""The binding of the operators beside the layer, on the CPU: which device and stream a call runs on,
and what is refused before the library is called."""
import contextlib
import os
import sys

import pytest
import torch

sys.path.insert(0, os.path.dirname(os.path.abspath(__file__)))
from paper_2608_14385_amd import deamoe as D  # noqa: E402


class OnSecond(torch.Tensor):
    """A CPU tensor that says it is on the second GPU."""

    def get_device(self):
        return 1


class Stream:
    def __init__(self, index, handle):
        self.device, self.cuda_stream = torch.device("cuda", index), handle


@pytest.fixture
def gpus(monkeypatch):
    """Two GPUs, the first of them current; yields a function that says what is current."""
    state = {"device": 0, 0: "default 0", 1: "default 1"}

    @contextlib.contextmanager
    def device(index):
        before, state["device"] = state["device"], index
        yield
        state["device"] = before

    @contextlib.contextmanager
    def stream(s):
        i = s.device.index
        before, state[i] = state[i], s.cuda_stream
        with device(i):
            yield
        state[i] = before

    monkeypatch.setattr(torch.cuda, "current_device", lambda: state["device"])
    monkeypatch.setattr(torch.cuda, "device", device)
    monkeypatch.setattr(torch.cuda, "stream", stream)
    monkeypatch.setattr(torch._C, "_cuda_getCurrentRawStream", lambda i: state[i], raising=False)
    return lambda: (state["device"], state[state["device"]])


def refused(f, *a, status=D.ERR_INVALID, **kw):
    with pytest.raises(D.DeamoeError) as e:
        f(*a, **kw)
    assert e.value.status == status, str(e.value)


@pytest.mark.parametrize("stream", [None, Stream(1, "side")])
def test_a_blocks_layer_runs_where_its_rows_are(gpus, monkeypatch, stream):
    """Norms and layer run on the same device and stream, that of x and the call, also where another
    device is the current one."""
    ran = []
    monkeypatch.setattr(D, "_run", lambda fn, dev, stream, *args: ran.append(("norm", dev, gpus())))

    def layer(u):
        ran.append(("layer", u.get_device(), gpus()))
        return u

    x, w = (torch.zeros(*s).as_subclass(OnSecond) for s in ((4, 8), (8,)))
    D.Block(layer, w, w)(x, stream=stream)
    here = (1, "default 1" if stream is None else "side")
    assert ran == [("norm", 1, here), ("layer", 1, here), ("norm", 1, here)]
    assert gpus() == (0, "default 0")


def test_a_call_runs_on_its_tensors_device(gpus):
    def fn(*args):
        return args, gpus()

    assert D._call(fn, 1, None, (7,)) == ((7, "default 1"), (1, "default 1"))
    assert D._call(fn, 1, Stream(1, "side"), (7,))[0] == (7, "side")
    assert D._call(fn, 0, None, (7,)) == ((7, "default 0"), (0, "default 0"))


def test_a_stream_of_another_device_is_refused(gpus):
    def fn(*args):
        raise AssertionError("called")

    far = Stream(0, "far")
    refused(D._call, fn, 1, far, ())
    refused(D._run_with_workspace, fn, 1, far, None, 64)
    x, w = (torch.zeros(*s).as_subclass(OnSecond) for s in ((4, 8), (8,)))
    refused(D.Block(fn, w, w), x, stream=far)
    pair = (torch.zeros(2, 4, 4, dtype=torch.uint8), torch.zeros(2, 4, 1))
    refused(D.W4Experts(pair, pair, pair), x, torch.zeros(4, 1, dtype=torch.int32), torch.zeros(4, 1), stream=far)


def test_every_missing_tensor_is_refused():
    i32, bf = torch.int32, torch.bfloat16
    ids, x, xs = torch.zeros(4, 2, dtype=i32), torch.zeros(4, 8, dtype=bf), torch.zeros(8, 8, dtype=bf)
    off, pair, w, v = torch.zeros(9, dtype=i32), torch.zeros(8, dtype=i32), torch.zeros(4, 2), torch.zeros(8, dtype=bf)
    codes, scale = torch.zeros(5, 64, dtype=torch.uint8), torch.zeros(5, 1)
    rows, out = torch.zeros(6, 128, dtype=bf), torch.zeros(6, 5, dtype=bf)
    for f, args in ((D.deamoe_dispatch, (ids, x, off, pair, ids, xs)), (D.deamoe_dispatch_backward, (ids, xs, x)),
                    (D.deamoe_combine, (ids, w, xs, x)), (D.deamoe_w4_linear, (rows, codes, scale, out)),
                    (D.deamoe_w4_swiglu, (rows, codes, scale, codes, scale, out)),
                    (D.deamoe_prenorm, (x, v, x)), (D.deamoe_prenorm_backward, (x, v, x, x, v.float())),
                    (D.deamoe_postnorm, (x, x, v, x)), (D.deamoe_postnorm_backward, (x, v, x, x, x, v.float()))):
        for i in range(len(args)):
            if f is D.deamoe_dispatch and i == 5:   # the lists alone
                continue
            refused(f, *args[:i], None, *args[i + 1:])


def test_sizes_past_32_bits_are_refused():
    """2^32 + 4 would reach the library as 4, which it would answer."""
    far, bf, un = (1 << 32) + 4, torch.bfloat16, D.ERR_UNSUPPORTED

    def meta(*shape, dtype=bf):
        return torch.empty(*shape, dtype=dtype, device="meta")

    for T, h in ((far, 8), (2, far)):
        x, v, f = meta(T, h), meta(h), meta(h, dtype=torch.float32)
        refused(D.deamoe_prenorm, x, v, x, status=un)
        refused(D.deamoe_prenorm_backward, x, v, x, x, f, status=un)
        refused(D.deamoe_postnorm, x, x, v, x, status=un)
        refused(D.deamoe_postnorm_backward, x, v, x, x, x, f, status=un)
        row, w = meta(T, 1, dtype=torch.int32), meta(T, 1, dtype=torch.float32)
        refused(D.deamoe_combine, row, w, x, x, status=un)
        refused(D.deamoe_combine_backward, row, w, x, x, x, w, status=un)
        refused(D.deamoe_dispatch_backward, row, x, x, status=un)
        refused(D.deamoe_dispatch, row, x, meta(5, dtype=torch.int32), meta(T, dtype=torch.int32), row, x, status=un)
    for M, n, R, K in ((far, 1, 8, 64), (2, 1, far, 64), (2, 1, 8, far - 4 + 64), (2, far, 8, 64)):
        codes, scale = meta(n, R, K // 2, dtype=torch.uint8), meta(n, R, K // 64)
        x, y, off = meta(M, K), meta(M, R), meta(n + 1, dtype=torch.int32)
        refused(D.deamoe_w4_linear, x, codes, scale, y, offset=off, status=un)
        refused(D.deamoe_w4_swiglu, x, codes, scale, codes, scale, y, offset=off, status=un)
    ids = meta(4, 2, dtype=torch.int32)
    refused(D.deamoe_dispatch, ids, None, meta(far + 1, dtype=torch.int32), meta(8, dtype=torch.int32), ids, status=un)
    refused(D.deamoe_dispatch_workspace_bytes, far, 2, 8, status=un)
    refused(D.deamoe_norm_workspace_bytes, far, 8, status=un)
