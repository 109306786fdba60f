"""Performance cases of the operators around and beside the decode layer.

Three operators, each with the directions a user runs:

* tokens sorted by expert (`dispatch`: the sort and the gathered rows; `dispatch_backward`)
  and brought back with their routing weights (`combine`; `combine_train` adds its gradient);
* products with 4-bit weights and group scales (`w4_linear`: one matrix, or the experts' down
  matrices; `w4_swiglu`: the experts' gate and up matrices with the activation);
* the norms around a block with its gate and residual scale (`prenorm`, `postnorm`, and
  `prenorm_train` and `postnorm_backward`, which return the gradients).

Sizes are those of the layer presets (hidden 1024 to 7168, 64 to 1280 experts, 6 to 10 experts
per token), for one token up to the batches of a prompt or a training step.
"""
from __future__ import annotations

import functools
import math

import torch

own = False

EPS = 1e-6
_TYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
_BYTES = {"f32": 4, "bf16": 2}


def _move(name, op, tokens, k, n, h, dtype="bf16", drop=0.0):
    return {"name": name, "op": op, "tokens": tokens, "k": k, "n": n, "h": h, "dtype": dtype,
            "drop": drop}


def _w4(name, op, tokens, rows, cols, group, k=0, n=1, scale="f32"):
    """k = 0: one dense matrix; else n experts, k of them per token."""
    return {"name": name, "op": op, "tokens": tokens, "k": k, "n": n, "rows": rows, "cols": cols,
            "group": group, "scale": scale}


def _norm(name, op, tokens, h, dtype="bf16", gate="none", following=False, res_scale=1.0):
    """gate: "none", "shared" ([h]) or "full" ([tokens, h]); following: the next block's pre-norm."""
    return {"name": name, "op": op, "tokens": tokens, "h": h, "dtype": dtype, "gate": gate,
            "following": following, "res_scale": res_scale}


def listed():
    return [
        # one user's decode step: 10 experts of a small model, launches and latency only
        _move("dispatch_t1", "dispatch", 1, 10, 672, 1024),
        # a prompt or training batch with a padded tail and dropped pairs
        _move("dispatch_t8192", "dispatch", 8192, 8, 128, 4096, drop=0.03),
        # the gradient of a ragged training batch in fp32
        _move("dispatch_backward_t4099", "dispatch_backward", 4099, 6, 64, 2048, dtype="f32"),
        # a decode batch on its way back to the tokens
        _move("combine_t61", "combine", 61, 8, 256, 7168),
        # a training batch: forward and gradient of rows and weights
        _move("combine_train_t8192", "combine_train", 8192, 8, 128, 4096, drop=0.03),
        # one token through one dense matrix, and a busy server's batch with an odd width
        _w4("w4_linear_t1", "w4_linear", 1, 7168, 7168, 128),
        _w4("w4_linear_t61", "w4_linear", 61, 2815, 2048, 64, scale="bf16"),
        # the experts of a decode batch, and of a prompt
        _w4("w4_swiglu_t16", "w4_swiglu", 16, 1536, 4096, 128, k=8, n=128),
        _w4("w4_swiglu_t2048", "w4_swiglu", 2048, 1280, 2048, 128, k=6, n=64),
        # between two blocks of a decode step: post-norm, residual and the next pre-norm
        _norm("postnorm_t16", "postnorm", 16, 7168, following=True),
        # a training step's block boundary with a learned gate on its way back, and a ragged fp32
        # batch in both directions
        _norm("postnorm_backward_t8192", "postnorm_backward", 8192, 4096, gate="shared",
              following=True, res_scale=0.5),
        _norm("prenorm_train_t2051", "prenorm_train", 2051, 2048, dtype="f32"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    top = [work(c) for c in listed()]
    most = {m: max(w[m] for w in top) for m in ("bytes", "flops")}
    while True:
        op = rng.choice(("dispatch", "dispatch_backward", "combine", "combine_train", "w4_linear",
                         "w4_linear", "w4_swiglu", "prenorm", "prenorm_train", "postnorm",
                         "postnorm_backward"))
        h = rng.choice((256, 1024, 2048, 4096, 5120, 7168, 8 * _log(rng, 32, 1024),
                        _log(rng, 200, 8200)))
        dtype = rng.choice(("bf16", "bf16", "f32"))
        if op in ("dispatch", "dispatch_backward", "combine", "combine_train"):
            n = rng.choice((16, 64, 128, 160, 256, 384, 672, 1280))
            c = _move("", op, _log(rng, 1, 16384), rng.randint(1, 10), n, h, dtype,
                      rng.choice((0.0, 0.0, 0.03, 0.25)))
        elif op in ("w4_linear", "w4_swiglu"):
            group = rng.choice((32, 64, 128, 128))
            cols = group * max(1, rng.choice((1024, 2048, 4096, 5120, 7168, _log(rng, 256, 8192))) // group)
            rows = rng.choice((384, 1024, 1536, 2048, 4096, 7168, _log(rng, 100, 8192)))
            experts = op == "w4_swiglu" or rng.random() < 0.3
            if experts:
                c = _w4("", op, _log(rng, 1, 2048), min(rows, 2048), cols, group,
                        rng.randint(1, 10), rng.choice((16, 64, 128)),
                        rng.choice(("f32", "bf16")))
            else:
                c = _w4("", op, _log(rng, 1, 2048), rows, cols, group, scale=rng.choice(("f32", "bf16")))
        else:
            post = op.startswith("postnorm")
            c = _norm("", op, _log(rng, 1, 16384), h, dtype,
                      rng.choice(("none", "shared", "full")) if post else "none",
                      post and rng.random() < 0.5, rng.choice((1.0, 0.5)) if post else 1.0)
        del c["name"]
        if all(work(c)[m] <= most[m] for m in most):
            return c


# ------------------------------------------------------------------- inputs


def _routing(g, T, k, n, drop):
    """[T, k] distinct experts and their normalised weights: random logits with some experts more
    popular; the last share of the tokens is padding, and as many single pairs are dropped (-1)."""
    popular = torch.arange(1, n + 1, device="cuda", dtype=torch.float32).pow(-0.3).log()
    logits = torch.randn(T, n, device="cuda", generator=g) + popular
    top, ids = logits.topk(k, dim=1)
    w = torch.softmax(top, 1)
    ids = ids.to(torch.int32)
    if drop:
        gone = torch.rand(T, k, device="cuda", generator=g) < drop
        gone |= (torch.arange(T, device="cuda") >= T - int(T * drop))[:, None]
        ids = torch.where(gone, torch.full_like(ids, -1), ids)
    return ids.contiguous(), w.contiguous()


def _lists(ids, n):
    """The sorted order of the pairs: offset [n + 1], pair [T * k] (row -> pair), row [T, k] (pair ->
    row), -1 where a pair is dropped."""
    T, k = ids.shape
    flat = ids.reshape(-1).long()
    held = (flat >= 0) & (flat < n)
    key = torch.where(held, flat, torch.full_like(flat, n))
    order = torch.argsort(key, stable=True)
    count = torch.zeros(n + 1, dtype=torch.int64, device=ids.device).scatter_add_(0, key, torch.ones_like(key))
    offset = torch.zeros(n + 1, dtype=torch.int64, device=ids.device)
    offset[1:] = count[:n].cumsum(0)
    at = torch.arange(T * k, device=ids.device)
    used = at < offset[n]
    pair = torch.where(used, order, torch.full_like(order, -1))
    row = torch.empty_like(order).scatter_(0, order, at)
    row = torch.where(held, row, torch.full_like(row, -1)).reshape(T, k)
    return offset.int(), pair.int(), row.int(), used


def _state(case, seed):
    g = torch.Generator(device="cuda").manual_seed(int(seed))
    op, T = case["op"], case["tokens"]

    def normal(*shape, dtype, scale=1.0):
        return (torch.randn(*shape, device="cuda", generator=g) * scale).to(dtype)

    if op in ("dispatch", "dispatch_backward", "combine", "combine_train"):
        k, n, h, t = case["k"], case["n"], case["h"], _TYPE[case["dtype"]]
        ids, w = _routing(g, T, k, n, case["drop"])
        if op == "dispatch":
            return {"ids": ids, "n": n, "x": normal(T, h, dtype=t),
                    "offset": torch.empty(n + 1, dtype=torch.int32, device="cuda"),
                    "pair": torch.empty(T * k, dtype=torch.int32, device="cuda"),
                    "row": torch.empty(T, k, dtype=torch.int32, device="cuda"),
                    "xs": torch.zeros(T * k, h, dtype=t, device="cuda")}
        s = {"row": _lists(ids, n)[2], "w": w}
        if op == "dispatch_backward":
            return s | {"dxs": normal(T * k, h, dtype=t), "dx": torch.empty(T, h, dtype=t, device="cuda")}
        s |= {"ys": normal(T * k, h, dtype=t), "y": torch.empty(T, h, dtype=t, device="cuda")}
        if op == "combine_train":
            s |= {"dy": normal(T, h, dtype=t), "dys": torch.zeros(T * k, h, dtype=t, device="cuda"),
                  "dw": torch.empty(T, k, device="cuda")}
        return s
    if op in ("w4_linear", "w4_swiglu"):
        k, n, R, K, group = case["k"], case["n"], case["rows"], case["cols"], case["group"]
        M, lead = (T * k, (n, R)) if k else (T, (R,))

        def matrix():   # codes of a normal matrix, scales around 1 / sqrt(K) over the codes' spread
            codes = torch.randint(0, 256, (*lead, K // 2), dtype=torch.uint8, device="cuda", generator=g)
            scale = torch.rand(*lead, K // group, device="cuda", generator=g) + 0.5
            return codes, (scale * (0.2 / math.sqrt(K))).to(_TYPE[case["scale"]])

        s = {"x": normal(M, K, dtype=torch.bfloat16), "T": T,
             "y": torch.zeros(M, R, dtype=torch.bfloat16, device="cuda"),
             "offset": _lists(_routing(g, T, k, n, 0.0)[0], n)[0] if k else None}
        s["codes"], s["scales"] = matrix()
        if op == "w4_swiglu":
            s["up_codes"], s["up_scales"] = matrix()
        return s
    h, t = case["h"], _TYPE[case["dtype"]]
    s = {"x": normal(T, h, dtype=t), "w": normal(h, dtype=t, scale=0.2) + 1.0,
         "res_scale": case["res_scale"], "gate": None, "w_next": None}
    if op in ("prenorm", "prenorm_train"):
        s["u"] = torch.empty_like(s["x"])
        if op == "prenorm_train":
            s |= {"du": normal(T, h, dtype=t), "dres": normal(T, h, dtype=t),
                  "dx": torch.empty_like(s["x"]), "dw": torch.empty(h, device="cuda")}
        return s
    s |= {"y": normal(T, h, dtype=t, scale=2.0), "z": torch.empty_like(s["x"])}
    if op == "postnorm_backward":
        s["z"] = normal(T, h, dtype=t, scale=1.5)
    if case["gate"] != "none":
        s["gate"] = normal(*((h,) if case["gate"] == "shared" else (T, h)), dtype=t, scale=0.5)
    if case["following"]:
        s |= {"w_next": normal(h, dtype=t, scale=0.2) + 1.0, "u": torch.empty_like(s["x"])}
    if op == "postnorm_backward":
        s |= {"dz": normal(T, h, dtype=t), "dx": torch.empty_like(s["x"]),
              "dy": torch.empty_like(s["x"]), "dw": torch.empty(h, device="cuda")}
        if case["gate"] != "none":
            s["dgate"] = torch.empty_like(s["gate"], dtype=t if case["gate"] == "full" else torch.float32)
        if case["following"]:
            s |= {"du": normal(T, h, dtype=t), "dw_next": torch.empty(h, device="cuda")}
    return s


def prepare(case, seed):
    return {"op": case["op"], **_state(case, seed)}


# -------------------------------------------------------------- the plain forms


def _plain_dispatch(s):
    offset, pair, row, used = _lists(s["ids"], s["n"])
    k = s["ids"].shape[1]
    xs = torch.where(used[:, None], s["x"][pair.long().clamp(min=0) // k], s["xs"])
    return {"offset": offset, "pair": pair, "row": row, "xs": xs}


def _gathered(row, rows):
    """[T, k, h] rows in 32 bits, zeros in the place of dropped pairs."""
    held = row >= 0
    got = rows[row.long().clamp(min=0)].float()
    return torch.where(held[..., None], got, torch.zeros((), device=got.device)), held


def _plain_dispatch_backward(s):
    return _gathered(s["row"], s["dxs"])[0].sum(1).to(s["dx"].dtype)


def _plain_combine(s):
    got, held = _gathered(s["row"], s["ys"])
    w = torch.where(held, s["w"], torch.zeros_like(s["w"]))
    return (w[..., None] * got).sum(1).to(s["y"].dtype)


def _plain_combine_backward(s):
    got, held = _gathered(s["row"], s["ys"])
    dy = s["dy"].float()
    dw = (got * dy[:, None]).sum(-1)
    at = s["row"].long()[held]
    s["dys"][at] = (s["w"][..., None] * dy[:, None])[held].to(s["dys"].dtype)
    return {"dys": s["dys"], "dw": dw}


def _plain_matrix(codes, scales, wide=torch.float32):
    """[..., R, K]: code 2j in the low, 2j + 1 in the high half of byte j, less 8, times the group's scale."""
    q = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2).to(wide) - 8
    groups = q.unflatten(-1, (scales.shape[-1], -1))
    return (groups * scales.to(wide)[..., None]).flatten(-2)


def _plain_product(s, codes, scales):
    x, w = s["x"].float(), _plain_matrix(codes, scales)
    if s["offset"] is None:
        return x @ w.T
    # every expert's rows padded to the batch's tokens: an expert has a token once at most
    first, end = s["offset"][:-1].long(), s["offset"][1:].long()
    at = first[:, None] + torch.arange(s["T"], device=x.device)
    got = torch.bmm(x[at.clamp(max=x.shape[0] - 1)], w.transpose(1, 2).contiguous())
    mine = torch.arange(x.shape[0], device=x.device)
    e = (mine[:, None] >= end).sum(1)
    return got[e, mine - first[e]]


def _plain_w4(s):
    a = _plain_product(s, s["codes"], s["scales"])
    if s["op"] == "w4_swiglu":
        a = a / (1 + torch.exp(-a)) * _plain_product(s, s["up_codes"], s["up_scales"])
    return a.to(s["y"].dtype)


def _plain_rms(v, wide=torch.float32):
    """v / sqrt(mean v^2 + eps) over the rows, and the factor."""
    v = v.to(wide)
    r = 1 / torch.sqrt((v * v).mean(-1, keepdim=True) + EPS)
    return v * r, r


def _plain_rms_backward(hat, r, d):
    return r * (d - hat * (d * hat).mean(-1, keepdim=True))


def _plain_prenorm(s):
    return (_plain_rms(s["x"])[0] * s["w"].float()).to(s["x"].dtype)


def _plain_prenorm_backward(s):
    hat, r = _plain_rms(s["x"])
    du = s["du"].float()
    dx = s["dres"].float() + _plain_rms_backward(hat, r, du * s["w"].float())
    return {"dx": dx.to(s["dx"].dtype), "dw": (du * hat).sum(0)}


def _plain_postnorm(s):
    n = _plain_rms(s["y"])[0] * s["w"].float()
    n = n if s["gate"] is None else n * s["gate"].float()
    z = (s["res_scale"] * s["x"].float() + n).to(s["x"].dtype)
    out = {"z": z}
    if s["w_next"] is not None:
        out["u"] = (_plain_rms(z)[0] * s["w_next"].float()).to(z.dtype)
    return out


def _plain_postnorm_backward(s):
    t = s["x"].dtype
    d, out = s["dz"].float(), {}
    if s["w_next"] is not None:
        zhat, rz = _plain_rms(s["z"])
        du = s["du"].float()
        d = d + _plain_rms_backward(zhat, rz, du * s["w_next"].float())
        out["dw_next"] = (du * zhat).sum(0)
    out["dx"] = (s["res_scale"] * d).to(t)
    hat, r = _plain_rms(s["y"])
    w, dn = s["w"].float(), d
    if s["gate"] is not None:
        dgate = d * (hat * w)
        out["dgate"] = dgate.sum(0) if s["gate"].dim() == 1 else dgate.to(t)
        dn = d * s["gate"].float()
    out["dw"] = (dn * hat).sum(0)
    out["dy"] = _plain_rms_backward(hat, r, dn * w).to(t)
    return out


def _run_plain(s):
    op = s["op"]
    if op == "dispatch":
        return _plain_dispatch(s)
    if op == "dispatch_backward":
        return _plain_dispatch_backward(s)
    if op == "combine":
        return _plain_combine(s)
    if op == "combine_train":
        return {"y": _plain_combine(s), **_plain_combine_backward(s)}
    if op in ("w4_linear", "w4_swiglu"):
        return _plain_w4(s)
    if op == "prenorm":
        return _plain_prenorm(s)
    if op == "prenorm_train":
        return {"u": _plain_prenorm(s), **_plain_prenorm_backward(s)}
    return _plain_postnorm(s) if op == "postnorm" else _plain_postnorm_backward(s)


# ----------------------------------------------------------- the framework's calls


def _run_own(s):
    from paper_2608_14385_amd import deamoe as D
    op = s["op"]
    if op == "dispatch":
        D.deamoe_dispatch(s["ids"], s["x"], s["offset"], s["pair"], s["row"], s["xs"])
        return {k: s[k] for k in ("offset", "pair", "row", "xs")}
    if op == "dispatch_backward":
        D.deamoe_dispatch_backward(s["row"], s["dxs"], s["dx"])
        return s["dx"]
    if op in ("combine", "combine_train"):
        D.deamoe_combine(s["row"], s["w"], s["ys"], s["y"])
        if op == "combine":
            return s["y"]
        D.deamoe_combine_backward(s["row"], s["w"], s["ys"], s["dy"], s["dys"], s["dw"])
        return {k: s[k] for k in ("y", "dys", "dw")}
    if op == "w4_linear":
        D.deamoe_w4_linear(s["x"], s["codes"], s["scales"], s["y"], offset=s["offset"])
        return s["y"]
    if op == "w4_swiglu":
        D.deamoe_w4_swiglu(s["x"], s["codes"], s["scales"], s["up_codes"], s["up_scales"], s["y"],
                           offset=s["offset"])
        return s["y"]
    if op in ("prenorm", "prenorm_train"):
        D.deamoe_prenorm(s["x"], s["w"], s["u"], eps=EPS)
        if op == "prenorm":
            return s["u"]
        D.deamoe_prenorm_backward(s["x"], s["w"], s["du"], s["dx"], s["dw"], dres=s["dres"], eps=EPS)
        return {k: s[k] for k in ("u", "dx", "dw")}
    if op == "postnorm":
        D.deamoe_postnorm(s["x"], s["y"], s["w"], s["z"], gate=s["gate"], res_scale=s["res_scale"],
                          w_next=s["w_next"], u=s.get("u"), eps=EPS)
        return {k: s[k] for k in ("z", "u") if k in s}
    D.deamoe_postnorm_backward(s["y"], s["w"], s["dz"], s["dx"], s["dy"], s["dw"], gate=s["gate"],
                               dgate=s.get("dgate"), res_scale=s["res_scale"],
                               z=s["z"] if s["w_next"] is not None else None, w_next=s["w_next"],
                               du=s.get("du"), dw_next=s.get("dw_next"), eps=EPS)
    return {k: s[k] for k in ("dx", "dy", "dw", "dgate", "dw_next") if k in s}


def run(state):
    return _run_own(state) if own else _run_plain(state)


# ------------------------------------------------------------- work of a pass


@functools.lru_cache(maxsize=None)
def _touched(T, k, n):
    """Mean number of experts that a batch of the drawn routing touches."""
    g = torch.Generator().manual_seed(1)
    popular = torch.arange(1, n + 1, dtype=torch.float32).pow(-0.3).log()
    return sum((torch.randn(T, n, generator=g) + popular).topk(k, dim=1).indices.unique().numel()
               for _ in range(4)) / 4


def work(case):
    op, T = case["op"], case["tokens"]
    if op in ("dispatch", "dispatch_backward", "combine", "combine_train"):
        k, h, b = case["k"], case["h"], _BYTES[case["dtype"]]
        tail = 1 - int(T * case["drop"]) / T
        pairs = T * k * tail * (1 - case["drop"])
        row, lists = h * b, 4 * T * k
        if op == "dispatch":
            return {"bytes": T * tail * row + pairs * row + 3 * lists + 4 * case["n"], "flops": 0}
        if op == "dispatch_backward":
            return {"bytes": T * row + pairs * row + lists, "flops": pairs * h}
        if op == "combine":
            return {"bytes": T * row + pairs * row + 2 * lists, "flops": 2 * pairs * h}
        return {"bytes": 2 * T * row + 2 * pairs * row + 3 * lists, "flops": 5 * pairs * h}
    if op in ("w4_linear", "w4_swiglu"):
        R, K, k = case["rows"], case["cols"], case["k"]
        mats = (_touched(T, k, case["n"]) if k else 1) * (2 if op == "w4_swiglu" else 1)
        M = T * k if k else T
        b = mats * (R * K / 2 + R * (K // case["group"]) * _BYTES[case["scale"]])
        return {"bytes": b + 2 * M * (K + R), "flops": 2.0 * M * R * K * (2 if op == "w4_swiglu" else 1)}
    h, row = case["h"], T * case["h"] * _BYTES[case["dtype"]]
    if op == "prenorm":
        return {"bytes": 2 * row, "flops": 4 * T * h}
    if op == "prenorm_train":   # x, du, dres in; u, dx out
        return {"bytes": 5 * row + 8 * h, "flops": 14 * T * h}
    full, nxt = case["gate"] == "full", case["following"]
    if op == "postnorm":        # x, y, gate in; z, u out
        return {"bytes": (3 + full + nxt) * row, "flops": (7 + 4 * nxt) * T * h}
    # y, dz, gate, z, du in; dx, dy, dgate out
    return {"bytes": (4 + 2 * full + 2 * nxt) * row + 16 * h, "flops": (14 + 12 * nxt) * T * h}


# -------------------------------------------------------------- correct results


def _exact_moves(case, s):
    op = case["op"]
    if op == "dispatch":
        T, k, n = case["tokens"], case["k"], case["n"]
        flat = s["ids"].flatten()
        pairs = torch.cat([(flat == e).nonzero().flatten() for e in range(n)])   # by expert, then pair
        held = (flat >= 0) & (flat < n)
        offset = torch.tensor([0] + [int((held & (flat <= e)).sum()) for e in range(n)], device="cuda")
        pair = torch.full((T * k,), -1, device="cuda")
        pair[:len(pairs)] = pairs
        row = torch.full((T * k,), -1, device="cuda")
        row[pairs] = torch.arange(len(pairs), device="cuda")
        xs = s["xs"].double()
        xs[:len(pairs)] = s["x"].double()[pairs // k]
        return {"offset": offset.int(), "pair": pair.int(), "row": row.int().view(T, k), "xs": xs}
    rows = s["dxs"] if op == "dispatch_backward" else s["ys"]
    total = torch.zeros(case["tokens"], case["h"], dtype=torch.float64, device="cuda")
    dys = s["dys"].double() if op == "combine_train" else None
    dw = torch.zeros(s["row"].shape, dtype=torch.float64, device="cuda")
    for i in range(case["k"]):   # a token has one row of every slot at most
        t = (s["row"][:, i] >= 0).nonzero().flatten()
        r = s["row"][t, i].long()
        p = s["w"][t, i].double()[:, None] if op != "dispatch_backward" else 1.0
        total[t] += p * rows[r].double()
        if dys is not None:
            dy = s["dy"][t].double()
            dys[r] = p * dy
            dw[t, i] = (rows[r].double() * dy).sum(1)
    return total if dys is None else {"y": total, "dys": dys, "dw": dw}


def _exact_w4(case, s):
    x = s["x"].double()
    y = s["y"].double()
    offset = s["offset"].tolist() if s["offset"] is not None else [0, len(x)]
    names = (("codes", "scales"), ("up_codes", "up_scales")) if case["op"] == "w4_swiglu" else (("codes", "scales"),)
    for e in range(len(offset) - 1):
        a, b = offset[e], offset[e + 1]
        if a == b:
            continue
        got = []
        for c, sc in names:
            codes, scales = (s[c], s[sc]) if s["offset"] is None else (s[c][e], s[sc][e])
            w = torch.empty(codes.shape[0], 2 * codes.shape[1], dtype=torch.float64, device="cuda")
            w[:, 0::2] = torch.remainder(codes, 16)
            w[:, 1::2] = torch.div(codes, 16, rounding_mode="floor")
            w = (w - 8) * scales.double().repeat_interleave(case["group"], 1)
            got.append(x[a:b] @ w.T)
        y[a:b] = got[0] if len(got) == 1 else got[0] * torch.sigmoid(got[0]) * got[1]
    return y


def _exact_norms(case, s):
    """Values by the formulas, gradients by differentiating them."""
    leaves = {k: s[k].double().requires_grad_() for k in ("x", "y", "w", "gate", "w_next") if s.get(k) is not None}

    def rms(v):
        return v * (v.pow(2).mean(-1, keepdim=True) + EPS).rsqrt()

    if case["op"].startswith("prenorm"):
        u = rms(leaves["x"]) * leaves["w"]
        if case["op"] == "prenorm":
            return u.detach()
        loss = (u * s["du"].double()).sum() + (leaves["x"] * s["dres"].double()).sum()
        dx, dw = torch.autograd.grad(loss, (leaves["x"], leaves["w"]))
        return {"u": u.detach(), "dx": dx, "dw": dw}
    z = s["res_scale"] * leaves["x"] + leaves.get("gate", 1.0) * rms(leaves["y"]) * leaves["w"]
    if case["op"] == "postnorm":
        out = {"z": z}
        if s["w_next"] is not None:
            out["u"] = rms(z) * leaves["w_next"]
        return {k: v.detach() for k, v in out.items()}
    # the gradient reaching z: its own, and what comes back through the next norm at the z in hand
    dz, out = s["dz"].double(), {}
    if s["w_next"] is not None:
        at, w_next = s["z"].double().requires_grad_(), leaves.pop("w_next")
        more, out["dw_next"] = torch.autograd.grad((rms(at) * w_next * s["du"].double()).sum(), (at, w_next))
        dz = dz + more
    out |= dict(zip(("d" + k for k in leaves), torch.autograd.grad((z * dz).sum(), list(leaves.values()))))
    return out


def exact(case, seed):
    s = _state(case, seed)
    if case["op"] in ("w4_linear", "w4_swiglu"):
        return _exact_w4(case, s)
    if "norm" in case["op"]:
        return _exact_norms(case, s)
    return _exact_moves(case, s)
