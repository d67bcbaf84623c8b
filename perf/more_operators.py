"""The cases of the operators for rows that go to different weights: what a
program that trains or serves a block of experts, or adapters of many requests
beside a shared projection, has the library do.

Kinds:

  sort         ids [t][slots] -> where each expert's rows start, the order of
               the rows, and each row's place; ids of no expert are dropped.
  rows_train   tokens copied to their experts' rows, the experts' rows weighted
               and summed back to tokens, and the gradients of both.
  rows_infer   the two without gradients.
  gated_train  h = act(x Wg_e^T) * (x Wu_e^T) for the rows of each expert e, then
               from gh the gradients of x, Wg and Wu.
  gated_infer  the forward alone.
  linear_train y = x W_e^T, then from gy the gradients of x and W.
  linear_infer the forward alone.
  lora_infer   y[t] + s_e (x[t] A_e^T) B_e^T, e the adapter of token t's request.
  lora_train   the same, then from gy the gradients of x, A and B.

`own` chooses between the library's kernels and a plain form in fp32.
"""
from __future__ import annotations

import math
import random

import torch

own = False

DEV = "cuda:0"
_T = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32, "i32": torch.int32, "i64": torch.int64}
_SIZE = {"f16": 2, "bf16": 2, "f32": 4, "i32": 4, "i64": 8}
_ACTS = ("silu", "gelu", "relu")


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------

def _sort(name, tokens, slots, groups, ids="i32", drop=0.0):
    return dict(name=name, kind="sort", tokens=tokens, slots=slots, groups=groups, ids=ids, drop=drop)


def _rows(name, kind, tokens, slots, groups, width, dtype, drop=0.0):
    return dict(name=name, kind=kind, tokens=tokens, slots=slots, groups=groups, width=width, dtype=dtype, drop=drop)


def _experts(name, kind, rows, groups, k, f, dtype, act="silu", drop=0.0):
    return dict(name=name, kind=kind, rows=rows, groups=groups, k=k, f=f, dtype=dtype, act=act, drop=drop)


def _lora(name, kind, m, requests, groups, rank, k, n, dtype, drop=0.0, wide=0):
    """requests: of equal share, each with one adapter; m of them is a token each."""
    return dict(name=name, kind=kind, m=m, requests=requests, groups=groups, rank=rank, k=k, n=n, dtype=dtype, drop=drop,
                wide=wide)


def listed():
    return [
        # the routing of 16 tokens being answered: latency alone
        _sort("sort_m16", 16, 4, 64),
        # the routing of a large training batch with many small experts, ids as an index sort gives them
        _sort("sort_m32768", 32768, 8, 128, "i64", 0.02),
        # rows of a training batch to their experts and back
        _rows("rows_train_bf16_m8192", "rows_train", 8192, 4, 32, 4096, "bf16"),
        # a few prompts, a width whose rows start at any 2-byte address, some tokens past their experts' capacity
        _rows("rows_infer_f16_ragged", "rows_infer", 517, 3, 17, 1027, "f16", 0.05),
        # the largest training step: 8192 tokens to 2 of 8 experts
        _experts("gated_train_bf16_n16384", "gated_train", 16384, 8, 2048, 4096, "bf16"),
        # many small experts, sizes that fill no tile, rows behind the last expert's
        _experts("gated_train_f16_ragged", "gated_train", 4099, 27, 1000, 531, "f16", "gelu", 0.03),
        # 16 tokens being answered, 2 experts each: bound by reading their weights
        _experts("gated_infer_bf16_n32", "gated_infer", 32, 16, 2048, 4096, "bf16"),
        # the experts' way back to the model's width
        _experts("linear_train_bf16_n8192", "linear_train", 8192, 16, 2048, 2048, "bf16"),
        # one token of one request beside a square projection: latency
        _lora("lora_infer_bf16_m1", "lora_infer", 1, 1, 8, 16, 4096, 4096, "bf16"),
        # 64 requests being answered, one token each, some without an adapter
        _lora("lora_infer_f16_m64", "lora_infer", 64, 64, 40, 16, 4096, 8192, "f16", 0.1),
        # prompts of several requests, odd sizes, rows of wider tensors
        _lora("lora_infer_bf16_ragged", "lora_infer", 2049, 7, 12, 24, 2051, 5001, "bf16", 0.0, 5),
        # a training step of a few adapters at once
        _lora("lora_train_bf16_m8192", "lora_train", 8192, 16, 4, 32, 4096, 4096, "bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _size(rng, lo, hi):
    """A size over [lo, hi], spread over its logarithm: a third each multiples of 64, multiples of 8 and any."""
    v, step = _log(rng, lo, hi), rng.choice((64, 8, 1))
    return max(step, v // step * step)


def draw(rng):
    kind = rng.choice(["sort", "rows_train", "rows_infer", "gated_train", "gated_infer", "linear_train", "linear_infer",
                       "lora_infer", "lora_infer", "lora_train"])
    dtype, drop = rng.choice(["f16", "bf16"]), rng.choice((0.0, 0.0, 0.03, 0.2))
    groups = _log(rng, 1, 160)
    if kind == "sort":
        c = _sort("", _log(rng, 1, 32768), rng.randint(1, 8), groups, rng.choice(("i32", "i64")), drop)
    elif kind in ("rows_train", "rows_infer"):
        slots, width = rng.randint(1, 8), _size(rng, 64, 8192)
        tokens = max(1, min(_log(rng, 1, 16384), 8192 * 4 * 4096 // (slots * width)))
        c = _rows("", kind, tokens, slots, groups, width, rng.choice((dtype, dtype, "f32")), drop)
    elif kind not in ("lora_infer", "lora_train"):
        k, f = _size(rng, 64, 4096), _size(rng, 64, 8192)
        groups = max(1, min(groups, 8 * 2048 * 4096 // (k * f)))
        rows = max(1, min(_log(rng, 1, 32768), 16384 * 2048 * 4096 // (k * f), 16384 * 4096 // max(k, f)))
        c = _experts("", kind, rows, groups, k, f, dtype, rng.choice(_ACTS), drop)
    else:
        k, n, rank = _size(rng, 64, 8192), _size(rng, 64, 8192), rng.choice((4, 8, 16, 24, 32, 64, 128))
        groups = max(1, min(groups, 64 * 8192 * 32 // (rank * max(k, n))))
        m = max(1, min(rng.choice([1, rng.randint(2, 64), _log(rng, 16, 16384)]), 8192 * 4096 // max(k, n),
                       8192 * 4096 * 64 // (rank * max(k, n))))
        c = _lora("", kind, m, rng.choice((m, _log(rng, 1, m))), groups, rank, k, n, dtype, drop, rng.choice((0, 0, 8, 5)))
    del c["name"]
    return c


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _normal(gen, shape, std, dtype, wide=0):
    """N(0, std^2) in the type; `wide` > 0: the leading columns of a tensor that has so many more."""
    t = torch.randn((*shape[:-1], shape[-1] + wide), generator=gen, device=DEV, dtype=torch.float32)
    return (t * std).to(dtype)[..., :shape[-1]]


def _drop(gen, ids, share):
    """Some of the ids replaced by -1."""
    if share == 0.0:
        return ids
    u = torch.rand(ids.shape, generator=gen, device=DEV)
    return torch.where(u < share, torch.full_like(ids, -1), ids)


def _route(gen, tokens, slots, groups):
    """Each token's experts: distinct (as far as there are so many) and of unequal favour."""
    favour = torch.randn((groups,), generator=gen, device=DEV) * 0.7
    score = torch.randn((tokens, groups), generator=gen, device=DEV) + favour
    some = min(slots, groups)
    ids = torch.topk(score, some, dim=1).indices
    return ids.repeat(1, -(-slots // some))[:, :slots].contiguous() if some < slots else ids


def _plan(ids, groups):
    """(offsets, order, place) of ids by comparisons and a stable sort, in 32-bit integers."""
    flat = ids.reshape(-1).long()
    key = torch.where((flat >= 0) & (flat < groups), flat, torch.full_like(flat, groups))
    order = torch.sort(key, stable=True).indices
    place = torch.empty_like(order)
    place[order] = torch.arange(len(flat), device=flat.device)
    place = torch.where(key < groups, place, torch.full_like(place, -1))
    counts = (key.unsqueeze(0) == torch.arange(groups, device=flat.device).unsqueeze(1)).sum(1)
    offsets = torch.cat([counts.new_zeros(1), counts.cumsum(0)])
    return offsets.int(), order.int(), place.view(ids.shape).int()


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed)
    s, kind = dict(case), case["kind"]
    if kind == "sort":
        ids = _route(gen, case["tokens"], case["slots"], case["groups"])
        s["ids"] = _drop(gen, ids, case["drop"]).to(_T[case["ids"]])
        return s
    t = _T[case["dtype"]]
    if kind in ("rows_train", "rows_infer"):
        tokens, slots, width = case["tokens"], case["slots"], case["width"]
        ids = _drop(gen, _route(gen, tokens, slots, case["groups"]), case["drop"])
        s["place"] = _plan(ids, case["groups"])[2]
        s["x"] = _normal(gen, (tokens, width), 1.0, t)
        s["ys"] = _normal(gen, (tokens * slots, width), 1.0, t)
        w = torch.rand((tokens, slots), generator=gen, device=DEV) + 0.05
        s["weights"] = w / w.sum(1, keepdim=True)
        # rows of no token stay as they are
        s["xs"] = torch.zeros((tokens * slots, width), dtype=t, device=DEV)
        if kind == "rows_train":
            s["gxs"] = _normal(gen, (tokens * slots, width), 0.1, t)
            s["gy"] = _normal(gen, (tokens, width), 0.1, t)
            s["gys"] = torch.zeros_like(s["xs"])
    elif kind in ("lora_infer", "lora_train"):
        m, groups, rank, k, n = (case[v] for v in ("m", "groups", "rank", "k", "n"))
        mine = _drop(gen, torch.randint(0, groups, (case["requests"],), generator=gen, device=DEV), case["drop"])
        # a request's tokens lie together
        ids = mine[torch.arange(m, device=DEV) * case["requests"] // m]
        s["offsets"], s["order"], _ = _plan(ids, groups)
        s["bounds"] = s["offsets"].tolist()
        s["x"] = _normal(gen, (m, k), 1.0, t, case["wide"])
        s["y"] = _normal(gen, (m, n), 1.0, t, case["wide"])
        s["a"] = _normal(gen, (groups, rank, k), k ** -0.5, t)
        s["b"] = _normal(gen, (groups, n, rank), 0.5 * rank ** -0.5, t)
        s["scale"] = torch.rand((groups,), generator=gen, device=DEV) + 0.5
        s["out"] = torch.empty((m, n), dtype=t, device=DEV)
        if kind == "lora_train":
            s["gy"] = _normal(gen, (m, n), 0.1, t)
    else:
        rows, groups, k, f = (case[v] for v in ("rows", "groups", "k", "f"))
        ids = _drop(gen, _route(gen, rows, 1, groups), case["drop"])
        s["offsets"] = _plan(ids, groups)[0]
        s["bounds"] = s["offsets"].tolist()
        s["x"] = _normal(gen, (rows, k), 1.0, t)
        s["w"] = [_normal(gen, (groups, f, k), k ** -0.5, t) for _ in range(2 if kind.startswith("gated") else 1)]
        # rows behind the last expert's stay as they are
        s["h"] = torch.zeros((rows, f), dtype=t, device=DEV)
        if kind.endswith("train"):
            s["gh"] = _normal(gen, (rows, f), 0.05, t)
            s["grads"] = [torch.zeros((rows, k), dtype=t, device=DEV)] + [torch.empty_like(w) for w in s["w"]]
    return s


# ---------------------------------------------------------------------------
# the plain forms, in fp32
# ---------------------------------------------------------------------------

def _act(g, act):
    if act == "silu":
        return g / (1.0 + torch.exp(-g))
    if act == "gelu":
        return 0.5 * g * (1.0 + torch.erf(g * 0.5 ** 0.5))
    return g.clamp_min(0.0)


def _act_grad(g, act):
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-g))
        return p * (1.0 + g * (1.0 - p))
    if act == "gelu":
        return 0.5 * (1.0 + torch.erf(g * 0.5 ** 0.5)) + g * torch.exp(-0.5 * g * g) * (2.0 * math.pi) ** -0.5
    return (g > 0).to(g.dtype)


def _scatter(rows, place, out):
    """out[place[t, s]] = rows[t, s]; out keeps its other rows."""
    keep = place.reshape(-1) >= 0
    out[place.reshape(-1)[keep].long()] = rows.reshape(-1, rows.shape[-1])[keep].to(out.dtype)
    return out


def _taken(rows, place):
    """rows[place[t, s]] in fp32, zero where there is none: [t][slots][width]."""
    v = rows[place.clamp_min(0).long()].float()
    return torch.where((place >= 0).unsqueeze(-1), v, torch.zeros((), device=v.device))


def _plain_rows(s):
    x, ys, place, w, t = s["x"], s["ys"], s["place"], s["weights"], s["x"].dtype
    xs = _scatter(x.unsqueeze(1).expand(-1, place.shape[1], -1), place, s["xs"])
    v = _taken(ys, place)
    y = (v * w.unsqueeze(-1)).sum(1).to(t)
    if s["kind"] == "rows_infer":
        return xs, y
    gy = s["gy"].float().unsqueeze(1)
    gys = _scatter(gy * w.unsqueeze(-1), place, s["gys"])
    return xs, _taken(s["gxs"], place).sum(1).to(t), y, gys, (v * gy).sum(-1)


def _plain_experts(s):
    train, gated, act, b = s["kind"].endswith("train"), len(s["w"]) == 2, s["act"], s["bounds"]
    h = s["h"]
    for e in range(s["groups"]):
        rows = slice(b[e], b[e + 1])
        if b[e] == b[e + 1]:
            if train:
                [g[e].zero_() for g in s["grads"][1:]]
            continue
        x, w = s["x"][rows].float(), [v[e].float() for v in s["w"]]
        g = x @ w[0].t()
        if gated:
            u, a = x @ w[1].t(), _act(g, act)
        h[rows] = (a * u if gated else g).to(h.dtype)
        if train:
            gh = s["gh"][rows].float()
            d = [gh * u * _act_grad(g, act), gh * a] if gated else [gh]
            s["grads"][0][rows] = sum(di @ wi for di, wi in zip(d, w)).to(h.dtype)
            for grad, di in zip(s["grads"][1:], d):
                grad[e] = (di.t() @ x).to(h.dtype)
    return (h, *s["grads"]) if train else h


def _plain_lora(s):
    t, b, order = s["x"].dtype, s["bounds"], s["order"].long()
    out, train = s["out"].copy_(s["y"]), s["kind"] == "lora_train"
    if train:
        gx, ga, gb = (torch.zeros(v.shape, dtype=t, device=DEV) for v in (s["x"], s["a"], s["b"]))
    for e in range(s["groups"]):
        if b[e] == b[e + 1]:
            continue
        rows = order[b[e]:b[e + 1]]
        x, A, B = s["x"][rows].float(), s["a"][e].float(), s["b"][e].float()
        mid = (x @ A.t()) * s["scale"][e]
        out[rows] = (s["y"][rows].float() + mid @ B.t()).to(t)
        if train:
            gy = s["gy"][rows].float()
            p = (gy @ B) * s["scale"][e]
            gx[rows], ga[e], gb[e] = (p @ A).to(t), (p.t() @ x).to(t), (gy.t() @ mid).to(t)
    return (out, gx, ga, gb) if train else out


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def _own(s):
    import paper_2003_04296_amd as q

    kind = s["kind"]
    if kind == "sort":
        return q.moe_sort(s["ids"], s["groups"])
    if kind in ("rows_train", "rows_infer"):
        xs = q.moe_gather(s["x"], s["place"], out=s["xs"])
        if kind == "rows_infer":
            return xs, q.moe_combine(s["ys"], s["place"], s["weights"])
        gx = q.moe_gather_backward(s["gxs"], s["place"])
        y = q.moe_combine(s["ys"], s["place"], s["weights"])
        gys, gw = q.moe_combine_backward(s["gy"], s["ys"], s["place"], s["weights"], out=(s["gys"], None))
        return xs, gx, y, gys, gw
    if kind in ("lora_infer", "lora_train"):
        args = s["a"], s["b"], s["offsets"], s["order"]
        out, mid = q.lora_forward(s["y"], s["x"], *args, s["scale"], keep_mid=kind == "lora_train", out=s["out"])
        if kind == "lora_infer":
            return out
        return (out, *q.lora_backward(s["x"], *args, mid, s["gy"], s["scale"]))
    if kind == "linear_infer":
        return q.moe_linear_forward(s["x"], *s["w"], s["offsets"], out=s["h"])
    if kind == "linear_train":
        y = q.moe_linear_forward(s["x"], *s["w"], s["offsets"], out=s["h"])
        return (y, *q.moe_linear_backward(s["x"], *s["w"], s["offsets"], s["gh"], out=s["grads"]))
    act = {"silu": q.ACT_SILU, "gelu": q.ACT_GELU, "relu": q.ACT_RELU}[s["act"]]
    h, pre = q.moe_gated_forward(s["x"], *s["w"], s["offsets"], act, keep_pre=kind == "gated_train", out=s["h"])
    if kind == "gated_infer":
        return h
    return (h, *q.moe_gated_backward(s["x"], *s["w"], s["offsets"], pre, s["gh"], act, out=s["grads"]))


def run(state):
    if own:
        return _own(state)
    kind = state["kind"]
    if kind == "sort":
        return _plan(state["ids"], state["groups"])
    return {"rows": _plain_rows, "lora": _plain_lora}.get(kind.split("_")[0], _plain_experts)(state)


def work(case):
    kind = case["kind"]
    if kind == "sort":
        # ids in, order and places out, a comparison each
        n = case["tokens"] * case["slots"]
        return {"bytes": n * (_SIZE[case["ids"]] + 8) + 4 * (case["groups"] + 1), "flops": n}
    size = _SIZE[case["dtype"]]
    if kind in ("rows_train", "rows_infer"):
        m, n, w = case["tokens"], case["tokens"] * case["slots"], case["width"]
        # x and the experts' rows in, those rows and y out; places and weights
        b, flops = size * w * (2 * m + 2 * n) + 8 * n, 2 * n * w
        if kind == "rows_train":
            # gy, the rows of gxs in, the rows of gys and gx out, the weights' gradient
            b, flops = b + size * w * (2 * m + 2 * n) + 4 * n, 6 * n * w
        return {"bytes": b, "flops": flops}
    if kind in ("lora_infer", "lora_train"):
        m, r, k, n = case["m"], case["rank"], case["k"], case["n"]
        used = min(case["groups"], case["requests"])  # adapters that have tokens, at most
        weights = size * used * r * (k + n)
        if kind == "lora_infer":
            return {"bytes": size * m * (k + 2 * n) + weights, "flops": 2 * m * r * (k + n)}
        return {"bytes": size * m * (2 * k + 3 * n) + weights + size * case["groups"] * r * (k + n),
                "flops": 6 * m * r * (k + n)}
    m, k, f, two = case["rows"], case["k"], case["f"], 2 if kind.startswith("gated") else 1
    weights = size * two * min(case["groups"], m) * k * f
    if kind.endswith("infer"):
        return {"bytes": size * m * (k + f) + weights, "flops": 2 * two * m * k * f}
    return {"bytes": size * 2 * m * (k + f) + weights + size * two * case["groups"] * k * f, "flops": 6 * two * m * k * f}


# ---------------------------------------------------------------------------
# the definition, in 64 bits
# ---------------------------------------------------------------------------

def _exact_gate(g, act):
    """act(g) and its derivative."""
    if act == "relu":
        on = (g > 0).double()
        return g * on, on
    if act == "silu":
        p = torch.sigmoid(g)
        return g * p, p + g * p * (1 - p)
    cdf = 0.5 * torch.erfc(-g / math.sqrt(2.0))
    return g * cdf, cdf + g * torch.exp(-g * g / 2) / math.sqrt(2 * math.pi)


def _exact_sort(s):
    """Expert after expert, row after row."""
    ids, groups = s["ids"].reshape(-1).tolist(), s["groups"]
    lists = [[] for _ in range(groups + 1)]
    for i, e in enumerate(ids):
        lists[e if 0 <= e < groups else groups].append(i)
    offsets, place = [0], [-1] * len(ids)
    for some in lists[:groups]:
        for j, i in enumerate(some):
            place[i] = offsets[-1] + j
        offsets.append(offsets[-1] + len(some))
    ints = lambda v: torch.tensor(v, dtype=torch.int32)
    return ints(offsets), ints([i for some in lists for i in some]), ints(place).view(s["ids"].shape)


def _exact_rows(s):
    """Slot after slot."""
    m, slots = s["place"].shape
    w, train = s["weights"].double(), s["kind"] == "rows_train"
    xs = torch.zeros(s["xs"].shape, dtype=torch.float64, device=DEV)
    y = torch.zeros(s["x"].shape, dtype=torch.float64, device=DEV)
    if train:
        gx, gys, gw, gy = torch.zeros_like(y), torch.zeros_like(xs), torch.zeros_like(w), s["gy"].double()
    for j in range(slots):
        at = torch.nonzero(s["place"][:, j] >= 0).squeeze(1)
        to = s["place"][at, j].long()
        xs[to] = s["x"][at].double()
        v = s["ys"][to].double()
        y[at] += w[at, j, None] * v
        if train:
            gx[at] += s["gxs"][to].double()
            gys[to] = w[at, j, None] * gy[at]
            gw[at, j] = (v * gy[at]).sum(1)
    return (xs, gx, y, gys, gw) if train else (xs, y)


def _exact_experts(s):
    train, double = s["kind"].endswith("train"), lambda v: torch.zeros(v.shape, dtype=torch.float64, device=DEV)
    h, grads = double(s["h"]), [double(v) for v in s["grads"]] if train else []
    for e in range(s["groups"]):
        i, j = s["bounds"][e], s["bounds"][e + 1]
        if i == j:
            continue
        x, w = s["x"][i:j].double(), [v[e].double() for v in s["w"]]
        p = [torch.mm(x, v.t().contiguous()) for v in w]
        gh = s["gh"][i:j].double() if train else None
        if len(w) == 2:
            a, slope = _exact_gate(p[0], s["act"])
            h[i:j] = a * p[1]
            d = [gh * p[1] * slope, gh * a] if train else []
        else:
            h[i:j], d = p[0], [gh]
        if train:
            for n, v in enumerate(d):
                grads[0][i:j] += torch.mm(v, w[n])
                grads[1 + n][e] = torch.mm(v.t().contiguous(), x)
    return (h, *grads) if train else h


def _exact_lora(s):
    train = s["kind"] == "lora_train"
    y = s["y"].double()
    if train:
        gx, ga, gb = (torch.zeros(s[v].shape, dtype=torch.float64, device=DEV) for v in ("x", "a", "b"))
    for e in range(s["groups"]):
        rows = s["order"][s["bounds"][e]:s["bounds"][e + 1]].long()
        if len(rows) == 0:
            continue
        x, a, b, c = s["x"][rows].double(), s["a"][e].double(), s["b"][e].double(), s["scale"][e].double()
        mid = torch.mm(x, a.t().contiguous())
        y[rows] += c * torch.mm(mid, b.t().contiguous())
        if train:
            gy = s["gy"][rows].double()
            p = torch.mm(gy, b)
            gx[rows] = c * torch.mm(p, a)
            ga[e], gb[e] = c * torch.mm(p.t().contiguous(), x), c * torch.mm(gy.t().contiguous(), mid)
    return (y, gx, ga, gb) if train else y


def exact(case, seed):
    s = prepare(case, seed)
    if case["kind"] == "sort":
        return _exact_sort(s)
    return {"rows": _exact_rows, "lora": _exact_lora}.get(case["kind"].split("_")[0], _exact_experts)(s)
