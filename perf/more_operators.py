"""Timed cases of training through the routed experts of one MoE block.

A token's rows are sorted by expert and the experts' outputs come back weighted
(``sort``, ``unsort``, ``unsort_step`` with the gradients), the products between
are a matrix product with bias, activation, factor and residual, of one weight or
of one per group of rows (``linear``, ``linear_step``), and the coefficients'
gradient goes through the gate's choice to its logits (``gate_grad``).  Each case
is one call of an operator, or for the steps the forward and backward pass.

Keys of a case: op, rows, and
  sort, unsort, unsort_step  k slots, E local experts of E * R, d;
        sort: q (MXFP8 rows, else bf16)
        unsort: ys / res / y formats ("none": absent), w (weighted; without
        weights it is the gradient of sort)
  linear, linear_step  d in, N out, G groups (0: one weight), zipf exponent of the
        groups' sizes, live rows of them (the others belong to no group), act,
        bias, mul, res, y format
  gate_grad  E experts, k slots, score, norm (normalised coefficients), scale
"""
from __future__ import annotations

import math

import numpy as np
import torch

own = False

DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "bf16": 2, "none": 0}
ACTS = ["none", "relu", "silu", "gelu", "gelu_tanh"]


def _sort(rows, k, E, R, d, q):
    return dict(op="sort", rows=rows, k=k, E=E, R=R, d=d, q=q)


def _unsort(rows, k, E, R, d, ys="bf16", res="bf16", y="bf16", w=True, op="unsort"):
    return dict(op=op, rows=rows, k=k, E=E, R=R, d=d, ys=ys, res=res, y=y, w=w)


def _linear(rows, d, N, G=0, zipf=0.0, live=None, act="none", bias=False, mul=False, res="none",
            y="bf16", op="linear"):
    return dict(op=op, rows=rows, d=d, N=N, G=G, zipf=zipf, live=rows if live is None else live,
                act=act, bias=bias, mul=mul, res=res, y=y)


def _gate(rows, E, k, score, norm, scale=1.0):
    return dict(op="gate_grad", rows=rows, E=E, k=k, score=score, norm=norm, scale=scale)


def listed():
    return [
        # a few decoded tokens on one of eight ranks of 32 experts: launch latency
        dict(name="sort_tokens", **_sort(13, 8, 32, 8, 7168, False)),
        # a training step's tokens, every expert here: each row is written eight times
        dict(name="sort_prefill", **_sort(8191, 8, 64, 1, 4096, False)),
        # the experts' rows of a few decoded tokens back onto the residual stream
        dict(name="unsort_tokens", **_unsort(9, 8, 64, 1, 7168)),
        # a training step's way back, and its gradients of rows and coefficients
        dict(name="unsort_step", **_unsort(8192, 6, 32, 1, 4096, op="unsort_step")),
        # one token's projection: the weight is streamed once
        dict(name="linear_token", **_linear(1, 7168, 2048, act="gelu", bias=True)),
        # a short prompt's projection back onto the residual stream
        dict(name="linear_ragged", **_linear(777, 2560, 6144, bias=True, res="bf16")),
        # one replica's prefill of the widest layer
        dict(name="linear_prefill", **_linear(8192, 7168, 2048, act="gelu_tanh", bias=True)),
        # 24 tokens' pairs on eight experts: three rows each, weights streamed
        dict(name="experts_tokens", **_linear(24, 4096, 2048, G=8, zipf=0.5, act="silu", mul=True)),
        # a dense layer's training step
        dict(name="linear_step", **_linear(4095, 4096, 2048, act="gelu", bias=True,
                                           op="linear_step")),
        # the gate projection of a training step's gated experts, some popular
        dict(name="experts_step", **_linear(8192, 4096, 2048, G=8, zipf=0.8, act="silu", mul=True,
                                            op="linear_step")),
        # a few rows' coefficients back to 256 sigmoid scores
        dict(name="gate_grad_tokens", **_gate(9, 256, 8, "sigmoid", True, 2.5)),
        # eight replicas' tokens of the 160-expert layer
        dict(name="gate_grad_prefill", **_gate(65536, 160, 8, "softmax", False)),
    ]


def _log_int(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    op = rng.choice(["sort", "sort", "unsort", "unsort", "unsort_step", "linear", "linear",
                     "linear", "linear_step", "linear_step", "gate_grad", "gate_grad"])
    rows = _log_int(rng, 1, 8192)
    if op in ("sort", "unsort", "unsort_step"):
        E, R = rng.choice([(8, 8), (32, 8), (16, 10), (64, 1), (12, 1), (160, 1)])
        k = rng.randint(1, 8)
        d = rng.choice([256, 1024, 2304, 4096, 32 * rng.randint(9, 95), _log_int(rng, 65, 4096)])
        if op == "sort":
            q = d % 32 == 0 and rng.random() < 0.5
            return _sort(rows, k, E, R, d, q)
        ys, res, y = rng.choice([("bf16", "bf16", "bf16"), ("bf16", "none", "f32"),
                                 ("f32", "f32", "f32"), ("bf16", "f32", "bf16")])
        if op == "unsort_step":
            return _unsort(rows, min(k, 6), E, R, d, "bf16", res, rng.choice(["bf16", "f32"]),
                           op=op)
        return _unsort(rows, k, E, R, d, ys, res, y, rng.random() < 0.6)
    if op == "gate_grad":
        return _gate(_log_int(rng, 1, 65536), rng.choice([64, 160, rng.randint(8, 256)]),
                     rng.randint(1, 8), rng.choice(["softmax", "sigmoid"]), rng.random() < 0.6,
                     rng.choice([1.0, 2.5]))
    d = rng.choice([256, 1024, 2048, 4096, 8 * rng.randint(20, 380)])
    N = rng.choice([128, 256, 1408, 2048, 4096, 8 * rng.randint(20, 300)])
    G = rng.choice([0, 0, 0, 8, 16, 32])
    rows = _log_int(rng, 1, 4095 if op == "linear_step" and G == 0 else 8192)
    kw = dict(G=G, act=rng.choice(ACTS[2:] + ["none"] if op == "linear_step" else ACTS),
              bias=rng.random() < 0.5, y=rng.choice(["bf16", "bf16", "f32"]),
              res=rng.choice(["none", "none", "bf16", "f32"]), mul=rng.random() < 0.3)
    if G:  # some sorted buffers are longer than the rows in them
        kw |= dict(zipf=rng.choice([0.0, 0.5, 1.2]), live=rng.choice([rows, rows, rows * 5 // 8]))
    return _linear(rows, d, N, op=op, **kw)


def row_bytes(d):
    """An MXFP8 row: d codes, d / 32 scales, padded to 16 bytes."""
    return (d + d // 32 + 15) // 16 * 16


def work(c):
    T, op = c["rows"], c["op"]
    if op in ("sort", "unsort", "unsort_step"):
        k, d = c["k"], c["d"]
        E = c["E"] * c["R"]
        P = T * min(k, E) / c["R"]  # expected pairs of this rank
        if op == "sort":
            row = row_bytes(d) if c["q"] else 2 * d
            here = T * (1 - math.prod((E - c["E"] - j) / (E - j) for j in range(min(k, E))))
            return {"bytes": (here + P) * row + 8 * T * k + 4 * P, "flops": T * k}
        n = P * d * SIZE[c["ys"]] + T * d * (SIZE[c["res"]] + SIZE[c["y"]]) + T * k * 8
        if op == "unsort":
            return {"bytes": n, "flops": 2 * P * d}
        return {"bytes": n + P * d * SIZE[c["ys"]] + T * d * SIZE[c["y"]] + T * k * 4,
                "flops": 5 * P * d}
    if op == "gate_grad":
        E, k = c["E"], c["k"]
        read = E if c["score"] == "softmax" and not c["norm"] else k
        return {"bytes": 4 * T * (E + read + 2 * k), "flops": T * (E + 10 * k)}
    P, d, N, G = c["live"], c["d"], c["N"], max(c["G"], 1)
    if c["G"]:
        G = min(G, P)
    once = 2 * P * d + P * N * (SIZE[c["y"]] + SIZE[c["res"]] + (2 if c["mul"] else 0))
    if op == "linear":
        return {"bytes": once + 2 * G * d * N, "flops": 2 * P * d * N}
    return {"bytes": once + 2 * P * d + P * N * (SIZE[c["y"]] + (2 if c["mul"] else 0))
            + 2 * (G + max(c["G"], 1)) * d * N, "flops": 6 * P * d * N}


# ------------------------------------------------------------------ inputs

def prepare(c, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    T, op = c["rows"], c["op"]

    def normal(*shape, std=1.0, dtype="bf16"):
        return torch.randn(*shape, device="cuda", generator=g).mul_(std).to(DTYPE[dtype])

    def rand(*shape):
        return torch.rand(*shape, device="cuda", generator=g)

    s = dict(case=c)
    if op in ("sort", "unsort", "unsort_step"):
        k, E, d = c["k"], c["E"], c["d"]
        # a token's experts differ; those of other ranks leave their slots empty
        ids = rand(T, E * c["R"]).topk(k, -1)[1].to(torch.int32)
        ids = torch.where(ids < E, ids, -1)
        if op == "sort":
            s["ids"] = ids
            if c["q"]:  # MXFP8 rows, as bytes
                s["x"] = torch.randint(0, 256, (T, row_bytes(d)), dtype=torch.uint8, device="cuda",
                                       generator=g)
            else:
                s["x"] = normal(T, d)
        else:
            s["place"] = _sort_plan(c, ids)["place"]
            s["ys"] = normal(T * k, d, dtype=c["ys"])
            w = rand(T, k) + 0.05
            s["w"] = w / w.sum(-1, keepdim=True) if c["w"] else None
            s["res"] = None if c["res"] == "none" else normal(T, d, std=2.0, dtype=c["res"])
            if op == "unsort_step":
                s["dy"] = normal(T, d, std=0.1, dtype=c["y"])
    elif op == "gate_grad":
        E, k = c["E"], c["k"]
        logits = normal(T, E, dtype="f32")
        # some rows have all but a few experts masked
        some = torch.arange(T, device="cuda") % 17 == 3
        logits.masked_fill_(some[:, None] & (rand(T, E) >= 0.02), -math.inf)
        top, ids = logits.topk(k, -1)
        s["logits"], s["dw"] = logits, normal(T, k, dtype="f32")
        s["ids"] = ids.masked_fill(top == -math.inf, -1).to(torch.int32)
    else:
        d, N, G, P = c["d"], c["N"], c["G"], c["live"]
        if G:
            r = np.random.default_rng(seed)
            p = r.permutation(np.arange(1, G + 1.0) ** -c["zipf"])
            s["counts"] = [int(n) for n in r.multinomial(P, p / p.sum())]
            s["offsets"] = torch.tensor([0] + list(np.cumsum(s["counts"])), dtype=torch.int32,
                                        device="cuda")
        else:
            s["counts"], s["offsets"] = [T], None
        w = [G] if G else []
        s["x"], s["W"] = normal(T, d), normal(*w, d, N, std=0.02)
        s["bias"] = normal(*w, N, std=0.2, dtype="f32") if c["bias"] else None
        s["mul"] = normal(T, N) if c["mul"] else None
        s["res"] = None if c["res"] == "none" else normal(T, N, dtype=c["res"])
        if op == "linear_step":
            s["dy"] = normal(T, N, std=0.01, dtype=c["y"])
    return s


# ---------------------------------------------------- the framework's calls

def _plan(s):
    """Descriptors, output buffers and workspace, as a program keeps them.  Rows
    that a call leaves as they are start as zeros."""
    from paper_2609_33252_amd import cep
    c = s["case"]
    T, op = c["rows"], c["op"]
    code = {"f32": cep.CEP_F32, "bf16": cep.CEP_BF16, "none": cep.CEP_BF16}
    p = dict(cep=cep)

    def zeros(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype, device="cuda")

    def space(n):
        return torch.empty(max(int(n), 16), dtype=torch.uint8, device="cuda")

    if op == "sort":
        k, E = c["k"], c["E"]
        row = s["x"][0].numel() * s["x"].element_size()
        p["desc"] = cep.make_expert_sort(rows=T, top_k=k, n_experts=E, capacity=T * k,
                                         row_bytes=row)
        p["plan"], p["pair"] = zeros(E + 2, dtype=torch.int32), zeros(T * k, dtype=torch.int32)
        p["place"] = zeros(T, k, dtype=torch.int32)
        p["x"] = zeros(T * k, s["x"].shape[1], dtype=s["x"].dtype)
        p["ws"] = space(cep.cep_expert_sort_workspace(p["desc"]))
    elif op in ("unsort", "unsort_step"):
        k, d = c["k"], c["d"]
        p["desc"] = cep.make_expert_unsort(rows=T, top_k=k, d=d, sorted_rows=T * k,
                                           ys_dtype=code[c["ys"]], res_dtype=code[c["res"]],
                                           y_dtype=code[c["y"]])
        p["y"] = zeros(T, d, dtype=DTYPE[c["y"]])
        if op == "unsort_step":
            p["dys"], p["dw"] = torch.zeros_like(s["ys"]), zeros(T, k, dtype=torch.float32)
    elif op == "gate_grad":
        p["desc"] = cep.make_gate(rows=T, n_experts=c["E"], top_k=c["k"],
                                  score=cep.CEP_SOFTMAX if c["score"] == "softmax"
                                  else cep.CEP_SIGMOID, normalize=int(c["norm"]), scale=c["scale"])
        p["dl"] = zeros(T, c["E"], dtype=torch.float32)
    else:
        back = op == "linear_step"
        act = dict(none=cep.CEP_IDENTITY, relu=cep.CEP_RELU, silu=cep.CEP_SILU, gelu=cep.CEP_GELU,
                   gelu_tanh=cep.CEP_GELU_TANH)[c["act"]]
        p["desc"] = cep.make_linear(rows=T, d_in=c["d"], d_out=c["N"], n_groups=c["G"], act=act,
                                    y_dtype=code[c["y"]], res_dtype=code[c["res"]],
                                    dx_dtype=cep.CEP_BF16, dw_dtype=cep.CEP_BF16)
        p["y"] = zeros(T, c["N"], dtype=DTYPE[c["y"]])
        if back:
            curved = c["act"] != "none" or c["mul"]
            p["pre"] = zeros(T, c["N"], dtype=torch.float32) if curved else None
            p["dx"], p["dW"] = zeros(T, c["d"]), torch.zeros_like(s["W"])
            p["db"] = torch.zeros_like(s["bias"]) if c["bias"] else None
            p["dm"] = torch.zeros_like(s["mul"]) if c["mul"] else None
        p["ws"] = space(cep.cep_linear_workspace(p["desc"], back))
    return p


def _run_own(s):
    if "plan" not in s:
        s["plan"] = _plan(s)
    p, op = s["plan"], s["case"]["op"]
    cep, desc = p["cep"], p["desc"]
    if op == "sort":
        cep.cep_expert_sort(desc, s["ids"], p["plan"], p["pair"], p["place"], p["ws"], x=s["x"],
                            out_x=p["x"])
        return dict(plan=p["plan"], pair=p["pair"], place=p["place"], x=p["x"])
    if op in ("unsort", "unsort_step"):
        cep.cep_expert_unsort(desc, s["ys"], s["place"], p["y"], w=s["w"], residual=s["res"])
        if op == "unsort":
            return dict(y=p["y"])
        cep.cep_expert_unsort_backward(desc, s["dy"], s["ys"], s["place"], s["w"], p["dys"],
                                       p["dw"])
        return dict(y=p["y"], dys=p["dys"], dw=p["dw"])
    if op == "gate_grad":
        cep.cep_gate_topk_backward(desc, s["logits"], s["ids"], s["dw"], p["dl"])
        return dict(dl=p["dl"])
    extra = dict(bias=s["bias"], mul=s["mul"], residual=s["res"], offsets=s["offsets"])
    if op == "linear":
        cep.cep_linear(desc, s["x"], s["W"], p["y"], p["ws"], **extra)
        return dict(y=p["y"])
    cep.cep_linear(desc, s["x"], s["W"], p["y"], p["ws"], preact=p["pre"], **extra)
    cep.cep_linear_backward(desc, s["dy"], s["x"], s["W"], p["ws"], dx=p["dx"], dw=p["dW"],
                            dbias=p["db"], preact=p["pre"], mul=s["mul"], dmul=p["dm"],
                            offsets=s["offsets"])
    return dict(y=p["y"], dx=p["dx"], dW=p["dW"], db=p["db"], dm=p["dm"])


# ---------------------------------------------------------- the plain forms

def _sort_plan(c, ids):
    T, k, E = c["rows"], c["k"], c["E"]
    flat = ids.flatten()
    here = flat >= 0
    key = torch.where(here, flat, E)
    order = key.sort(stable=True)[1]
    counts = (key[:, None] == torch.arange(E, device=ids.device)).sum(0)
    plan = torch.cat([counts.new_zeros(1), counts.cumsum(0), counts.new_zeros(1)])
    place = torch.empty_like(order)
    place[order] = torch.arange(T * k, device=ids.device)
    live = torch.arange(T * k, device=ids.device) < plan[E]
    return dict(plan=plan.to(torch.int32), live=live,
                pair=torch.where(live, order, 0).to(torch.int32),
                place=torch.where(here, place, -1).view(T, k).to(torch.int32))


def _sorted(c, ids, x):
    p = _sort_plan(c, ids)
    rows = x[p["pair"].long() // c["k"]]
    return dict(plan=p["plan"], pair=p["pair"], place=p["place"],
                x=torch.where(p["live"][:, None], rows, torch.zeros((), dtype=x.dtype,
                                                                    device=x.device)))


def _unsort_plain(c, ys, place, w, res, dy=None):
    T, k, d = c["rows"], c["k"], c["d"]
    y = torch.zeros(T, d, device=ys.device) if res is None else res.float()
    here = place >= 0
    coef = here.float() if w is None else torch.where(here, w, 0.0)
    at = place.clamp_min(0).long()
    for j in range(k):
        y = y + coef[:, j, None] * ys[at[:, j]].float()
    out = dict(y=y.to(DTYPE[c["y"]]))
    if dy is not None:
        dy = dy.float()
        dys = torch.zeros(T * k + 1, d, dtype=ys.dtype, device=ys.device)
        dw = torch.zeros(T, k, device=ys.device)
        for j in range(k):
            dys[torch.where(here[:, j], place[:, j].long(), T * k)] = \
                (coef[:, j, None] * dy).to(ys.dtype)
            dw[:, j] = torch.where(here[:, j], (dy * ys[at[:, j]].float()).sum(-1), 0.0)
        out |= dict(dys=dys[:T * k], dw=dw)
    return out


def _gate_grad(c, logits, ids, dw):
    E, soft = c["E"], c["score"] == "softmax"
    here = ids >= 0
    at = ids.clamp_min(0).long()
    picked = logits.gather(1, at)
    g = torch.where(here, dw * c["scale"], 0.0)
    dense = torch.zeros_like(logits)
    if soft and not c["norm"]:
        top = logits.max(-1, keepdim=True)[0]
        p = torch.exp(logits - torch.where(top == -math.inf, 0.0, top))
        p = p / p.sum(-1, keepdim=True).clamp_min(1e-30)
        dense.scatter_add_(1, at, g)
        return dict(dl=p * (dense - (p * dense).sum(-1, keepdim=True)))
    if soft:
        top = torch.where(here, picked, -math.inf).max(-1, keepdim=True)[0]
        score = torch.where(here, torch.exp(picked - top), 0.0)
        rest = 1.0
    else:
        score = torch.where(here, 1.0 / (1.0 + torch.exp(-picked)), 0.0)
        rest = 1.0 / (1.0 + torch.exp(picked))
    if c["norm"]:
        total = score.sum(-1, keepdim=True)
        coef = torch.where(total > 0, score / total, 0.0)
        v = coef * rest * (g - (coef * g).sum(-1, keepdim=True))
    else:
        v = g * score * rest
    return dict(dl=dense.scatter_add_(1, at, torch.where(here, v, 0.0)))


def _act(name, z):
    """act(z) and its slope, float32."""
    if name == "none":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp_min(0.0), (z > 0).float()
    if name == "silu":
        s = 1.0 / (1.0 + torch.exp(-z))
        return z * s, s * (1.0 + z * (1.0 - s))
    if name == "gelu":
        phi = 0.5 * torch.erfc(-z * math.sqrt(0.5))
        return z * phi, phi + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi)
    a, b = math.sqrt(2 / math.pi), 0.044715  # the tangent as a logistic function
    s = 1.0 / (1.0 + torch.exp(-2 * a * (z + b * z ** 3)))
    return z * s, s + z * s * (1.0 - s) * 2 * a * (1.0 + 3 * b * z * z)


def _linear_plain(c, x, W, bias, mul, res, counts, dy=None):
    T, N, bf = c["rows"], c["N"], torch.bfloat16
    W = W if c["G"] else W[None]
    bias = bias if bias is None or c["G"] else bias[None]
    y = torch.zeros(T, N, dtype=DTYPE[c["y"]], device=x.device)
    back = dy is not None
    if back:
        dx, dW = torch.zeros_like(x), torch.zeros_like(W)
        db = None if bias is None else torch.zeros_like(bias)
        dm = None if mul is None else torch.zeros_like(mul)
    at = 0
    for g, n in enumerate(counts):
        r = slice(at, at + n)
        at += n
        if n == 0:
            continue
        xg, wg = x[r].float(), W[g].float()
        z = xg @ wg
        if bias is not None:
            z = z + bias[g]
        a, slope = _act(c["act"], z)
        v = a if mul is None else a * mul[r].float()
        y[r] = (v if res is None else v + res[r].float()).to(y.dtype)
        if back:
            up = dy[r].float()
            if mul is not None:
                dm[r] = (up * a).to(bf)
                up = up * mul[r].float()
            dz = up * slope
            dx[r], dW[g] = (dz @ wg.T).to(bf), (xg.T @ dz).to(bf)
            if db is not None:
                db[g] = dz.sum(0)
    if not back:
        return dict(y=y)
    return dict(y=y, dx=dx, dW=dW if c["G"] else dW[0],
                db=db if db is None or c["G"] else db[0], dm=dm)


def run(s):
    if own:
        return _run_own(s)
    c = s["case"]
    if c["op"] == "sort":
        return _sorted(c, s["ids"], s["x"])
    if c["op"] in ("unsort", "unsort_step"):
        return _unsort_plain(c, s["ys"], s["place"], s["w"], s["res"], s.get("dy"))
    if c["op"] == "gate_grad":
        return _gate_grad(c, s["logits"], s["ids"], s["dw"])
    return _linear_plain(c, s["x"], s["W"], s["bias"], s["mul"], s["res"], s["counts"],
                         s.get("dy"))


# --------------------------------------------------- definitions in 64 bits

def exact(c, seed):
    s = prepare(c, seed)
    op, T = c["op"], c["rows"]
    v = {k: t.double() for k, t in s.items()
         if isinstance(t, torch.Tensor) and t.is_floating_point()}
    if op == "sort":
        out = dict(plan=None, pair=None, place=None, x=None)
        if not c["q"]:
            k, ids = c["k"], s["ids"].cpu().numpy().reshape(-1)
            src = np.concatenate([np.flatnonzero(ids == e) for e in range(c["E"])]) // k
            x = torch.zeros(T * k, c["d"], dtype=torch.float64, device="cuda")
            x[:len(src)] = v["x"][torch.from_numpy(src).cuda()]
            out["x"] = x
        return out
    if op in ("unsort", "unsort_step"):
        k = c["k"]
        slot = s["place"].reshape(-1).long()
        some = (slot >= 0).nonzero()[:, 0]  # the pairs, and their rows and tokens
        row, tok = slot[some], some // k
        coef = torch.ones(T * k, dtype=torch.float64, device="cuda") if s["w"] is None \
            else v["w"].reshape(-1)
        y = torch.zeros(T, c["d"], dtype=torch.float64, device="cuda")
        for j in range(k):  # one slot of every token at a time
            mine = some % k == j
            y.index_add_(0, tok[mine], v["ys"][row[mine]] * coef[some[mine]][:, None])
        out = dict(y=y + v["res"] if s["res"] is not None else y)
        if op == "unsort_step":
            dys = torch.zeros_like(v["ys"])
            dw = torch.zeros(T * k, dtype=torch.float64, device="cuda")
            for j in range(k):
                mine = some % k == j
                up = v["dy"][tok[mine]]
                dys[row[mine]] = up * coef[some[mine]][:, None]
                dw[some[mine]] = (up * v["ys"][row[mine]]).sum(1)
            out |= dict(dys=dys, dw=dw.reshape(T, k))
        return out
    if op == "gate_grad":
        # the Jacobian of the chosen coefficients applied to dw
        l, ids = v["logits"], s["ids"].long()
        none = torch.full((T, 1), -math.inf, dtype=torch.float64, device="cuda")
        at = torch.where(ids < 0, c["E"], ids)  # empty slots: a masked expert past the last
        l = torch.cat([l, none], 1)
        picked = l.gather(1, at)
        up = v["dw"] * c["scale"] * (ids >= 0)
        dl = torch.zeros_like(l)
        if c["score"] == "softmax" and not c["norm"]:
            p = torch.softmax(l, 1).nan_to_num(0.0)
            dot = (p.gather(1, at) * up).sum(1, keepdim=True)
            dl = dl.scatter_add(1, at, up * p.gather(1, at)) - p * dot
        else:
            p = torch.sigmoid(picked)
            if c["score"] == "softmax":
                q = torch.softmax(picked, 1).nan_to_num(0.0)
                dv = q * up - q * (q * up).sum(1, keepdim=True)
            elif c["norm"]:
                q = (p / p.sum(1, keepdim=True)).nan_to_num(0.0)
                dv = (q * up - q * (q * up).sum(1, keepdim=True)) * torch.sigmoid(-picked)
            else:
                dv = up * p * torch.sigmoid(-picked)
            dl = dl.scatter_add(1, at, dv.nan_to_num(0.0))
        return dict(dl=dl[:, :c["E"]])
    f64 = dict(dtype=torch.float64, device="cuda")
    group = torch.repeat_interleave(torch.arange(len(s["counts"])), torch.tensor(s["counts"])).cuda()
    W = v["W"].reshape(-1, c["d"], c["N"])
    bias = v["bias"].reshape(-1, c["N"]) if c["bias"] else None
    y, dx = torch.zeros(T, c["N"], **f64), torch.zeros(T, c["d"], **f64)
    dm, dW = torch.zeros(T, c["N"], **f64), torch.zeros_like(W)
    db = torch.zeros(len(W), c["N"], **f64)
    for e in range(len(W)):
        rows = (group == e).nonzero()[:, 0]
        x = v["x"][rows]
        z = torch.matmul(x, W[e])
        if bias is not None:
            z += bias[e]
        if c["act"] == "none":
            a, slope = z, 1.0
        elif c["act"] == "relu":
            a, slope = torch.where(z > 0, z, 0.0), torch.where(z > 0, 1.0, 0.0)
        elif c["act"] == "silu":
            a = z / (1 + torch.exp(-z))
            slope = torch.sigmoid(z) + a * torch.sigmoid(-z)
        elif c["act"] == "gelu":
            cdf = torch.special.ndtr(z)
            a, slope = z * cdf, cdf + z * torch.exp(-z.square() / 2) / (2 * math.pi) ** 0.5
        else:
            t = torch.tanh((2 / math.pi) ** 0.5 * (z + 0.044715 * z.pow(3)))
            inner = (2 / math.pi) ** 0.5 * (1 + 0.134145 * z.square())
            a, slope = z * (1 + t) / 2, (1 + t) / 2 + z * (1 - t.square()) / 2 * inner
        m = v["mul"][rows] if c["mul"] else 1.0
        y[rows] = a * m + (v["res"][rows] if s["res"] is not None else 0.0)
        if op == "linear_step":
            up = v["dy"][rows]
            dm[rows] = up * a
            dz = up * m * slope
            dx[rows] = torch.matmul(dz, W[e].t().contiguous())
            dW[e] = torch.matmul(x.t().contiguous(), dz)
            db[e] = dz.sum(0)
    if op == "linear":
        return dict(y=y)
    return dict(y=y, dx=dx, dW=dW.reshape(s["W"].shape),
                db=db.reshape(s["bias"].shape) if c["bias"] else None, dm=dm if c["mul"] else None)
