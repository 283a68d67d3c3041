"""Plain float64 forms of the operators that train through the routed experts."""
import math

import numpy as np
import torch

ACTS = ("identity", "relu", "silu", "gelu", "gelu_tanh")  # by code
LIPSCHITZ = (1.0, 1.0, 1.1, 1.13, 1.13)  # bounds of |act'|


def expert_sort(ids, E):
    """plan, pair, place (numpy)."""
    flat = ids.reshape(-1)
    lists = [np.flatnonzero(flat == e) for e in range(E)]
    pair = np.concatenate(lists).astype(np.int32)
    place = np.full(flat.size, -1, np.int32)
    place[pair] = np.arange(pair.size)
    bad = int(((flat < -1) | (flat >= E)).sum())
    plan = np.array([0, *np.cumsum([len(l) for l in lists]), bad], np.int32)
    return plan, pair, place.reshape(ids.shape)


def expert_unsort(ys, place, w, res):
    """y, and the sum of the addends' magnitudes."""
    T, k = place.shape
    y = torch.zeros(T, ys.shape[1], dtype=torch.float64, device=ys.device)
    if res is not None:
        y += res.double()
    mag = y.abs()
    for t_j in range(k):
        here = (place[:, t_j] >= 0) & (place[:, t_j] < ys.shape[0])
        rows = ys[place[here, t_j].long()].double()
        if w is not None:
            rows = rows * w[here, t_j].double()[:, None]
        y[here] += rows
        mag[here] += rows.abs()
    return y, mag


def expert_unsort_grad(dy, ys, place, w):
    """dys (NaN where no pair's), dw, and the sum of |dy ys| of each pair."""
    T, k = place.shape
    dy, ysd = dy.double(), ys.double()
    dys = torch.full(ys.shape, math.nan, dtype=torch.float64, device=ys.device)
    dw = torch.zeros(T, k, dtype=torch.float64, device=ys.device)
    mag = torch.zeros_like(dw)
    for j in range(k):
        here = (place[:, j] >= 0) & (place[:, j] < ys.shape[0])
        at = place[here, j].long()
        up = dy[here]
        dys[at] = up if w is None else up * w[here, j].double()[:, None]
        dw[here, j] = (up * ysd[at]).sum(1)
        mag[here, j] = (up * ysd[at]).abs().sum(1)
    return dys, dw, mag


def act(code, z):
    """act(z) and its slope in float64."""
    name = ACTS[code]
    if name == "identity":
        return z, torch.ones_like(z)
    if name == "relu":
        return z.clamp_min(0), (z > 0).double()
    if name == "silu":
        s = torch.sigmoid(z)
        return z * s, s * (1 + z * torch.sigmoid(-z))
    if name == "gelu":
        phi = torch.special.ndtr(z)
        return z * phi, phi + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
    a = math.sqrt(2 / math.pi)
    t = 2 * a * (z + 0.044715 * z ** 3)
    s = torch.sigmoid(t)
    return z * s, s + z * s * torch.sigmoid(-t) * 2 * a * (1 + 3 * 0.044715 * z * z)


def groups_of(offsets, rows):
    """(group, slice) of every group; one of all rows without offsets."""
    if offsets is None:
        return [(0, slice(0, rows))]
    return [(g, slice(offsets[g], offsets[g + 1])) for g in range(len(offsets) - 1)]


def linear(x, w, bias, mul, res, code, offsets):
    """z, y and the sum of |x w| (zeros in rows of no group)."""
    rows, N = x.shape[0], w.shape[-1]
    z = torch.zeros(rows, N, dtype=torch.float64, device=x.device)
    mag, y = torch.zeros_like(z), torch.zeros_like(z)
    ws = w if offsets is not None else w[None]
    for g, r in groups_of(offsets, rows):
        z[r] = x[r].double() @ ws[g].double()
        mag[r] = x[r].double().abs() @ ws[g].double().abs()
        if bias is not None:
            b = bias[g] if offsets is not None else bias
            z[r] += b.double()
            mag[r] += b.double().abs()
        y[r] = act(code, z[r])[0]
        if mul is not None:
            y[r] *= mul[r].double()
        if res is not None:
            y[r] += res[r].double()
    return z, y, mag


def linear_grad(dy, x, w, z, mul, code, offsets):
    """dict of dz, dx, dw, db, dm."""
    rows, N = dy.shape
    ws = (w if offsets is not None else w[None]).double()
    a, slope = act(code, z.double())
    up = dy.double() if mul is None else dy.double() * mul.double()
    dz, dm = up * slope, dy.double() * a
    dx = torch.zeros(rows, x.shape[1], dtype=torch.float64, device=x.device)
    dw = torch.zeros_like(ws)
    db = torch.zeros(ws.shape[0], N, dtype=torch.float64, device=x.device)
    for g, r in groups_of(offsets, rows):
        dx[r] = dz[r] @ ws[g].T.contiguous()
        dw[g] = x[r].double().T.contiguous() @ dz[r]
        db[g] = dz[r].sum(0)
    return dict(dz=dz, dm=dm, dx=dx, dw=dw.reshape(w.shape), db=db if offsets is not None else db[0])


def gate_grad(logits, ids, dw, score="softmax", normalize=True, scale=1.0):
    """numpy, row by row, from the coefficients' Jacobian."""
    T, E = logits.shape
    out = np.zeros((T, E))
    for t in range(T):
        l = logits[t].astype(np.float64)
        l = np.where(np.isnan(l), -np.inf, np.minimum(l, np.finfo(np.float32).max))
        slots = [(i, dw[t, j] * scale) for j, i in enumerate(ids[t])
                 if 0 <= i < E and l[i] > -np.inf]
        if not slots:
            continue
        at = np.array([i for i, _ in slots])
        g = np.array([v for _, v in slots], np.float64)
        if score == "softmax":
            p = np.exp(l - l.max())
            p /= p.sum()
            if not normalize:
                G = np.zeros(E)
                np.add.at(G, at, g)
                out[t] = p * (G - (p[at] * g).sum())
                continue
            c = np.exp(l[at] - l[at].max())
            c /= c.sum()
            v = c * (g - (c * g).sum())
        else:
            with np.errstate(over="ignore"):
                s, rest = 1 / (1 + np.exp(-l[at])), 1 / (1 + np.exp(l[at]))
            if normalize:
                c = s / s.sum() if s.sum() > 0 else 0 * s
                v = c * (g - (c * g).sum()) * rest
            else:
                v = g * s * rest
        np.add.at(out[t], at, v)
    return out
