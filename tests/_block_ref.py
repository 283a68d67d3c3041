"""Plain float64 forms of the operators around the routed experts."""
import numpy as np
import torch


def rms_norm(x, res, w, eps):
    s = x.double() if res is None else x.double() + res.double()
    inv = 1.0 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    return s, s * inv * w.double()


def rms_norm_grad(s, w, dy, dres, eps):
    s, w, dy = s.double(), w.double(), dy.double()
    inv = 1.0 / torch.sqrt((s * s).mean(-1, keepdim=True) + eps)
    n, a = s * inv, dy * w
    dx = inv * (a - n * (a * n).mean(-1, keepdim=True))
    if dres is not None:
        dx = dx + dres.double()
    return dx, (dy * n).sum(0)


def gate(logits, k, score="softmax", bias=None, groups=1, topg=1, normalize=True, scale=1.0):
    """numpy, row by row; keys compared exactly, the lower expert on ties."""
    T, E = logits.shape
    ids, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    for t in range(T):
        l = logits[t].astype(np.float64)
        l = np.where(np.isnan(l), -np.inf, np.minimum(l, np.finfo(np.float32).max))
        shut = l == -np.inf
        if score == "softmax":
            key = l.copy()
            p = np.exp(l - l.max()) if not shut.all() else np.zeros(E)
            p = np.where(shut, 0.0, p)
            if not normalize and p.sum() > 0:
                p = p / p.sum()
        else:
            with np.errstate(over="ignore"):
                p = np.where(shut, 0.0, 1.0 / (1.0 + np.exp(-l)))
            key = np.where(shut, -np.inf, p + (0.0 if bias is None else bias.astype(np.float64)))
        if groups > 1:
            g = key.reshape(groups, -1)
            top = -np.sort(-np.pad(g, ((0, 0), (0, 1)), constant_values=-np.inf), axis=1)[:, :2]
            total = np.where(top[:, 0] == -np.inf, -np.inf,
                             top[:, 0] + np.where(top[:, 1] == -np.inf, 0.0, top[:, 1]))
            kept = np.argsort(-total, kind="stable")[:topg]
            mask = np.zeros(groups, bool)
            mask[kept] = True
            key = np.where(np.repeat(mask, E // groups), key, -np.inf)
        order = [e for e in np.argsort(-key, kind="stable")[:k] if key[e] > -np.inf]
        ids[t, :len(order)] = order
        w[t, :len(order)] = p[order]
        if normalize:
            total = w[t].sum()
            w[t] = w[t] / total if total > 0 else 0.0
    return ids, w * scale


def dispatch(ids, w, R, per):
    """[(token, local ids, weights)] of every sent row, plan."""
    rows, offsets, pairs = [], [0], []
    for r in range(R):
        n = 0
        for t in range(ids.shape[0]):
            here = (ids[t] >= r * per) & (ids[t] < (r + 1) * per)
            if here.any():
                rows.append((t, np.where(here, ids[t] - r * per, -1), np.where(here, w[t], 0.0)))
                n += int(here.sum())
        offsets.append(len(rows))
        pairs.append(n)
    bad = int(((ids < -1) | (ids >= R * per)).sum())
    return rows, np.array(offsets + pairs + [bad], np.int32)


def gated_ffn(x, wg, wu, wd):
    x, wg, wu, wd = x.double(), wg.double(), wu.double(), wd.double()
    g, u = x @ wg, x @ wu
    h = g * torch.sigmoid(g) * u
    return g, u, h, h @ wd


def gated_ffn_grad(dy, x, wg, wu, wd):
    g, u, h, _ = gated_ffn(x, wg, wu, wd)
    dy, x = dy.double(), x.double()
    s = torch.sigmoid(g)
    dh = dy @ wd.double().T.contiguous()
    dg, du = dh * u * s * (1 + g * (1 - s)), dh * g * s
    xt = x.T.contiguous()
    return dict(dg=dg, du=du, dh=dh, h=h,
                dx=dg @ wg.double().T.contiguous() + du @ wu.double().T.contiguous(),
                dwg=xt @ dg, dwu=xt @ du, dwd=h.T.contiguous() @ dy)
