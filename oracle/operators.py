"""Plain fp64 forms of the routing to a fixed number of experts, the experts' products on a given
choice and the residual layer norm (numpy; test infrastructure only)."""
import numpy as np


def _clean(z):
    z = np.asarray(z, np.float64)
    z = np.where(z == np.inf, float(np.finfo(np.float32).max), z)
    return np.where(np.isnan(z), -np.inf, z)


def _sigmoid(z):
    e = np.exp(-np.abs(z))
    return np.where(z >= 0, 1.0 / (1.0 + e), e / (1.0 + e))


def log_scores(z, sigmoid):
    """log s of one row; -inf for experts that take no part."""
    live = z > -np.inf
    out = np.full(z.shape, -np.inf)
    if not live.any():
        return out
    v = z[live]
    out[live] = (np.minimum(v, 0.0) - np.log1p(np.exp(-np.abs(v))) if sigmoid
                 else v - v.max() - np.log(np.exp(v - v.max()).sum()))
    return out


def route_topk(g, k, n_groups=1, top_groups=1, sel_bias=None, scale=1.0, sigmoid=False,
               renorm=False, top2=False):
    """(idx [T, k], w [T, k]) of the logits g [T, E]."""
    T, E = g.shape
    Gs = E // n_groups
    idx, w = np.full((T, k), -1, np.int32), np.zeros((T, k))
    bias = None if sel_bias is None else _clean(sel_bias)
    for t in range(T):
        z = _clean(g[t])
        ls = log_scores(z, sigmoid)
        s = np.exp(ls)
        c = z.copy() if bias is None else s + bias
        part = z > -np.inf if bias is None else (z > -np.inf) & (bias > -np.inf)
        by = s if top2 and bias is None else c
        if n_groups > 1:
            worth = []
            for a in range(n_groups):
                v = sorted((by[e] for e in range(a * Gs, (a + 1) * Gs) if part[e]), reverse=True)
                if v:
                    worth.append((-(v[0] + (v[1] if top2 and len(v) > 1 else 0.0)), a))
            stay = {a for _, a in sorted(worth)[:top_groups]}
            part = part & np.array([e // Gs in stay for e in range(E)])
        order = sorted((-c[e], e) for e in range(E) if part[e])[:k]
        for j, (_, e) in enumerate(order):
            idx[t, j] = e
        n = len(order)
        if n:
            l = ls[idx[t, :n]]
            w[t, :n] = np.exp(l - l.max()) / np.exp(l - l.max()).sum() if renorm else np.exp(l)
    return idx, w * scale


def route_topk_grad(g, idx, dw, scale=1.0, sigmoid=False, renorm=False):
    """d(sum w dw) / dg with the choice held fixed."""
    T, E = g.shape
    out = np.zeros((T, E))
    for t in range(T):
        z = _clean(g[t])
        ls = log_scores(z, sigmoid)
        slots = [(e, a) for e, a in zip(idx[t], np.asarray(dw[t], np.float64))
                 if 0 <= e < E and z[e] > -np.inf]
        if not slots:
            continue
        e, a = np.array([s[0] for s in slots]), np.array([s[1] for s in slots])
        q = np.exp(ls[e])
        if renorm:
            q = np.exp(ls[e] - ls[e].max())
            q = q / q.sum()
            a = a - (q * a).sum()
        v = q * a
        if sigmoid:
            v = v * _sigmoid(-z[e])
        np.add.at(out[t], e, v)
        if not sigmoid and not renorm:
            out[t] -= np.exp(ls) * (q * a).sum()
    return out * scale


def layernorm(r, eps, w=None, b=None):
    """(u, mu, rstd) of the rows of r."""
    r = np.asarray(r, np.float64)
    mu = r.mean(1, keepdims=True)
    rstd = 1.0 / np.sqrt(((r - mu) ** 2).mean(1, keepdims=True) + eps)
    u = (r - mu) * rstd
    if w is not None:
        u = u * np.asarray(w, np.float64)
    if b is not None:
        u = u + np.asarray(b, np.float64)
    return u, mu, rstd


def layernorm_grad(r, du, dres, eps, w=None):
    """(dx, dw, db)."""
    du = np.asarray(du, np.float64)
    hat, _, rstd = layernorm(r, eps)
    a = du if w is None else du * np.asarray(w, np.float64)
    dx = rstd * (a - a.mean(1, keepdims=True) - hat * (a * hat).mean(1, keepdims=True))
    if dres is not None:
        dx = dx + np.asarray(dres, np.float64)
    return dx, (du * hat).sum(0), du.sum(0)


def routed_ffn(x, idx, gate_w, W_in, W_up, W_out, b_in=None, b_out=None):
    """(y, bound): y = sum_j w_j FFN_{idx_j}(x) with 128 neurons per expert (W_up None: the GELU
    MLP), and how far an evaluation may be off that rounds as follows: x and the weights exact in
    bf16; sums over d and over the chosen neurons in fp32, in chains of at most n = 128 additions
    each; the activation in fp32 (8 roundings); h to 16 bits (two bf16 numbers); y in fp32."""
    x, W_in, W_out = (np.asarray(a, np.float64) for a in (x, W_in, W_out))
    T, E = x.shape[0], W_in.shape[0] // 128
    half = 2.0 ** -24
    y, bound = np.zeros((T, W_out.shape[0])), np.zeros((T, W_out.shape[0]))
    if b_out is not None:
        y += np.asarray(b_out, np.float64)
        bound += 128 * half * np.abs(b_out)
    for e in range(E):
        hit = idx == e
        wt = (hit * (1.0 if gate_w is None else np.where(hit, gate_w, 0.0))).sum(1)
        wa = (hit * (1.0 if gate_w is None else np.abs(np.where(hit, gate_w, 0.0)))).sum(1)
        t = np.nonzero(hit.any(1))[0]
        if not len(t):
            continue
        n = slice(128 * e, 128 * e + 128)
        a, da = x[t] @ W_in[n].T, 128 * half * (np.abs(x[t]) @ np.abs(W_in[n]).T)
        if W_up is None:
            if b_in is not None:
                a = a + np.asarray(b_in, np.float64)[n]
            h = 0.5 * a * (1 + np.tanh(np.sqrt(2 / np.pi) * (a + 0.044715 * a ** 3)))
            dh = 1.2 * da + 8 * half * np.abs(a)  # |GELU'| < 1.2
        else:
            up = np.asarray(W_up, np.float64)[n]
            b, db = x[t] @ up.T, 128 * half * (np.abs(x[t]) @ np.abs(up).T)
            f = a * _sigmoid(a)
            h = f * b
            dh = 1.1 * da * np.abs(b) + np.abs(f) * db + 8 * half * np.abs(a * b)  # |SiLU'| < 1.1
        y[t] += wt[t, None] * (h @ W_out[:, n].T)
        dh = dh + (2.0 ** -16 + 128 * half) * np.abs(h)
        bound[t] += wa[t, None] * (dh @ np.abs(W_out[:, n]).T)
    return y, bound
