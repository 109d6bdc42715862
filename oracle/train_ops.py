"""Plain fp64 oracle of the operators for training other models: packed attention, RMS norm with the residual's addition,
distillation from a teacher's top logits, embedding lookup and the gradient of its table.  numpy, one record / row / token at
a time, backward passes written out by hand."""
import numpy as np


def visible(n, causal, window):
    """[n, n] truth values: does query i (row) see key j (column)"""
    i, j = np.arange(n)[:, None], np.arange(n)[None, :]
    see = np.ones((n, n), bool)
    if causal:
        see = j <= i
        if window:
            see &= i - j < window
    return see


def attention_record(q, k, v, scale, see, do=None):
    """One record, one head: q, k, v [n, D].  Returns o, lse and, with do, (dq, dk, dv)."""
    s = np.where(see, scale * (q @ k.T), -np.inf)
    m = s.max(1, keepdims=True)
    e = np.exp(s - m)
    p = e / e.sum(1, keepdims=True)
    o, lse = p @ v, m[:, 0] + np.log(e.sum(1))
    if do is None:
        return o, lse
    dp = do @ v.T
    ds = p * (dp - (do * o).sum(1, keepdims=True))
    return o, lse, scale * (ds @ k), scale * (ds.T @ q), p.T @ do


def attention(q, k, v, starts, scale, causal, window, do=None):
    """q [T, H, D], k, v [T, Hk, D]; starts: n_seq + 1 rows.  Returns a dict of o, lse [H, T], dq, dk, dv; rows outside every
    record are NaN."""
    T, H, D = q.shape
    Hk = k.shape[1]
    q, k, v = (np.asarray(t, np.float64) for t in (q, k, v))
    out = {"o": np.full((T, H, D), np.nan), "lse": np.full((H, T), np.nan)}
    if do is not None:
        do = np.asarray(do, np.float64)
        out.update(dq=np.full((T, H, D), np.nan), dk=np.full((T, Hk, D), np.nan), dv=np.full((T, Hk, D), np.nan))
    for a, b in zip(starts[:-1], starts[1:]):
        if a == b:
            continue
        see = visible(b - a, causal, window)
        if do is not None:
            out["dk"][a:b] = 0.0
            out["dv"][a:b] = 0.0
        for h in range(H):
            g = h // (H // Hk)
            r = attention_record(q[a:b, h], k[a:b, g], v[a:b, g], scale, see, None if do is None else do[a:b, h])
            out["o"][a:b, h], out["lse"][h, a:b] = r[0], r[1]
            if do is not None:
                out["dq"][a:b, h] = r[2]
                out["dk"][a:b, g] += r[3]
                out["dv"][a:b, g] += r[4]
    return out


def rmsnorm_fwd(x, res, gamma, eps):
    """returns s = x + res, rho [T], u"""
    s = np.asarray(x, np.float64) + (0.0 if res is None else np.asarray(res, np.float64))
    rho = 1.0 / np.sqrt((s * s).mean(1) + eps)
    return s, rho, s * rho[:, None] * np.asarray(gamma, np.float64)


def rmsnorm_bwd(du, h, rho, gamma, dres):
    """returns dh, dgamma"""
    du, h, gamma = (np.asarray(t, np.float64) for t in (du, h, gamma))
    xh = h * np.asarray(rho, np.float64)[:, None]
    g = du * gamma
    dh = np.asarray(rho, np.float64)[:, None] * (g - xh * (g * xh).mean(1, keepdims=True))
    return dh + (0.0 if dres is None else np.asarray(dres, np.float64)), (du * xh).sum(0)


def _log_softmax(z):
    m = z.max()
    return z - m - np.log(np.exp(z - m).sum())


def distill(z, ids, top, tau, kd, labels, ce, w):
    """z [T, V], ids / top [T, k], labels [T] or None, w [T] or None.  Returns loss_tok, loss, dz."""
    z = np.asarray(z, np.float64)
    T, V = z.shape
    w = np.full(T, 1.0 / T) if w is None else np.asarray(w, np.float64)
    loss_tok, dz = np.zeros(T), np.zeros((T, V))
    for t in range(T):
        if w[t] == 0:
            continue
        used = [(int(i), float(x)) for i, x in zip(ids[t], top[t]) if 0 <= i < V and x != -np.inf]
        if used:
            lp = _log_softmax(np.array([x for _, x in used], np.float64) / tau)
            lq = _log_softmax(z[t] / tau)
            g = np.exp(lq)
            for (i, _), l in zip(used, lp):
                p = np.exp(l)
                loss_tok[t] += kd * tau * tau * p * (l - lq[i])
                g[i] -= p
            dz[t] += w[t] * kd * tau * g
        if labels is not None and 0 <= labels[t] < V:
            lq = _log_softmax(z[t])
            loss_tok[t] -= ce * lq[labels[t]]
            g = np.exp(lq)
            g[labels[t]] -= 1.0
            dz[t] += w[t] * ce * g
    return loss_tok, float((w * loss_tok).sum()), dz


def embed_fwd(tokens, table, scale):
    out = np.zeros((len(tokens), table.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < table.shape[0]:
            out[t] = scale * np.asarray(table[v], np.float64)
    return out


def embed_bwd(tokens, dout, vocab, scale):
    g = np.zeros((vocab, dout.shape[1]))
    for t, v in enumerate(tokens):
        if 0 <= v < vocab:
            g[v] += scale * np.asarray(dout[t], np.float64)
    return g
