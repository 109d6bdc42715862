"""Pins of the oracle of packed attention, RMS norm, distillation and embedding: torch's own fp64 operators with
autograd, and central differences of the written-out values."""
import numpy as np
import pytest
import torch
import torch.nn.functional as F

from oracle import train_ops as to


def _t(a):
    return torch.tensor(np.asarray(a), dtype=torch.float64, requires_grad=True)


def _differences(f, x, g, rng, n=12, h=1e-5):
    """f(x) against its gradient g at n places"""
    for _ in range(n):
        i = tuple(rng.integers(0, s) for s in x.shape)
        a, b = x.copy(), x.copy()
        a[i] += h
        b[i] -= h
        d = (f(a) - f(b)) / (2 * h)
        assert abs(d - g[i]) <= 1e-7 * max(1.0, abs(d)), (i, d, g[i])


@pytest.mark.parametrize("lens,H,Hk,causal,window", [([5, 0, 1, 9], 4, 2, 1, 0), ([7, 3], 3, 3, 0, 0), ([12], 4, 1, 1, 3)])
def test_attention(lens, H, Hk, causal, window):
    rng = np.random.default_rng(3)
    D, starts = 8, np.concatenate([[2], 2 + np.cumsum(lens)])
    T = int(starts[-1]) + 3
    q, k, v = rng.normal(size=(T, H, D)), rng.normal(size=(T, Hk, D)), rng.normal(size=(T, Hk, D))
    do = rng.normal(size=(T, H, D))
    r = to.attention(q, k, v, starts, 0.3, causal, window, do)
    tq, tk, tv = _t(q), _t(k), _t(v)
    total = 0.0
    for a, b in zip(starts[:-1], starts[1:]):
        n = int(b - a)
        if n == 0:
            continue
        mask = torch.ones(n, n).tril(0 if causal else n).bool()
        if window:
            mask &= ~torch.ones(n, n).tril(-window).bool()
        rep = lambda t: t[a:b].repeat_interleave(H // Hk, 1).transpose(0, 1)
        o = F.scaled_dot_product_attention(tq[a:b].transpose(0, 1), rep(tk), rep(tv), attn_mask=mask, scale=0.3).transpose(0, 1)
        assert np.abs(o.detach().numpy() - r["o"][a:b]).max() < 1e-12
        s = (tq[a:b].transpose(0, 1) @ rep(tk).transpose(1, 2) * 0.3).masked_fill(~mask, -np.inf)
        assert np.abs(torch.logsumexp(s, -1).detach().numpy() - r["lse"][:, a:b]).max() < 1e-12
        total = total + (o * torch.tensor(do[a:b])).sum()
    total.backward()
    on = slice(int(starts[0]), int(starts[-1]))
    for name, t in (("dq", tq), ("dk", tk), ("dv", tv)):
        assert np.abs(t.grad.numpy()[on] - r[name][on]).max() < 1e-12, name
        assert np.isnan(r[name][:2]).all() and np.isnan(r[name][on.stop:]).all()
    f = lambda kk: float(np.nansum(to.attention(q, kk, v, starts, 0.3, causal, window)["o"] * do))
    g = np.nan_to_num(r["dk"])
    _differences(f, k, g, rng)


@pytest.mark.parametrize("with_res", [False, True])
def test_rmsnorm(with_res):
    rng = np.random.default_rng(4)
    x, gamma, du = rng.normal(size=(6, 24)), rng.normal(size=24), rng.normal(size=(6, 24))
    res = rng.normal(size=(6, 24)) if with_res else None
    s, rho, u = to.rmsnorm_fwd(x, res, gamma, 1e-3)
    tx, tg = _t(x if res is None else x + res), _t(gamma)
    y = F.rms_norm(tx, (24,), tg, 1e-3)
    assert np.abs(y.detach().numpy() - u).max() < 1e-12
    (y * torch.tensor(du)).sum().backward()
    dres = rng.normal(size=(6, 24))
    dh, dgamma = to.rmsnorm_bwd(du, s, rho, gamma, dres)
    assert np.abs(tx.grad.numpy() + dres - dh).max() < 1e-12 and np.abs(tg.grad.numpy() - dgamma).max() < 1e-12
    _differences(lambda t: float((to.rmsnorm_fwd(t, None, gamma, 1e-3)[2] * du).sum()), s, dh - dres, rng)


@pytest.mark.parametrize("tau", [1.0, 2.5])
def test_distill(tau):
    rng = np.random.default_rng(5)
    T, V, k = 7, 30, 4
    z, top = rng.normal(size=(T, V)) * 2, rng.normal(size=(T, k)) * 3
    ids = np.stack([rng.permutation(V)[:k] for _ in range(T)])
    ids[1, 2:] = [-1, V]                       # unused entries
    ids[2] = -1                                # none at all
    ids[3, 1] = ids[3, 0]                      # one id twice
    top[4, 0] = -np.inf
    labels = np.array([3, -1, 5, V, 0, 2, 9])
    w = np.array([0.5, 1.0, 0.25, 2.0, 1.0, 0.0, 1.0])
    loss_tok, loss, dz = to.distill(z, ids, top, tau, 0.7, labels, 0.3, w)
    tz = _t(z)
    total = 0.0
    for t in range(T):
        if w[t] == 0:
            assert loss_tok[t] == 0 and not dz[t].any()
            continue
        ok = (ids[t] >= 0) & (ids[t] < V) & (top[t] > -np.inf)
        l = torch.zeros((), dtype=torch.float64)
        if ok.any():
            p = torch.zeros(V, dtype=torch.float64)
            pj = torch.softmax(torch.tensor(top[t][ok] / tau), -1)
            p.index_add_(0, torch.tensor(ids[t][ok]), pj)
            # sum_j p_j log p_j over the entries (an id given twice keeps its two entropy terms)
            cross = -(p * F.log_softmax(tz[t] / tau, -1)).sum()
            l = l + 0.7 * tau ** 2 * (cross + (pj * pj.log()).sum())
        if 0 <= labels[t] < V:
            l = l + 0.3 * F.cross_entropy(tz[t][None], torch.tensor([labels[t]]))
        assert abs(float(l.detach()) - loss_tok[t]) < 1e-12
        total = total + w[t] * l
    total.backward()
    assert abs(float(total.detach()) - loss) < 1e-12 and np.abs(tz.grad.numpy() - dz).max() < 1e-12
    _differences(lambda x: to.distill(x, ids, top, tau, 0.7, labels, 0.3, w)[1], z, dz, rng)


def test_embed():
    rng = np.random.default_rng(6)
    table, dout = rng.normal(size=(9, 8)), rng.normal(size=(11, 8))
    tokens = np.array([3, 3, -1, 0, 8, 9, 3, 1 << 30, 0, 2, -(1 << 31)])
    tt = _t(table)
    ok = (tokens >= 0) & (tokens < 9)
    y = F.embedding(torch.tensor(np.where(ok, tokens, 0)), tt) * 1.5 * torch.tensor(ok)[:, None]
    assert np.abs(y.detach().numpy() - to.embed_fwd(tokens, table, 1.5)).max() == 0
    (y * torch.tensor(dout)).sum().backward()
    assert np.abs(tt.grad.numpy() - to.embed_bwd(tokens, dout, 9, 1.5)).max() < 1e-12
