"""Distillation loss on the GPU against the fp64 oracle, element by element.

Bounds: an exponential's argument (z - max) log2(e) / tau is off by 2^-22 of its size, log-sum-exp by 2^-22 of its own size and the sums'
chains (V / 1024 + 16 additions) by 2^-24 each, so a probability q is off by r = 2^-22 (|z - max| / tau + |log q| + 8) + (V / 1024 + 16) 2^-24
of itself; a gradient of bf16 by 2^-8 of itself on top."""
import numpy as np
import pytest

from oracle import train_ops as to
from paper_2407_00952_amd import binding as B
from paper_2407_00952_amd import synth
from gpu_util import say

pytestmark = pytest.mark.gpu
MARK = 5.0


def inputs(T, V, k, seed, dtype):
    rng = np.random.default_rng(seed)
    z = (rng.standard_normal((T, V)) * 2).astype(np.float32)
    ids = np.stack([rng.permutation(V)[:k] if k <= V else rng.integers(0, V, k) for _ in range(T)]).astype(np.int32)
    top = (8 + 3 * rng.standard_normal((T, k))).astype(np.float32)
    np.put_along_axis(z, ids.astype(np.int64), np.take_along_axis(z, ids.astype(np.int64), 1) + 2, 1)
    if dtype == "bf16":
        z = synth.round_bf16(z)
    labels = rng.integers(0, V, T).astype(np.int32)
    w = rng.uniform(0.5, 1.5, T).astype(np.float32) / T
    return z, ids, top, labels, w


def gpu(z, ids, top, tau, kd, labels, ce, w, dtype="fp32", pad=(0, 0), offset=0, grad=True, in_place=False):
    """pad: elements behind a row of the logits and of the gradient; offset: elements in front of both buffers"""
    import torch
    T, V = z.shape
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16

    def buf(extra):
        flat = torch.full((offset + T * (V + extra) + 64,), MARK, dtype=dt, device="cuda")
        return flat, flat[offset:offset + T * (V + extra)].view(T, V + extra)

    zf, zt = buf(pad[0])
    zt[:, :V] = torch.from_numpy(z).cuda()
    gf, gt = (zf, zt) if in_place else buf(pad[1])
    dev = lambda a: None if a is None else torch.from_numpy(a).cuda()
    loss_tok = torch.full((T,), MARK, dtype=torch.float32, device="cuda")
    loss = torch.full((1,), MARK, dtype=torch.float32, device="cuda")
    B.slora_distill_loss(T, V, B.DTYPE_F32 if dtype == "fp32" else B.DTYPE_BF16, zt, zt.shape[1], ids.shape[1], dev(ids), dev(top), tau,
                         kd, dev(labels), ce, dev(w), loss_tok, loss, gt if grad else None, gt.shape[1])
    torch.cuda.synchronize()
    assert bool((gt[:, V:] == MARK).all()) and bool((gf[:offset] == MARK).all()) and bool((gf[offset + gt.numel():] == MARK).all())
    if not grad:
        assert bool((gt == MARK).all())
    return loss_tok.cpu().numpy().astype(np.float64), float(loss), gt[:, :V].float().cpu().numpy().astype(np.float64)


def check(z, ids, top, tau, kd, labels, ce, w, dtype="fp32", label="", **kw):
    T, V = z.shape
    lt, loss, dz = gpu(z, ids, top, tau, kd, labels, ce, w, dtype, **kw)
    olt, oloss, odz = to.distill(z, ids, top, tau, kd, labels, ce, w)
    ww = np.full(T, 1.0 / T) if w is None else w.astype(np.float64)
    zz = z.astype(np.float64)
    zz = np.where(ww[:, None] == 0, 0.0, zz)                  # (rows of weight 0 have the value 0 and, times their weight, the bound 0)
    m = zz.max(1, keepdims=True)
    chain = (V / 1024 + 16) * 2.0 ** -24
    lim, scale_tok = np.zeros((T, V)), np.zeros(T)
    for t_, f in ((tau, kd * tau), (1.0, ce)):
        a = np.maximum(m - zz, 0) / t_
        a = np.where(np.isfinite(a), a, 0.0)
        q = np.exp(np.where(np.isfinite(zz), -a, -np.inf))
        s = q.sum(1, keepdims=True)
        lq = a + np.log(s)
        lim += ww[:, None] * f * (q / s) * (2.0 ** -22 * (a + lq + 8) + chain)
        size = np.abs(m[:, 0]) / t_ + np.log(s)[:, 0] + 8
        scale_tok += (kd * tau * tau if f == kd * tau and t_ == tau else 0) * size + (ce if t_ == 1.0 else 0) * size
    # the teacher's own probabilities: off by the same rule, their spread below 2^6
    np.add.at(lim, (np.arange(T)[:, None], np.where((ids >= 0) & (ids < V), ids, 0)), (ww * kd * tau)[:, None] * 2.0 ** -22 * 80)
    if labels is not None:
        lim[np.arange(T), np.clip(labels, 0, V - 1)] += ww * ce * 2.0 ** -22
    if dtype == "bf16":
        lim += 2.0 ** -8 * np.abs(odz)
    tmax = np.where((ids >= 0) & (ids < V) & np.isfinite(top), np.abs(top), 0).max(1) / tau
    lim_tok = 2.0 ** -21 * (scale_tok + kd * tau * tau * (tmax + 8)) * (ww != 0)
    rg = np.nan_to_num(np.abs(dz - odz) / (lim + 1e-30), nan=np.inf).max()
    rt = np.nan_to_num(np.abs(lt - olt) / (lim_tok + 1e-30), nan=np.inf).max()
    rl = abs(loss - oloss) / ((np.abs(ww) * lim_tok).sum() + 2.0 ** -23 * abs(oloss) + 1e-30)
    say("   %s T=%d V=%d k=%d tau=%g: errors over their bounds: gradient %.2f, rows %.2f, loss %.2f" % (label, T, V, ids.shape[1], tau, rg, rt, rl))
    assert rg <= 1 and rt <= 1 and rl <= 1


@pytest.mark.parametrize("T,V,k,tau,kd,ce,dtype,pad,offset", [
    (1, 1, 1, 1.0, 1.0, 1.0, "fp32", (0, 0), 0),
    (3, 7, 3, 2.0, 0.5, 0.5, "bf16", (0, 0), 1),
    (5, 50, 50, 1.0, 1.0, 0.0, "bf16", (6, 14), 0),
    (4, 1000, 20, 4.0, 1.0, 0.25, "fp32", (24, 0), 0),
    (6, 1003, 8, 0.5, 1.0, 1.0, "bf16", (0, 0), 3),            # dense odd rows: every alignment
    (6, 1003, 8, 2.0, 1.0, 1.0, "fp32", (0, 1), 1),            # the gradient's rows aligned unlike the logits'
    (5, 4096, 64, 1.0, 0.7, 0.3, "bf16", (0, 0), 0),
    (5, 4097, 64, 2.0, 0.7, 0.3, "bf16", (0, 3), 5),
    (3, 8193, 5, 2.0, 1.0, 0.0, "fp32", (0, 0), 0),
    (3, 16385, 100, 1.0, 1.0, 0.5, "fp32", (7, 0), 0),
    (2, 50257, 1024, 2.0, 1.0, 0.5, "bf16", (0, 0), 0),
    (2, 65536, 3, 2.0, 1.0, 0.5, "bf16", (0, 0), 0),
    (2, 65545, 3, 2.0, 1.0, 0.5, "bf16", (0, 0), 0),
    (2, 131073, 700, 1.5, 1.0, 0.5, "bf16", (0, 0), 2),
    (2, 65537, 9, 2.0, 1.0, 0.5, "fp32", (0, 0), 0),
    (2, 140001, 9, 2.0, 1.0, 0.5, "fp32", (3, 3), 1),
])
def test_against_the_oracle(T, V, k, tau, kd, ce, dtype, pad, offset):
    z, ids, top, labels, w = inputs(T, V, k, V + k, dtype)
    check(z, ids, top, tau, kd, labels, ce, w, dtype, "plain", pad=pad, offset=offset)


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_rows_with_missing_parts(dtype):
    """No used entry, no label, neither; ids outside the vocabulary, one id in several entries, the label among them; weights of 0
    on rows that hold NaN; teacher logits of -inf; masked words of -inf and of the type's lowest value."""
    T, V, k = 12, 600, 6
    z, ids, top, labels, w = inputs(T, V, k, 40, dtype)
    ids[0] = -1
    labels[1] = -1
    ids[2], labels[2] = [V, -1, 2 ** 31 - 1, -2 ** 31, V + 1, -5], V
    ids[3, 3:] = -1
    top[3, 3:] = np.nan
    ids[4, [0, 2, 5]] = ids[4, 1]
    labels[5] = ids[5, 2]
    ids[6] = ids[6, 0]
    labels[6] = ids[6, 0]
    w[7], z[7], top[7] = 0.0, np.nan, np.nan
    top[8, 1:] = -np.inf
    top[9] = -np.inf
    keep = np.concatenate([ids[10], [labels[10]]])
    rest = np.setdiff1d(np.arange(V), keep)
    z[10, rest[:300]] = -np.inf
    low = -3.0e38 if dtype == "fp32" else float(synth.round_bf16(np.array([-3.0e38], np.float32))[0])
    rest = np.setdiff1d(np.arange(V), np.concatenate([ids[11], [labels[11]]]))
    z[11, rest[:300]] = low
    for tau in (1.0, 2.0, 0.5):
        check(z, ids, top, tau, 0.6, labels, 0.4, w, dtype, "missing parts")
        check(z, ids, top, tau, 0.6, None, 0.4, w, dtype, "no labels")


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("V,pad,offset", [(1, (0, 0), 0), (3, (0, 0), 1), (7, (0, 2), 1), (17, (0, 0), 3), (100, (3, 1), 2), (1003, (0, 0), 5),
                                          (4099, (0, 5), 0)])
def test_rows_of_weight_zero_at_every_alignment(V, pad, offset, dtype):
    T, k = 18, 1
    z, ids, top, labels, w = inputs(T, V, k, V, dtype)
    w[::2], z[::2] = 0.0, np.nan
    check(z, ids, top, 2.0, 0.6, labels, 0.4, w, dtype, "weights of 0", pad=pad, offset=offset)


def test_row_of_masked_words_only_and_huge_logits():
    z, ids, top, labels, w = inputs(3, 100, 4, 41, "fp32")
    z[1] = -np.inf
    z[2] = 1e30                                               # all equal: uniform
    lt, loss, dz = gpu(z, ids, top, 1.0, 1.0, labels, 1.0, w)
    assert np.isnan(lt[1]) and np.isnan(loss) and np.isnan(dz[1]).all()
    assert abs(lt[2] - to.distill(np.zeros((1, 100)), ids[2:], top[2:], 1.0, 1.0, labels[2:], 1.0, None)[0][0]) < 1e-4
    assert np.isfinite(dz[[0, 2]]).all()


def test_loss_alone_in_place_and_equal_weights():
    for dtype in ("fp32", "bf16"):
        z, ids, top, labels, w = inputs(9, 777, 5, 42, dtype)
        a = gpu(z, ids, top, 2.0, 1.0, labels, 0.5, None, dtype)
        b = gpu(z, ids, top, 2.0, 1.0, labels, 0.5, None, dtype, grad=False)
        c = gpu(z, ids, top, 2.0, 1.0, labels, 0.5, None, dtype, in_place=True)
        d = gpu(z, ids, top, 2.0, 1.0, labels, 0.5, np.full(9, np.float32(1.0) / np.float32(9)), dtype)
        assert np.array_equal(a[0], b[0]) and a[1] == b[1]
        assert np.array_equal(a[0], c[0]) and np.array_equal(a[2], c[2])
        assert np.array_equal(a[0], d[0]) and np.array_equal(a[2], d[2])
        check(z, ids, top, 2.0, 1.0, labels, 0.5, None, dtype, "equal weights")


def test_gradient_against_differences():
    z, ids, top, labels, w = inputs(4, 90, 5, 43, "fp32")
    _, _, dz = gpu(z, ids, top, 2.0, 1.0, labels, 0.5, w)
    rng = np.random.default_rng(1)
    d = rng.standard_normal(z.shape).astype(np.float32) * np.float32(0.05)
    hi, lo = (z + d).astype(np.float32), (z - d).astype(np.float32)
    f = lambda x: gpu(x, ids, top, 2.0, 1.0, labels, 0.5, w, grad=False)[1]
    g = lambda x: to.distill(x, ids, top, 2.0, 1.0, labels, 0.5, w)[1]
    step = hi.astype(np.float64) - lo
    curve = abs(g(hi) - g(lo) - (to.distill(z, ids, top, 2.0, 1.0, labels, 0.5, w)[2] * step).sum())
    assert abs(f(hi) - f(lo) - (dz * step).sum()) <= curve + 2.0 ** -20 * 20
