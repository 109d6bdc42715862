"""Packed attention where scores are large, against the fp64 oracle.

Rounding of scores, with E = 2^-24 |lse|.  Forward: the exponent s c - m of an element is rounded once and the maximum m is the same for a
row, so o is as exact as with small scores; lse = (m + log2 l) ln 2 passes three roundings (four where scores are multiplied and rounded
before their maximum is taken) and two rounded constants, 4 E (5 E) together.
Backward: P is formed from lse, which is multiplied by a rounded constant and rounded once more (2 E): P is off by a factor of
exp(+-6 E), the same for all keys of a query, and never above 1."""
import numpy as np
import pytest

from oracle import train_ops as to
from paper_2407_00952_amd import synth
from gpu_util import say
from test_gpu_attention_packed import FP32, U, Call, bounds, make

pytestmark = pytest.mark.gpu


def run(q, k, v, do, starts, scale, causal, window):
    c = Call(q, k, v, do, starts, scale, causal, window, "dense")
    c.fwd()
    c.bwd()
    return c.results()


def over(got, ref, lim):
    return float(np.nan_to_num(np.abs(got - ref) / (lim + 1e-300), nan=np.inf).max())


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("common", [1 << 10, 1 << 14, -(1 << 14), 1 << 17, 1 << 20])
def test_a_large_common_part(common, D):
    """Scores of `common` and some units: P does not depend on `common`, only its rounding does.  Products and sums of q k are
    multiples of 1/4 below 2^21, so exact in fp32."""
    starts, H, Hk, T = np.array([0, 70, 71, 300]), 2, 1, 300
    rng = np.random.default_rng(D + 1)
    _, _, v, do = make(T, H, Hk, D, 5)
    q, k = np.zeros((T, H, D), np.float32), np.zeros((T, Hk, D), np.float32)
    q[..., :16] = 2.0 ** np.ceil(np.log2(abs(common) / 16) / 2)
    k[..., :16] = common / 16 / q[0, 0, 0]
    q[..., 16:32], k[..., 16:32] = rng.integers(-2, 3, (T, H, 16)), rng.integers(-2, 3, (T, Hk, 16)) * 0.25
    assert (synth.round_bf16(q) == q).all() and (synth.round_bf16(k) == k).all()
    ref = to.attention(q, k, v, starts, 1.0, 1, 0, do)
    got, lim = run(q, k, v, do, starts, 1.0, 1, 0), bounds(q, k, v, do, starts, 1.0, 1, 0, ref, 2.0 ** -16)
    E = 2.0 ** -24 * np.abs(ref["lse"]).max()
    p_off = np.expm1(6 * E)
    # P off by a factor: dv by p_off P^T |do|, dq and dk by p_off of sum |dS| |k|, sum |dS| |q|
    for a, z in zip(starts[:-1], starts[1:]):
        see = to.visible(z - a, 1, 0)
        for h in range(H):
            p = np.where(see, np.exp((q[a:z, h] @ k[a:z, 0].astype(np.float64).T) - ref["lse"][h, a:z][:, None]), 0.0)
            ds = np.abs(p * (do[a:z, h] @ v[a:z, 0].astype(np.float64).T - (do[a:z, h] * ref["o"][a:z, h]).sum(1, keepdims=True)))
            lim["dv"][a:z, 0] += p_off * (p.T @ np.abs(do[a:z, h]))
            lim["dq"][a:z, h] += p_off * (ds @ np.abs(k[a:z, 0]))
            lim["dk"][a:z, 0] += p_off * (ds.T @ np.abs(q[a:z, h]))
    worst = {n: over(got[n], ref[n], lim[n]) for n in ("o", "dq", "dk", "dv")}
    worst["lse"] = float(np.abs(got["lse"] - ref["lse"]).max() / (2.0 ** -16 + 4 * E))
    say("   scores around %g, D=%d: errors over their bounds %s" % (common, D, {n: "%.2f" % w for n, w in worst.items()}))
    assert all(w <= 1 for w in worst.values()), worst


@pytest.mark.parametrize("lens,D,causal,window", [([300, 1, 64], 64, 1, 0), ([200, 130], 128, 1, 0), ([257], 64, 0, 0),
                                                  ([400, 33], 64, 1, 40), ([330], 128, 1, 129)])
@pytest.mark.parametrize("size", [1e6, 1e8, 1e10, 1e30, -1e10, -1e30])
def test_far_scores(size, lens, D, causal, window):
    """Scores that are 0 or `size` (keys along the axes, a query along one of them): each query takes the keys of the larger score that it
    sees in equal parts.  Exact in the forward whatever the size; the backward's P lies between 0 and 1, so that |dv| <= sum |do|, and
    results are finite."""
    starts = np.concatenate([[0], np.cumsum(lens)])
    T, H, Hk = int(starts[-1]), 4, 2
    rng = np.random.default_rng(T + D)
    _, _, v, do = make(T, H, Hk, D, 6)
    q, k = np.zeros((T, H, D), np.float32), np.zeros((T, Hk, D), np.float32)
    at = np.arange(T)
    q[at[:, None], np.arange(H), rng.integers(0, D, (T, H))] = 1.0
    k[at[:, None], np.arange(Hk), rng.integers(0, D, (T, Hk))] = np.sign(size)
    q[at % 7 == 3] *= 201.0 / 128                             # (scores that are no powers of two: products that are rounded)
    scale = float(np.float32(abs(size)))
    ref = to.attention(q, k, v, starts, scale, causal, window, do)
    got = run(q, k, v, do, starts, scale, causal, window)
    lim_o, most_dv = np.zeros(ref["o"].shape), np.zeros(ref["dv"].shape)
    for a, z in zip(starts[:-1], starts[1:]):
        see = to.visible(z - a, causal, window)
        for h in range(H):
            p = np.where(see, np.exp(scale * (q[a:z, h].astype(np.float64) @ k[a:z, h // 2].T) - ref["lse"][h, a:z][:, None]), 0.0)
            p /= p.sum(1, keepdims=True)                      # (at 1e30 lse of 64 bits leaves no digit of P)
            lim_o[a:z, h] = (U + FP32) * (np.abs(ref["o"][a:z, h]) + p @ np.abs(v[a:z, h // 2]))
            most_dv[a:z, h // 2] += see.T @ np.abs(do[a:z, h])
    worst = {"o": over(got["o"], ref["o"], lim_o), "dv": over(got["dv"], 0.0, most_dv * (1 + U + FP32)),
             "lse": over(got["lse"], ref["lse"], 2.0 ** -16 + 5 * 2.0 ** -24 * np.abs(ref["lse"]))}
    say("   scores of %g, D=%d: over their bounds %s" % (size, D, {n: "%.2f" % w for n, w in worst.items()}))
    assert all(w <= 1 for w in worst.values()), worst
    assert np.isfinite(got["dq"]).all() and np.isfinite(got["dk"]).all()
