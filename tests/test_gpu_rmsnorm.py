"""RMS norm with the residual's addition on the GPU against the fp64 oracle, element by element.

Bounds: a result in bf16 is off by 2^-8 of itself, one in fp32 by 2^-24, and the fp32 arithmetic before it by n 2^-24 of the absolute sums,
n = the longest chain of additions (d / 64 + 8 within a row, T over the rows for dgamma), plus 16 roundings of factors."""
import numpy as np
import pytest

from oracle import train_ops as to
from paper_2407_00952_amd import binding as B
from paper_2407_00952_amd import synth
from gpu_util import say

pytestmark = pytest.mark.gpu
E24 = 2.0 ** -24
UB = {"bf16": 2.0 ** -8, "fp32": E24}


def run(T, d, res, codes, extra=0, dgamma=True, dres=True, in_place=False, eps=1e-5, scale=1.0, seed=1):
    import torch
    rng = np.random.default_rng(seed)
    f = lambda *s: rng.standard_normal(s).astype(np.float32)
    rt = torch.float32 if res == "fp32" else torch.bfloat16
    ty = B.DTYPE_F32 if res == "fp32" else B.DTYPE_BF16
    rnd = (lambda a: a) if res == "fp32" else synth.round_bf16
    x, gamma = synth.round_bf16(f(T, d) * np.float32(scale)), synth.round_bf16(1 + 0.3 * f(d))
    x[::3, d // 2] *= 16
    r = None if res is None else rnd(2 * f(T, d) * np.float32(scale))
    du, dr = synth.round_bf16(f(T, d)), None if (res is None or not dres) else rnd(f(T, d))

    def strided(a):
        t = torch.full((T, d + extra), 7.0, dtype=torch.bfloat16, device="cuda")
        t[:, :d] = B.to_device_bf16(a)
        return t

    dev = lambda a: None if a is None else torch.from_numpy(a).cuda().to(rt)
    tx, tg, tdu = strided(x), B.to_device_bf16(gamma), strided(du)
    tr, tdr = dev(r), dev(dr)
    h = None if r is None else (tr if in_place else torch.empty_like(tr))
    u = torch.full((T, d + extra), 7.0, dtype=torch.bfloat16, device="cuda")
    q = torch.zeros((T, d), dtype=torch.uint8, device="cuda") if codes else None
    qs = torch.zeros((T, d // 32), dtype=torch.uint8, device="cuda") if codes else None
    rho = torch.zeros(T, dtype=torch.float32, device="cuda")
    B.slora_rmsnorm_fwd(T, d, ty, tx, d + extra, tr, tg, eps, h, u, d + extra, q, qs, rho)
    nws = B.slora_rmsnorm_bwd_ws_bytes(T, d)
    ws = torch.full((nws,), 0xFF, dtype=torch.uint8, device="cuda")
    hh = tx[:, :d].contiguous() if h is None else h
    dh = tdr if in_place and tdr is not None else torch.zeros((T, d), dtype=rt if res else torch.bfloat16, device="cuda")
    dx = torch.full((T, d + extra), 7.0, dtype=torch.bfloat16, device="cuda")
    dg = torch.full((d,), 7.0, dtype=torch.float32, device="cuda") if dgamma else None
    B.slora_rmsnorm_bwd(T, d, ty, tdu, d + extra, hh, rho, tg, tdr, dh, dx, d + extra, dg, ws if dgamma else None, nws)
    torch.cuda.synchronize()
    if extra:
        assert bool((u[:, d:] == 7.0).all()) and bool((dx[:, d:] == 7.0).all())
    if codes:
        # the codes are those of the bf16 result, bit for bit
        cq, cs = torch.zeros_like(q), torch.zeros_like(qs)
        B.slora_mx_quantize(T, d, u[:, :d].contiguous(), d, cq, cs)
        torch.cuda.synchronize()
        assert torch.equal(cq, q) and torch.equal(cs, qs)
    n = lambda t: t.float().cpu().numpy().astype(np.float64)
    s, rh, uu = to.rmsnorm_fwd(x, r, gamma, eps)
    worst = {}

    def hold(name, got, ref, lim):
        worst[name] = float(np.nan_to_num(np.abs(got - ref) / (lim + 1e-300), nan=np.inf).max())

    chain = (d / 64 + 24) * E24
    hold("u", n(u[:, :d]), uu, (UB["bf16"] + chain) * np.abs(uu))
    hold("rho", n(rho), rh, chain * rh)
    if h is not None:
        hold("h", n(h), s, UB[res] * np.abs(s))
    # the backward from what the forward stored
    hn, rn = n(hh), n(rho)
    odh, odg = to.rmsnorm_bwd(du, hn, rn, gamma, dr)
    xh, g = np.abs(hn * rn[:, None]), np.abs(du.astype(np.float64) * gamma)
    size = rn[:, None] * (g + xh * (g * xh).mean(1, keepdims=True)) + (0 if dr is None else np.abs(dr))
    hold("dh", n(dh), odh, UB[res or "bf16"] * np.abs(odh) + chain * size)
    hold("dx", n(dx[:, :d]), odh, UB["bf16"] * np.abs(odh) + chain * size)
    if dgamma:
        hold("dgamma", n(dg), odg, (T + 16) * E24 * (np.abs(du) * xh).sum(0))
    say("   T=%d d=%d %s: errors over their bounds %s" % (T, d, res, {k: "%.2f" % v for k, v in worst.items()}))
    assert all(w <= 1.0 for w in worst.values()), worst


# every kernel width (chunks x threads of a row) at its ends, one row, rows that fill no block
@pytest.mark.parametrize("T,d,res,codes", [
    (1, 8, None, False), (1, 32, "bf16", True), (3, 64, "fp32", True), (5, 504, "bf16", False), (7, 512, None, True), (4, 520, "fp32", False),
    (9, 1024, "fp32", True), (6, 1032, "bf16", False), (2, 1536, "bf16", True), (5, 1600, None, True), (3, 2048, "fp32", True),
    (3, 2056, "fp32", False), (2, 4096, "bf16", True), (3, 4128, "fp32", True), (2, 6144, None, False), (2, 6176, "bf16", True),
    (3, 8192, "fp32", False), (2, 8200, "bf16", False), (2, 12288, "fp32", True), (2, 12296, None, False), (1, 16384, "bf16", True),
    (3, 120, "bf16", False), (17, 128, "fp32", True), (33, 136, None, False), (15, 160, "fp32", True), (23, 256, "bf16", True),
    (9, 264, "fp32", False), (2, 16, None, False), (10007, 128, None, False), (5003, 224, "bf16", True),
    (4099, 96, "bf16", True), (9001, 64, "fp32", False), (1500, 2080, "bf16", False)])
def test_against_the_oracle(T, d, res, codes):
    run(T, d, res, codes)


def test_strides_and_partial_calls():
    run(37, 256, "fp32", True, extra=24, dgamma=False)
    run(37, 256, "bf16", False, extra=8, dres=False)
    run(5, 2304, None, True, extra=16)


def test_in_place_residual_stream():
    run(33, 1024, "fp32", True, in_place=True)
    run(33, 4096, "bf16", False, in_place=True)


def test_tiny_and_huge_rows():
    run(5, 256, "fp32", False, scale=1e-12, eps=1e-30)
    run(5, 256, "bf16", True, scale=1e12)
    run(5, 256, "bf16", True, scale=2.0 ** -60, eps=0.0)


def test_zero_row_and_no_rows():
    import torch
    d = 64
    x, g = torch.zeros((2, d), dtype=torch.bfloat16, device="cuda"), torch.ones(d, dtype=torch.bfloat16, device="cuda")
    u, q, s = torch.ones_like(x), torch.ones((2, d), dtype=torch.uint8, device="cuda"), torch.ones((2, 2), dtype=torch.uint8, device="cuda")
    B.slora_rmsnorm_fwd(2, d, B.DTYPE_BF16, x, d, None, g, 1e-5, None, u, d, q, s, None)
    dg = torch.ones(d, dtype=torch.float32, device="cuda")
    n = B.slora_rmsnorm_bwd_ws_bytes(0, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.slora_rmsnorm_bwd(0, d, B.DTYPE_BF16, x, d, x, dg, g, None, u, None, 0, dg, ws, n)
    torch.cuda.synchronize()
    assert not u.any() and not q.any() and not s.any() and not dg.any()
