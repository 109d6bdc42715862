"""Embedding lookup and the gradient of its table on the GPU: the lookup bit for bit (one fp32 product, one rounding), the gradient
against the fp64 oracle with n 2^-24 of the absolute sum, n = the occurrences of the token + 4."""
import numpy as np
import pytest

from oracle import train_ops as to
from paper_2407_00952_amd import binding as B
from paper_2407_00952_amd import synth
from gpu_util import say

pytestmark = pytest.mark.gpu


def tokens_of(kind, T, V, rng):
    if kind == "uniform":
        t = rng.integers(0, V, T)
    elif kind == "zipf":
        t = np.minimum(np.exp(rng.uniform(size=T) * np.log(V + 1)).astype(np.int64) - 1, V - 1)
    elif kind == "one":
        t = np.full(T, V - 1)
    elif kind == "two":
        t = np.where(np.arange(T) < T // 2 + 7, 0, V - 1)
    else:                                                     # nothing but padding
        t = np.where(np.arange(T) % 2 == 0, -1, V)
    t = t.astype(np.int64)
    if kind in ("uniform", "zipf") and T > 4:
        t[rng.integers(0, T, max(T // 20, 1))] = rng.choice([-1, V, 2 ** 31 - 1, -2 ** 31], max(T // 20, 1))
    return t.astype(np.int32)


def run(T, V, d, dtype, kind, scale=1.5, extra=0, seed=2):
    import torch
    rng = np.random.default_rng(seed)
    tok = tokens_of(kind, T, V, rng)
    dt = torch.float32 if dtype == "fp32" else torch.bfloat16
    ty = B.DTYPE_F32 if dtype == "fp32" else B.DTYPE_BF16
    rnd = (lambda a: a) if dtype == "fp32" else synth.round_bf16
    table, dout = rnd(rng.standard_normal((V, d)).astype(np.float32)), rnd(rng.standard_normal((T, d)).astype(np.float32))
    tt, ttok = torch.from_numpy(table).cuda().to(dt), torch.from_numpy(tok).cuda()
    pad = (tok < 0) | (tok >= V)
    dout[pad] = np.nan                                        # rows of padding are not read
    td = torch.full((T, d + extra), float("nan"), dtype=dt, device="cuda")
    td[:, :d] = torch.from_numpy(dout).cuda().to(dt)
    out = torch.full((T, d + extra), 9.0, dtype=dt, device="cuda")
    B.slora_embed_fwd(T, V, d, ty, ttok, tt, scale, out, d + extra)
    g = torch.full((V, d), 9.0, dtype=torch.float32, device="cuda")
    n = B.slora_embed_bwd_ws_bytes(T, V, d)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    B.slora_embed_bwd(T, V, d, ty, ttok, td, d + extra, scale, 0, g, ws, n)
    before = torch.from_numpy(rng.standard_normal((V, d)).astype(np.float32)).cuda()
    acc = before.clone()
    B.slora_embed_bwd(T, V, d, ty, ttok, td, d + extra, scale, 1, acc, ws, n)
    torch.cuda.synchronize()
    ref = np.where(pad[:, None], np.float32(0), table[np.where(pad, 0, tok)] * np.float32(scale)).astype(np.float32)
    assert np.array_equal(out[:, :d].float().cpu().numpy(), rnd(ref)) and bool((out[:, d:] == 9.0).all())
    dout[pad] = 0.0
    count = np.bincount(tok[~pad], minlength=V)[:, None]
    size = to.embed_bwd(tok, np.abs(dout), V, abs(scale))
    want = to.embed_bwd(tok, dout, V, scale)
    got, plus, old = (t.cpu().numpy().astype(np.float64) for t in (g, acc, before))
    lim = (count + 4) * 2.0 ** -24
    e = np.nan_to_num(np.abs(got - want) / (lim * size + 1e-30), nan=np.inf).max()
    e2 = np.nan_to_num(np.abs(plus - old - want) / (lim * (size + np.abs(old)) + 1e-30), nan=np.inf).max()
    say("   %s T=%d V=%d d=%d %s: errors over their bounds %.2f, added %.2f" % (kind, T, V, d, dtype, e, e2))
    assert e <= 1 and e2 <= 1
    absent = count[:, 0] == 0
    assert not got[absent].any() and np.array_equal(plus[absent], old[absent])


@pytest.mark.parametrize("T,V,d,dtype,kind", [
    (1, 1, 8, "fp32", "uniform"), (1, 300, 64, "bf16", "uniform"), (37, 50257, 64, "bf16", "zipf"), (64, 7, 520, "fp32", "zipf"),
    (65, 255, 8, "bf16", "uniform"), (1000, 256, 72, "fp32", "uniform"), (1023, 257, 64, "bf16", "zipf"), (1025, 65535, 8, "bf16", "uniform"),
    (2047, 65536, 8, "fp32", "zipf"), (2049, 65537, 16, "bf16", "uniform"), (4097, 3, 1032, "bf16", "zipf"), (5000, 1, 24, "fp32", "one"),
    (5000, 90000, 16, "bf16", "one"), (6000, 100, 64, "fp32", "two"), (300, 100, 64, "bf16", "none"), (20011, 5003, 128, "bf16", "zipf"),
    (40000, 200, 32, "fp32", "zipf"), (140001, 70001, 8, "bf16", "zipf")])
def test_against_the_oracle(T, V, d, dtype, kind):
    run(T, V, d, dtype, kind)


@pytest.mark.parametrize("T,V,d", [(70, 5, 65536), (300, 2, 4104), (129, 40, 2056)])
def test_wide_rows(T, V, d):
    run(T, V, d, "bf16", "zipf")


@pytest.mark.parametrize("T", [2000, 5000])
def test_the_largest_vocabulary(T):
    """2^24 words: one more pass of the sort than any vocabulary below, every pass over values that small integers sum exactly."""
    import torch
    V, d = 1 << 24, 8
    gen = torch.Generator(device="cuda").manual_seed(5)
    words = torch.randint(0, V, (T // 3,), generator=gen, device="cuda")
    tok = words[torch.randint(0, T // 3, (T,), generator=gen, device="cuda")].to(torch.int32)
    tok[0], tok[1], tok[2], tok[3] = V - 1, 0, V, -1
    dout = torch.randint(-8, 9, (T, d), generator=gen, device="cuda").to(torch.float32)
    n = B.slora_embed_bwd_ws_bytes(T, V, d)
    ws = torch.full((n,), 0xFF, dtype=torch.uint8, device="cuda")
    got = torch.full((V, d), 9.0, dtype=torch.float32, device="cuda")
    B.slora_embed_bwd(T, V, d, B.DTYPE_F32, tok, dout, d, 2.0, 0, got, ws, n)
    word = (tok >= 0) & (tok < V)
    want = np.zeros((V, d), np.float32)
    np.add.at(want, tok[word].cpu().numpy(), 2.0 * dout[word].cpu().numpy())
    assert np.array_equal(got.cpu().numpy(), want)
    table = torch.randint(-8, 9, (V, d), generator=gen, device="cuda").to(torch.bfloat16)
    out = torch.full((T, d), 9.0, dtype=torch.bfloat16, device="cuda")
    B.slora_embed_fwd(T, V, d, B.DTYPE_BF16, tok, table, 0.5, out, d)
    assert torch.equal(out, torch.where(word[:, None], table[torch.where(word, tok, 0).long()] * 0.5, torch.zeros_like(out)))


def test_strides_and_scales():
    run(500, 99, 200, "bf16", "zipf", scale=-0.25, extra=16)
    run(500, 99, 200, "fp32", "zipf", scale=0.0, extra=8)


def test_no_tokens_and_equal_bits():
    import torch
    g = torch.ones((5, 64), dtype=torch.float32, device="cuda")
    n = B.slora_embed_bwd_ws_bytes(0, 5, 64)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.slora_embed_bwd(0, 5, 64, B.DTYPE_BF16, ws, g, 64, 1.0, 0, g, ws, n)
    torch.cuda.synchronize()
    assert not g.any()
    T, V, d = 9000, 40, 64
    tok = torch.randint(0, V, (T,), device="cuda", dtype=torch.int32)
    x = torch.randn((T, d), dtype=torch.float32, device="cuda")
    n = B.slora_embed_bwd_ws_bytes(T, V, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    outs = []
    for fill in (0, 255):
        ws.fill_(fill)
        g = torch.empty((V, d), dtype=torch.float32, device="cuda")
        B.slora_embed_bwd(T, V, d, B.DTYPE_F32, tok, x, d, 1.0, 0, g, ws, n)
        outs.append(g)
    torch.cuda.synchronize()
    assert torch.equal(*outs)
