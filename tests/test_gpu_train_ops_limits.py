"""The operators for training other models at the ends of their ranges: the most rows, records, words and columns that a call takes."""
import pytest

from paper_2407_00952_amd import binding as B
from gpu_util import say

pytestmark = pytest.mark.gpu
U = 2.0 ** -8                                                 # half a step of bf16, relative


def gen(seed):
    import torch
    return torch.Generator(device="cuda").manual_seed(seed)


def f32(*shape):
    import torch
    return torch.empty(shape, dtype=torch.float32, device="cuda")


def worst(got, want, lim):
    import torch
    return float(torch.nan_to_num((got.double() - want).abs() / (lim + 1e-30), nan=float("inf")).max())


def test_attention_with_eight_million_records():
    """Records of two tokens (every third one has one), as many as the grid takes.  Token 1 of a record: P = (1 - p, p), so
    o = v0 + p (v1 - v0), dS = +-p (1 - p) do (v1 - v0).  P, dS and every result are rounded to bf16 (U each), exp and the sums add 2^-18."""
    import torch
    H, D, N = 1, 64, (1 << 23) - (1 << 20)
    g = gen(1)
    lens = torch.where(torch.arange(N, device="cuda") % 3 == 0, 1, 2)
    start = torch.cat([lens.new_zeros(1), lens.cumsum(0)]).to(torch.int32)
    T = int(start[-1])
    q, k, v, do = (torch.empty((T, D), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for _ in range(4))
    o, lo, dq, dk, dv = (torch.full_like(q, 77.0) for _ in range(5))
    lse = f32(1, T)
    n = B.slora_attention_bwd_ws_bytes(T, H, H, D)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    scale = 0.125
    head = (N, T, H, H, D, scale, 1, 0, q, D, k, D, v, D, start)
    B.slora_attention_fwd(*head, o, lo, D, lse)
    B.slora_attention_bwd(*head, o, lo, D, lse, do, D, dq, D, dk, D, dv, D, ws, n)
    torch.cuda.synchronize()
    bad = [0.0] * 5
    for a in range(0, N, 1 << 20):                            # a part of the records at a time, in fp64
        b = min(a + (1 << 20), N)
        two, first = lens[a:b] == 2, start[a:b].long()
        i, j = first[two], first[two] + 1
        one = first[~two]
        assert torch.equal(o[one], v[one]) and torch.equal(o[i], v[i]) and torch.equal(dv[one], do[one])
        f = lambda t, at: t[at].double()
        s0, s1 = (scale * (f(q, j) * f(k, at)).sum(1, keepdim=True) for at in (i, j))
        p = torch.sigmoid(s1 - s0)
        v0, v1, d0, d1 = f(v, i), f(v, j), f(do, i), f(do, j)
        bad[0] = max(bad[0], worst(o[j], v0 + p * (v1 - v0), 2.1 * U * ((1 - p) * v0.abs() + p * v1.abs())))
        bad[1] = max(bad[1], worst(lse[0, j, None], torch.logaddexp(s0, s1), 2.0 ** -18 * (1 + s0.abs() + s1.abs())))
        bad[2] = max(bad[2], worst(dv[i], d0 + (1 - p) * d1, 2.1 * U * (d0.abs() + (1 - p) * d1.abs())))
        ds = p * (1 - p) * (d1 * (v1 - v0)).sum(1, keepdim=True)
        # dS = P (dP - delta), delta = rowsum(do o).  o is held to 2^-16 but is the sum of rounded probabilities, (1 - p)(1 + e0) v0 +
        # p (1 + e1) v1 with |e| <= U: delta is off by (1 - p) e0 do v0 + p e1 do v1, which neither side of the difference cancels
        delta = U * ((1 - p) * (d1 * v0).sum(1, keepdim=True).abs() + p * (d1 * v1).sum(1, keepdim=True).abs())
        size = 2.1 * U * ds.abs() + delta + 2.0 ** -15 * (d1.abs() * (v0.abs() + v1.abs())).sum(1, keepdim=True)
        k0, k1, q1 = f(k, i), f(k, j), f(q, j)
        bad[3] = max(bad[3], worst(dq[j], scale * ds * (k1 - k0), scale * size * (k0.abs() + k1.abs()) + U * (scale * ds * (k1 - k0)).abs()))
        bad[4] = max(bad[4], worst(dk[j], scale * ds * q1, scale * size * q1.abs() + U * (scale * ds * q1).abs()))
    say("   attention, %d records: errors over their bounds %s" % (N, " ".join("%.2f" % x for x in bad)))
    assert max(bad) <= 1


def test_rmsnorm_with_the_most_rows():
    import torch
    T, d = (1 << 23) - 1, 8
    g = gen(2)
    x, du = (torch.empty((T, d), dtype=torch.bfloat16, device="cuda").normal_(0, 1, generator=g) for _ in range(2))
    gamma = torch.empty(d, dtype=torch.bfloat16, device="cuda").normal_(1, 0.1, generator=g)
    u, dx = torch.full_like(x, 77.0), torch.full_like(x, 77.0)
    rho, dgamma = f32(T), f32(d)
    n = B.slora_rmsnorm_bwd_ws_bytes(T, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    B.slora_rmsnorm_fwd(T, d, B.DTYPE_BF16, x, d, None, gamma, 1e-5, None, u, d, None, None, rho)
    B.slora_rmsnorm_bwd(T, d, B.DTYPE_BF16, du, d, x, rho, gamma, None, None, dx, d, dgamma, ws, n)
    torch.cuda.synchronize()
    xd, dd, gd = x.double(), du.double(), gamma.double()
    r = torch.rsqrt((xd * xd).mean(1, keepdim=True) + 1e-5)
    e_u = worst(u, xd * r * gd, 1.001 * U * (xd * r * gd).abs())
    h, t = xd * r, dd * gd
    m = (t * h).mean(1, keepdim=True)
    e_x = worst(dx, r * (t - h * m), 1.001 * U * (r * (t - h * m)).abs() + 2.0 ** -20 * r * (t.abs() + h.abs() * (t * h).abs().mean(1, keepdim=True)))
    # a lane adds a row of each 2048 to its sum, then 512 blocks of 4
    e_g = worst(dgamma, (dd * h).sum(0), (T / 2048 + 520) * 2.0 ** -24 * (dd * h).abs().sum(0))
    say("   rms norm, %d rows: errors over their bounds %.2f %.2f %.2f" % (T, e_u, e_x, e_g))
    assert max(e_u, e_x, e_g) <= 1


@pytest.mark.parametrize("T,V,ce", [((1 << 22) - 1, 3, 0.5), (2, 1 << 24, 0.5), (2, 1 << 24, 0.0)])
def test_distillation_with_the_most_rows_and_words(T, V, ce):
    """Bounds as in the operator's own tests: a probability is off by 2^-22 (|z| range / tau + |log q| + 8) and V / 1024 + 16 roundings."""
    import torch
    g = gen(3)
    k, tau, kd = 1, 2.0, 1.0
    z = f32(T, V).normal_(0, 1, generator=g)
    ids = torch.randint(0, V, (T, k), generator=g, device="cuda").to(torch.int32)
    lab = torch.randint(0, V, (T,), generator=g, device="cuda").to(torch.int32)
    top = f32(T, k).zero_()
    w = f32(T).uniform_(0, 1, generator=g) / T
    lt, loss, dz = f32(T), f32(1), torch.full_like(z, 77.0)
    B.slora_distill_loss(T, V, B.DTYPE_F32, z, V, k, ids, top, tau, kd, lab, ce, w, lt, loss, dz, V)
    torch.cuda.synchronize()
    zd, wd = z.double(), w.double()[:, None]
    row = torch.arange(T, device="cuda")
    lq, l1 = (torch.log_softmax(zd / t, 1) for t in (tau, 1.0))
    want = -kd * tau * tau * lq[row, ids[:, 0].long()] - ce * l1[row, lab.long()]
    rel = 2.0 ** -22 * (12 + 24 + 8) + (V / 1024 + 16) * 2.0 ** -24
    grad = wd * (kd * tau * lq.exp() + ce * l1.exp())
    lim = rel * grad.abs()
    for at, f in ((ids[:, 0].long(), kd * tau), (lab.long(), ce)):
        grad[row, at] -= wd[:, 0] * f
        lim[row, at] += 2.0 ** -22 * wd[:, 0] * f
    e_t = worst(lt, want, rel * (kd * tau * tau + ce) + 2.0 ** -21 * want.abs())
    e_z = worst(dz, grad, lim)
    total = (wd[:, 0] * want).sum()
    e_l = float((loss[0].double() - total).abs() / ((wd[:, 0] * (rel * 5 + 2.0 ** -21 * want.abs())).sum() + 2.0 ** -23 * total.abs()))
    say("   distillation, %d rows of %d: errors over their bounds %.2f %.2f %.2f" % (T, V, e_t, e_z, e_l))
    assert max(e_t, e_z, e_l) <= 1


def test_embedding_gradient_with_the_most_tokens():
    """Sums of 1 and -1, exact in any order: 2^24 tokens of 50 words, one of them half of all."""
    import torch
    T, V, d = 1 << 24, 50, 8
    g = gen(4)
    tok = torch.randint(-1, V + 1, (T,), generator=g, device="cuda").to(torch.int32)
    tok[torch.rand(T, generator=g, device="cuda") < 0.5] = 7
    dout = (2 * torch.randint(0, 2, (T, d), generator=g, device="cuda") - 1).to(torch.bfloat16)
    n = B.slora_embed_bwd_ws_bytes(T, V, d)
    ws = torch.empty(n, dtype=torch.uint8, device="cuda")
    got = f32(V, d).fill_(9.0)
    B.slora_embed_bwd(T, V, d, B.DTYPE_BF16, tok, dout, d, 0.5, 0, got, ws, n)
    torch.cuda.synchronize()
    want = torch.stack([dout[tok == v].double().sum(0) for v in range(V)]) * 0.5
    assert torch.equal(got.double(), want)
