"""Calls that move more than 128 MiB store their results past the caches, in instances of the kernels of their own.  Rows do not depend
on each other, so such a call has to give the bits that calls on parts of its rows give, which stay below."""
import pytest

from paper_2407_00952_amd import binding as B
from gpu_util import say

pytestmark = pytest.mark.gpu
BF, F32, EPS = B.DTYPE_BF16, B.DTYPE_F32, 1e-5
LIMIT = 128 << 20
MARK = 7.0


def dtype_of(ty):
    import torch
    return torch.float32 if ty == F32 else torch.bfloat16


def normal(shape, dtype, seed, mean=0.0, std=1.0):
    import torch
    g = torch.Generator(device="cuda").manual_seed(seed)
    return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(mean, std, generator=g).to(dtype)


def marked(shape, dtype):
    import torch
    return torch.full(shape, MARK, dtype=dtype, device="cuda")


def thirds(T):
    """rows of three calls that move less than half of what one on all rows does"""
    return [(T * i // 3, T * (i + 1) // 3) for i in range(3)]


def equal(name, whole, parts):
    import torch
    assert torch.equal(whole, parts), "%s: %d elements differ" % (name, int((whole != parts).sum()))


# every width of the kernels (threads and chunks of a row)
@pytest.mark.parametrize("d", [128, 256, 512, 1024, 1504, 2048, 4096, 5120, 8192, 12288, 16384])
@pytest.mark.parametrize("res", [None, BF, F32])
def test_rmsnorm(d, res):
    import torch
    bf = torch.bfloat16
    e = {None: 0, BF: 2, F32: 4}[res]
    fwd, bwd = 2 + 2 * e + 3, 2 + 2 * (e or 2) + (e or 2)     # bytes an element: x, residual in and out, u, codes; du, h, dres, dh
    T = LIMIT // (d * min(fwd, bwd)) + 50
    assert T * d * fwd > LIMIT and T * d * bwd > LIMIT and (T // 3 + 1) * d * (max(fwd, bwd) + 2) < LIMIT
    ty, rt = (BF if res is None else res), dtype_of(BF if res is None else res)
    x, r, gamma = normal((T, d), bf, 1), None if res is None else normal((T, d), rt, 2, std=2.0), normal((d,), bf, 3, 1.0, 0.3)
    du, dres = normal((T, d), bf, 4), normal((T, d), rt, 5)
    u8 = lambda n: torch.full((T, n), 9, dtype=torch.uint8, device="cuda")

    def run(ranges, in_place):
        o = dict(u=marked((T, d), bf), q=u8(d), s=u8(d // 32), rho=marked((T,), torch.float32), dx=marked((T, d), bf))
        o["h"] = None if r is None else (r.clone() if in_place else marked((T, d), rt))
        o["dh"] = dres.clone() if in_place else marked((T, d), rt)
        src, dsrc = (o["h"] if in_place and r is not None else r), (o["dh"] if in_place else dres)
        at = lambda t, a, b: None if t is None else t[a:b]
        for a, b in ranges:
            B.slora_rmsnorm_fwd(b - a, d, ty, x[a:b], d, at(src, a, b), gamma, EPS, at(o["h"], a, b), o["u"][a:b], d, o["q"][a:b],
                                o["s"][a:b], o["rho"][a:b])
        h = x if r is None else o["h"]
        o["dgamma"] = []
        for a, b in ranges:
            n = B.slora_rmsnorm_bwd_ws_bytes(b - a, d)
            ws = torch.empty(n, dtype=torch.uint8, device="cuda")
            dg = marked((d,), torch.float32)
            B.slora_rmsnorm_bwd(b - a, d, ty, du[a:b], d, h[a:b], o["rho"][a:b], gamma, dsrc[a:b], o["dh"][a:b], o["dx"][a:b], d, dg, ws, n)
            o["dgamma"].append(dg)
        torch.cuda.synchronize()
        return o

    say("rms norm [%d, %d], residual %s" % (T, d, {None: "none", BF: "bf16", F32: "fp32"}[res]))
    whole, parts, place = run([(0, T)], False), run(thirds(T), False), run([(0, T)], True)
    for n in ("u", "q", "s", "rho", "h", "dh", "dx"):
        if whole[n] is not None:
            equal(n, whole[n], parts[n])
            equal(n + " in place", whole[n], place[n])
    # dgamma adds up T products in fp32, in an order that depends on T: each sum is off by at most T 2^-24 of the absolute sum
    want, size = torch.zeros(d, dtype=torch.float64, device="cuda"), torch.zeros(d, dtype=torch.float64, device="cuda")
    h = x if r is None else whole["h"]
    for a in range(0, T, 4096):
        t = du[a:a + 4096].double() * h[a:a + 4096].double() * whole["rho"][a:a + 4096, None].double()
        want += t.sum(0)
        size += t.abs().sum(0)
    for o in (whole, parts):
        got = sum(g.double() for g in o["dgamma"])
        assert bool(((got - want).abs() <= (T + 16) * 2.0 ** -24 * size).all())


@pytest.mark.parametrize("ty,V", [(BF, 5003), (BF, 50257), (BF, 100003), (BF, 140001), (F32, 3001), (F32, 32003), (F32, 50257), (F32, 70001)])
@pytest.mark.parametrize("tau,labelled", [(1.0, True), (2.0, True), (4.0, True), (1.5, True), (2.0, False)])
def test_distillation(ty, V, tau, labelled):
    """every form of a row (few threads, registers of both sizes, read twice), dense rows at every alignment, a quarter of them of weight 0"""
    import torch
    dt, e, k = dtype_of(ty), 4 if ty == F32 else 2, 9
    T = LIMIT // (2 * e * V) + 9
    g = torch.Generator(device="cuda").manual_seed(V)
    z = normal((T, V), dt, V + 1, std=2.0)
    ids = torch.randint(0, V, (T, k), generator=g, device="cuda").to(torch.int32)
    ids[:, 4] = ids[:, 2]                                     # an id in two entries
    ids[::5, 7] = -1
    top = normal((T, k), torch.float32, V + 2, std=3.0)
    labels = torch.where(torch.arange(T, device="cuda") % 3 == 0, ids[:, 1], torch.randint(0, V, (T,), generator=g, device="cuda").to(torch.int32))
    w = torch.where(torch.rand(T, generator=g, device="cuda") < 0.25, 0.0, 1.0 / T).to(torch.float32)
    assert 2 * e * T * V > LIMIT and 2 * e * (T // 3 + 1) * V < LIMIT

    def run(ranges, out=None):
        lt, dz = marked((T,), torch.float32), marked((T, V), dt) if out is None else out
        src, losses = z if out is None else out, []
        for a, b in ranges:
            loss = marked((1,), torch.float32)
            B.slora_distill_loss(b - a, V, ty, src[a:b], V, k, ids[a:b], top[a:b], tau, 0.6, labels[a:b] if labelled else None, 0.4,
                                 w[a:b], lt[a:b], loss, dz[a:b], V)
            losses.append(loss)
        torch.cuda.synchronize()
        return lt, dz, sum(float(x) for x in losses)

    say("distillation [%d, %d]" % (T, V))
    whole, parts, place = run([(0, T)]), run(thirds(T)), run([(0, T)], z.clone())
    for other in (parts, place):
        equal("rows", whole[0], other[0])
        equal("gradient", whole[1], other[1])
    assert bool((whole[1][w == 0] == 0).all())
    # the loss of a call is one sum in 64 bits, rounded once
    assert abs(whole[2] - parts[2]) <= 4 * 2.0 ** -24 * float((w.double() * whole[0].double().abs()).sum())
    assert whole[2] == place[2]


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("d", [64, 128, 256, 1024, 2056])
def test_embedding_lookup(ty, d):
    import torch
    dt, e, V = dtype_of(ty), 4 if ty == F32 else 2, 1003
    T = LIMIT // (e * d) + 77
    assert e * d * (T // 3 + 1 + V) < LIMIT
    g = torch.Generator(device="cuda").manual_seed(d)
    tok = torch.randint(-3, V + 3, (T,), generator=g, device="cuda").to(torch.int32)
    table = normal((V, d), dt, d + 1)
    whole, parts = marked((T, d), dt), marked((T, d), dt)
    B.slora_embed_fwd(T, V, d, ty, tok, table, 1.5, whole, d)
    for a, b in thirds(T):
        B.slora_embed_fwd(b - a, V, d, ty, tok[a:b], table, 1.5, parts[a:b], d)
    torch.cuda.synchronize()
    equal("rows", whole, parts)
    word = (tok >= 0) & (tok < V)
    want = (table.float() * 1.5).to(dt)[tok.clamp(0, V - 1).long()].masked_fill_(~word[:, None], 0.0)
    equal("rows", whole, want)


@pytest.mark.parametrize("ty", [BF, F32])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_embedding_gradient(ty, accumulate):
    """columns do not depend on each other either: calls on a quarter of them (1024 and more have the same order of sums)"""
    import torch
    dt, d, V, T, n = dtype_of(ty), 4096, 9001, 12000, 1024
    e = 4 if ty == F32 else 2
    g = torch.Generator(device="cuda").manual_seed(9)
    tok = torch.randint(-3, V + 3, (T,), generator=g, device="cuda").to(torch.int32)
    tok[::4], tok[1::40] = 17, 8000                            # tokens in 3000 and in 300 places
    dout, old = normal((T, d), dt, 10), normal((V, d), torch.float32, 11)
    assert 4 * V * d + e * T * d > LIMIT and (8 * min(V, T) + e * T) * n < LIMIT
    ws_n = B.slora_embed_bwd_ws_bytes(T, V, d)
    ws = torch.empty(ws_n, dtype=torch.uint8, device="cuda")
    whole, parts = old.clone(), old.clone()
    B.slora_embed_bwd(T, V, d, ty, tok, dout, d, 0.5, accumulate, whole, ws, ws_n)
    for c in range(0, d, n):
        p = old[:, c:c + n].contiguous()
        B.slora_embed_bwd(T, V, n, ty, tok, dout[:, c:c + n], d, 0.5, accumulate, p, ws, ws_n)
        parts[:, c:c + n] = p
    torch.cuda.synchronize()
    equal("gradient", whole, parts)
    count = torch.bincount(tok[(tok >= 0) & (tok < V)].long(), minlength=V)
    assert bool((whole[count == 0] == (old[count == 0] if accumulate else 0.0)).all())
