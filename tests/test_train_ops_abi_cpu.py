"""What the operators for training other models refuse, before anything touches a GPU."""
import pytest

from paper_2407_00952_amd import binding as B

P = 0x10000          # aligned, never dereferenced by the host-side checks


def refused(f, code=B.SLORA_EINVAL):
    with pytest.raises(B.SloraError) as e:
        f()
    assert e.value.code == code


def attn(bwd=False, **kw):
    a = dict(n_seq=3, T=100, n_head=4, n_kv_head=2, head_dim=64, scale=0.125, causal=1, window=0, q=P, ldq=512, k=P, ldk=512,
             v=P, ldv=512, seq_start=P, o=P, o_lo=None, ldo=256, lse=P)
    if bwd:
        a.update(dout=P, lddo=256, dq=P, lddq=512, dk=P, lddk=512, dv=P, lddv=512, ws=P,
                 ws_bytes=B.slora_attention_bwd_ws_bytes(100, 4, 2, 64))
    a.update(kw)
    return (B.slora_attention_bwd if bwd else B.slora_attention_fwd)(**a, stream=0)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("bad", [
    dict(n_seq=-1), dict(T=-1), dict(T=(1 << 24) + 1), dict(n_head=0), dict(n_head=1025, n_kv_head=1), dict(n_kv_head=3), dict(n_kv_head=0),
    dict(head_dim=32), dict(head_dim=96), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(causal=2),
    dict(window=-1), dict(causal=0, window=8), dict(q=None), dict(k=None), dict(v=None), dict(seq_start=None), dict(o=None), dict(lse=None),
    dict(q=P + 8), dict(k=P + 2), dict(v=P + 4), dict(seq_start=P + 2), dict(o=P + 8), dict(o_lo=P + 8), dict(lse=P + 2), dict(ldq=248),
    dict(ldq=260), dict(ldk=120), dict(ldv=1 << 24), dict(ldo=248), dict(n_seq=1 << 24, n_head=1024, n_kv_head=2, ldq=1 << 17, ldo=1 << 17),
    dict(T=1 << 24, n_head=128, ldq=8192, ldo=8192)])
def test_attention_refuses(bwd, bad):
    refused(lambda: attn(bwd, **bad))


@pytest.mark.parametrize("bad", [dict(dout=None), dict(dq=None), dict(dk=None), dict(dv=None), dict(ws=None), dict(dout=P + 8), dict(dq=P + 8),
                                 dict(dk=P + 8), dict(dv=P + 8), dict(ws=P + 128), dict(lddo=128), dict(lddq=128), dict(lddk=64),
                                 dict(lddv=64), dict(lddk=132)])
def test_attention_backward_refuses(bad):
    refused(lambda: attn(True, **bad))


def test_attention_workspace():
    assert B.slora_attention_bwd_ws_bytes(100, 4, 3, 64) == 0 and B.slora_attention_bwd_ws_bytes(100, 4, 2, 80) == 0
    assert B.slora_attention_bwd_ws_bytes(-1, 4, 2, 64) == 0
    n = B.slora_attention_bwd_ws_bytes(100, 4, 2, 64)
    assert n >= 4 * 4 * 100 and n % 256 == 0
    refused(lambda: attn(True, ws_bytes=n - 1), B.SLORA_ENOSPC)
    attn(n_seq=0), attn(T=0), attn(True, n_seq=0), attn(True, T=0)          # nothing to do, no launch
    # the scratch for some tokens serves fewer
    for H, Hk, D in ((32, 8, 128), (16, 1, 64), (40, 8, 64), (12, 12, 64), (7, 1, 128)):
        sizes = [B.slora_attention_bwd_ws_bytes(t, H, Hk, D) for t in list(range(0, 3000)) + list(range(3000, 70000, 61))]
        assert sizes[0] > 0 and all(a <= b for a, b in zip(sizes, sizes[1:]))


def norm(bwd=False, **kw):
    if bwd:
        a = dict(T=10, d=64, res_dtype=B.DTYPE_F32, du=P, lddu=64, h=P, rho=P, gamma=P, dres=P, dh=P, dx=None, lddx=0, dgamma=P, ws=P,
                 ws_bytes=B.slora_rmsnorm_bwd_ws_bytes(10, 64))
    else:
        a = dict(T=10, d=64, res_dtype=B.DTYPE_F32, x=P, ldx=64, res=P, gamma=P, eps=1e-5, h=P, u=P, ldu=64, codes=P, scales=P, rho=P)
    a.update(kw)
    return (B.slora_rmsnorm_bwd if bwd else B.slora_rmsnorm_fwd)(**a, stream=0)


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(T=1 << 23), dict(d=0), dict(d=12), dict(d=16392), dict(d=40, ldx=64), dict(res_dtype=2), dict(eps=-1.0),
    dict(eps=float("nan")), dict(x=None), dict(gamma=None), dict(u=None, codes=None, scales=None), dict(scales=None), dict(codes=None),
    dict(res=None), dict(ldx=56), dict(ldx=68), dict(ldu=56), dict(ldu=66), dict(x=P + 8), dict(res=P + 8), dict(gamma=P + 8), dict(h=P + 8),
    dict(u=P + 8), dict(codes=P + 4), dict(rho=P + 2)])
def test_rmsnorm_refuses(bad):
    refused(lambda: norm(**bad))


@pytest.mark.parametrize("bad", [
    dict(T=-1), dict(T=1 << 23), dict(d=0), dict(d=20), dict(d=16392), dict(res_dtype=2), dict(du=None), dict(h=None), dict(rho=None), dict(gamma=None),
    dict(dh=None), dict(ws=None), dict(lddu=56), dict(lddu=66), dict(dx=P, lddx=60), dict(du=P + 8), dict(h=P + 8), dict(gamma=P + 8),
    dict(dres=P + 8), dict(dh=P + 8), dict(dx=P + 8, lddx=64), dict(dgamma=P + 2), dict(ws=P + 64)])
def test_rmsnorm_backward_refuses(bad):
    refused(lambda: norm(True, **bad))


def test_rmsnorm_workspace():
    assert B.slora_rmsnorm_bwd_ws_bytes(10, 12) == 0 and B.slora_rmsnorm_bwd_ws_bytes(-1, 64) == 0
    refused(lambda: norm(True, ws_bytes=B.slora_rmsnorm_bwd_ws_bytes(10, 64) - 1), B.SLORA_ENOSPC)
    norm(T=0), norm(True, T=0, dgamma=None, ws=None, ws_bytes=0)            # nothing to do, no launch
    for d in (8, 1024, 2048, 2056, 16384):
        n = [B.slora_rmsnorm_bwd_ws_bytes(t, d) for t in range(0, 9000, 7)]
        assert n[0] > 0 and all(a <= b for a, b in zip(n, n[1:]))


def distill(**kw):
    a = dict(T=5, vocab=100, dtype=B.DTYPE_BF16, logits=P, ldl=100, k=4, t_ids=P, t_logits=P, tau=2.0, kd=1.0, labels=None, ce=0.0,
             row_weight=None, loss_tok=P, loss=P, dlogits=2 * P, ldd=100)
    a.update(kw)
    return B.slora_distill_loss(**a, stream=0)


@pytest.mark.parametrize("bad", [
    dict(T=0), dict(T=-1), dict(T=1 << 22), dict(vocab=0), dict(vocab=(1 << 24) + 1, ldl=1 << 25), dict(k=0), dict(k=B.MAX_TOP + 1),
    dict(dtype=2), dict(logits=None), dict(t_ids=None), dict(t_logits=None), dict(loss_tok=None), dict(loss=None), dict(tau=0.0),
    dict(tau=-1.0), dict(tau=float("nan")), dict(tau=float("inf")), dict(tau=1e-16),
    dict(tau=2e15), dict(kd=2e30), dict(ce=2e30), dict(kd=-0.5), dict(kd=float("nan")), dict(ce=-1.0), dict(ce=float("inf")),
    dict(ldl=99), dict(ldd=99), dict(dlogits=P, ldd=104), dict(logits=P + 1), dict(dtype=B.DTYPE_F32, logits=P + 2),
    dict(dlogits=2 * P + 1), dict(t_ids=P + 2), dict(t_logits=P + 2), dict(labels=P + 1), dict(row_weight=P + 2), dict(loss_tok=P + 2),
    dict(loss=P + 1)])
def test_distill_refuses(bad):
    refused(lambda: distill(**bad))


def embed(bwd=False, **kw):
    a = dict(T=5, vocab=100, d=64, dtype=B.DTYPE_BF16, tokens=P)
    if bwd:
        a.update(dout=P, ldd=64, scale=1.0, accumulate=0, dtable=P, ws=P, ws_bytes=B.slora_embed_bwd_ws_bytes(5, 100, 64))
    else:
        a.update(table=P, scale=1.0, out=P, ldo=64)
    a.update(kw)
    return (B.slora_embed_bwd if bwd else B.slora_embed_fwd)(**a, stream=0)


@pytest.mark.parametrize("bwd", [False, True])
@pytest.mark.parametrize("bad", [dict(T=-1), dict(T=(1 << 24) + 1), dict(vocab=0), dict(vocab=(1 << 24) + 1), dict(d=0), dict(d=12),
                                 dict(d=65544), dict(dtype=2), dict(tokens=None), dict(tokens=P + 2)])
def test_embed_refuses(bwd, bad):
    refused(lambda: embed(bwd, **bad))


@pytest.mark.parametrize("bwd,bad", [(False, dict(table=None)), (False, dict(out=None)), (False, dict(ldo=56)), (False, dict(ldo=66)),
                                     (False, dict(table=P + 8)), (False, dict(out=P + 8)), (True, dict(dout=None)),
                                     (True, dict(dtable=None)), (True, dict(ws=None)), (True, dict(ldd=56)), (True, dict(ldd=66)),
                                     (True, dict(accumulate=2)), (True, dict(dout=P + 8)), (True, dict(dtable=P + 8)),
                                     (True, dict(ws=P + 16))])
def test_embed_refuses_in_one_direction(bwd, bad):
    refused(lambda: embed(bwd, **bad))


def test_embed_workspace():
    assert B.slora_embed_bwd_ws_bytes(5, 100, 12) == 0 and B.slora_embed_bwd_ws_bytes(-1, 100, 64) == 0
    refused(lambda: embed(True, ws_bytes=B.slora_embed_bwd_ws_bytes(5, 100, 64) - 1), B.SLORA_ENOSPC)
    embed(T=0), embed(True, T=0, accumulate=1)                              # nothing to do, no launch
    for V, d in ((100, 8), (50257, 1024), (1 << 24, 64)):
        n = [B.slora_embed_bwd_ws_bytes(t, V, d) for t in list(range(0, 3000, 7)) + list(range(3000, 200000, 997))]
        assert n[0] > 0 and all(a <= b for a, b in zip(n, n[1:]))
