"""More that the operators for training other models refuse before anything touches a GPU."""
import pytest

from paper_2407_00952_amd import binding as B
from test_train_ops_abi_cpu import P, attn, distill, embed, norm, refused


@pytest.mark.parametrize("kd,tau", [(1e30, 1e15), (1e30, 1.01), (1.1, 1e15), (1e10, 1.1e10), (1e20, 1e6), (1e30, 2.0)])
def test_distillation_refuses_a_factor_beyond_its_range(kd, tau):
    """kd tau^2, which the loss is multiplied by, passes 1e30: fp32 would hold infinities instead of it, and 0 * inf where p = q"""
    refused(lambda: distill(kd=kd, tau=tau))


def test_rmsnorm_backward_refuses_a_strided_h():
    """The forward reads x with a stride, the backward reads h dense; without a residual h is x.  Handed on as it is, a view of wider rows
    would be read as other rows."""
    import torch
    wide = torch.zeros((10, 96), dtype=torch.bfloat16)
    for h in (wide[:, :64], wide[::2, :64], wide.t()[:64].t(), wide.view(10, 96)[:, 32:]):
        refused(lambda: norm(True, res_dtype=B.DTYPE_BF16, h=h, dres=None))


def test_rmsnorm_backward_takes_a_dense_h():
    """dense in any shape, an address, nothing to do: not refused (no rows, so nothing is launched)"""
    import torch
    dense = torch.zeros((10, 64), dtype=torch.bfloat16)
    for h in (dense, dense.view(2, 5, 64), dense.view(-1), dense[3:], P):
        norm(True, T=0, res_dtype=B.DTYPE_BF16, h=h, dres=None, dgamma=None, ws=None, ws_bytes=0)


def test_calls_with_nothing_to_do_take_empty_tensors():
    """an empty torch tensor has the address 0: no rows, no pointers to them"""
    import torch
    e = torch.empty((0, 64), dtype=torch.bfloat16)
    assert e.data_ptr() == 0
    attn(T=0, q=e, k=e, v=e, o=e, lse=e)
    attn(n_seq=0, T=0, q=e, k=e, v=e, o=e, lse=e)
    attn(True, T=0, q=e, k=e, v=e, o=e, lse=e, dout=e, dq=e, dk=e, dv=e)
    norm(T=0, x=e, res=e, h=e, u=e, codes=e, scales=e, rho=e)
    norm(T=0, x=e, res=None, h=None, u=e, codes=None, scales=None, rho=None)
    norm(True, T=0, du=e, h=e, rho=e, dres=e, dh=e, dgamma=None, ws=None, ws_bytes=0)
    embed(T=0, tokens=e, out=e)
    embed(True, T=0, tokens=e, dout=e, accumulate=1)


def test_calls_with_nothing_to_do_keep_their_other_checks():
    for bad in (dict(head_dim=32), dict(scale=0.0), dict(causal=2), dict(n_kv_head=3)):
        refused(lambda: attn(T=0, **bad))
        refused(lambda: attn(True, T=0, **bad))
    for bad in (dict(d=12), dict(res_dtype=2)):
        refused(lambda: norm(T=0, **bad))
        refused(lambda: norm(True, T=0, **bad))
    refused(lambda: norm(T=0, eps=-1.0))
    refused(lambda: norm(True, T=0, dgamma=P + 2))
    refused(lambda: embed(T=0, d=12))
    for bad in (dict(d=12), dict(accumulate=2), dict(dtable=None), dict(dtable=P + 8)):
        refused(lambda: embed(True, T=0, **bad))
