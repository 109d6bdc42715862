"""More that the operators for training other models refuse before anything touches a GPU."""
import pytest

from paper_2407_00952_amd import binding as B
from test_train_ops_abi_cpu import P, distill, norm, refused


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
