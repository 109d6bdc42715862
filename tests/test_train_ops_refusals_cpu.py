"""More that the operators for training other models refuse before anything touches a GPU."""
import pytest

from paper_2407_00952_amd import binding as B
from test_train_ops_abi_cpu import distill, refused


@pytest.mark.parametrize("kd,tau", [(1e30, 1e15), (1e30, 1.01), (1.1, 1e15), (1e10, 1.1e10), (1e20, 1e6), (1e30, 2.0)])
def test_distillation_refuses_a_factor_beyond_its_range(kd, tau):
    """kd tau^2, which the loss is multiplied by, passes 1e30: fp32 would hold infinities instead of it, and 0 * inf where p = q"""
    refused(lambda: distill(kd=kd, tau=tau))
