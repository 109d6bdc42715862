"""The training step's own gradients against differences of its own loss: what the library wrote into dtable, dg1 and dg2 says how the loss
moves when the table or a norm's gamma moves."""
import numpy as np
import pytest

from gpu_util import say
from test_gpu_train_step import Step, reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("name", ["table", "g1", "g2"])
def test_gradient_against_differences_of_the_loss(name):
    """A central difference along the fp64 model's gradient, 8 long to each side.  Three things part it from <gradient, step>: the step is
    no infinitesimal one (the fp64 model's difference against its own gradient says by how much), each of the two losses is off by up
    to 4e-3 of itself and the gradient by up to 12 * 2^-8 of its 2-norm (the bounds of the step's comparison with one model).  Together
    they stay below six tenths of the difference (the table 0.22, g1 0.52, g2 0.13), so that a gradient that is off by as much fails."""
    import torch
    st = Step(3)
    st.run()
    torch.cuda.synchronize()
    got = {"table": st.dtable, "g1": st.dg1, "g2": st.dg2}[name].double().cpu()
    loss, dt, d1, d2 = reference(st)
    want = {"table": dt, "g1": d1, "g2": d2}[name]
    tensor = getattr(st, name)
    base, losses, moved_to, model = tensor.double().cpu(), [], [], []
    for sign in (8.0, -8.0):
        tensor.copy_((base + sign * want / want.norm()).to(torch.bfloat16))
        st.np[name] = tensor.float().cpu().numpy()
        st.run()
        losses.append(float(st.loss))
        moved_to.append(tensor.double().cpu())
        model.append(reference(st)[0])
    step = moved_to[0] - moved_to[1]
    along, difference = float((got * step).sum()), losses[0] - losses[1]
    curve = abs(model[0] - model[1] - float((want * step).sum()))
    lim = curve + 4e-3 * sum(abs(x) for x in model) + 12 * 2.0 ** -8 * float(step.norm() * want.norm())
    say("   %s: along the gradient %.4f, difference of the loss %.4f, allowed %.4f" % (name, along, difference, lim))
    assert lim < 0.6 * abs(model[0] - model[1])
    assert abs(along - difference) <= lim
