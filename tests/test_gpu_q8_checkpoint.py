"""GCN2(checkpoint8=True): the backward pass takes the codes of the forward pass
right before it, whatever that was, and its mask is exact at every level."""
import numpy as np
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd import inputs as I
from tests.test_gpu_q8_model import LEVELS, f64, make

pytestmark = pytest.mark.gpu

# O3 trains in bf16: binary16's Adam divides by second moments that round to 0
TRAINED = LEVELS[:-1] + [("O3", G.GCN_BF16)]
GRADIENTS = ("grad", "loss", "n_correct", "overflow")


def pair(level, prec, **kw):
    wl = I.workload("er2k", 0, n_override=600)
    return [make(wl, prec, level, dropout=0.0, checkpoint8=True, **kw) for _ in range(2)]


def same(a, b, what):
    torch.cuda.synchronize()
    assert a.overflow.item() == 0, what
    for t in GRADIENTS:
        assert torch.equal(getattr(a, t), getattr(b, t)), (what, t)
    assert torch.equal(a.dZ1[:, :a.f_h], b.dZ1[:, :b.f_h]), what
    assert b.grad.any(), what


@pytest.mark.parametrize("level,prec", TRAINED)
def test_backward_behind_an_evaluation(level, prec):
    """Without dropout an evaluation computes what a training pass does, and so does the backward pass behind it:
    the same bits, on a new model, after steps that kept other codes, and when it is asked twice."""
    a, b = pair(level, prec)
    for step in range(3):
        a.forward(step, training=False)
        b.forward(step)
        a.loss_and_backward()
        b.loss_and_backward()
        same(a, b, step)
        a.loss_and_backward()
        same(a, b, (step, "again"))
        for m in (a, b):
            m.optimizer_step()
            m.step(step)


def test_backward_behind_answers_from_8_bits():
    """forward8()'s H1 is what its backward pass is taken from, behind an evaluation too."""
    a, b = pair("O2", G.GCN_F16)
    for m in (a, b):
        m.step(0)
        m.quantize()
    a.forward8()
    b.forward(1, training=False)
    b.forward8()
    a.loss_and_backward()
    b.loss_and_backward()
    same(a, b, "forward8")


@pytest.mark.parametrize("level,prec", [("O0", G.GCN_F32), ("O2", G.GCN_F16)])
def test_backward_beside_captured_epochs(level, prec):
    """Recording an epoch runs nothing and keeps nothing; a replayed one keeps its own H1."""
    a, b = pair(level, prec, device_epoch=True)
    a.step(0)
    b.step(0)
    a.forward(0, training=False)
    a.capture()
    b.forward(0)
    a.loss_and_backward()
    b.loss_and_backward()
    same(a, b, "captured between")
    for m in (a, b):
        m.optimizer_step()
    for k in range(3):
        a.forward(0, training=False)
        a.replay()
        b.step(0)
        a.loss_and_backward()
        b.loss_and_backward()
        same(a, b, k)
