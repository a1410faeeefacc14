"""GCN2(checkpoint8=True): the backward pass takes the codes of the forward pass
right before it, whatever that was, and its mask is exact at every level."""
import numpy as np
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd import inputs as I
from tests.test_gpu_q8 import LEAST
from tests.test_gpu_q8_model import LEVELS, f64, make, wide_workload

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


@pytest.mark.parametrize("dense", [False, True])
def test_answers_at_o1_leave_the_training_step_alone(dense):
    """forward8() reads the features as codes, which hold numbers beyond the 16-bit type: no 16-bit copy of them is
    made, and the flag of the training step is not raised; what cannot be held raises that of the answers."""
    wl = dict(I.workload("er2k", 0, n_override=600))
    wl["X"] = np.array(wl["X"], np.float32)
    wl["X"][3, 5] = 1e6                    # times weights below 1e-2: products inside binary16's range
    wl["W1"] = wl["W1"] * np.float32(1e-2 / np.abs(wl["W1"]).max())
    m = make(wl, G.GCN_F16, "O1", dense=dense)
    m.quantize()
    m.X.zero_()
    m.forward8()
    torch.cuda.synchronize()
    assert not m.X.any() and m.overflow.item() == 0 and m.scores_overflow.item() == 0
    s1, x = f64(m.SG1[3, :m.f_h]), f64(m.X32[3, :m.f_in])
    # a feature's and a weight's code are within one step of their rows' largest value over 127
    w, wtop = f64(m.W1w()[:, :m.f_h]), np.abs(f64(m.W1w()[:, :m.f_h])).max(0)
    err = 1e6 / 127 * np.abs(w).sum(0) + wtop / 127 * np.abs(x).sum() + x.size * 1e6 / 127 * wtop / 127
    assert np.all(np.abs(s1 - x @ w) <= err + 2.0 ** -11 * np.abs(x @ w) + 2.0 ** -24) and np.abs(s1).max() > 0
    (m.g.dense if dense else m.g.values).view(-1)[0] = 1e6
    m.forward8()
    torch.cuda.synchronize()
    assert m.overflow.item() == 0 and m.scores_overflow.item() == 1


@pytest.mark.parametrize("level,prec", LEVELS)
def test_mask(level, prec):
    """dZ1 is 0 exactly where H1 is, in every type, and nowhere else but where its own value rounds to 0: values
    that a code's half step would round to 0 count too."""
    m = make(wide_workload(), prec, level, checkpoint8=True)
    m.forward(0)
    h1 = m.H1[:, :m.f_h].clone()
    m.loss_and_backward()
    torch.cuda.synchronize()
    dz, on = m.dZ1[:, :m.f_h], h1 > 0
    assert not dz[~on].any()
    assert (on & (h1.double() < 0.5 * m.H1s.double()[:, None])).any()
    gs, w = f64(m.SG2[:, :m.C]), f64(m.W2w()[:, :m.C])
    # C products added in fp32, cut off at the worst, and the two roundings by 1 / (1 - p)
    err = (m.C + 4) * 2.0 ** -23 * (np.abs(gs) @ np.abs(w).T) * 2
    sure = on.cpu().numpy() & (np.abs(gs @ w.T * 2) > err + LEAST[prec])
    learns = on.cpu().numpy() & gs.any(1, keepdims=True)      # rows beside one with a label
    assert np.mean(sure[learns]) > 0.9 and np.all(f64(dz)[sure] != 0)


def test_recorded_passes_run_nothing():
    """A forward pass recorded between an evaluation and its backward pass changes neither; graphs of an evaluation and
    of a backward pass, in one or two, do what the passes do."""
    a, b = pair("O2", G.GCN_F16, device_epoch=True)
    for m in (a, b):
        m.step(0)

    def record(*calls):
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            for call in calls:
                call()
        return graph

    a.forward(0, training=False)
    fwd = record(lambda: a.forward(0))
    b.forward(0)
    a.loss_and_backward()
    b.loss_and_backward()
    same(a, b, "recorded between")
    bwd = record(a.loss_and_backward)                        # behind the recorded training pass: reads its codes
    both = record(lambda: a.forward(0, training=False), a.loss_and_backward)
    for k in range(3):
        for m in (a, b):
            m.optimizer_step()
        fwd.replay()
        bwd.replay()
        b.forward(0)
        b.loss_and_backward()
        same(a, b, ("two graphs", k))
        for m in (a, b):
            m.optimizer_step()
        both.replay()
        b.forward(0)
        b.loss_and_backward()
        same(a, b, ("one graph", k))
