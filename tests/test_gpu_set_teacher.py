"""GCN2.set_teacher: what no step could run with is refused at once, and steps
on any stream find the teacher whole."""
import numpy as np
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd import inputs as I
from tests.test_gpu_student import make

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def wl():
    return I.workload("er2k", 0, n_override=512)


def teacher_of(wl, K=8):
    m = make(wl, 1, seed=5)
    m.forward(0, training=False)
    v, c = m.top_logits(K)
    return v[:, :K].contiguous(), c[:, :K].contiguous()


@pytest.mark.parametrize("bad", [
    dict(mask=np.zeros(512, np.uint8)), dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=2.0 ** -11),
    dict(temperature=1025.0), dict(temperature=float("nan")), dict(weight=0.0), dict(weight=-1.0),
    dict(weight=float("inf")), dict(weight=float("nan")), dict(weight=1e-60), dict(weight=1e60),
    dict(top_classes=None)],
    ids=lambda d: next(iter(d)))
def test_refusals(wl, bad):
    v, c = teacher_of(wl)
    m = make(wl, 1)
    m.set_teacher(v, c, weight=0.25)
    kept = m.teacher
    with pytest.raises(ValueError):
        m.set_teacher(**dict(dict(top_values=v, top_classes=c), **bad))
    assert m.teacher is kept                      # the teacher it had still teaches
    m.step(0)
    torch.cuda.synchronize()
    assert m.overflow.item() == 0 and np.isfinite(m.distill_loss.item())


def test_ends_of_the_ranges(wl):
    v, c = teacher_of(wl)
    m = make(wl, 0)
    for T in (G.MIN_TEMPERATURE, G.MAX_TEMPERATURE):
        m.set_teacher(v, c, temperature=T, weight=1e-3)
        m.forward(0)
        m.loss_and_backward()
        torch.cuda.synchronize()
        assert m.overflow.item() == 0


def test_views_off_alignment(wl):
    """A contiguous view whose memory starts off 16 bytes is copied."""
    v, c = teacher_of(wl)
    vv = torch.empty(v.numel() + 1, dtype=v.dtype, device="cuda")[1:].view_as(v).copy_(v)
    cc = torch.empty(c.numel() + 1, dtype=c.dtype, device="cuda")[1:].view_as(c).copy_(c)
    a, b = make(wl, 1), make(wl, 1)
    a.set_teacher(v, c)
    b.set_teacher(vv, cc)
    for m in (a, b):
        m.step(0)
    torch.cuda.synchronize()
    assert torch.equal(a.grad, b.grad) and torch.equal(a.distill_loss, b.distill_loss)


@pytest.mark.parametrize("K", [5, 8])
def test_step_on_another_stream(wl, K):
    """The copies that set_teacher makes (K not a multiple of 8) lie behind
    other work of the current stream; a step on another stream waits for them."""
    v, c = teacher_of(wl, K)
    a, b = make(wl, 1), make(wl, 1)
    a.set_teacher(v, c)
    a.step(0)
    busy = torch.ones(1 << 26, device="cuda")
    side = torch.cuda.Stream()
    b.set_teacher(v, c)                           # a first teacher, replaced while its step may run
    b.forward(0)
    torch.cuda.synchronize()
    b.loss_and_backward(side)
    for _ in range(200):
        busy.mul_(1.0)
    b.set_teacher(v, c)
    b.loss_and_backward(side)
    torch.cuda.synchronize()
    assert torch.equal(a.distill_loss, b.distill_loss) and torch.equal(a.grad, b.grad)
