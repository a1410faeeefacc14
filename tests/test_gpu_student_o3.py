"""A student at level O3 (every tensor in 16 bits, no loss scale) and with
fp32 masters (O2) on the same teacher: gradients against the float64 oracle,
and the optimiser's steps with it."""
import numpy as np
import pytest
import torch

from oracle import gcn_oracle as O
from oracle import scores_oracle as S
from paper_2010_12635_amd import inputs as I
from tests.parity import assert_close
from tests.test_gpu_student import make

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", [1, 2])
def test_student_gradients_o3(prec):
    print(f"[student] O3 prec={prec}", flush=True)
    wl = I.workload("er2k", 0, n_override=512)
    n, K, T, w = wl["n"], 4, 2.0, 0.5
    C, F = wl["W2"].shape[1], wl["W1"].shape[1]
    teacher = make(wl, prec, seed=5, level="O3")
    teacher.forward(0, training=False)
    tv, tc = teacher.top_logits(K)
    wv, wc = S.top_logits(teacher.Z2[:, :C].double().cpu().numpy(), K)
    assert np.array_equal(tc[:, :K].cpu().numpy(), wc)
    mask = torch.as_tensor((np.arange(n) % 3 != 0).astype(np.uint8)).cuda()
    m = make(wl, prec, level="O3")
    m.set_teacher(tv, tc, mask, T, w)
    m.forward(0)
    m.loss_and_backward()
    torch.cuda.synchronize()
    # from the logits that the student holds: the losses and dZ2 (loss scale 1)
    z2 = m.Z2[:, :C].double().cpu().numpy()
    ce, d_ce, _ = O.softmax_ce(z2, wl["labels"], wl["mask"], 1.0)
    kd, dz2, db2 = S.distill(z2, wv, wc, T, w, 1.0, mask.cpu().numpy(), base=d_ce)
    assert m.overflow.item() == 0
    assert_close(m.loss.cpu().numpy(), np.array([ce]), prec, "cross-entropy")
    assert_close(m.distill_loss.cpu().numpy(), np.array([kd]), prec, "distillation")
    assert_close(m.dZ2[:, :C].float().cpu().numpy(), dz2, prec, "dZ2")
    assert_close(m.db2()[:C].cpu().numpy(), db2, prec, "db2")
    # the backward pass from the tensors that the student holds
    g = O.graph(n, wl["src"], wl["dst"])
    h1 = m.H1[:, :F].double().cpu().numpy()
    w2 = m.W2w()[:, :C].double().cpu().numpy()
    _, dw2, _, dz1 = O.layer_bwd(g, O.norm_values(g), h1, w2, dz2, "relu", 0.5)
    assert_close(m.dW2()[:, :C].cpu().numpy(), dw2, prec, "dW2")
    assert_close(m.db1()[:F].cpu().numpy(), dz1.sum(0), prec, "db1")


@pytest.mark.parametrize("prec", [1, 2])
def test_student_steps_o3(prec):
    """Captured epochs with a teacher at O3 give the eager bits, NaN included
    (16-bit Adam sends most weights there: test_gpu_precision.py)."""
    wl = I.workload("er2k", 0, n_override=512)
    teacher = make(wl, prec, seed=5, level="O3")
    teacher.forward(0, training=False)
    tv, tc = teacher.top_logits(8)
    eager, rep = (make(wl, prec, level="O3", device_epoch=True) for _ in range(2))
    start = eager.working.clone()
    for m in (eager, rep):
        m.set_teacher(tv, tc, temperature=3.0, weight=2.0)
    rep.capture()
    for k in range(4):
        eager.step(0)
        rep.replay()
        torch.cuda.synchronize()
        for t in ("working", "m", "v", "scaler", "grad", "loss", "distill_loss"):
            a, b = (getattr(m, t).view(torch.uint8) for m in (eager, rep))
            assert torch.equal(a, b), (k, t)
    assert not torch.equal(eager.working, start)
