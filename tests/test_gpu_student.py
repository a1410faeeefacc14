"""Teacher and student as a program runs them: a trained model's top scores,
a student that learns from them beside its labels, labels drawn from the
student for vertices without one, and a captured epoch of it all.

The student's gradients are checked against the float64 oracle's chain rule
with the tolerances of the parity tests."""
import numpy as np
import pytest
import torch

from oracle import gcn_oracle as O
from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd import inputs as I
from paper_2010_12635_amd.model import DeviceGraph, GCN2
from tests.parity import assert_close

pytestmark = pytest.mark.gpu


def make(wl, prec, seed=0, level=None, **kw):
    fp32_graph = level == "O1"
    dg = DeviceGraph(wl["n"], wl["src"], wl["dst"], prec=G.GCN_F32 if fp32_graph else prec)
    rng = np.random.default_rng(seed)
    w1, w2 = (w + 0.3 * rng.standard_normal(w.shape).astype(np.float32) * np.abs(w).max() * (seed > 0)
              for w in (wl["W1"], wl["W2"]))
    return GCN2(dg, wl["X"], wl["labels"], wl["mask"], w1, w2, wl["b1"], wl["b2"], prec=prec, dropout=0.5,
                seed=wl["dropout_seed"], loss_scale=1024.0 if prec else 1.0, level=level, **kw)


@pytest.mark.parametrize("level,prec", [("O0", 0), ("O1", 1), ("O2", 1), ("O2", 2)])
def test_student_gradients(level, prec):
    print(f"[student] {level} prec={prec}", flush=True)
    wl = I.workload("er2k", 0, n_override=512)
    n, K, T, w = wl["n"], 4, 2.0, 0.5
    teacher = make(wl, prec, seed=5, level=level)
    teacher.forward(0, training=False)
    tv, tc = teacher.top_logits(K)
    C = wl["W2"].shape[1]
    zt = teacher.Z2[:, :C].double().cpu().numpy()
    wv, wc = S.top_logits(zt, K)
    assert np.array_equal(tc[:, :K].cpu().numpy(), wc) and np.array_equal(tv[:, :K].double().cpu().numpy(), wv)
    assert (tc[:, K:] == -1).all()
    mask = torch.as_tensor((np.arange(n) % 3 != 0).astype(np.uint8)).cuda()
    m = make(wl, prec, level=level)
    m.set_teacher(tv[:, :K].contiguous(), tc[:, :K].contiguous(), mask, T, w)
    m.forward(0)
    m.loss_and_backward()
    torch.cuda.synchronize()

    g = O.graph(n, wl["src"], wl["dst"])
    vals = O.norm_values(g)
    x = wl["X"].astype(np.float64)
    _, _, h1 = O.layer_fwd(g, vals, x, wl["W1"], wl["b1"], "relu", 0.5, True, wl["dropout_seed"], 0, 0)
    _, z2, _ = O.layer_fwd(g, vals, h1, wl["W2"], wl["b2"], "none")
    scale = 1024.0 if prec else 1.0
    ce, d_ce, _ = O.softmax_ce(z2, wl["labels"], wl["mask"], scale)
    kd, dz2, _ = S.distill(z2, wv, wc, T, w, scale, mask.cpu().numpy(), base=d_ce)
    # the backward pass is checked from the hidden layer that the student holds:
    # a pre-activation within its rounding of 0 may lie on either side of 0, and
    # ReLU's derivative there is then the held value's, not the exact one's
    h1 = m.H1[:, :wl["W1"].shape[1]].double().cpu().numpy()
    _, dw2, db2, dz1 = O.layer_bwd(g, vals, h1, wl["W2"], dz2, "relu", 0.5)
    _, dw1, db1, _ = O.layer_bwd(g, vals, x, wl["W1"], dz1, "none", 0.0, need_dh=False)
    F = wl["W1"].shape[1]
    assert m.overflow.item() == 0
    assert_close(m.loss.cpu().numpy(), np.array([ce]), prec, "cross-entropy")
    assert_close(m.distill_loss.cpu().numpy(), np.array([kd]), prec, "distillation")
    dZ = m.dZ2f if level == "O1" else m.dZ2
    assert_close(dZ[:, :C].float().cpu().numpy(), dz2, prec, "dZ2")
    assert_close(m.dW2()[:, :C].cpu().numpy(), dw2, prec, "dW2")
    assert_close(m.db2()[:C].cpu().numpy(), db2, prec, "db2")
    assert_close(m.dW1()[:, :F].cpu().numpy(), dw1, prec, "dW1")
    assert_close(m.db1()[:F].cpu().numpy(), db1, prec, "db1")


@pytest.mark.parametrize("prec", [0, 1])
def test_labels_for_self_training(prec):
    wl = I.workload("er2k", 0, n_override=512)
    m = make(wl, prec)
    m.forward(0, training=False)
    C = wl["W2"].shape[1]
    unlabelled = (m.mask == 0).to(torch.uint8)
    given = m.labels.clone()
    u = torch.rand(m.n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    prob = torch.full((m.n,), -1.0, device="cuda")
    m.sample_labels(u, m.labels, prob, unlabelled, temperature=0.5, top_k=5, top_p=0.9)
    z = m.Z2[:, :C].double().cpu().numpy()
    wy, _ = S.sample_labels(z, u.double().cpu().numpy(), 0.5, 5, float(np.float32(0.9)), 0.0,
                            unlabelled.cpu().numpy(), given.cpu().numpy())
    assert np.array_equal(m.labels.cpu().numpy(), wy)
    labelled = unlabelled == 0
    assert torch.equal(m.labels[labelled], given[labelled]) and (prob[labelled] == -1).all()
    # the drawn labels train the model
    m.mask.fill_(1)
    m.n_mask = m.n
    m.step(0)
    torch.cuda.synchronize()
    assert m.overflow.item() == 0 and np.isfinite(m.loss.item())


@pytest.mark.parametrize("prec", [0, 1])
def test_captured_student(prec):
    """An epoch with a teacher, and draws of labels after it, captured and
    replayed: every replay gives the eager bits."""
    wl = I.workload("er2k", 0, n_override=512)
    teacher = make(wl, prec, seed=5)
    teacher.forward(0, training=False)
    tv, tc = teacher.top_logits(8)
    eager, rep = (make(wl, prec, device_epoch=True) for _ in range(2))
    for m in (eager, rep):
        m.set_teacher(tv, tc, temperature=3.0, weight=2.0)
        m.drawn = torch.zeros(m.n, dtype=torch.int32, device="cuda")
        m.prob = torch.zeros(m.n, device="cuda")
    u = torch.rand(wl["n"], generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")
    rep.capture()
    with pytest.raises(ValueError):
        rep.set_teacher(None, None)
    draws = torch.cuda.CUDAGraph()
    with torch.cuda.graph(draws):
        rep.sample_labels(u, rep.drawn, rep.prob, temperature=0.7, top_p=0.8)
    for k in range(5):
        eager.step(0)
        eager.sample_labels(u, eager.drawn, eager.prob, temperature=0.7, top_p=0.8)
        rep.replay()
        draws.replay()
        torch.cuda.synchronize()
        assert float(torch.arange(4096, device="cuda", dtype=torch.float32).sum()) == 4096 * 4095 / 2
        for t in ("master", "m", "v", "scaler", "grad", "loss", "distill_loss", "drawn", "prob"):
            assert torch.equal(getattr(eager, t), getattr(rep, t)), (k, t)
        assert (rep.drawn >= 0).all()


def test_student_without_a_teacher_is_unchanged():
    wl = I.workload("er2k", 0, n_override=512)
    a, b = make(wl, 1), make(wl, 1)
    tv, tc = a.top_logits(8) if a.forward(0, training=False) is None else (None, None)
    b.set_teacher(tv, tc)
    b.set_teacher(None, None)
    for m in (a, b):
        m.step(0)
    torch.cuda.synchronize()
    assert torch.equal(a.master, b.master) and torch.equal(a.loss, b.loss)


def test_bad_scores_do_not_skip_a_step():
    wl = I.workload("er2k", 0, n_override=512)
    m = make(wl, 1)
    m.forward(0, training=False)
    m.Z2[3, 2] = float("nan")
    m.top_logits(8)
    y = torch.zeros(m.n, dtype=torch.int32, device="cuda")
    m.sample_labels(torch.full((m.n,), 0.5, device="cuda"), y)
    assert m.scores_overflow.item() == 1 and y[3].item() == -1 and (y >= 0).sum().item() == m.n - 1
    m.step(0)
    assert m.scaler_state()["step"] == 1


def test_refusals():
    wl = I.workload("er2k", 0, n_override=512)
    m = make(wl, 1)
    m.forward(0, training=False)
    tv, tc = m.top_logits(8)
    for v, c in ((tv[1:], tc[1:]), (tv, tc.long()), (tv.double(), tc), (tv[:, :5], tc[:, :5]), (tv.cpu(), tc.cpu()),
                 (tv, tc[:, :4].contiguous())):
        with pytest.raises(ValueError):
            m.set_teacher(v, c)
    with pytest.raises(ValueError):
        m.set_teacher(tv, tc, mask=np.ones(7, np.uint8))
    wide = torch.zeros((m.n, 264), dtype=tv.dtype, device="cuda")
    with pytest.raises(ValueError):
        m.set_teacher(wide, wide.to(torch.int32))
    u = torch.rand(m.n, device="cuda")
    for bad in (dict(u=u.double()), dict(u=u[1:]), dict(labels=m.labels.long()), dict(mask=m.labels),
                dict(prob=u.half()), dict(u=u.cpu())):
        with pytest.raises(ValueError):
            m.sample_labels(**dict(dict(u=u, labels=m.labels), **bad))
    with pytest.raises(G.GcnError):
        m.sample_labels(u, m.labels, top_p=0.0)
    with pytest.raises(G.GcnError):
        m.top_logits(300)
