"""The operators on class scores as programs call them: one after the other,
captured and replayed, on another stream than the current one, side by side on
two streams, on more rows than one pass of the grid takes, and repeated (the
same bits every time)."""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu


class Program:
    """Teacher scores -> top logits -> student's loss and gradient -> labels."""

    def __init__(self, n, C, K, prec, seed, top_k=0, top_p=0.9, min_p=0.01):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.C, self.K, self.prec, self.ld = n, C, K, prec, round8(C)
        self.filters = (top_k, float(np.float32(top_p)), float(np.float32(min_p)))
        dt = G.torch_dtype(prec)
        self.zt, self.zs = ((torch.randn((n, self.ld), generator=gen, device="cuda") * 3).to(dt) for _ in range(2))
        self.u = torch.rand(n, generator=gen, device="cuda")
        ldk = round8(K)
        self.v = torch.zeros((n, ldk), dtype=dt, device="cuda")
        self.c = torch.zeros((n, ldk), dtype=torch.int32, device="cuda")
        self.loss = torch.zeros(1, device="cuda")
        self.d = torch.zeros((n, self.ld), dtype=dt, device="cuda")
        self.y = torch.zeros(n, dtype=torch.int32, device="cuda")
        self.prob = torch.zeros(n, device="cuda")
        self.ov = torch.zeros(1, dtype=torch.int32, device="cuda")
        self.ws = torch.full((max(G.gcn_top_logits_workspace_size(n, C, K, prec),
                                  G.gcn_distill_workspace_size(n, C, K, prec),
                                  G.gcn_sample_labels_workspace_size(n, C, prec)),), 0xFF, dtype=torch.uint8,
                             device="cuda")

    def run(self, stream=None):
        n, C, ld, prec, K, ldk = self.n, self.C, self.ld, self.prec, self.K, self.v.shape[1]
        G.gcn_top_logits(n, C, ld, prec, self.zt, K, ldk, self.v, self.c, self.ov, self.ws, stream)
        G.gcn_distill(n, C, ld, prec, self.zs, K, ldk, prec, self.v, self.c, None, n, 2.0, 1.0, None, None, self.loss,
                      self.d, self.ov, self.ws, stream)
        G.gcn_sample_labels(n, C, ld, prec, self.zs, None, self.u, 0.8, *self.filters, self.y, self.prob, self.ov,
                            self.ws, stream)

    def outputs(self):
        return dict(v=self.v[:, :self.K], c=self.c[:, :self.K], loss=self.loss, d=self.d[:, :self.C], y=self.y,
                    prob=self.prob, ov=self.ov)

    def take(self):
        return {k: t.clone() for k, t in self.outputs().items()}

    def clear(self):
        for t in self.outputs().values():
            t.zero_()


def same(a, b):
    for k in a:
        assert torch.equal(a[k], b[k]), k


CASES = [(300, 64, 8, 1, {}), (200, 700, 20, 2, {}), (5, 3000, 16, 0, {}), (3, 70001, 40, 1, {}),
         (4, 40000, 256, 0, dict(top_k=400)), (260, 9001, 64, 2, dict(top_k=50)), (6, 20011, 5, 1, dict(top_p=1.0, min_p=0.0))]


@pytest.mark.parametrize("n,C,K,prec,filters", CASES)
def test_program(n, C, K, prec, filters):
    """In sequence, against the oracle; then again, on a side stream and from
    a graph: the same bits."""
    print(f"[program] n={n} C={C} K={K} prec={prec} {filters}", flush=True)
    P = Program(n, C, K, prec, C, **filters)
    P.run()
    first = P.take()
    zt, zs = (t[:, :C].double().cpu().numpy() for t in (P.zt, P.zs))
    wv, wc = S.top_logits(zt, K)
    assert np.array_equal(first["c"].cpu().numpy(), wc) and np.array_equal(first["v"].double().cpu().numpy(), wv)
    wl, wg, _ = S.distill(zs, wv, wc, 2.0)
    # the parts' bounds are derived in test_gpu_scores.py; here: 2^-18 of the
    # loss's terms (at most 2 ln C + 30 each) and half a step of the type
    assert abs(first["loss"].item() - wl) <= 2.0 ** -18 * 4 * (2 * np.log(C) + 30)
    half = {0: 2.0 ** -24, 1: 2.0 ** -11, 2: 2.0 ** -8}[prec]
    tiny = {0: 0.0, 1: 2.0 ** -25, 2: 0.0}[prec]
    err = np.abs(first["d"].double().cpu().numpy() - wg)
    assert (err <= half * np.abs(wg) + 2.0 ** -17 * np.abs(wg).max() + tiny).all()
    wy, _ = S.sample_labels(zs, P.u.double().cpu().numpy(), float(np.float32(0.8)), *P.filters)
    assert np.array_equal(first["y"].cpu().numpy(), wy)
    assert first["ov"].item() == 0
    P.clear()
    P.run()
    same(first, P.take())
    side = torch.cuda.Stream()
    P.clear()
    side.wait_stream(torch.cuda.current_stream())
    P.run(side)
    side.synchronize()
    same(first, P.take())
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        P.run()
    for _ in range(4):
        P.clear()
        junk = torch.arange(4096, device="cuda", dtype=torch.float32).sum()
        graph.replay()
        torch.cuda.synchronize()
        assert float(junk) == 4096 * 4095 / 2
        same(first, P.take())


def test_two_streams_at_once():
    """Two programs with buffers of their own on two streams."""
    a, b = Program(2000, 64, 8, 1, 1), Program(9, 50001, 64, 2, 2)
    want = []
    for p in (a, b):
        p.run()
        want.append(p.take())
        p.clear()
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        a.run(s1)
        b.run(s2)
    torch.cuda.synchronize()
    same(want[0], a.take())
    same(want[1], b.take())


def test_more_rows_than_the_grid():
    """Narrow rows past 65536 workgroups: the workgroups walk on.  Two classes:
    the answers are closed forms."""
    n, C, ld = 65536 * 4 * 256 + 12345, 2, 8
    print(f"[program] n={n}", flush=True)
    z = torch.empty((n, ld), dtype=torch.float16, device="cuda")
    i = torch.arange(n, device="cuda")
    z[:, 0] = 1.0
    z[:, 1] = torch.where(i % 3 == 0, 2.0, 0.5).half()
    win = (i % 3 == 0).int()
    v = torch.zeros((n, 8), dtype=torch.float16, device="cuda")
    c = torch.full((n, 8), -9, dtype=torch.int32, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(G.gcn_top_logits_workspace_size(n, C, 1, 1), G.gcn_sample_labels_workspace_size(n, C, 1),
                         G.gcn_distill_workspace_size(n, C, 1, 1)), dtype=torch.uint8, device="cuda")
    G.gcn_top_logits(n, C, ld, 1, z, 1, 8, v, c, ov, ws)
    assert torch.equal(c[:, 0], win) and (c[:, 1:] == -9).all()
    assert torch.equal(v[:, 0], torch.maximum(z[:, 0], z[:, 1]))
    # p(class 0) = 1 / (1 + e^1) where class 1 leads, 1 / (1 + e^-0.5) elsewhere
    u = torch.where(i % 2 == 0, 0.25, 0.75).float()
    y = torch.full((n,), -9, dtype=torch.int32, device="cuda")
    G.gcn_sample_labels(n, C, ld, 1, z, None, u, 1.0, 0, 1.0, 0.0, y, None, ov, ws)
    p0 = torch.where(i % 3 == 0, 1 / (1 + np.e), 1 / (1 + np.exp(-0.5)))
    assert torch.equal(y, (u >= p0).int())
    del u, y, v
    # the teacher names the leading class: cross-entropy against it
    loss = torch.zeros(1, device="cuda")
    d = torch.full((n, ld), 9.0, dtype=torch.float16, device="cuda")
    t = torch.zeros((n, 8), dtype=torch.float16, device="cuda")
    scale = torch.full((1,), float(n), device="cuda")
    G.gcn_distill(n, C, ld, 1, z, 1, 8, 1, t, c, None, n, 1.0, 1.0, scale, None, loss, d, ov, ws)
    ones = int(win.sum().item())
    want = (ones * np.log1p(np.exp(-1.0)) + (n - ones) * np.log1p(np.exp(-0.5))) / n
    # n terms in chains of at most 2^12: within 2^-11 by the worst bound, and
    # rounding errors of one sign only would reach it
    assert abs(loss.item() - want) <= 2.0 ** -11 * want
    for k, val in ((0, 1 / (1 + np.exp(-1.0)) - 1), (1, 1 / (1 + np.exp(-0.5)) - 1)):
        lead = d[i % 3 == 0, 1] if k == 0 else d[i % 3 != 0, 0]
        assert (lead - val).abs().max().item() <= 2.0 ** -11
    assert ov.item() == 0


@pytest.mark.parametrize("C", [1022, 1023, 1024, 1025, 511, 512, 513, 255, 257])
@pytest.mark.parametrize("prec", [0, 1, 2])
def test_either_side_of_a_kernel(C, prec):
    """The widths at which another kernel takes over."""
    print(f"[program] C={C} prec={prec}", flush=True)
    for filters in ({}, dict(top_k=30), dict(top_p=1.0, min_p=0.0)):
        P = Program(9, C, 20, prec, C, **filters)
        P.run()
        zt, zs = (t[:, :C].double().cpu().numpy() for t in (P.zt, P.zs))
        _, wc = S.top_logits(zt, 20)
        wy, _ = S.sample_labels(zs, P.u.double().cpu().numpy(), float(np.float32(0.8)), *P.filters)
        assert np.array_equal(P.c[:, :20].cpu().numpy(), wc)
        assert np.array_equal(P.y.cpu().numpy(), wy)
        assert P.ov.item() == 0


@pytest.mark.parametrize("prec", [0, 1, 2])
@pytest.mark.parametrize("C", [3000, 30011])
def test_spread_scores(C, prec):
    """Long rows whose mass lies on few, many, nearly all or exactly equal
    classes: every way in which the border of top-p is found."""
    n = 8
    rng = np.random.default_rng(C)
    k = np.arange(C)
    rows = [rng.standard_normal(C) * 3, rng.standard_normal(C) * 0.3, np.zeros(C), -k / C, np.where(k % 2, 0.0, -30.0),
            rng.standard_normal(C) * 8, np.sort(rng.standard_normal(C) * 3), np.where(k < C // 2, 1.0, 1.0 - 2.0 ** -6)]
    ld = round8(C)
    z = torch.full((n, ld), float("nan"), dtype=G.torch_dtype(prec), device="cuda")
    z[:, :C] = torch.as_tensor(np.stack(rows).astype(np.float32)).cuda().to(z.dtype)
    zh = z[:, :C].double().cpu().numpy()
    ws = torch.empty(G.gcn_sample_labels_workspace_size(n, C, prec), dtype=torch.uint8, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    y = torch.zeros(n, dtype=torch.int32, device="cuda")
    pr = torch.zeros(n, device="cuda")
    for top_k, top_p, min_p in ((0, 0.9, 0.0), (0, 0.3, 0.0), (0, 0.9999, 0.0), (0, 1.0, 0.2), (1000, 0.7, 0.0), (300, 1.0, 0.0),
                                (C - 1, 0.99, 0.001)):
        for T in (1.0, 5.0):
            print(f"[program] spread C={C} prec={prec} k={top_k} p={top_p} m={min_p} T={T}", flush=True)
            u = torch.as_tensor(rng.random(n).astype(np.float32)).cuda()
            G.gcn_sample_labels(n, C, ld, prec, z, None, u, T, top_k, top_p, min_p, y, pr, ov, ws)
            wy, wp = S.sample_labels(zh, u.double().cpu().numpy(), T, top_k, float(np.float32(top_p)),
                                     float(np.float32(min_p)))
            assert np.array_equal(y.cpu().numpy(), wy), (top_k, top_p, min_p, T)
            # see check_sample in test_gpu_scores.py
            assert (np.abs(pr.double().cpu().numpy() - wp) <= 2.0 ** -17 * wp).all()
    assert ov.item() == 0


@pytest.mark.parametrize("prec", [0, 1, 2])
@pytest.mark.parametrize("C", [7, 64, 300, 5000])
def test_nan_of_either_sign(C, prec):
    """NaN is no score whatever its sign and payload: left out of the top
    scores, no label drawn from its row, reported by both."""
    n, K, ld = 6, 5, round8(C)
    rng = np.random.default_rng(C)
    z = torch.as_tensor(rng.standard_normal((n, ld)).astype(np.float32)).cuda().to(G.torch_dtype(prec))
    bits = z.view(torch.int32 if prec == 0 else torch.int16)
    quiet = {0: 0x7FC00001, 1: 0x7E01, 2: 0x7FC1}[prec]
    low = -(1 << 31) if prec == 0 else -(1 << 15)
    bits[1, C // 2] = quiet
    bits[3, C - 1] = quiet + low                     # the same with a sign
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    for row, flagged in ((1, True), (3, True), (2, False)):
        ov.zero_()
        one = z[row:row + 1].contiguous()
        ws = torch.empty(max(G.gcn_top_logits_workspace_size(1, C, K, prec),
                             G.gcn_sample_labels_workspace_size(1, C, prec)), dtype=torch.uint8, device="cuda")
        v = torch.zeros((1, 8), dtype=z.dtype, device="cuda")
        c = torch.zeros((1, 8), dtype=torch.int32, device="cuda")
        G.gcn_top_logits(1, C, ld, prec, one, K, 8, v, c, ov, ws)
        wv, wc = S.top_logits(one[:, :C].double().cpu().numpy(), K)
        assert np.array_equal(c[:, :K].cpu().numpy(), wc) and np.array_equal(v[:, :K].double().cpu().numpy(), wv)
        assert ov.item() == int(flagged)
        for k, p in ((0, 1.0), (0, 0.9), (3, 0.9)):
            ov.zero_()
            y = torch.zeros(1, dtype=torch.int32, device="cuda")
            u = torch.full((1,), 0.5, device="cuda")
            G.gcn_sample_labels(1, C, ld, prec, one, None, u, 1.0, k, p, 0.0, y, None, ov, ws)
            assert (y.item() == -1) == flagged and ov.item() == int(flagged)


@pytest.mark.parametrize("C", [7, 64, 3000])
@pytest.mark.parametrize("value", [float("nan"), float("inf")])
def test_teacher_that_is_not_finite(C, value):
    """A teacher's NaN or +inf makes the loss non-finite and is reported; rows
    outside the mask are not looked at."""
    n, K, ld = 5, 3, round8(C)
    z = torch.zeros((n, ld), device="cuda")
    v = torch.zeros((n, 8), device="cuda")
    c = torch.full((n, 8), -1, dtype=torch.int32, device="cuda")
    c[:, :K] = torch.arange(K, device="cuda")
    v[2, 1] = value
    ws = torch.empty(G.gcn_distill_workspace_size(n, C, K, 0), dtype=torch.uint8, device="cuda")
    mask = torch.ones(n, dtype=torch.uint8, device="cuda")
    for out in (False, True):
        mask[2] = 0 if out else 1
        ov = torch.zeros(1, dtype=torch.int32, device="cuda")
        loss, d = torch.zeros(1, device="cuda"), torch.zeros((n, ld), device="cuda")
        G.gcn_distill(n, C, ld, 0, z, K, 8, 0, v, c, mask, n - out, 1.0, 1.0, None, None, loss, d, ov, ws)
        assert ov.item() == (0 if out else 1)
        assert bool(torch.isfinite(loss).item()) == out
        # K of C equal scores named: ln(C / K)
        if out:
            assert abs(loss.item() - np.log(C / K)) < 1e-6 * np.log(C)
            assert torch.isfinite(d[:, :C]).all() and (d[2] == 0).all()
