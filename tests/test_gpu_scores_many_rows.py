"""More long rows than one launch takes (262144 workgroups): every kernel of
the operators on class scores that gives a row a workgroup, or several, of its
own.  Equal scores but for one class a row: the answers are closed forms."""
import numpy as np
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu
N, C = (1 << 18) * 2 + 37, 513
LD = round8(C)


def rows(n, classes, ld, dtype, lead):
    i = torch.arange(n, device="cuda")
    at = i * 7 % classes
    z = torch.zeros((n, ld), dtype=dtype, device="cuda")
    z[i, at] = lead
    return z, at


@pytest.mark.parametrize("K", [5, 40, 70])
def test_top(K):
    print(f"[many rows] top K={K}", flush=True)
    z, at = rows(N, C, LD, torch.float32, 3.0)
    v = torch.full((N, round8(K)), 9.0, device="cuda")
    c = torch.full((N, round8(K)), 9, dtype=torch.int32, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.gcn_top_logits_workspace_size(N, C, K, 0), dtype=torch.uint8, device="cuda")
    G.gcn_top_logits(N, C, LD, 0, z, K, round8(K), v, c, ov, ws)
    assert torch.equal(c[:, 0], at.int()) and (v[:, 0] == 3).all() and (v[:, 1:K] == 0).all()
    j = torch.arange(K - 1, device="cuda")[None]
    assert torch.equal(c[:, 1:K], (j + (j >= at[:, None])).int()) and ov.item() == 0


@pytest.mark.parametrize("k,p", [(20, 1.0), (40, 0.9), (300, 0.9), (0, 0.9), (0, 1.0)])
def test_sample(k, p):
    """The leading class weighs more than all others: u below its share draws
    it wherever it stands, since what comes before it weighs nothing much."""
    print(f"[many rows] sample k={k} p={p}", flush=True)
    z, at = rows(N, C, LD, torch.float32, 30.0)
    u = torch.full((N,), 0.5, device="cuda")
    y = torch.full((N,), -9, dtype=torch.int32, device="cuda")
    pr = torch.full((N,), -9.0, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.gcn_sample_labels_workspace_size(N, C, 0), dtype=torch.uint8, device="cuda")
    G.gcn_sample_labels(N, C, LD, 0, z, None, u, 1.0, k, p, 0.0, y, pr, ov, ws)
    assert torch.equal(y, at.int()) and (pr > 0.999).all() and (pr <= 1).all() and ov.item() == 0


def test_distill():
    print("[many rows] distill", flush=True)
    z, at = rows(N, C, LD, torch.float32, 3.0)
    v = torch.zeros((N, 8), device="cuda")
    c = torch.full((N, 8), -1, dtype=torch.int32, device="cuda")
    c[:, 0] = at.int()
    loss = torch.zeros(1, device="cuda")
    d = torch.full((N, LD), 9.0, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    scale = torch.full((1,), float(N), device="cuda")
    ws = torch.empty(G.gcn_distill_workspace_size(N, C, 1, 0), dtype=torch.uint8, device="cuda")
    G.gcn_distill(N, C, LD, 0, z, 1, 8, 0, v, c, None, N, 1.0, 1.0, scale, None, loss, d, ov, ws)
    s = np.exp(3.0) + C - 1
    # 513 additions, a quotient and the scale: within 2^-14
    assert abs(loss.item() - (np.log(s) - 3.0)) <= 2.0 ** -12 * np.log(s)
    i = torch.arange(N, device="cuda")
    lead = d[i, at]
    assert (lead - (np.exp(3.0) / s - 1)).abs().max().item() <= 2.0 ** -14
    d[i, at] = 1 / s
    assert (d[:, :C] * s - 1).abs().max().item() <= 2.0 ** -14 and ov.item() == 0


def test_distill_segments():
    """Two segments a row, the loss alone."""
    n, classes = (1 << 17) + 5, 65544
    print(f"[many rows] distill segments n={n}", flush=True)
    z, at = rows(n, classes, classes, torch.bfloat16, 8.0)
    v = torch.zeros((n, 8), dtype=torch.bfloat16, device="cuda")
    c = torch.full((n, 8), -1, dtype=torch.int32, device="cuda")
    c[:, 0] = at.int()
    loss = torch.zeros(1, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(G.gcn_distill_workspace_size(n, classes, 1, 2), dtype=torch.uint8, device="cuda")
    s = np.exp(8.0) + classes - 1
    z[n - 1, at[n - 1]] = 0.0
    # one row at a time: the last, of equal scores, and those beside the launches' border
    for row, want in ((n - 1, np.log(classes)), (n - 2, np.log(s) - 8.0), (1 << 17, np.log(s) - 8.0),
                      ((1 << 17) - 1, np.log(s) - 8.0), (0, np.log(s) - 8.0)):
        mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
        mask[row] = 1
        G.gcn_distill(n, classes, classes, 2, z, 1, 8, 2, v, c, mask, 1, 1.0, 1.0, None, None, loss, None, ov, ws)
        # chains of at most 2^9 additions: within 2^-14
        assert abs(loss.item() - want) <= 2.0 ** -14 * np.log(s) and ov.item() == 0, row
