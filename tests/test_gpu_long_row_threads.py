"""Long rows on either side of every width, row count, number of entries and
top-k at which a workgroup of another size takes over.  References on the GPU:
a stable sort, and for draws the definition in float64."""
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu
VE = {0: 4, 1: 8, 2: 8}


def make_rows(n, C, prec, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    z = (torch.randn((n, round8(C)), generator=gen, device="cuda") * 3).to(G.torch_dtype(prec))
    z[:, C:] = float("nan")
    z[n // 2, :C] = z[n // 2, :C].round()         # a row of many equal scores
    return z, torch.rand(n, generator=gen, device="cuda")


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("vecs", [1024, 4096, 8192])
@pytest.mark.parametrize("n", [3, 513])
def test_top(n, vecs, prec):
    for C in (vecs * VE[prec], vecs * VE[prec] + 1):
        z, _ = make_rows(n, C, prec, C)
        v, i = torch.sort(z[:, :C], dim=1, descending=True, stable=True)
        for K in (1, 32, 64, 65, 128, 129, 256):
            print(f"[threads] top n={n} C={C} K={K} prec={prec}", flush=True)
            tv = torch.zeros((n, round8(K)), dtype=z.dtype, device="cuda")
            tc = torch.zeros((n, round8(K)), dtype=torch.int32, device="cuda")
            ov = torch.zeros(1, dtype=torch.int32, device="cuda")
            ws = torch.empty(G.gcn_top_logits_workspace_size(n, C, K, prec), dtype=torch.uint8, device="cuda")
            G.gcn_top_logits(n, C, z.shape[1], prec, z, K, round8(K), tv, tc, ov, ws)
            assert torch.equal(tc[:, :K], i[:, :K].int()) and torch.equal(tv[:, :K], v[:, :K])
            assert ov.item() == 0


def draw64(z, u, T, k, p):
    """Labels in float64, and whether no sum lies next to a border."""
    z = z.double()
    C = z.shape[1]
    v, i = torch.sort(z, dim=1, descending=True, stable=True)
    w = torch.exp((v - v[:, :1]) / T)
    keep = torch.ones_like(w, dtype=torch.bool)
    if 0 < k < C:
        keep[:, k:] = False
        w[:, k:] = 0.0
    sure = torch.ones(z.shape[0], dtype=torch.bool, device="cuda")
    if p < 1.0:
        run = torch.cumsum(w, 1)
        want = p * run[:, -1:]
        keep &= run - w < want
        sure &= ((run - want).abs() > 1e-11 * want).all(1)
    kept = torch.zeros_like(keep).scatter_(1, i, keep)
    w = torch.where(kept, torch.exp((z - v[:, :1]) / T), 0.0)
    run = torch.cumsum(w, 1)
    want = u[:, None].double() * run[:, -1:]
    sure &= ((run - want).abs() > 1e-11 * run[:, -1:]).all(1)
    return (run <= want).sum(1).int(), sure


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("vecs", [512, 2048, 8192])
@pytest.mark.parametrize("n", [3, 513, 1025])
def test_sample(n, vecs, prec):
    for C in (vecs * VE[prec], vecs * VE[prec] + 1):
        z, u = make_rows(n, C, prec, C + 1)
        ws = torch.empty(G.gcn_sample_labels_workspace_size(n, C, prec), dtype=torch.uint8, device="cuda")
        for k, p in ((5, 1.0), (128, 0.75), (129, 0.75), (256, 1.0), (257, 0.75), (0, 0.75), (0, 1.0)):
            print(f"[threads] sample n={n} C={C} k={k} p={p} prec={prec}", flush=True)
            y = torch.full((n,), -7, dtype=torch.int32, device="cuda")
            ov = torch.zeros(1, dtype=torch.int32, device="cuda")
            G.gcn_sample_labels(n, C, z.shape[1], prec, z, None, u, 1.0, k, p, 0.0, y, None, ov, ws)
            want, sure = draw64(z[:, :C], u, 1.0, k, p)
            assert torch.equal(y[sure], want[sure]) and ov.item() == 0
            assert int((~sure).sum()) <= n // 8 + 1   # the row of equal scores, others by chance


@pytest.mark.parametrize("prec,C,n", [(1, 16, 70000 * 64), (1, 200, 16400 * 16), (1, 400, 16400 * 8), (1, 900, 16400 * 4),
                                      (0, 64, 16400 * 32), (0, 400, 16400 * 4)])
def test_sample_in_lane_groups(prec, C, n):
    """Rows enough for two an iteration where the rule takes two, filters or not."""
    z, u = make_rows(n, C, prec, C)
    z[n // 2] = 0.0
    ws = torch.empty(G.gcn_sample_labels_workspace_size(n, C, prec), dtype=torch.uint8, device="cuda")
    for k, p in ((0, 1.0), (C // 2, 0.75)):
        print(f"[threads] groups n={n} C={C} k={k} p={p} prec={prec}", flush=True)
        y = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        ov = torch.zeros(1, dtype=torch.int32, device="cuda")
        G.gcn_sample_labels(n, C, z.shape[1], prec, z, None, u, 1.0, k, p, 0.0, y, None, ov, ws)
        for a in range(0, n, 1 << 18):
            want, sure = draw64(z[a:a + (1 << 18), :C], u[a:a + (1 << 18)], 1.0, k, p)
            assert torch.equal(y[a:a + (1 << 18)][sure], want[sure])
        assert ov.item() == 0
