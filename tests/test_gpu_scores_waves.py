"""Long rows' draws where the waves of a workgroup are far apart in time: rows
just past a lane group's width, where a pass over the row is a few
instructions, and as many rows at once as the chip holds, each with scores of
its own level, so that what one wave takes from another at the wrong moment
changes the answer.  Labels against the float64 oracle, and the same bits in
every repetition."""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu


def draws(z, C, prec, u, T, k, p, m):
    n = z.shape[0]
    ws = torch.empty(G.gcn_sample_labels_workspace_size(n, C, prec), dtype=torch.uint8, device="cuda")
    ov = torch.zeros(1, dtype=torch.int32, device="cuda")
    out = []
    for _ in range(4):
        y = torch.full((n,), -7, dtype=torch.int32, device="cuda")
        pr = torch.full((n,), -7.0, device="cuda")
        G.gcn_sample_labels(n, C, z.shape[1], prec, z, None, u, T, k, p, m, y, pr, ov, ws)
        out.append((y, pr))
    assert ov.item() == 0
    for y, pr in out[1:]:
        assert torch.equal(y, out[0][0]) and torch.equal(pr, out[0][1])
    return out[0]


@pytest.mark.parametrize("prec", [0, 1, 2])
def test_many_short_rows_under_top_k(prec):
    """256 < top_k < C: the lowest score of the row is looked for right after
    its largest."""
    n, C = 1500, 1025 if prec else 513
    k = 260 if prec == 0 else 500
    rng = np.random.default_rng(prec)
    z = rng.standard_normal((n, C)) * 2 + 20 * rng.standard_normal((n, 1))
    zt = torch.full((n, round8(C)), float("nan"), dtype=G.torch_dtype(prec), device="cuda")
    zt[:, :C] = torch.as_tensor(z.astype(np.float32)).cuda().to(zt.dtype)
    zh = zt[:, :C].double().cpu().numpy()
    u = rng.random(n).astype(np.float32)
    for p, T in ((1.0, 1.0), (0.9, 2.0)):
        print(f"[waves] top_k={k} prec={prec} p={p} T={T}", flush=True)
        y, _ = draws(zt, C, prec, torch.as_tensor(u).cuda(), T, k, p, 0.0)
        wy, _ = S.sample_labels(zh, u.astype(np.float64), T, k, float(np.float32(p)), 0.0)
        assert np.array_equal(y.cpu().numpy(), wy)


@pytest.mark.parametrize("prec", [0, 1, 2])
@pytest.mark.parametrize("C", [1025, 2049, 9001])
def test_doubt_without_a_border(C, prec):
    """No top-k and no top-p: every row's u lies on a running sum exactly, so
    that the draw in 32 bits is in doubt and the one in 64 bits follows it at
    once.  Scores are equal in a power of two of classes and out of the row in
    the others: the answers are whole numbers."""
    n, half = 700, 512
    print(f"[waves] doubt C={C} prec={prec}", flush=True)
    rng = np.random.default_rng(C)
    z = np.full((n, C), -np.inf)
    at = np.stack([np.sort(rng.permutation(C)[:half]) for _ in range(n)])
    z[np.arange(n)[:, None], at] = rng.integers(-3, 4, (n, 1))
    zt = torch.full((n, round8(C)), float("nan"), dtype=G.torch_dtype(prec), device="cuda")
    zt[:, :C] = torch.as_tensor(z.astype(np.float32)).cuda().to(zt.dtype)
    j = rng.integers(0, half, n)
    y, pr = draws(zt, C, prec, torch.as_tensor((j / half).astype(np.float32)).cuda(), 0.5, 0, 1.0, 0.0)
    assert np.array_equal(y.cpu().numpy(), at[np.arange(n), j])
    assert (pr == 1 / half).all()


@pytest.mark.parametrize("prec,C,n", [(1, 1024, 4000), (2, 1024, 4000), (0, 512, 4000), (1, 64, 30000)])
def test_many_draws_in_lane_groups(prec, C, n):
    """Thousands of rows a case, the widest rows of a lane group among them:
    the labels are those of 64 bits, the few rows near a border too."""
    print(f"[waves] groups n={n} C={C} prec={prec}", flush=True)
    rng = np.random.default_rng(C + prec)
    z = rng.standard_normal((n, C)) * np.where(np.arange(n) % 2, 3.0, 0.2)[:, None]
    zt = torch.full((n, round8(C)), float("nan"), dtype=G.torch_dtype(prec), device="cuda")
    zt[:, :C] = torch.as_tensor(z.astype(np.float32)).cuda().to(zt.dtype)
    zh = zt[:, :C].double().cpu().numpy()
    u = rng.random(n).astype(np.float32)
    for k, p, m in ((0, 1.0, 0.0), (C // 2, 0.9, 0.0)):
        y, _ = draws(zt, C, prec, torch.as_tensor(u).cuda(), 0.9, k, p, m)
        wy, _ = S.sample_labels(zh, u.astype(np.float64), float(np.float32(0.9)), k, float(np.float32(p)), m)
        assert np.array_equal(y.cpu().numpy(), wy)


@pytest.mark.parametrize("prec", [0, 1, 2])
@pytest.mark.parametrize("C", [64, 900, 1300, 9001, 50001])
def test_u_next_to_running_sums(C, prec):
    """u is the fp32 number nearest to a running sum's share, or its neighbour:
    32 bits cannot tell on which side of it the draw falls, 64 bits can."""
    n = 200 if C < 9000 else 40
    print(f"[waves] next to sums C={C} prec={prec}", flush=True)
    rng = np.random.default_rng(C)
    z = rng.standard_normal((n, C)) * np.where(np.arange(n) % 2, 2.0, 0.3)[:, None]
    zt = torch.full((n, round8(C)), float("nan"), dtype=G.torch_dtype(prec), device="cuda")
    zt[:, :C] = torch.as_tensor(z.astype(np.float32)).cuda().to(zt.dtype)
    zh = zt[:, :C].double().cpu().numpy()
    w = np.exp(zh - zh.max(1, keepdims=True))
    run = np.cumsum(w, 1) / w.sum(1, keepdims=True)
    u = run[np.arange(n), rng.integers(0, C - 1, n)].astype(np.float32)
    u = np.where(np.arange(n) % 3 == 0, np.nextafter(u, np.float32(0)), u)
    # a share p of the sum can be the definition's to 2^-53 only: sums that
    # equal u to 12 digits decide nothing
    sure = np.abs(run - u.astype(np.float64)[:, None]).min(1) > 1e-12
    assert sure.sum() > 0.9 * n
    y, _ = draws(zt, C, prec, torch.as_tensor(u).cuda(), 1.0, 0, 1.0, 0.0)
    wy, _ = S.sample_labels(zh, u.astype(np.float64), 1.0)
    assert np.array_equal(y.cpu().numpy()[sure], wy[sure])


@pytest.mark.parametrize("prec", [0, 2])
def test_same_bits_whatever_the_timing(prec):
    """Sums that threads add to as they come: rows of nearly equal scores (all
    classes in the histograms), of few different ones and of large top-k, many
    times over beside another stream's work."""
    n, C = 48, 30011
    rng = np.random.default_rng(prec)
    rows = [rng.standard_normal(C) * 0.1, rng.integers(0, 5, C) / 3.0, rng.standard_normal(C) * 3,
            np.where(rng.random(C) < 0.5, 0.0, 1.0 / 3.0)]
    z = np.stack([rng.permutation(rows[i % 4]) for i in range(n)])
    zt = torch.full((n, round8(C)), float("nan"), dtype=G.torch_dtype(prec), device="cuda")
    zt[:, :C] = torch.as_tensor(z.astype(np.float32)).cuda().to(zt.dtype)
    u = torch.as_tensor(rng.random(n).astype(np.float32)).cuda()
    side = torch.cuda.Stream()
    busy = torch.ones(1 << 24, device="cuda")
    for k, p, m in ((0, 0.75, 0.0), (5000, 0.5, 0.0), (0, 0.999, 0.01)):
        print(f"[waves] timing prec={prec} k={k} p={p}", flush=True)
        first = draws(zt, C, prec, u, 1.0, k, p, m)
        for _ in range(6):
            with torch.cuda.stream(side):
                busy.mul_(1.0)
            y, pr = draws(zt, C, prec, u, 1.0, k, p, m)
            assert torch.equal(y, first[0]) and torch.equal(pr, first[1])
        torch.cuda.synchronize()
