"""Scores of the smallest magnitudes, subnormal numbers among them, are ordered
like any others, and their classes' probabilities are all but equal; column sums
of the distillation gradient with padding behind the classes on every way they
are added up."""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8
from tests.test_gpu_scores import E, distill, host, put, run_sample, run_top

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", [0, 1, 2])
@pytest.mark.parametrize("n,C", [(9, 7), (9, 64), (5, 300), (5, 1000), (4, 5000), (3, 40000)])
def test_subnormal_scores(n, C, prec):
    """Whole multiples of the smallest subnormal number, of both signs."""
    print(f"[tiny] n={n} C={C} prec={prec}", flush=True)
    rng = np.random.default_rng(C)
    bits = rng.integers(0, 100, (n, C)) + np.where(rng.random((n, C)) < 0.5, 0, -2 ** 31 if prec == 0 else -2 ** 15)
    z = torch.zeros((n, round8(C)), dtype=G.torch_dtype(prec))
    z[:, :C] = torch.as_tensor(bits.astype(np.int32 if prec == 0 else np.int16)).view(z.dtype)
    zt = z.cuda()
    zh = host(zt, C)
    assert np.abs(zh).max() < 2.0 ** -17 and len(np.unique(zh)) > 1
    K = min(C, 40)
    v, c, ov = run_top(zt, n, C, zt.shape[1], prec, K)
    wv, wc = S.top_logits(zh, K)
    assert np.array_equal(c[:, :K].cpu().numpy(), wc) and np.array_equal(host(v, K), wv) and ov.item() == 0
    u = rng.random(n).astype(np.float32)
    # weights exp(x), |x| < 2^-6: a sum of C of them; no sum near a border is asked for
    for k, p in ((1, 1.0), (C // 2, 1.0), (300, 1.0)):
        y, _, ov = run_sample(zt, n, C, prec, torch.as_tensor(u).cuda(), 1.0, k, p)
        wy, _ = S.sample_labels(zh, u.astype(np.float64), 1.0, k, p)
        assert np.array_equal(y.cpu().numpy(), wy) and ov.item() == 0


@pytest.mark.parametrize("n,C,extra", [(500, 7, 16), (40000, 64, 24), (300000, 64, 8), (300000, 200, 64), (9, 256, 128)])
@pytest.mark.parametrize("prec", [0, 1])
def test_column_sums_with_padding(n, C, extra, prec):
    """Few, many and very many workgroups; the sums are whole numbers."""
    print(f"[tiny] column sums n={n} C={C} prec={prec}", flush=True)
    ld = round8(C) + extra
    zt = put(np.zeros((n, C)), prec, ld)
    vt = torch.zeros((n, 8), dtype=zt.dtype, device="cuda")
    ct = torch.full((n, 8), -1, dtype=torch.int32, device="cuda")
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mask[0] = 1                                   # nothing named: no row counts
    rng = np.random.default_rng(C)
    base = torch.as_tensor(rng.integers(-3, 4, (n, C)).astype(np.float32)).cuda()
    bt = torch.full((n, ld), float("nan"), dtype=zt.dtype, device="cuda")
    bt[:, :C] = base
    loss, d, cs, ov = distill(zt, vt, ct, n, C, 1, prec, prec, 1.0, 1.0, mask, 1, 1.0, bt, False, True)
    assert torch.equal(d[:, :C].float(), base) and loss.item() == 0 and ov.item() == 0
    assert torch.equal(cs[:C], base.sum(0)) and (cs[C:] == 0).all()
