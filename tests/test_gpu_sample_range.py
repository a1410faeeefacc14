"""gcn_sample_labels on long rows whose scores lie further apart than fp32
reaches: the largest less the smallest is infinite there, while every score is
an ordinary one of its row's order."""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from tests.test_gpu_scores import NAMES, host, put, run_sample
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", [0, 2], ids=NAMES.get)
@pytest.mark.parametrize("C", [1500, 3000, 40000])
def test_range_past_fp32(C, prec):
    n = 12
    rng = np.random.default_rng(C)
    z = np.full((n, C), -2.0e38)
    for i in range(n):
        z[i, rng.permutation(C)[:300 + 50 * (i % 3)]] = 2.0e38
    z[4] = np.where(z[4] > 0, 2.0e38 - 1.0e36 * rng.integers(0, 3, C), -2.0e38 + 1.0e36 * rng.integers(0, 60, C))
    z[5, ::7] = -np.inf
    zt = put(z, prec, round8(C))
    zh = host(zt, C)
    for k, p, m in ((400, 0.5, 0.0), (320, 0.9, 0.0), (1000, 0.5, 0.0), (C - 1, 0.25, 0.0), (400, 1.0, 0.5),
                    (0, 0.5, 0.0), (20, 0.5, 0.0)):
        print(f"[sample range] C={C} {NAMES[prec]} k={k} p={p} m={m}", flush=True)
        u = rng.random(n).astype(np.float32)
        y, pr, ov = run_sample(zt, n, C, prec, torch.as_tensor(u).cuda(), 1.0, k, p, m)
        wy, wp = S.sample_labels(zh, u.astype(np.float64), 1.0, k, float(np.float32(p)), float(np.float32(m)))
        assert np.array_equal(y.cpu().numpy(), wy), (k, p, m)
        # weights are 0 or 1 and their sums whole: only the quotient rounds
        assert (np.abs(pr.double().cpu().numpy() - wp) <= 2.0 ** -24 * wp).all()
        assert ov.item() == 0
