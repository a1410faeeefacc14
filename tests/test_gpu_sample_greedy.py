"""Draws at temperature 0: the first class of the order, without random
numbers."""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd import inputs as I
from tests.test_gpu_scores import host, put, run_sample, scores
from tests.test_gpu_student import make
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("prec", [0, 1, 2])
@pytest.mark.parametrize("C", [1, 7, 64, 600, 3000, 40000])
def test_without_u(C, prec):
    rng = np.random.default_rng(C)
    for kind in ("normal", "ties", "absent"):
        print(f"[greedy] C={C} prec={prec} {kind}", flush=True)
        zt = put(scores(rng, 9, C, kind), prec, round8(C))
        y, pr, ov = run_sample(zt, 9, C, prec, None, 0.0, 0, 0.5, 0.1)
        wy, wp = S.sample_labels(host(zt, C), np.full(9, 2.0), 0.0, 0, 0.5, 0.1)
        assert np.array_equal(y.cpu().numpy(), wy) and np.array_equal(pr.double().cpu().numpy(), wp)
        assert ov.item() == 0


def test_model_without_u():
    m = make(I.workload("er2k", 0, n_override=512), 1)
    m.forward(0, training=False)
    y = torch.full((m.n,), -9, dtype=torch.int32, device="cuda")
    m.sample_labels(None, y, temperature=0.0)
    _, c = m.top_logits(1)
    assert torch.equal(y, c[:, 0])
    with pytest.raises(G.GcnError):
        m.sample_labels(None, y, temperature=1.0)
