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
