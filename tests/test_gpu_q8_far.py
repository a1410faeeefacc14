"""Rows in 8 bits whose codes or gradients lie 2^25 bytes and more apart (64 rows
span 2^31): every type and width takes the same kernels there."""
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from tests.test_gpu_q8 import NAN, PRECS, backward, padded, round8, round16

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("far", ["codes", "gradient"])
@pytest.mark.parametrize("n,M,N", [(70, 40, 7), (66, 17, 30), (130, 33, 40), (65, 130, 64), (70, 40, 100), (67, 9, 200)])
@pytest.mark.parametrize("prec", PRECS)
def test_backward(prec, n, M, N, far):
    """Whole numbers: |dW| <= 255 * 2 n / 4 and |dZ| <= 4 N have under 24 bits, so every sum is exact."""
    dt = G.torch_dtype(prec)
    size = dt.itemsize
    gen = torch.Generator(device="cuda").manual_seed(n + N)
    for kind, act in (("relu", G.GCN_ACT_RELU), ("signed", G.GCN_ACT_NONE)):
        q = torch.randint(-127 if kind == "signed" else 0, 128 if kind == "signed" else 256, (n, M), generator=gen,
                          device="cuda", dtype=torch.int32)
        q *= torch.randint(0, 2, (n, M), generator=gen, device="cuda", dtype=torch.int32)
        g = torch.randint(-2, 3, (n, N), generator=gen, device="cuda")
        w = torch.randint(-1, 2, (M, N), generator=gen, device="cuda")
        tq = torch.full((n, 1 << 25 if far == "codes" else round16(M)), 0x5a, dtype=torch.uint8, device="cuda")
        tq[:, :M] = (q & 255).to(torch.uint8)
        tg = torch.empty((n, (1 << 25) // size if far == "gradient" else round8(N)), dtype=dt, device="cuda")
        tg[:, :round8(N)] = NAN
        tg[:, :N] = g.to(dt)
        p = 0.5 if act else 0.0
        dW, dZ, db, ov = backward(tq, torch.full((n,), 0.25, device="cuda"), padded(w, dt, round8(N)), tg, prec, kind, n, M,
                                  N, act, p)
        z = g.double() @ w.double().t().contiguous()
        if act:
            z = z * (q > 0) * 2
        assert torch.equal(dW[:, :N].double(), 0.25 * (q.double().t().contiguous() @ g.double())), kind
        assert not dW[:, N:].any() and ov.item() == 0
        assert torch.equal(dZ[:, :M], z.to(dt)) and torch.equal(db[:M].double(), z.sum(0)), kind
