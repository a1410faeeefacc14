"""Every kernel that the launch rules of the 8-bit product and backward pass can
choose, where a workgroup walks more than one tile: exactly on whole numbers, and
for long sums of other numbers within the roundings they are made of."""
import numpy as np
import pytest
import torch

from paper_2010_12635_amd import gcn as G
from tests import test_gpu_q8 as T
from tests.test_gpu_q8 import HALF_STEP, LEAST, PRECS, padded, quantize, round8, round16

pytestmark = pytest.mark.gpu


# weights in LDS: blocks of 128, 64, 32 and (fp32) 16 columns, by 1, 2 and more steps of 64 along k, with more 16-row
# tiles than the launch has waves
@pytest.mark.parametrize("n,K,N", [(70001, 64, 128), (70001, 100, 128), (70001, 500, 128), (70003, 300, 100),
                                   (140001, 64, 64), (140001, 128, 40), (140001, 250, 50), (140001, 480, 60), (280001, 64, 30),
                                   (280001, 128, 30), (270001, 200, 20), (540001, 60, 7), (560001, 128, 16),
                                   (530001, 150, 16)])
@pytest.mark.parametrize("prec", PRECS)
def test_product(prec, n, K, N):
    T.test_product_many_rows(prec, n, K, N)


# one pass: up to 16, 32, 64, 128 and 256 columns of G by up to 32, 64 and 128 of H
@pytest.mark.parametrize("n,M,N", [(200001, 16, 13), (100001, 50, 16), (40000, 130, 9), (300000, 32, 30),
                                   (100001, 60, 30), (400000, 32, 40), (100000, 64, 40), (10000, 20, 100),
                                   (24000, 32, 128), (60000, 32, 100), (60001, 64, 128), (50000, 30, 280),
                                   (70000, 64, 270), (9000, 2000, 2600)])
@pytest.mark.parametrize("prec", PRECS)
def test_backward(prec, n, M, N):
    T.test_backward_many_rows(prec, n, M, N)


# past them: dZ by the row-streaming product, with blocks of 16 to 128 columns of H
@pytest.mark.parametrize("N", [140, 300, 700, 1500])
@pytest.mark.parametrize("n,M", [(3000, 8), (3001, 20), (3002, 40), (3003, 60), (3004, 100), (3005, 130), (40000, 48)])
@pytest.mark.parametrize("prec", PRECS)
def test_backward_wide(prec, n, M, N):
    T.test_backward_many_rows(prec, n, M, N)


@pytest.mark.parametrize("signs", ["mixed", "positive"])
@pytest.mark.parametrize("n,M,N", [(1 << 18, 128, 64), (1 << 17, 2048, 16), (100001, 1000, 100), (90001, 1000, 200),
                                   (1 << 17, 256, 300)])
@pytest.mark.parametrize("prec", PRECS)
def test_long_sums(prec, n, M, N, signs):
    """Tens of tiles a workgroup.  Numbers of one sign are where roundings that cut off would add up to a bias."""
    dt = G.torch_dtype(prec)
    gen = torch.Generator(device="cuda").manual_seed(n + M + N)
    h = torch.randn((n, M), generator=gen, device="cuda").clamp(min=0) * 2
    w = torch.randn((M, N), generator=gen, device="cuda") / M ** 0.5
    g = torch.randn((n, N), generator=gen, device="cuda") * 0.05
    if signs == "positive":
        w, g = w.abs(), g.abs()
    h, w, g = padded(h, dt, round8(M)), padded(w, dt, round8(N)), padded(g, dt, round8(N))
    q, s, _ = quantize(h, M, prec, "relu", round16(M))
    p = float(np.float32(0.3))
    dW, dZ, db, ov = T.backward(q, s, w, g, prec, "relu", n, M, N, G.GCN_ACT_RELU, p)
    G.gcn_dequantize(n, M, G.GCN_Q8_RELU, q, q.shape[1], s, prec, h, h.shape[1], ov)
    hb, wd, gd = h[:, :M].double(), w[:, :N].double(), g[:, :N].double()
    ht, wt = hb.t().contiguous(), wd.t().contiguous()
    want_w, want_z = ht @ gd, torch.where(hb > 0, gd @ wt / (1 - p), 0.0)
    # k products added one after another in fp32 err by k 2^-24 times the sum of their sizes, twice that where the
    # matrix instructions cut off instead of rounding; keep rounds twice more
    assert ((dW[:, :N].double() - want_w).abs() <= (n + 2) * 2.0 ** -23 * (ht @ gd.abs())).all()
    err = (N + 4) * 2.0 ** -23 * torch.where(hb > 0, gd.abs() @ wt.abs(), 0.0) / (1 - p)
    assert ((dZ[:, :M].double() - want_z).abs() <= err + HALF_STEP[prec] * (want_z.abs() + err) + LEAST[prec]).all()
    want_b = want_z.sum(0)
    assert ((db[:M].double() - want_b).abs() <= err.sum(0) + (n + 2) * 2.0 ** -24 * want_z.abs().sum(0)).all()
    # and as near as the framework's fp32 products are held to, however long the sums
    for got, ref in ((dW[:, :N], want_w), (db[:M], want_b)):
        assert (got.double() - ref).abs().max() <= 1e-5 * ref.abs().max()
    assert ov.item() == 0
