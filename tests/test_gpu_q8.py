"""Rows in 8 bits on the GPU: codes and scales bit for bit against the oracle,
the 8-bit product and the backward pass exactly on whole numbers (every sum of
theirs is exact in 32 bits) and within bounds on others."""
import numpy as np
import pytest
import torch

from oracle import q8_oracle as Q
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import DeviceGraph, round8
from tests.parity import hub_graph

pytestmark = pytest.mark.gpu

KINDS = {"signed": G.GCN_Q8_SIGNED, "relu": G.GCN_Q8_RELU}
PRECS = [G.GCN_F32, G.GCN_F16, G.GCN_BF16]
HALF_STEP = {G.GCN_F32: 2.0 ** -24, G.GCN_F16: 2.0 ** -11, G.GCN_BF16: 2.0 ** -8}
LEAST = {G.GCN_F32: 2.0 ** -149, G.GCN_F16: 2.0 ** -24, G.GCN_BF16: 2.0 ** -133}
NAN, INF = float("nan"), float("inf")


def round16(x):
    return (x + 15) // 16 * 16


def padded(a, dtype, ld, fill=NAN):
    """a (numpy or tensor, rounded to dtype) in the first columns of a device
    matrix of ld columns; the others hold what must not matter."""
    a = torch.as_tensor(a)
    t = torch.full((a.shape[0], ld), fill, dtype=dtype, device="cuda")
    t[:, :a.shape[1]] = a.to("cuda").to(dtype)
    return t


def codes(q, kind, ld, fill=0x5a):
    t = torch.full((q.shape[0], ld), fill, dtype=torch.uint8, device="cuda")
    t[:, :q.shape[1]] = torch.as_tensor((q & 0xff).astype(np.uint8)).cuda()
    return t


def read_codes(t, f, kind):
    c = t[:, :f].cpu().numpy()
    return (c.view(np.int8) if kind == "signed" else c).astype(np.int64)


def flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def f64(t, f=None):
    return (t if f is None else t[:, :f]).double().cpu().numpy()


def quantize(h, f, prec, kind, ld_q, stream=None):
    n = h.shape[0]
    q = torch.full((n, ld_q), 0x33, dtype=torch.uint8, device="cuda")
    s = torch.full((n,), 7.0, device="cuda")
    ov = flag()
    G.gcn_quantize(n, f, prec, h, h.shape[1], KINDS[kind], q, ld_q, s, ov, stream)
    return q, s, ov


# ------------------------------------------------------------ codes, scales ----

SPECIAL = [
    [0.0] * 6, [1.0, 0.5, 0.25, -0.125, 0, 3], [-1.0, -2, -3, -4, -5, -6], [127.0, 0.5, 1.5, 2.5, -2.5, -0.5],
    [255.0, 0.5, 1.5, 2.5, -2.5, 126.5], [1e-7, -1e-7, 0, 0, 0, 0], [6e4, 1, 1e-3, -6e4, 1e-7, 0],
    [NAN, 1, 2, 3, 4, 5], [1, 2, INF, 3, 4, 5], [1, 2, 3, -INF, 4, 5], [-0.0, 0.0, -0.0, 0, 0, -0.0],
    [7.9375, 4.40625, 2.53125, -2.65625, 0.78125, 3.15625], [1, 2, 3, 4, 5, NAN]]
EXTREME = {  # the largest and smallest numbers of a type
    G.GCN_F16: [65504.0, 2.0 ** -24, -65504.0, 2.0 ** -14, 1.0, 0],
    G.GCN_BF16: [3.3895e38, 1e-38, -3.3895e38, 1.0, 1e-40, 0],
    G.GCN_F32: [3.4028235e38, 1e-45, -3.4028235e38, 1.0, 1.2e-38, 0]}
TINY = {G.GCN_F16: [2.0 ** -24, 0, 2.0 ** -24, 0, 0, -(2.0 ** -24)], G.GCN_BF16: [1e-40, -1e-40, 9.2e-41, 0, 1e-38, 0],
        G.GCN_F32: [1e-45, -1e-45, 1e-44, 2e-38, 1e-40, 0]}


@pytest.mark.parametrize("kind", list(KINDS))
@pytest.mark.parametrize("prec", PRECS)
def test_special_rows(prec, kind):
    rows = torch.tensor(SPECIAL + [EXTREME[prec], TINY[prec], TINY[prec][:5] + [0]], dtype=torch.float64)
    h = padded(rows, G.torch_dtype(prec), 8)
    q, s, ov = quantize(h, 6, prec, kind, 16)
    want_q, want_s = Q.quantize(f64(h, 6), kind)
    assert np.array_equal(f64(s), want_s, equal_nan=True)
    assert np.array_equal(read_codes(q, 6, kind), want_q)
    assert ov.item() == 1
    back = torch.full((len(rows), 8), 5.0, dtype=h.dtype, device="cuda")
    ov = flag()
    G.gcn_dequantize(len(rows), 6, KINDS[kind], q, 16, s, prec, back, 8, ov)
    want = torch.as_tensor(want_q * want_s[:, None]).to(h.dtype).double().numpy()   # exact in 32 bits, rounded once
    assert np.array_equal(f64(back, 6), want, equal_nan=True) and ov.item() == 1


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("n,f", [(1, 1), (3, 7), (70, 8), (33, 9), (1000, 16), (5, 31), (129, 40), (257, 64), (65, 100),
                                 (300, 128), (41, 255), (50, 256), (20, 500), (9, 512), (7, 513), (6, 1111), (5, 2047),
                                 (5, 2048), (3, 2049), (3, 4100), (2, 8200), (1, 65536)])
def test_codes_and_scales(prec, n, f):
    rng = np.random.default_rng(n * 131 + f)
    for kind in KINDS:
        h = rng.standard_normal((n, f)) * np.exp(rng.normal(0, 2, (n, 1)))
        h[rng.random((n, f)) < 0.2] = 0.0
        t = padded(h, G.torch_dtype(prec), round8(f) + 8)
        q, s, ov = quantize(t, f, prec, kind, round16(f) + 16)
        want_q, want_s = Q.quantize(f64(t, f), kind)
        assert np.array_equal(f64(s), want_s), kind
        assert np.array_equal(read_codes(q, f, kind), want_q), kind
        assert ov.item() == 0
        assert (q[:, round16(f):] == 0x33).all()               # what lies past the padding of 16 stays
        back = torch.full((n, round8(f) + 16), 5.0, dtype=t.dtype, device="cuda")
        G.gcn_dequantize(n, f, KINDS[kind], q, q.shape[1], s, prec, back, back.shape[1], ov)
        want = torch.as_tensor(want_q * want_s[:, None]).to(t.dtype).double().numpy()
        assert np.array_equal(f64(back, f), want), kind
        assert (back[:, round8(f):] == 5.0).all() and ov.item() == 0
        if kind == "relu":
            assert np.array_equal(want_q > 0, f64(t, f) > 0)


def test_many_rows():
    """More rows than one pass of the launch takes."""
    n, f = 8192 * 256 + 77, 3
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    h = torch.randint(-127, 128, (n, 8), generator=g, device="cuda").half()
    h[:, 0] = 127.0
    q, s, ov = quantize(h, f, G.GCN_F16, "signed", 16)
    assert (s == 1.0).all() and ov.item() == 0
    assert torch.equal(q.view(torch.int8)[:, :f].half(), h[:, :f])
    back = torch.zeros_like(h)
    G.gcn_dequantize(n, f, G.GCN_Q8_SIGNED, q, 16, s, G.GCN_F16, back, 8, ov)
    assert torch.equal(back[:, :f], h[:, :f])


@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("f_in,f_out", [(1, 1), (7, 3), (16, 7), (17, 16), (128, 40), (300, 33), (500, 64), (1000, 5),
                                        (2048, 130)])
def test_weights(prec, f_in, f_out):
    rng = np.random.default_rng(f_in + f_out)
    w = rng.standard_normal((f_in, f_out)) / np.sqrt(f_in)
    w[:, f_out // 2] = 0.0
    t = padded(w, G.torch_dtype(prec), round8(f_out) + 8)
    ld = round16(f_in) + 16
    wq = torch.full((f_out, ld), 0x33, dtype=torch.uint8, device="cuda")
    ws = torch.full((f_out,), 7.0, device="cuda")
    wsum = torch.full((f_out,), 7, dtype=torch.int32, device="cuda")
    ov = flag()
    G.gcn_quantize_weights(f_in, f_out, prec, t, t.shape[1], wq, ld, ws, wsum, ov)
    q, s = Q.quantize(f64(t, f_out).T, "signed")
    assert np.array_equal(read_codes(wq, f_in, "signed"), q) and np.array_equal(f64(ws), s)
    assert np.array_equal(wsum.cpu().numpy(), q.sum(1)) and ov.item() == 0
    assert (wq[:, round16(f_in):] == 0x33).all()
    t[f_in // 2, f_out - 1] = INF
    G.gcn_quantize_weights(f_in, f_out, prec, t, t.shape[1], wq, ld, ws, wsum, ov)
    assert ov.item() == 1 and np.isnan(ws[-1].item()) and wsum[-1].item() == 0
    assert np.array_equal(f64(ws[:-1]), s[:-1])


# ------------------------------------------------------------------ product ----

SIZES = [(1, 1, 1), (1, 16, 7), (1, 500, 64), (3, 2048, 130), (5, 33, 9), (16, 64, 16), (17, 65, 17), (31, 129, 8),
         (63, 100, 40), (64, 128, 64), (65, 300, 33), (130, 16, 128), (200, 500, 257), (256, 2000, 300), (300, 40, 1),
         (1000, 128, 128), (1025, 513, 65), (2049, 256, 256), (3000, 64, 7), (5000, 130, 40), (700, 2048, 520),
         (513, 1500, 513), (4100, 256, 300)]


def product(q, s, wq, ws, wsum, prec, kind, n, K, N, ld_s, stream=None):
    S = torch.full((n, ld_s), 5.0, dtype=G.torch_dtype(prec), device="cuda")
    ov = flag()
    G.gcn_transform_q8(n, K, N, KINDS[kind], q, q.shape[1], s, wq, wq.shape[1], ws, wsum, prec, S, ld_s, ov, stream)
    return S, ov


def check_product(S, want, prec, N, ov):
    # the sum to fp32, its product with the scales' mantissas and theirs, and the result: four
    # roundings to 24 bits, one to the type
    got = f64(S, N)
    tol = np.abs(want) * (HALF_STEP[prec] + 4.01 * 2.0 ** -24) + LEAST[prec]
    assert np.all(np.abs(got - want) <= tol), np.max(np.abs(got - want) / np.maximum(tol, 1e-300))
    assert ov.item() == 0


@pytest.mark.parametrize("n,K,N", SIZES)
@pytest.mark.parametrize("prec", PRECS)
def test_product(prec, n, K, N):
    rng = np.random.default_rng(n + 7 * K + 31 * N)
    for kind in KINDS:
        lo, hi = (-127, 128) if kind == "signed" else (0, 256)
        q = rng.integers(lo, hi, (n, K))
        w = rng.integers(-127, 128, (N, K))
        s = rng.uniform(0.5, 2.0, n).astype(np.float32) * np.float32(2.0 ** -9 / K)
        ws = rng.uniform(0.5, 2.0, N).astype(np.float32) * np.float32(2.0 ** -7)
        tq, tw = codes(q, kind, round16(K) + 16), codes(w, "signed", round16(K), fill=0x77)
        ts, tws = torch.as_tensor(s).cuda(), torch.as_tensor(ws).cuda()
        wsum = torch.as_tensor(w.sum(1).astype(np.int32)).cuda() if kind == "relu" else None
        S, ov = product(tq, ts, tw, tws, wsum, prec, kind, n, K, N, round8(N) + 8)
        check_product(S, Q.product(q, s.astype(np.float64), w, ws.astype(np.float64)), prec, N, ov)
        assert (S[:, round8(N):] == 5.0).all()


@pytest.mark.parametrize("n,K,N", [(20000, 100, 128), (20000, 500, 128), (20000, 512, 100), (33001, 577, 130),
                                   (50000, 530, 200), (65001, 600, 250), (16384, 4100, 300), (5000, 640, 40)])
@pytest.mark.parametrize("prec", PRECS)
def test_product_many_rows(prec, n, K, N):
    """As test_product, with the reference in float64 on the GPU (whole sums below 2^53: exact)."""
    gen = torch.Generator(device="cuda").manual_seed(n + K + N)
    for kind in KINDS:
        lo, hi = (-127, 128) if kind == "signed" else (0, 256)
        q = torch.randint(lo, hi, (n, K), generator=gen, device="cuda", dtype=torch.int32)
        w = torch.randint(-127, 128, (N, K), generator=gen, device="cuda", dtype=torch.int32)
        s = (0.5 + 1.5 * torch.rand(n, generator=gen, device="cuda")) * (2.0 ** -9 / K)
        ws = (0.5 + 1.5 * torch.rand(N, generator=gen, device="cuda")) * 2.0 ** -7
        tq = torch.full((n, round16(K) + 16), 0x5a, dtype=torch.uint8, device="cuda")
        tw = torch.full((N, round16(K)), 0x77, dtype=torch.uint8, device="cuda")
        tq[:, :K], tw[:, :K] = (q & 255).to(torch.uint8), (w & 255).to(torch.uint8)
        wsum = w.sum(1, dtype=torch.int32) if kind == "relu" else None
        S, ov = product(tq, s, tw, ws, wsum, prec, kind, n, K, N, round8(N) + 8)
        want = q.double() @ w.double().t().contiguous() * s.double()[:, None] * ws.double()
        tol = want.abs() * (HALF_STEP[prec] + 4.01 * 2.0 ** -24) + LEAST[prec]
        assert ((S[:, :N].double() - want).abs() <= tol).all(), kind
        assert (S[:, round8(N):] == 5.0).all() and ov.item() == 0


@pytest.mark.parametrize("n,K,N", [(1, 65536, 3), (40, 65536, 20), (300, 65536, 70)])
def test_product_largest_sums(n, K, N):
    """Sums next to the 32-bit border: every code at its largest."""
    q = np.full((n, K), 255)
    w = np.full((N, K), 127)
    w[1::2] = -127
    one = np.ones(max(n, N), np.float32)
    S, ov = product(codes(q, "relu", K), torch.as_tensor(one[:n]).cuda(), codes(w, "signed", K),
                    torch.as_tensor(one[:N]).cuda(), torch.as_tensor(w.sum(1).astype(np.int32)).cuda(), G.GCN_F32, "relu",
                    n, K, N, round8(N))
    check_product(S, Q.product(q, one[:n].astype(np.float64), w, one[:N].astype(np.float64)), G.GCN_F32, N, ov)


@pytest.mark.parametrize("n,N", [(1, 7), (20, 40), (300, 70)])
def test_product_scales_out_of_range(n, N):
    """A product of scales below or above the fp32 range whose results are in it; rows without a scale."""
    K = 64
    rng = np.random.default_rng(n)
    q, w = rng.integers(0, 256, (n, K)), rng.integers(-127, 128, (N, K))
    wsum = torch.as_tensor(w.sum(1).astype(np.int32)).cuda()
    for a, b in ((2.0 ** -126, 2.0 ** 110), (2.0 ** 120, 2.0 ** -110), (2.0 ** -100, 2.0 ** -40), (2.0 ** 64, 2.0 ** 40)):
        s, ws = np.full(n, a, np.float32), np.full(N, b, np.float32)
        S, ov = product(codes(q, "relu", K), torch.as_tensor(s).cuda(), codes(w, "signed", K), torch.as_tensor(ws).cuda(),
                        wsum, G.GCN_F32, "relu", n, K, N, round8(N))
        check_product(S, Q.product(q, s.astype(np.float64), w, ws.astype(np.float64)), G.GCN_F32, N, ov)
    s = np.ones(n, np.float32)
    s[n // 2] = NAN
    # in fp32: the sums, up to 64 * 255 * 127 = 2.1e6, lie beyond fp16
    S, ov = product(codes(q, "relu", K), torch.as_tensor(s).cuda(), codes(w, "signed", K), torch.ones(N, device="cuda"),
                    wsum, G.GCN_F32, "relu", n, K, N, round8(N))
    assert ov.item() == 1 and torch.isnan(S[n // 2, :N]).all()
    assert torch.isfinite(S[torch.arange(n, device="cuda") != n // 2][:, :N].float()).all()


# ----------------------------------------------------------------- backward ----

BWD_SIZES = [(1, 1, 1), (1, 40, 7), (2, 16, 16), (3, 128, 64), (15, 9, 3), (16, 64, 32), (17, 65, 33), (63, 100, 7),
             (64, 128, 64), (65, 130, 40), (129, 17, 130), (200, 512, 16), (255, 33, 256), (500, 500, 64), (1000, 16, 7),
             (1025, 256, 64), (3001, 128, 40), (4096, 64, 128), (777, 300, 257), (900, 2048, 16), (300, 70, 600),
             (20000, 128, 64), (6000, 200, 200), (1030, 33, 300), (2100, 250, 520), (1100, 40, 2600),
             (20000, 20, 66), (26000, 40, 70), (18000, 500, 66), (81000, 128, 100)]


def backward(q, s, w, g, prec, kind, n, M, N, act, p, below=True, colsum=True, ld_dz=None, stream=None, ws=None):
    ld_dz = ld_dz or round8(M)
    dW = torch.full((M, w.shape[1]), 7.0, device="cuda")
    dZ = torch.full((n, ld_dz), 5.0, dtype=G.torch_dtype(prec), device="cuda") if below else None
    db = torch.full((round8(M) + 8,), 7.0, device="cuda") if below and colsum else None
    ov = flag()
    if ws is None:
        ws = torch.full((G.gcn_transform_bwd_q8_workspace_size(n, M, N, prec) // 4,), NAN, device="cuda")
    G.gcn_transform_bwd_q8(n, M, N, prec, KINDS[kind], q, q.shape[1], s, w, w.shape[1], g, g.shape[1], act, p, dW, dZ,
                           ld_dz, db, ov, ws, stream)
    return dW, dZ, db, ov


def whole_case(rng, n, M, N, prec, kind):
    """Whole numbers whose every sum of products has fewer than 24 bits."""
    lo, hi = (-127, 128) if kind == "signed" else (0, 256)
    q = rng.integers(lo, hi, (n, M))
    q[rng.random((n, M)) < 0.4] = 0
    s = 2.0 ** rng.integers(-3, 1, n)
    g = rng.integers(-2, 3, (n, N)) * 0.25
    w = rng.integers(-1, 2, (M, N)) * 1.0
    dt = G.torch_dtype(prec)
    return (q, s, w, g, codes(q, kind, round16(M) + 16), torch.as_tensor(s.astype(np.float32)).cuda(),
            padded(w, dt, round8(N) + 8), padded(g, dt, round8(N) + 16))


@pytest.mark.parametrize("n,M,N", BWD_SIZES)
@pytest.mark.parametrize("prec", PRECS)
def test_backward_whole_numbers(prec, n, M, N):
    """127 * 2 * n / 4 * 8 and the like stay below 2^24: all sums are exact, and the results are those of the
    definition, rounded once."""
    rng = np.random.default_rng(n + 3 * M + 7 * N)
    for kind, act in (("relu", G.GCN_ACT_RELU), ("signed", G.GCN_ACT_NONE), ("relu", G.GCN_ACT_NONE)):
        q, s, w, g, tq, ts, tw, tg = whole_case(rng, n, M, N, prec, kind)
        p = 0.5 if act == G.GCN_ACT_RELU else 0.0
        dW, dZ, db, ov = backward(tq, ts, tw, tg, prec, kind, n, M, N, act, p, ld_dz=round8(M) + 8)
        want = Q.transform_bwd(q * s[:, None], w, g, q > 0 if act else None, p)
        assert np.array_equal(f64(dW, N), want[0]), (kind, act)
        assert not dW[:, N:].any()
        assert torch.equal(dZ[:, :M].cpu(), torch.as_tensor(want[1]).to(dZ.dtype)), (kind, act)
        assert (dZ[:, round8(M):] == 5.0).all()
        assert np.array_equal(f64(db)[:M], want[2]) and not db[M:round8(M)].any() and (db[round8(M):] == 7.0).all()
        assert ov.item() == 0
    # the weight gradient alone, and without column sums: the same bits
    dW1, _, _, ov = backward(tq, ts, tw, tg, prec, kind, n, M, N, act, p, below=False)
    dW2, dZ2, _, ov2 = backward(tq, ts, tw, tg, prec, kind, n, M, N, act, p, colsum=False)
    assert torch.equal(dW1, dW) and torch.equal(dW2, dW) and torch.equal(dZ2[:, :M], dZ[:, :M])
    assert ov.item() == 0 and ov2.item() == 0


@pytest.mark.parametrize("n,M,N", [(60000, 256, 250), (60001, 128, 100), (100000, 16, 16), (30000, 2048, 13),
                                   (90000, 100, 30), (70000, 60, 200), (50000, 256, 64), (200000, 30, 130),
                                   (60000, 130, 300)])
@pytest.mark.parametrize("prec", PRECS)
def test_backward_many_rows(prec, n, M, N):
    """Several tiles a workgroup, with the reference in float64 on the GPU: whole numbers whose sums stay below
    2^24 (|dW| <= 15 n, |dZ| <= 2 N, |db| as asserted), so all are exact."""
    gen = torch.Generator(device="cuda").manual_seed(n + M + N)
    dt = G.torch_dtype(prec)
    for kind, act, p in (("relu", G.GCN_ACT_RELU, 0.5), ("signed", G.GCN_ACT_NONE, 0.0)):
        q = torch.randint(-15 if kind == "signed" else 0, 16, (n, M), generator=gen, device="cuda", dtype=torch.int32)
        q *= torch.randint(0, 2, (n, M), generator=gen, device="cuda", dtype=torch.int32)
        g = torch.randint(-1, 2, (n, N), generator=gen, device="cuda").double()
        w = torch.randint(-1, 2, (M, N), generator=gen, device="cuda").double()
        tq = torch.full((n, round16(M)), 0x5a, dtype=torch.uint8, device="cuda")
        tq[:, :M] = (q & 255).to(torch.uint8)
        dW, dZ, db, ov = backward(tq, torch.ones(n, device="cuda"), padded(w, dt, round8(N)), padded(g, dt, round8(N)),
                                  prec, kind, n, M, N, act, p)
        z = g @ w.t().contiguous()
        if act:
            z = z * (q > 0) * 2
        assert z.abs().sum(0).max() < 2 ** 24
        assert torch.equal(dW[:, :N].double(), q.t().contiguous().double() @ g), kind
        assert torch.equal(dZ[:, :M], z.to(dt)), kind
        assert torch.equal(db[:M].double(), z.sum(0)) and ov.item() == 0, kind


@pytest.mark.parametrize("n,M,N", [(3000, 128, 64), (700, 500, 64), (1500, 40, 300), (5000, 24, 7)])
@pytest.mark.parametrize("prec", PRECS)
def test_backward_numbers(prec, n, M, N):
    rng = np.random.default_rng(n + M + N)
    dt = G.torch_dtype(prec)
    h = padded(np.maximum(rng.standard_normal((n, M)), 0) * 2, dt, round8(M))
    q, s, _ = quantize(h, M, prec, "relu", round16(M))
    w = padded(rng.standard_normal((M, N)) / np.sqrt(M), dt, round8(N))
    g = padded(rng.standard_normal((n, N)) * 0.05, dt, round8(N))
    p = float(np.float32(0.3))
    dW, dZ, db, ov = backward(q, s, w, g, prec, "relu", n, M, N, G.GCN_ACT_RELU, p)
    back = torch.zeros_like(h)
    G.gcn_dequantize(n, M, G.GCN_Q8_RELU, q, q.shape[1], s, prec, back, back.shape[1], ov)
    hb, wd, gd = f64(back, M), f64(w, N), f64(g, N)
    want = Q.transform_bwd(hb, wd, gd, hb > 0, p)
    # k products added one after another in fp32 err by k 2^-24 times the sum of their sizes, twice that where
    # the matrix instructions cut off instead of rounding; keep rounds twice more
    size = np.abs(hb).T @ np.abs(gd)
    assert np.all(np.abs(f64(dW, N) - want[0]) <= (n + 2) * 2.0 ** -23 * size)
    dz_err = (N + 4) * 2.0 ** -23 * np.where(hb > 0, np.abs(gd) @ np.abs(wd).T, 0) / (1 - p)
    assert np.all(np.abs(f64(dZ, M) - want[1]) <= dz_err + HALF_STEP[prec] * (np.abs(want[1]) + dz_err) + LEAST[prec])
    assert np.all(np.abs(f64(db)[:M] - want[2]) <= dz_err.sum(0) + (n + 2) * 2.0 ** -24 * np.abs(want[1]).sum(0))
    # and as near as the framework's fp32 products are held to
    for got, ref in ((f64(dW, N), want[0]), (f64(db)[:M], want[2])):
        assert np.max(np.abs(got - ref)) <= 1e-5 * np.max(np.abs(ref))
    assert ov.item() == 0


@pytest.mark.parametrize("n,M,N", [(500, 40, 24), (300, 30, 300)])
def test_backward_overflow(n, M, N):
    rng = np.random.default_rng(5)
    for prec in (G.GCN_F16, G.GCN_F32):
        for what in ("gradient", "scale", "large"):
            _, _, _, _, tq, ts, tw, tg = whole_case(rng, n, M, N, prec, "relu")
            if what == "gradient":
                tg[n - 1, N - 1] = INF
            elif what == "scale":
                ts[n // 2] = NAN
            else:
                tg[0, 0] = 6e4 if prec == G.GCN_F16 else 3e38
                tw[:, 0] = 2.0
                tq[0, :M] = 1
            *_, ov = backward(tq, ts, tw, tg, prec, "relu", n, M, N, G.GCN_ACT_RELU, 0.5)
            assert ov.item() == 1, what


@pytest.mark.parametrize("n,M,N", [(1, 40, 7), (1, 130, 64), (1, 33, 300)])
@pytest.mark.parametrize("prec", [G.GCN_F32, G.GCN_BF16])
def test_backward_largest_numbers(prec, n, M, N):
    """A row up to the type's largest number and weights near it, where the results are far inside the range: one
    product each by a power of two, so they are exact."""
    dt = G.torch_dtype(prec)
    rng = np.random.default_rng(M)
    h = padded(rng.choice([-1.0, 1.0, 0.5], (n, M)) * torch.finfo(dt).max, dt, round8(M))
    q, s, ov = quantize(h, M, prec, "signed", round16(M))
    back = torch.zeros_like(h)
    G.gcn_dequantize(n, M, G.GCN_Q8_SIGNED, q, q.shape[1], s, prec, back, back.shape[1], ov)
    g = np.zeros((n, N))
    g[:, N - 1] = 2.0 ** -40
    w = rng.integers(-3, 4, (M, N)) * 2.0 ** 126
    dW, dZ, db, ov2 = backward(q, s, padded(w, dt, round8(N)), padded(g, dt, round8(N)), prec, "signed", n, M, N,
                               G.GCN_ACT_NONE, 0.0)
    assert np.array_equal(f64(dW, N), f64(back, M).T @ g)
    assert np.array_equal(f64(dZ, M), g @ w.T)
    ones = torch.ones_like(q)
    dW, dZ, db, ov3 = backward(ones, torch.ones(n, device="cuda"), padded(w, dt, round8(N)), padded(g, dt, round8(N)), prec,
                               "relu", n, M, N, G.GCN_ACT_RELU, 0.75)
    assert np.array_equal(f64(dZ, M), g @ w.T * 4)
    assert ov.item() == 0 and ov2.item() == 0 and ov3.item() == 0


# ------------------------------------------------------------- the layer's ----

@pytest.mark.parametrize("prec", PRECS)
@pytest.mark.parametrize("storage", ["csr", "tiled", "dense"])
def test_layer(prec, storage):
    """gcn_layer_bwd_q8 against gcn_layer_bwd on the rows taken back: the same aggregation, the same mask."""
    n, M, N = 1500, 100, 37
    rng = np.random.default_rng(11)
    src, dst = hub_graph(n, 4 * n, [(3, 600), (17, 200)], 4)
    dg = DeviceGraph(n, src, dst, prec=prec, dense=storage != "csr", tiled=storage == "tiled", heavy_threshold=48,
                     chunk_nnz=96)
    dt = G.torch_dtype(prec)
    h = padded(np.maximum(rng.standard_normal((n, M)), 0), dt, round8(M), 0.0)
    q, s, ov = quantize(h, M, prec, "relu", round16(M))
    G.gcn_dequantize(n, M, G.GCN_Q8_RELU, q, q.shape[1], s, prec, h, h.shape[1], ov)
    w = padded(rng.standard_normal((M, N)) / 10, dt, round8(N), 0.0)
    dz = padded(rng.standard_normal((n, N)), dt, round8(N), 0.0)
    L = G.GcnLayer(M, N, round8(M), round8(N), G.GCN_ACT_NONE, 0.0, 1, 0)
    out = []
    for q8 in (False, True):
        o = dict(dW=torch.full((M, round8(N)), 7.0, device="cuda"), db=torch.full((round8(N),), 7.0, device="cuda"),
                 dZ=torch.zeros((n, round8(M)), dtype=dt, device="cuda"),
                 dbb=torch.full((round8(M),), 7.0, device="cuda"), GS=torch.zeros((n, round8(N)), dtype=dt, device="cuda"))
        if q8:
            ws = torch.empty(G.gcn_layer_bwd_q8_workspace_size(dg.adj, L, prec), dtype=torch.uint8, device="cuda")
            G.gcn_layer_bwd_q8(dg.adj, L, prec, G.GCN_Q8_RELU, q, q.shape[1], s, w, dz, G.GCN_ACT_RELU, 0.5, o["dW"],
                               o["db"], o["dZ"], o["GS"], ov, ws, dbias_below=o["dbb"])
        else:
            ws = torch.empty(G.gcn_layer_workspace_size(dg.adj, L, prec), dtype=torch.uint8, device="cuda")
            G.gcn_layer_bwd(dg.adj, L, prec, h, w, dz, G.GCN_ACT_RELU, 0.5, o["dW"], o["db"], o["dZ"], o["GS"], ov, ws,
                            dbias_below=o["dbb"])
        out.append(o)
    a, b = out
    assert ov.item() == 0 and torch.equal(a["db"], b["db"])
    for k in ("GS", "dW", "dZ", "dbb"):
        x, y = f64(a[k].reshape(-1, 1)), f64(b[k].reshape(-1, 1))
        tol = {"GS": HALF_STEP[prec], "dZ": HALF_STEP[prec]}.get(k, 0.0) * 2 + 2e-5
        if k == "dbb":      # there summed as stored
            tol += HALF_STEP[prec] * 4
        assert np.max(np.abs(x - y)) <= tol * np.max(np.abs(x)), k


# ----------------------------------------------- streams, graphs, two at once ----

@pytest.mark.parametrize("prec", [G.GCN_F32, G.GCN_F16])
def test_captured_and_replayed(prec):
    """Quantize, product and backward in one graph, replayed over new inputs with eager work between."""
    n, M, N = 1200, 72, 24
    dt = G.torch_dtype(prec)
    rng = np.random.default_rng(2)
    h = padded(np.zeros((n, M)), dt, round8(M), 0.0)
    w = padded(rng.standard_normal((M, N)), dt, round8(N), 0.0)
    g = padded(np.zeros((n, N)), dt, round8(N), 0.0)
    q = torch.zeros((n, round16(M)), dtype=torch.uint8, device="cuda")
    s = torch.zeros(n, device="cuda")
    wq = torch.zeros((N, round16(M)), dtype=torch.uint8, device="cuda")
    wsc, wsum = torch.zeros(N, device="cuda"), torch.zeros(N, dtype=torch.int32, device="cuda")
    S = torch.zeros((n, round8(N)), dtype=dt, device="cuda")
    dW, db = torch.zeros((M, round8(N)), device="cuda"), torch.zeros(round8(M), device="cuda")
    dZ = torch.zeros((n, round8(M)), dtype=dt, device="cuda")
    ov = flag()
    ws = torch.empty(G.gcn_transform_bwd_q8_workspace_size(n, M, N, prec), dtype=torch.uint8, device="cuda")

    def program():
        G.gcn_quantize(n, M, prec, h, round8(M), G.GCN_Q8_RELU, q, q.shape[1], s, ov)
        G.gcn_quantize_weights(M, N, prec, w, round8(N), wq, wq.shape[1], wsc, wsum, ov)
        G.gcn_transform_q8(n, M, N, G.GCN_Q8_RELU, q, q.shape[1], s, wq, wq.shape[1], wsc, wsum, prec, S, round8(N), ov)
        G.gcn_transform_bwd_q8(n, M, N, prec, G.GCN_Q8_RELU, q, q.shape[1], s, w, round8(N), g, round8(N),
                               G.GCN_ACT_RELU, 0.5, dW, dZ, round8(M), db, ov, ws)

    outs = (q[:, :M], s, S[:, :N], dW, dZ[:, :M], db)         # padding past the widths may keep what it holds
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        program()
    for k in range(4):
        h[:, :M] = torch.as_tensor(rng.standard_normal((n, M))).cuda().to(dt)
        g[:, :N] = torch.as_tensor(rng.standard_normal((n, N))).cuda().to(dt)
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in outs]
        for t in outs:
            t.fill_(3)
        program()
        torch.cuda.synchronize()
        for a, b in zip(got, outs):
            assert torch.equal(a, b), k
    assert ov.item() == 0


def test_other_streams():
    """The same calls on two streams at once, each with its own workspace."""
    rng = np.random.default_rng(9)
    n, M, N, prec = 3000, 128, 64, G.GCN_F16
    q, s, w, g, tq, ts, tw, tg = whole_case(rng, n, M, N, prec, "relu")
    want = Q.transform_bwd(q * s[:, None], w, g, q > 0, 0.5)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream(), torch.cuda.Stream()]
    size = G.gcn_transform_bwd_q8_workspace_size(n, M, N, prec) // 4
    spaces = [torch.full((size,), NAN, device="cuda") for _ in streams]
    torch.cuda.synchronize()
    outs = []
    for _ in range(3):
        for st, ws in zip(streams, spaces):
            with torch.cuda.stream(st):
                outs.append(backward(tq, ts, tw, tg, prec, "relu", n, M, N, G.GCN_ACT_RELU, 0.5, stream=st, ws=ws))
    torch.cuda.synchronize()
    for dW, dZ, db, ov in outs:
        assert np.array_equal(f64(dW, N), want[0]) and np.array_equal(f64(db)[:M], want[2])
        assert torch.equal(dZ[:, :M].cpu(), torch.as_tensor(want[1]).half()) and ov.item() == 0
