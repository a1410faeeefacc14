"""Rows in 8 bits past 2^31 elements, and many rows of few columns: the last rows
against calls on those rows alone, bit for bit."""
import pytest
import torch

from paper_2010_12635_amd import gcn as G

pytestmark = pytest.mark.gpu

N_ROWS, F_IN, F_OUT, LAST = (1 << 20) + 83, 2064, 24, 777


def flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def test_past_2_31_elements():
    n, f, N, prec = N_ROWS, F_IN, F_OUT, G.GCN_F16
    assert n * f > 1 << 31
    gen = torch.Generator(device="cuda").manual_seed(1)
    h = torch.empty((n, f), dtype=torch.float16, device="cuda")
    for a in range(0, n, 1 << 17):
        b = min(n, a + (1 << 17))
        h[a:b] = torch.randn((b - a, f), generator=gen, device="cuda").clamp(min=0)
    q = torch.zeros((n, f), dtype=torch.uint8, device="cuda")
    s = torch.zeros(n, device="cuda")
    ov = flag()
    G.gcn_quantize(n, f, prec, h, f, G.GCN_Q8_RELU, q, f, s, ov)
    at = n - LAST
    q1, s1 = torch.zeros((LAST, f), dtype=torch.uint8, device="cuda"), torch.zeros(LAST, device="cuda")
    G.gcn_quantize(LAST, f, prec, h[at:], f, G.GCN_Q8_RELU, q1, f, s1, ov)
    assert torch.equal(q[at:], q1) and torch.equal(s[at:], s1)
    back = torch.zeros_like(h)
    G.gcn_dequantize(n, f, G.GCN_Q8_RELU, q, f, s, prec, back, f, ov)
    one = torch.zeros((LAST, f), dtype=torch.float16, device="cuda")
    G.gcn_dequantize(LAST, f, G.GCN_Q8_RELU, q1, f, s1, prec, one, f, ov)
    assert torch.equal(back[at:], one)
    assert (back[at:].float() - h[at:].float()).abs().max() <= 1.01 * s1.max()
    del h

    # the product
    w = torch.randint(-127, 128, (N, f), generator=gen, device="cuda", dtype=torch.int8)
    ws, wsum = torch.full((N,), 2.0 ** -10, device="cuda"), w.sum(1, dtype=torch.int32)
    S = torch.zeros((n, N), dtype=torch.float16, device="cuda")
    G.gcn_transform_q8(n, f, N, G.GCN_Q8_RELU, q, f, s, w, f, ws, wsum, prec, S, N, ov)
    S1 = torch.zeros((LAST, N), dtype=torch.float16, device="cuda")
    G.gcn_transform_q8(LAST, f, N, G.GCN_Q8_RELU, q[at:], f, s1, w, f, ws, wsum, prec, S1, N, ov)
    assert torch.equal(S[at:], S1) and S1.abs().max() > 0

    # the backward pass, all of its gradient in the last rows and whole numbers: exact sums
    s.fill_(0.125)
    g = torch.zeros((n, N), dtype=torch.float16, device="cuda")
    g[at:] = torch.randint(-2, 3, (LAST, N), generator=gen, device="cuda").half()
    W = torch.randint(-1, 2, (f, N), generator=gen, device="cuda").half()
    out = []
    for rows, qq, ss, gg in ((n, q, s, g), (LAST, q[at:], s[at:].clone(), g[at:])):
        dW, db = torch.zeros((f, N), device="cuda"), torch.zeros(f, device="cuda")
        dZ = torch.zeros((rows, f), dtype=torch.float16, device="cuda")
        ws_ = torch.empty(G.gcn_transform_bwd_q8_workspace_size(rows, f, N, prec), dtype=torch.uint8, device="cuda")
        G.gcn_transform_bwd_q8(rows, f, N, prec, G.GCN_Q8_RELU, qq, f, ss, W, N, gg, N, G.GCN_ACT_RELU, 0.5, dW, dZ, f, db,
                               ov, ws_)
        out.append((dW, db, dZ[-LAST:].clone(), dZ[:at].any().item() if rows == n else False))
        del dZ
    assert torch.equal(out[0][0], out[1][0]) and torch.equal(out[0][1], out[1][1]) and torch.equal(out[0][2], out[1][2])
    assert not out[0][3] and out[0][0].abs().max() > 0 and ov.item() == 0


@pytest.mark.parametrize("prec", [G.GCN_F32, G.GCN_F16, G.GCN_BF16])
def test_rows_behind_the_last_stay(prec):
    """Outputs allocated for more rows than the call has."""
    n, f, N, more = 777, 130, 40, 64
    dt = G.torch_dtype(prec)
    gen = torch.Generator(device="cuda").manual_seed(2)
    h = torch.randn((n + more, 136), generator=gen, device="cuda").to(dt)
    q = torch.full((n + more, 144), 7, dtype=torch.uint8, device="cuda")
    s = torch.full((n + more,), 7.0, device="cuda")
    ov = flag()
    G.gcn_quantize(n, f, prec, h, 136, G.GCN_Q8_RELU, q, 144, s, ov)
    assert (q[n:] == 7).all() and (s[n:] == 7.0).all()
    back = torch.full((n + more, 136), 7.0, dtype=dt, device="cuda")
    G.gcn_dequantize(n, f, G.GCN_Q8_RELU, q, 144, s, prec, back, 136, ov)
    assert (back[n:] == 7.0).all()
    for rows in (1, 16, 50, n):
        w = torch.randint(-127, 128, (N, 144), generator=gen, device="cuda", dtype=torch.int8)
        S = torch.full((n + more, N), 7.0, dtype=dt, device="cuda")
        G.gcn_transform_q8(rows, f, N, G.GCN_Q8_RELU, q, 144, s, w, 144, torch.full((N,), 2.0 ** -12, device="cuda"),
                           w[:, :f].sum(1, dtype=torch.int32), prec, S, N, ov)
        assert (S[rows:] == 7.0).all() and not (S[:rows] == 7.0).all()
    for N in (40, 300):
        g, W = (torch.randn((k, round_up(N)), generator=gen, device="cuda").to(dt) for k in (n + more, f))
        dW, dZ = torch.zeros((f, round_up(N)), device="cuda"), torch.full((n + more, 136), 7.0, dtype=dt, device="cuda")
        ws = torch.empty(G.gcn_transform_bwd_q8_workspace_size(n, f, N, prec), dtype=torch.uint8, device="cuda")
        G.gcn_transform_bwd_q8(n, f, N, prec, G.GCN_Q8_RELU, q, 144, s, W, W.shape[1], g, g.shape[1], G.GCN_ACT_RELU, 0.0, dW,
                               dZ, 136, None, ov, ws)
        assert (dZ[n:] == 7.0).all()
    assert ov.item() == 0


def round_up(x):
    return (x + 7) // 8 * 8


@pytest.mark.parametrize("prec", [G.GCN_F32, G.GCN_F16])
def test_rows_far_apart(prec):
    """Codes whose rows lie 2^25 bytes apart (a tile of 64 rows spans 2^31): the same bits as with rows side by side
    where every sum is exact."""
    n, f, N = 70, 40, 24
    dt = G.torch_dtype(prec)
    gen = torch.Generator(device="cuda").manual_seed(3)
    q = torch.randint(0, 256, (n, 48), generator=gen, device="cuda", dtype=torch.uint8)
    q[torch.rand((n, 48), generator=gen, device="cuda") < 0.4] = 0
    far = torch.zeros((n, 1 << 25), dtype=torch.uint8, device="cuda")
    far[:, :48] = q
    s = torch.full((n,), 0.25, device="cuda")
    g = torch.randint(-2, 3, (n, N), generator=gen, device="cuda").to(dt)
    W = torch.randint(-1, 2, (f, N), generator=gen, device="cuda").to(dt)
    ws = torch.empty(G.gcn_transform_bwd_q8_workspace_size(n, f, N, prec), dtype=torch.uint8, device="cuda")
    ov, out = flag(), []
    for codes in (q, far):
        dW, db = torch.zeros((f, N), device="cuda"), torch.zeros(f, device="cuda")
        dZ = torch.zeros((n, f), dtype=dt, device="cuda")
        G.gcn_transform_bwd_q8(n, f, N, prec, G.GCN_Q8_RELU, codes, codes.shape[1], s, W, N, g, N, G.GCN_ACT_RELU, 0.5, dW,
                               dZ, f, db, ov, ws)
        out.append((dW, db, dZ))
    assert all(torch.equal(a, b) for a, b in zip(*out)) and ov.item() == 0 and out[0][0].any()
    w8 = torch.randint(-127, 128, (N, 48), generator=gen, device="cuda", dtype=torch.int8)
    S = [torch.zeros((n, N), dtype=dt, device="cuda") for _ in range(2)]
    for t, codes in zip(S, (q, far)):
        G.gcn_transform_q8(n, f, N, G.GCN_Q8_RELU, codes, codes.shape[1], s, w8, 48, torch.full((N,), 2.0 ** -12, device="cuda"),
                           w8[:, :f].sum(1, dtype=torch.int32), prec, t, N, ov)
    assert torch.equal(*S) and S[0].any()
