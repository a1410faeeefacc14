"""gcn_top_logits, gcn_distill and gcn_sample_labels against the float64 oracle.

Top scores and labels are whole numbers and have to be equal.  Bounds of the
floating outputs, with e = 2^-24 (half a step of fp32, relative):

* A probability p_c = exp(x_c) / s, x_c = (z_c - max) / T.  x_c carries the
  roundings of the difference, of log2(e) / T (3: the constant, 1 / T, their
  product) and of the product: 5 e |x_c| absolute, so a factor exp(5 e |x|);
  the base-2 exponential 4 e (2 units in the last place).  s adds C terms in
  chains of at most D adds: D e.  Quotient (as reciprocal times), scale and
  the constants of the scale: 8 e.  With |x_c| p_c <= X p_c this is
  p_c (5 X + 5 Xmean + D + 16) e, and Xmean (the x averaged with weights p)
  is at most ln C.  q_j likewise over its K entries.
* A gradient is scale (p_c - q_c) (+ base) and is rounded once to its type:
  half a step of the type, plus half the smallest subnormal step.
* A row's loss sum q (y - x) - ln r + ln s: each term's error is bounded by
  (|y| + |x_c|) e times 8, and the logarithms by 4 e |ln| plus their
  arguments' relative error; the mean over rows of chains of D2 adds is
  within (D2 + 4) e of the sum of the rows' losses.
"""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8

pytestmark = pytest.mark.gpu
E = 2.0 ** -24
NAMES = {0: "f32", 1: "f16", 2: "bf16"}


def put(a, prec, ld, fill=float("nan")):
    """a (n x f) on the GPU with leading dimension ld; padding columns hold
    NaN, which no call may use."""
    t = torch.full((a.shape[0], ld), fill, dtype=G.torch_dtype(prec), device="cuda")
    t[:, :a.shape[1]] = torch.as_tensor(np.asarray(a, np.float32)).cuda().to(t.dtype)
    return t


def host(t, f=None):
    t = t if f is None else t[:, :f]
    return t.double().cpu().numpy()


def flag():
    return torch.zeros(1, dtype=torch.int32, device="cuda")


def scratch(nbytes):
    """Filled with NaN bits: stale contents must not matter."""
    return torch.full((nbytes,), 0xFF, dtype=torch.uint8, device="cuda")


def scores(rng, n, C, kind):
    if kind == "normal":
        return rng.standard_normal((n, C)) * 2.5
    if kind == "ties":                       # few different values
        return rng.integers(-2, 3, (n, C)).astype(np.float64)
    if kind == "equal":
        return np.full((n, C), -1.25)
    if kind == "absent":                     # most classes out of the row, some rows empty
        z = rng.standard_normal((n, C)) * 3
        z[rng.random((n, C)) < 0.7] = -np.inf
        z[rng.integers(0, n, max(1, n // 5))] = -np.inf
        return z
    if kind == "lowest":                     # the type's lowest number is a score like any other
        z = rng.standard_normal((n, C)) * 3
        z[rng.random((n, C)) < 0.6] = -65504.0
        z[0] = -65504.0
        return z
    if kind == "peaked":                     # one class far ahead
        z = rng.standard_normal((n, C))
        z[np.arange(n), rng.integers(0, C, n)] += 60
        return z
    if kind == "signs":                      # zeros of both signs
        return np.where(rng.random((n, C)) < 0.5, 0.0, -0.0)
    raise ValueError(kind)


SHAPES = [(1, 1), (3, 2), (33, 7), (70, 8), (19, 9), (300, 16), (65, 33), (1000, 40), (130, 64), (37, 65), (9, 129),
          (17, 255), (12, 256), (11, 257), (6, 511), (6, 512), (7, 513), (5, 1500), (3, 4097), (2, 20011), (2, 66001)]


# ------------------------------------------------------------- top scores ----

def run_top(zt, n, C, ld, prec, K, ld_top=None, stream=None):
    ld_top = ld_top or round8(K)
    v = torch.full((n, ld_top), 77.0, dtype=G.torch_dtype(prec), device="cuda")
    c = torch.full((n, ld_top), 77, dtype=torch.int32, device="cuda")
    ov = flag()
    ws = scratch(G.gcn_top_logits_workspace_size(n, C, K, prec))
    G.gcn_top_logits(n, C, ld, prec, zt, K, ld_top, v, c, ov, ws, stream)
    return v, c, ov


def check_top(zt, n, C, ld, prec, K, want_flag=0, ld_top=None):
    v, c, ov = run_top(zt, n, C, ld, prec, K, ld_top)
    z = host(zt, C)
    wv, wc = S.top_logits(z, K)
    assert np.array_equal(c[:, :K].cpu().numpy(), wc)
    assert np.array_equal(host(v, K), wv)
    assert (c[:, K:] == 77).all() and (v[:, K:] == 77).all()
    assert ov.item() == want_flag


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("n,C", SHAPES)
def test_top_sizes(n, C, prec):
    rng = np.random.default_rng(n * 1000 + C)
    for K in sorted({1, 2, min(C, 5), min(C, 8), min(C, 9), min(C, 64), min(C, 256)}):
        print(f"[top] n={n} C={C} K={K} {NAMES[prec]}", flush=True)
        check_top(put(scores(rng, n, C, "normal"), prec, round8(C)), n, C, round8(C), prec, K)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("kind", ["ties", "equal", "absent", "lowest", "peaked", "signs"])
@pytest.mark.parametrize("n,C,K", [(50, 7, 3), (50, 7, 20), (40, 64, 8), (40, 64, 64), (9, 300, 70), (5, 2500, 200),
                                   (3, 40000, 256)])
def test_top_kinds(n, C, K, kind, prec):
    print(f"[top] {kind} n={n} C={C} K={K} {NAMES[prec]}", flush=True)
    rng = np.random.default_rng(C + K)
    check_top(put(scores(rng, n, C, kind), prec, round8(C) + 16), n, C, round8(C) + 16, prec, K, ld_top=round8(K) + 8)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("C", [6, 90, 700, 30000])
def test_top_nan_and_infinity(C, prec):
    print(f"[top] nan C={C} {NAMES[prec]}", flush=True)
    rng = np.random.default_rng(C)
    z = scores(rng, 5, C, "normal")
    z[1, C // 2] = np.nan
    check_top(put(z, prec, round8(C)), 5, C, round8(C), prec, 4, want_flag=1)
    z[1, C // 2] = np.inf
    check_top(put(z, prec, round8(C)), 5, C, round8(C), prec, 4, want_flag=1)
    z[:] = np.nan
    check_top(put(z, prec, round8(C)), 5, C, round8(C), prec, 4, want_flag=1)


# ------------------------------------------------------------ distillation ----

def teacher(rng, n, C, K, top_prec, ld_top):
    """Entries in any order, some absent, some rows empty, classes that occur
    twice."""
    v = rng.standard_normal((n, K)) * 3
    c = rng.integers(0, C, (n, K)).astype(np.int32)       # with replacement
    c[rng.random((n, K)) < 0.2] = -1
    v[rng.random((n, K)) < 0.1] = -np.inf
    if n > 2:
        c[n // 2] = -1
    vt = put(v, top_prec, ld_top)
    ct = torch.full((n, ld_top), 2 ** 30, dtype=torch.int32, device="cuda")
    ct[:, :K] = torch.as_tensor(c).cuda()
    return vt, ct, host(vt, K), c


def distill(zt, vt, ct, n, C, K, prec, top_prec, T, w=1.0, mask=None, n_mask=None, scale=None, base=None,
            in_place=False, colsum=False, forward_only=False):
    ld = zt.shape[1]
    loss = torch.full((1,), 77.0, device="cuda")
    d = None if forward_only else base if in_place else torch.full_like(zt, 77.0)
    cs = torch.full((ld,), 77.0, device="cuda") if colsum else None
    ov = flag()
    ws = scratch(G.gcn_distill_workspace_size(n, C, K, prec))
    sc = None if scale is None else torch.full((1,), scale, device="cuda")
    G.gcn_distill(n, C, ld, prec, zt, K, vt.shape[1], top_prec, vt, ct, mask, n if n_mask is None else n_mask, T, w,
                  sc, base, loss, d, ov, ws, dlogits_colsum=cs)
    return loss, d, cs, ov


def distill_bounds(z, v, c, T, w, n_mask, scale, prec, counted):
    """Bounds of the gradient (n x C), of the loss and of the column sums
    without the base (see the head of the file)."""
    n, C = z.shape
    chain = C / 256 + 24
    with np.errstate(invalid="ignore", over="ignore"):
        x = np.maximum((z - z.max(1, keepdims=True)) / T, -1e3)
        p = np.exp(x)
        p /= p.sum(1, keepdims=True)
    rel_p = (5 * np.abs(x) + 5 * np.log(C) + chain + 16) * E
    gb = p * rel_p
    lb = np.zeros(n)
    for i in np.flatnonzero(counted):
        here = (c[i] >= 0) & (c[i] < C) & (v[i] > -np.inf)
        t = v[i][here] / T
        t = t - t.max()
        q = np.exp(t)
        q /= q.sum()
        rel_q = (5 * np.abs(t) + 5 * np.log(len(t)) + len(t) + 16) * E
        np.add.at(gb[i], c[i][here], q * (rel_q + len(t) * E))
        xi = np.abs(x[i, c[i][here]])
        lb[i] = (q * ((np.abs(t) + xi) * (8 * E + rel_q))).sum() + (len(t) + 4) * E * (q * (np.abs(t) + xi)).sum() \
            + 2 * (5 * np.log(C) + chain + 16 + len(t)) * E + 4 * E * (np.log(C) + np.log(len(t)))
    gb[~counted] = 0
    f = scale * w * T / n_mask
    return gb * f, lb[counted].sum() * w * T * T / n_mask


HALF = {0: 2.0 ** -24, 1: 2.0 ** -11, 2: 2.0 ** -8}
TINY = {0: 2.0 ** -149, 1: 2.0 ** -25, 2: 2.0 ** -134}


def check_distill(rng, n, C, K, prec, top_prec=None, T=1.0, w=1.0, masked=False, scale=None, base=False, colsum=False,
                  kind="normal", extra_ld=0, in_place=False):
    top_prec = prec if top_prec is None else top_prec
    ld = round8(C) + extra_ld
    zt = put(scores(rng, n, C, kind), prec, ld)
    z = host(zt, C)
    vt, ct, v, c = teacher(rng, n, C, K, top_prec, round8(K) + extra_ld)
    m = mt = None
    if masked:
        m = (rng.random(n) < 0.6).astype(np.uint8) * 255
        m[0] = 1
        mt = torch.as_tensor(m).cuda()
    n_mask = n if m is None else int(np.count_nonzero(m))
    b = bt = None
    if base:
        bt = put(rng.standard_normal((n, C)) * 0.1, prec, ld)
        b = host(bt, C)
    T, w = float(np.float32(T)), float(np.float32(w))
    loss, d, cs, ov = distill(zt, vt, ct, n, C, K, prec, top_prec, T, w, mt, n_mask, scale, bt, in_place, colsum)
    s = 1.0 if scale is None else scale
    wl, wg, wcs = S.distill(z, v, c, T, w, s, m, n_mask, b)
    counted = ((c >= 0) & (v > -np.inf)).any(1) & (np.ones(n, bool) if m is None else m != 0)
    gb, lb = distill_bounds(z, v, c, T, w, n_mask, s, prec, counted)
    gb = gb + (4 * E * np.abs(wg) + 2 * E * np.abs(b) if base else 4 * E * np.abs(wg))
    got = host(d, C)
    err = np.abs(got - wg)
    bound = gb + HALF[prec] * (np.abs(wg) + gb) + TINY[prec]
    assert np.isfinite(got).all()
    assert (err <= bound).all(), (np.unravel_index(np.argmax(err - bound), err.shape), err.max(), (err / bound).max())
    chain = n / 64 + 64
    assert abs(loss.item() - wl) <= lb + (chain + 8) * E * abs(wl) + (chain + 8) * E * lb, (loss.item(), wl, lb)
    if colsum:
        size = np.abs(wg).sum(0)
        assert (np.abs(cs[:C].double().cpu().numpy() - wcs) <= gb.sum(0) + (chain + 8) * E * (size + gb.sum(0))
                + 1e-40).all()
        assert (cs[C:] == 0).all()
    assert ov.item() == 0
    # the loss alone, the same bits
    l2, _, _, ov = distill(zt, vt, ct, n, C, K, prec, top_prec, T, w, mt, n_mask, scale, forward_only=True)
    assert torch.equal(loss, l2) and ov.item() == 0


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("n,C", SHAPES)
def test_distill_sizes(n, C, prec):
    rng = np.random.default_rng(n * 1000 + C + prec)
    for i, K in enumerate(sorted({1, 3, 8, 17, 100})):
        print(f"[distill] n={n} C={C} K={K} {NAMES[prec]}", flush=True)
        narrow = C <= (256 if prec == 0 else 512)
        check_distill(rng, n, C, K, prec, top_prec=(prec + i) % 3, T=[1.0, 2.0, 0.5, 4.0, 1.3][i],
                      w=[1.0, 0.25][i % 2], masked=i in (1, 4), scale=[None, 128.0][i % 2], base=i in (2, 4),
                      colsum=narrow, extra_ld=8 * (i == 3), in_place=i == 4)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("kind", ["ties", "equal", "lowest", "peaked"])
@pytest.mark.parametrize("n,C,K", [(60, 7, 3), (50, 64, 8), (9, 400, 40), (4, 9000, 64)])
def test_distill_kinds(n, C, K, kind, prec):
    print(f"[distill] {kind} n={n} C={C} K={K} {NAMES[prec]}", flush=True)
    check_distill(np.random.default_rng(C), n, C, K, prec, T=2.0, kind=kind, base=True)


@pytest.mark.parametrize("C", [7, 64, 500, 3000])
def test_distill_absent_student_classes(C):
    """A class that is out of the student's row has probability 0; a teacher
    that does not name it has a finite loss, one that does an infinite one."""
    n, K = 6, 3
    rng = np.random.default_rng(C)
    z = rng.standard_normal((n, C))
    z[:, 1] = -np.inf
    zt = put(z, 0, round8(C))
    c = np.tile(np.array([0, 2, 3], np.int32), (n, 1))
    ct = torch.as_tensor(np.pad(c, ((0, 0), (0, 5)), constant_values=-1)).cuda()
    vt = put(rng.standard_normal((n, K)), 0, 8)
    loss, d, _, ov = distill(zt, vt, ct, n, C, K, 0, 0, 1.0)
    wl, wg, _ = S.distill(host(zt, C), host(vt, K), c, 1.0)
    assert ov.item() == 0 and (d[:, 1] == 0).all()
    assert np.abs(host(d, C) - wg).max() < 2e-6 and abs(loss.item() - wl) < 1e-5 * wl
    ct[2, 1] = 1
    loss, d, _, ov = distill(zt, vt, ct, n, C, K, 0, 0, 1.0)
    assert loss.item() == float("inf") and ov.item() == 1
    assert torch.isfinite(d[:, :C]).all()


@pytest.mark.parametrize("prec", [0, 1], ids=NAMES.get)
@pytest.mark.parametrize("C", [7, 64, 3000])
def test_distill_flags(C, prec):
    n, K = 8, 4
    rng = np.random.default_rng(C)
    z = rng.standard_normal((n, C))
    ld = round8(C)
    vt, ct, v, c = teacher(rng, n, C, K, prec, 8)
    ct[0, :K] = torch.arange(K, device="cuda")
    ct[:, K:] = -1
    # a class past the end is left out and reported
    ct[0, 1] = C
    loss, d, _, ov = distill(put(z, prec, ld), vt, ct, n, C, K, prec, prec, 1.0)
    c = ct[:, :K].cpu().numpy()
    wl, wg, _ = S.distill(host(put(z, prec, ld), C), v, c, 1.0)
    assert ov.item() == 1 and np.isfinite(host(d, C)).all()
    assert np.abs(host(d, C) - wg).max() <= (4 * HALF[prec] + 1e-6) / n
    ct[0, 1] = 0
    # NaN and infinity in a row that counts; a row outside the mask may hold anything
    for bad in (float("nan"), float("inf")):
        zb = z.copy()
        zb[0, C // 2] = bad
        loss, d, _, ov = distill(put(zb, prec, ld), vt, ct, n, C, K, prec, prec, 1.0)
        assert ov.item() == 1 and not np.isfinite(loss.item())
        mask = torch.ones(n, dtype=torch.uint8, device="cuda")
        mask[0] = 0
        loss, d, _, ov = distill(put(zb, prec, ld), vt, ct, n, C, K, prec, prec, 1.0, mask=mask, n_mask=n - 1)
        assert ov.item() == 0 and np.isfinite(loss.item()) and (d[0, :C] == 0).all()
    # a gradient past the type's range
    if prec == 1:
        _, _, _, ov = distill(put(z, prec, ld), vt, ct, n, C, K, prec, prec, 1.0, scale=1e9)
        assert ov.item() == 1


# ------------------------------------------------------------ drawn labels ----

def run_sample(zt, n, C, prec, u, T, k=0, p=1.0, m=0.0, mask=None, labels=None, prob=True):
    y = torch.full((n,), -7, dtype=torch.int32, device="cuda") if labels is None else labels.clone()
    pr = torch.full((n,), -7.0, device="cuda") if prob else None
    ov = flag()
    ws = scratch(G.gcn_sample_labels_workspace_size(n, C, prec))
    G.gcn_sample_labels(n, C, zt.shape[1], prec, zt, mask, u, T, k, p, m, y, pr, ov, ws)
    return y, pr, ov


def check_sample(rng, n, C, prec, T, k=0, p=1.0, m=0.0, kind="normal", masked=False, u=None):
    ld = round8(C)
    zt = put(scores(rng, n, C, kind), prec, ld)
    z = host(zt, C)
    u = rng.random(n).astype(np.float32) if u is None else np.full(n, u, np.float32)
    T, p, m = (float(np.float32(x)) for x in (T, p, m))
    mask = mt = None
    if masked:
        mask = (rng.random(n) < 0.5).astype(np.uint8) * 7
        mt = torch.as_tensor(mask).cuda()
    y, pr, ov = run_sample(zt, n, C, prec, torch.as_tensor(u).cuda(), T, k, p, m, mt)
    wy, wp = S.sample_labels(z, u.astype(np.float64), T, k, p, m, mask)
    got = y.cpu().numpy()
    assert np.array_equal(got, wy), (np.flatnonzero(got != wy)[:5], got[got != wy][:5], wy[got != wy][:5])
    # a weight exp(x) carries 3 E |x| log2(e) + 4 E, the kept weights' sum 2^-18
    # at most (the bound that a draw in 32 bits is certified with), the
    # quotient 4 E; what 32 bits hold only as a subnormal number may come out
    # as 0.  |x| is at most ln C - ln prob above the sum's own ln C.
    x = np.where(wp > 0, -np.log(np.maximum(wp, 1e-300)), 0) + np.log(C)
    assert (np.abs(pr.double().cpu().numpy() - wp) <= (2.0 ** -18 + (5 * x + 8) * E) * np.abs(wp) + 2.0 ** -126).all()
    assert ov.item() == 0
    y2, _, _ = run_sample(zt, n, C, prec, torch.as_tensor(u).cuda(), T, k, p, m, mt, prob=False)
    assert torch.equal(y, y2)


FILTERS = [(0, 1.0, 0.0), (1, 1.0, 0.0), (3, 1.0, 0.0), (0, 0.9, 0.0), (0, 1.0, 0.05), (20, 0.8, 0.02), (0, 0.05, 0.0),
           (0, 0.995, 0.0), (300, 0.99, 0.0), (0, 1.0, 1.0)]


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("n,C", SHAPES)
def test_sample_sizes(n, C, prec):
    rng = np.random.default_rng(n * 1000 + C + prec)
    for i, (k, p, m) in enumerate(FILTERS):
        T = [1.0, 0.7, 1.5, 0.05, 10.0][i % 5]
        print(f"[sample] n={n} C={C} T={T} k={k} p={p} m={m} {NAMES[prec]}", flush=True)
        check_sample(rng, n, C, prec, T, k, p, m, masked=i % 3 == 2)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("kind", ["ties", "equal", "absent", "lowest", "peaked", "signs"])
@pytest.mark.parametrize("n,C", [(40, 7), (50, 64), (9, 300), (9, 512), (5, 2500), (3, 40000)])
def test_sample_kinds(n, C, kind, prec):
    rng = np.random.default_rng(C)
    for k, p, m in FILTERS:
        print(f"[sample] {kind} n={n} C={C} k={k} p={p} m={m} {NAMES[prec]}", flush=True)
        check_sample(rng, n, C, prec, 0.8, k, p, m, kind=kind)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("C", [1, 5, 64, 200, 1000, 33000])
def test_sample_ends(C, prec):
    """The smallest and the largest u, T at both ends and T = 0."""
    rng = np.random.default_rng(C)
    for u in (0.0, 2.0 ** -149, 1 - 2.0 ** -24):
        for T in (0.0, G.MIN_TEMPERATURE, 1.0, G.MAX_TEMPERATURE):
            for k, p in ((0, 1.0), (4, 1.0), (0, 0.7)):
                print(f"[sample] ends C={C} u={u} T={T} k={k} p={p} {NAMES[prec]}", flush=True)
                check_sample(rng, 6, C, prec, T, k, p, u=u, kind="ties" if k else "normal")


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("C", [4, 16, 64, 512, 1024, 16384])
def test_sample_on_the_border(C, prec):
    """Equal scores: u C and top_p C are whole numbers, so every running sum
    meets its border exactly."""
    n = 64
    rng = np.random.default_rng(C)
    zt = put(np.full((n, C), 0.5), prec, round8(C))
    u = (rng.integers(0, C, n) / C).astype(np.float32)
    for p, k in ((1.0, 0), (0.5, 0), (0.25, 0), (0.75, C // 2)):
        print(f"[sample] border C={C} p={p} k={k} {NAMES[prec]}", flush=True)
        y, _, ov = run_sample(zt, n, C, prec, torch.as_tensor(u).cuda(), 1.0, k, p)
        kept = int(np.ceil(p * (k or C)))
        want = np.floor(u.astype(np.float64) * kept).astype(np.int32)
        assert np.array_equal(y.cpu().numpy(), want) and ov.item() == 0


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("C", [7, 64, 700, 30000])
def test_sample_flags(C, prec):
    n = 6
    rng = np.random.default_rng(C)
    z = scores(rng, n, C, "normal")
    z[1, C // 2] = np.nan
    z[3, C - 1] = np.inf
    u = torch.full((n,), 0.5, device="cuda")
    u[4] = 1.0
    u[5] = float("nan")
    for T in (1.0, 0.0):
        y, pr, ov = run_sample(put(z, prec, round8(C)), n, C, prec, u, T, 0, 0.9)
        bad = [1, 3, 4, 5] if T else [1, 3]
        assert ov.item() == 1
        for i in range(n):
            assert (y[i].item() == -1 and pr[i].item() == 0) == (i in bad), (i, T)
    # a bad row that the mask leaves out is not looked at
    mask = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mask[[0, 2]] = 1
    y, pr, ov = run_sample(put(z, prec, round8(C)), n, C, prec, u, 1.0, 0, 0.9, mask=mask)
    assert ov.item() == 0 and (y[[1, 3, 4, 5]] == -7).all() and (pr[[1, 3, 4, 5]] == -7).all()
    assert (y[[0, 2]] >= 0).all()
