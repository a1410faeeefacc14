"""gcn_distill on scores that are large against the temperature, up to the
type's lowest number, in lane groups and in longer rows alike.

Bounds, with e = 2^-24: a power's exponent (t - max) / T carries the roundings
of the difference, of log2(e) / T (the constant, 1 / T, their product) and of
the product, 5 e |t - max| / T, however large t itself is; the base-2
exponential 4 e, sums of D adds D e.  So a teacher's weight is within
(5 |y| + 5 ln K + K + 16) e of itself and a student's probability within
(5 |x| + 5 ln C + D + 16) e, as for scores of ordinary size
(test_gpu_scores.py); a loss's term q (y - x) adds 8 e (|y| + |x|) q.  What a
bound on p leaves beyond that is a whole step at most: p is at most 1.
"""
import numpy as np
import pytest
import torch

from oracle import scores_oracle as S
from paper_2010_12635_amd import gcn as G
from paper_2010_12635_amd.model import round8
from tests.test_gpu_scores import E, HALF, NAMES, TINY, distill, host, put

pytestmark = pytest.mark.gpu
LOWEST = {p: float(torch.finfo(G.torch_dtype(p)).min) for p in (0, 1, 2)}
# lane groups, a workgroup a row (two widths), segments
SIZES = [(5, 64), (5, 256), (6, 700), (5, 4001), (3, 70001)]


def softmax(t):
    w = np.exp(t - t.max())
    return w / w.sum()


def check(z, v, c, prec, top_prec, T, finite=True):
    """z n x C, v and c n x K (no class twice, none absent)."""
    n, C = z.shape
    K = v.shape[1]
    zt, vt = put(z, prec, round8(C)), put(v, top_prec, round8(K))
    ct = torch.full((n, round8(K)), -1, dtype=torch.int32, device="cuda")
    ct[:, :K] = torch.as_tensor(c.astype(np.int32)).cuda()
    z, v = host(zt, C), host(vt, K)
    loss, d, _, ov = distill(zt, vt, ct, n, C, K, prec, top_prec, T)
    want_loss, want, _ = S.distill(z, v, c, T)
    chain = C / 256 + 24
    bound, loss_bound = np.zeros((n, C)), 0.0
    for i in range(n):
        x = (z[i] - z[i].max()) / T
        y = (v[i] - v[i].max()) / T
        p, q = softmax(x), softmax(y)
        rel_q = (5 * np.abs(y) + 5 * np.log(K) + K + 16) * E
        bound[i] = np.minimum(p * (5 * np.abs(x) + 5 * np.log(C) + chain + 16) * E, 1.0)
        bound[i, c[i]] += np.minimum(q * rel_q, 1.0)
        xc = np.abs(x[c[i]])
        terms = np.where(q > 0, q * (np.abs(y) + xc), 0.0)
        loss_bound += (terms * (rel_q + (8 + K) * E)).sum() + 2 * (5 * np.log(C) + chain + 16 + K) * E \
            + 4 * E * (np.log(C) + np.log(K))
    bound *= T / n
    bound += 8 * E * np.abs(want)
    got = host(d, C)
    assert np.isfinite(got).all()
    err = np.abs(got - want)
    lim = bound + HALF[prec] * (np.abs(want) + bound) + TINY[prec]
    assert (err <= lim).all(), (np.unravel_index(np.argmax(err - lim), err.shape), err.max(), (err / lim).max())
    loss_bound = loss_bound * T * T / n + 80 * E * abs(want_loss)
    assert abs(loss.item() - want_loss) <= loss_bound, (loss.item(), want_loss, loss_bound)
    assert ov.item() == 0


def classes(rng, n, C, K):
    return np.stack([rng.permutation(C)[:K] for _ in range(n)])


@pytest.mark.parametrize("prec,top_prec", [(0, 0), (1, 1), (2, 2), (0, 1), (1, 0)])
@pytest.mark.parametrize("n,C", SIZES)
def test_large_teacher(n, C, prec, top_prec):
    """The teacher's scores far from 0: its weights still sum to 1."""
    rng = np.random.default_rng(C + prec)
    for level, spread, T, K in ((20.0, 0.3, 0.05, 8), (20.0, 0.01, G.MIN_TEMPERATURE, 8), (3000.0, 4.0, 1.0, 30),
                                (-60000.0, 0.0, G.MIN_TEMPERATURE, 1), (60000.0, 200.0, 3.3, 5)):
        print(f"[range] teacher {level} T={T} n={n} C={C} {NAMES[prec]} {NAMES[top_prec]}", flush=True)
        v = level + spread * rng.standard_normal((n, K))
        check(rng.standard_normal((n, C)) * T, v, classes(rng, n, C, K), prec, top_prec, T)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("n,C", SIZES)
def test_teacher_of_lowest_scores(n, C, prec):
    """Entries of the lowest finite number are entries like any other: alone in
    a row they share its weight."""
    rng = np.random.default_rng(C)
    for T in (1.0, G.MIN_TEMPERATURE, 2.0):
        print(f"[range] lowest teacher T={T} n={n} C={C} {NAMES[prec]}", flush=True)
        v = np.full((n, 4), LOWEST[prec])
        v[1, 2] = 1.0                             # one entry far above the others
        check(rng.standard_normal((n, C)) * min(T, 1.0), v, classes(rng, n, C, 4), prec, prec, T)


@pytest.mark.parametrize("prec", [0, 1, 2], ids=NAMES.get)
@pytest.mark.parametrize("n,C", SIZES)
def test_student_of_lowest_scores(n, C, prec):
    """Rows masked with the type's lowest number: nothing weighs there unless
    nothing else is left, and then all weigh the same."""
    rng = np.random.default_rng(C)
    for T in (1.0, G.MIN_TEMPERATURE, 1.3, 3.0):
        print(f"[range] lowest student T={T} n={n} C={C} {NAMES[prec]}", flush=True)
        z = rng.standard_normal((n, C)) * min(T, 1.0)
        c = classes(rng, n, C, 4)
        v = rng.standard_normal((n, 4)) * T
        away = rng.random((n, C)) < 0.6
        np.put_along_axis(away, c, False, 1)
        z[away] = LOWEST[prec]
        z[1] = LOWEST[prec]
        check(z, v, c, prec, prec, T)
        check(np.full((n, C), LOWEST[prec]), v, c, prec, prec, T)


@pytest.mark.parametrize("n,C", SIZES)
def test_named_lowest_score(n, C):
    """A teacher that names a class of the lowest score: a loss near the end of
    the range, but a finite one, and a gradient of ordinary size."""
    rng = np.random.default_rng(C)
    for T in (1.0, 4.0):
        print(f"[range] named T={T} n={n} C={C}", flush=True)
        z = rng.standard_normal((n, C))
        c = classes(rng, n, C, 3)
        z[0, c[0, 1]] = LOWEST[0] if T == 1.0 else LOWEST[0] / 8
        check(z, rng.standard_normal((n, 3)), c, 0, 0, T)


@pytest.mark.parametrize("prec", [0, 2], ids=NAMES.get)
@pytest.mark.parametrize("n,C", SIZES)
def test_large_student(n, C, prec):
    """Scores far from 0 whose differences are of ordinary size against the
    temperature, and the largest numbers of both signs together."""
    rng = np.random.default_rng(C)
    for level, step, T in ((1.0e7, 1.0, 0.5), (-1.0e7, 1.0, 0.25), (1.0e7, 2.0 ** -9, G.MIN_TEMPERATURE),
                           (1.0e30, 0.0, 1.0), (-3.0e38, 0.0, 0.3)):
        print(f"[range] student {level} T={T} n={n} C={C} {NAMES[prec]}", flush=True)
        z = level + step * rng.integers(-3, 4, (n, C))
        c = classes(rng, n, C, 5)
        z = np.asarray(torch.as_tensor(z.astype(np.float32)).to(G.torch_dtype(prec)).double())
        top = z.max(1)
        for i in range(n):                        # bf16 keeps 8 bits: the differences may be large
            z[i, c[i]] = top[i]
        check(z, rng.standard_normal((n, 5)) * T, c, prec, prec, T)
    z = rng.standard_normal((n, C))
    c = classes(rng, n, C, 2)
    z[:, :] = -LOWEST[prec] * np.where(rng.random((n, C)) < 0.5, 1.0, -1.0)
    z[np.arange(n)[:, None], c] = -LOWEST[prec]
    check(z, rng.standard_normal((n, 2)), c, prec, prec, 1.0)


@pytest.mark.parametrize("prec", [0, 1], ids=NAMES.get)
@pytest.mark.parametrize("C", [32768, 32769, 65535, 65536, 65537])
def test_either_side_of_segments(C, prec):
    """The widths and row counts at which rows are cut into segments."""
    rng = np.random.default_rng(C)
    for n in (2, 191, 192):
        print(f"[range] segments n={n} C={C} {NAMES[prec]}", flush=True)
        z = rng.standard_normal((n, C)) * 3
        check(z, rng.standard_normal((n, 6)) * 2, rng.integers(0, C - 6, (n, 1)) + np.arange(6), prec, prec, 1.5)
