"""Refusals of the operators on class scores: every bad argument is named by a
status before anything is launched (no GPU is touched)."""
import os

import pytest
import torch  # noqa: F401  (loads the HIP runtime libgcn links against)

from paper_2010_12635_amd import gcn as G

pytestmark = pytest.mark.skipif(not os.path.exists(G.LIB_PATH), reason="libgcn.so not built")

INVALID, SHAPE, ALIGN, UNSUPPORTED, WORKSPACE = 1, 2, 3, 4, 6
NAN, INF = float("nan"), float("inf")


def top(n=10, C=7, ld=8, prec=1, z=0x1000, K=3, ld_top=8, v=0x2000, c=0x3000, ov=0x4000, ws=0x5000, wb=1 << 30):
    return G.lib().gcn_top_logits(n, C, ld, prec, z, K, ld_top, v, c, ov, ws, wb, None)


def distill(n=10, C=7, ld=8, prec=1, z=0x1000, K=3, ld_top=8, tp=1, v=0x2000, c=0x3000, mask=None, nm=10, T=1.0,
            w=1.0, s=None, base=None, loss=0x4000, d=0x6000, cs=None, ov=None, ws=0x5000, wb=1 << 30):
    return G.lib().gcn_distill(n, C, ld, prec, z, K, ld_top, tp, v, c, mask, nm, T, w, s, base, loss, d, cs, ov, ws,
                               wb, None)


def sample(n=10, C=7, ld=8, prec=1, z=0x1000, mask=None, u=0x2000, T=1.0, k=0, p=1.0, m=0.0, y=0x3000, pr=0x4000,
           ov=None, ws=0x5000, wb=1 << 30):
    return G.lib().gcn_sample_labels(n, C, ld, prec, z, mask, u, T, k, p, m, y, pr, ov, ws, wb, None)


@pytest.mark.parametrize("call", [top, distill, sample])
@pytest.mark.parametrize("args,status", [
    (dict(prec=3), INVALID), (dict(prec=-1), INVALID), (dict(n=0), SHAPE), (dict(n=-5), SHAPE), (dict(C=0), SHAPE),
    (dict(ld=6), SHAPE), (dict(ld=12), ALIGN), (dict(C=(1 << 30) + 1, ld=(1 << 30) + 8), UNSUPPORTED),
    (dict(n=1 << 31), UNSUPPORTED), (dict(z=None), INVALID), (dict(z=0x1008), ALIGN), (dict(ws=None), WORKSPACE),
    (dict(ws=0x5004), ALIGN), (dict(wb=0), WORKSPACE)])
def test_rows(call, args, status):
    if "n" in args:
        args = dict(args, **({"nm": 1} if call is distill else {}))
    assert call(**args) == status


@pytest.mark.parametrize("call", [top, distill])
@pytest.mark.parametrize("args,status", [
    (dict(K=0), SHAPE), (dict(K=9), SHAPE), (dict(ld_top=12), ALIGN), (dict(K=G.MAX_TOP + 1, ld_top=512), UNSUPPORTED),
    (dict(v=None), INVALID), (dict(c=None), INVALID), (dict(v=0x2002), ALIGN), (dict(c=0x3004), ALIGN)])
def test_entries(call, args, status):
    assert call(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(tp=3), INVALID), (dict(nm=0), SHAPE), (dict(nm=11), SHAPE), (dict(T=0.0), INVALID), (dict(T=-1.0), INVALID),
    (dict(T=2.0 ** -11), INVALID), (dict(T=1025.0), INVALID), (dict(T=NAN), INVALID), (dict(w=0.0), INVALID),
    (dict(w=INF), INVALID), (dict(w=NAN), INVALID), (dict(loss=None), INVALID), (dict(d=None, base=0x7000), INVALID),
    (dict(d=None, cs=0x7000), INVALID), (dict(base=0x7004), ALIGN), (dict(d=0x6004), ALIGN), (dict(cs=0x7004), ALIGN),
    (dict(C=513, ld=520, cs=0x7000), UNSUPPORTED), (dict(C=257, ld=264, prec=0, cs=0x7000), UNSUPPORTED)])
def test_distill(args, status):
    assert distill(**args) == status


@pytest.mark.parametrize("args,status", [
    (dict(T=-1.0), INVALID), (dict(T=2.0 ** -11), INVALID), (dict(T=2000.0), INVALID), (dict(T=NAN), INVALID),
    (dict(k=-1), INVALID), (dict(p=0.0), INVALID), (dict(p=1.5), INVALID), (dict(p=NAN), INVALID),
    (dict(m=-0.1), INVALID), (dict(m=1.1), INVALID), (dict(m=NAN), INVALID), (dict(u=None), INVALID),
    (dict(y=None), INVALID), (dict(u=0x2004), ALIGN), (dict(y=0x3004), ALIGN), (dict(pr=0x4004), ALIGN)])
def test_sample(args, status):
    assert sample(**args) == status


def test_workspace_sizes():
    for f, tail in ((G.gcn_top_logits_workspace_size, (5, 1)), (G.gcn_distill_workspace_size, (5, 1)),
                    (G.gcn_sample_labels_workspace_size, (1,))):
        assert f(1, 1, *tail) > 0 and f(1 << 21, 64, *tail) > 0 and f(3, 131072, *tail) > 0
        for bad in ((0, 7), (7, 0)):
            with pytest.raises(G.GcnError) as e:
                f(*bad, *tail)
            assert e.value.status == SHAPE
        with pytest.raises(G.GcnError) as e:
            f(7, 7, *tail[:-1], 3)
        assert e.value.status == INVALID
    with pytest.raises(G.GcnError) as e:
        G.gcn_top_logits_workspace_size(7, 7, 257, 1)
    assert e.value.status == UNSUPPORTED
