"""The oracle's cross-entropy on rows without a label: against the sum over the
others, by hand and by differences."""
import numpy as np

from oracle import gcn_oracle as O


def test_negative_labels_are_left_out():
    rng = np.random.default_rng(0)
    z = rng.standard_normal((6, 4))
    y = np.array([0, -1, 3, 2, -1, 1])
    mask = np.array([1, 1, 1, 0, 0, 1])
    loss, d, good = O.softmax_ce(z, y, mask, 2.0)
    p = np.exp(z) / np.exp(z).sum(1, keepdims=True)
    rows = [0, 2, 5]
    assert np.isclose(loss, -np.log(p[rows, y[rows]]).sum() / 4, rtol=1e-14)
    want = np.zeros_like(z)
    for i in rows:
        want[i] = p[i]
        want[i, y[i]] -= 1
    assert np.allclose(d, want * 2 / 4, rtol=0, atol=1e-15)
    assert good == sum(int(np.argmax(z[i]) == y[i]) for i in rows)
    for i in range(6):
        e = np.zeros_like(z)
        e[i, 1] = 1e-6
        num = (O.softmax_ce(z + e, y, mask, 2.0)[0] - O.softmax_ce(z - e, y, mask, 2.0)[0]) / 2e-6
        assert abs(2 * num - d[i, 1]) < 1e-8     # the loss does not carry the scale
