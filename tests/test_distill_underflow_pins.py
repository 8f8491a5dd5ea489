"""Pins of the distillation oracle where the teacher's mass is too small for fp32, without a device."""
import numpy as np

from oracle import distill as O


def test_mass_below_the_normal_range_counts_as_none_in_the_loss():
    z = np.array([[0.5, -np.inf, 1.0]])
    idx = np.array([[0, 1, 2]])
    for t, infinite in ((-1e4, False), (-100.0, False), (-88.0, False), (-87.0, True), (-30.0, True)):
        loss, dz, p, _ = O.distill(z, idx, np.array([[0.0, t, -1.0]]), 1.0)
        assert np.isinf(loss[0]) == infinite and np.isfinite(dz).all() and not dz[0, 1] > 0
    # relative to the largest entry, and in units of the temperature
    assert np.isinf(O.distill(z, idx, np.array([[-1e4, -1e4 - 150.0, -1e4]]), 2.0)[0][0])
    loss = O.distill(z, idx, np.array([[-1e4, -1e4 - 200.0, -1e4]]), 2.0)[0][0]
    # two entries of one half each are left
    lq = z[0] / 2 - np.log(np.exp(z[0] / 2).sum())
    assert np.isclose(loss, 4 * (np.log(0.5) - 0.5 * (lq[0] + lq[2])))


def test_what_is_left_out_is_nothing_beside_the_rest():
    rng = np.random.default_rng(3)
    z, t = rng.standard_normal((1, 50)) * 3, rng.standard_normal((1, 20))
    idx = rng.choice(50, 20, replace=False)[None]
    want = O.distill(z, idx[:, :12], t[:, :12], 1.5)
    t[:, 12:] = -200.0
    got = O.distill(z, idx, t, 1.5)
    assert np.isclose(got[0][0], want[0][0], rtol=1e-14) and np.allclose(got[1], want[1], rtol=0, atol=1e-16)
