"""Pins of the distillation oracle, and the argument checks of the loss, without a device."""
import numpy as np
import pytest

from oracle import distill as O


def _row(seed=0, R=3, V=17, J=4):
    rng = np.random.default_rng(seed)
    z, t = rng.standard_normal((R, V)), rng.standard_normal((R, J))
    idx = np.stack([rng.choice(V, J, replace=False) for _ in range(R)])
    return z, idx, t


def test_gradient_against_differences():
    z, idx, t = _row()
    idx[1, 2] = idx[1, 0]      # an index twice
    idx[2, 1:3] = -1           # entries that do not count
    w = np.array([0.5, 2.0, 1.0])
    loss, dz, _, _ = O.distill(z, idx, t, 1.7, w)
    h = 1e-5
    for r in range(3):
        for v in range(17):
            up, down = z.copy(), z.copy()
            up[r, v] += h
            down[r, v] -= h
            diff = w[r] * (O.distill(up, idx, t, 1.7)[0][r] - O.distill(down, idx, t, 1.7)[0][r]) / (2 * h)
            assert abs(diff - dz[r, v]) < 1e-8
    assert np.allclose(dz.sum(1), 0, atol=1e-12)


def test_whole_vocabulary_is_the_divergence():
    z, _, _ = _row(1)
    t = np.random.default_rng(5).standard_normal(z.shape)
    idx = np.tile(np.arange(17), (3, 1))
    loss, _, p, lq = O.distill(z, idx, t, 2.0)
    assert np.allclose(loss, 4.0 * (p * (np.log(p) - lq)).sum(1)) and np.all(loss > 0)
    same, dz, _, _ = O.distill(z, idx, z, 2.0)
    assert np.allclose(same, 0, atol=1e-14) and np.allclose(dz, 0, atol=1e-14)


def test_odd_rows():
    z, idx, t = _row(2)
    idx[0] = -1
    t[1] = -np.inf
    z[2, idx[2, 0]] = -np.inf
    loss, dz, _, _ = O.distill(z, idx, t, 1.0)
    assert loss[0] == 0 and not dz[0].any() and loss[1] == 0 and not dz[1].any() and loss[2] == np.inf and np.isfinite(dz[2]).all()


def _call(B, name, z=1 << 20, zt=0, rows=2, vocab=10, ldz=10, idx=1 << 21, ib=8, t=1 << 22, tt=0, top=3, tau=1.0, loss=1 << 23, stats=1 << 24,
          weight=None, dz=1 << 25, lddz=10):
    a = (z, zt, rows, vocab, ldz, idx, ib, t, tt, top, tau)
    if name == "forward":
        return B.lib.idkm_distill_forward(*a, loss, stats, None)
    if name == "backward":
        return B.lib.idkm_distill_backward(*a, stats, weight, dz, lddz, None)
    return B.lib.idkm_distill_step(*a, weight, loss, dz, lddz, None)


@pytest.mark.parametrize("name", ["forward", "backward", "step"])
@pytest.mark.parametrize("change,status", [
    (dict(z=None), "NULL"), (dict(idx=None), "NULL"), (dict(t=None), "NULL"), (dict(zt=3), "UNSUPPORTED"), (dict(tt=7), "UNSUPPORTED"),
    (dict(ib=2), "UNSUPPORTED"), (dict(top=0), "UNSUPPORTED"), (dict(top=257), "UNSUPPORTED"), (dict(rows=0), "SHAPE"), (dict(vocab=0), "SHAPE"),
    (dict(ldz=9), "SHAPE"), (dict(rows=1 << 30, vocab=1 << 30, ldz=1 << 30, lddz=1 << 30), "SHAPE"), (dict(tau=0.0), "PARAM"),
    (dict(tau=float("nan")), "PARAM"), (dict(tau=float("inf")), "PARAM"), (dict(z=(1 << 20) + 2), "ALIGN"), (dict(idx=(1 << 21) + 4), "ALIGN"),
    (dict(stats=(1 << 24) + 2, loss=(1 << 23) + 2), "ALIGN")])
def test_refusals(name, change, status):
    from paper_2312_07759_b200 import binding as B
    assert _call(B, name, **change) == getattr(B, "ERR_" + status)


def test_refusals_of_outputs():
    from paper_2312_07759_b200 import binding as B
    assert _call(B, "forward", loss=None) == B.ERR_NULL and _call(B, "step", loss=None) == B.ERR_NULL
    assert _call(B, "backward", stats=None) == B.ERR_NULL and _call(B, "backward", dz=None) == B.ERR_NULL
    assert _call(B, "step", dz=None) == B.ERR_NULL and _call(B, "step", lddz=9) == B.ERR_SHAPE
    assert _call(B, "step", dz=1 << 20, lddz=12) == B.ERR_PARAM and _call(B, "backward", dz=(1 << 25) + 2) == B.ERR_ALIGN


def test_binding_refuses_what_does_not_fit_together():
    import torch
    from paper_2312_07759_b200 import binding as B
    z, idx, t = torch.zeros(2, 10), torch.zeros(2, 3, dtype=torch.int64), torch.zeros(2, 3)
    for bad in [(z, idx.float(), t), (z, idx[:1], t), (z, idx, t[:, :2]), (z.t(), idx, t), (z[0], idx, t)]:
        with pytest.raises((ValueError, IndexError)):
            B.distill_forward(*bad, 1.0)
    with pytest.raises(ValueError):
        B.distill_forward(z, idx, t, 1.0)      # not on a device
    with pytest.raises(ValueError):
        B.distill_step(z, idx, t, 1.0, torch.zeros(3))
    with pytest.raises(ValueError):
        B.distill_backward(z, idx, t, 1.0, torch.zeros(2))
    with pytest.raises(B.IdkmError):
        B.distill_forward(z.double(), idx, t, 1.0)
