"""Teacher's mass below what fp32 holds, on classes that the student masks (B200 only): it counts as none.  Tolerances: those of
test_gpu_distill.py; what is left out is below 2^-126 of the largest probability, in the loss and in the gradient."""
import pytest

from test_gpu_distill import TYPES, _all_ways, _inputs, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("R,V,J", [(9, 1003, 5), (9, 1003, 40), (9, 60001, 100), (9, 151937, 256), (9, 300007, 64)])
@pytest.mark.parametrize("tau", [1.0, 3.0])
def test_teacher_mass_that_underflows_counts_as_none(t, R, V, J, tau):
    import torch
    z, idx, tl, w = _inputs(torch, R, V, J, t)
    tl.clamp_(-4, 4)
    tl[:, 0] = 2.0                              # of the row's largest entries
    last = J - 1

    def mask(r, j, logit):
        tl[r, j] = logit
        z[r, idx[r, j]] = -float("inf")

    mask(0, last, -1e4)
    mask(1, last, torch.finfo(torch.float32).min)
    mask(2, last, 2.0 - 100 * tau)              # e^-100: below 2^-126
    mask(3, last, 2.0 - 70 * tau)               # e^-70: counts, the loss is infinite
    for j in range(J // 2, J):                  # (whole warps of entries, each one's largest among them)
        mask(4, j, -1e4 - j)
    for j in range(J // 2, J):                  # ... among them one that counts
        mask(5, j, -1e4 if j < last else 2.0 - 60 * tau)
    for j in range(1, J):                       # a second entry that its warp has a larger one beside, but underflows itself
        if j != last:
            tl[6, j] = 2.0 - 60 * tau
    mask(6, last, 2.0 - 120 * tau)
    tl[7, 0] = -1e4                             # the largest entry of all, whatever its size
    for j in range(J):
        mask(7, j, -1e4 - 200 * tau * j)
    for j in range(J // 2, J):                  # (the student masks with its type's lowest value)
        tl[8, j] = -1e4 - j
        z[8, idx[8, j]] = torch.finfo(z.dtype).min
    ref = _reference(z, idx, tl, tau, w)
    loss, dz = _all_ways(torch, z, idx, tl, tau, w, ref)
    assert torch.isfinite(loss[[0, 1, 2, 4, 6, 8]]).all() and torch.isinf(loss[[3, 5, 7]]).all() and torch.isfinite(dz.float()).all()
