"""Masked classes in the distillation loss and its gradient (B200 only): at temperatures whose log2(e) / tau is rounded up as well as
down, and where the teacher has next to nothing on them.  Tolerances: those of test_gpu_distill.py."""
import pytest

from test_gpu_distill import TYPES, _all_ways, _inputs, _reference

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tau", [0.3, 0.7, 1.0, 1.5, 2.0, 2.5, 3.0, 5.0, 6.0, 10.0, 20.0])
def test_masked_classes_have_no_gradient_at_any_temperature(t, tau):
    import torch
    from paper_2312_07759_b200 import binding as B
    z, idx, tl, w = _inputs(torch, 9, 1003, 24, t)
    z[:, ::3] = -float("inf")
    z[4, 1::3] = torch.finfo(z.dtype).min
    idx[0] = idx[0] // 3 * 3 + 1                # no entry on a masked class: a finite loss
    idx[1] = idx[1] // 3 * 3                    # every entry on one
    idx[2, 5:] = -1
    idx[4] = idx[4] // 3 * 3 + 2                # (none on the classes of the lowest value)
    ref = _reference(z, idx, tl, tau, w)
    loss, dz = _all_ways(torch, z, idx, tl, tau, w, ref)
    assert torch.isfinite(loss[0]) and loss[1] == float("inf")
    _, stats = B.distill_forward(z, idx, tl, tau)
    back = B.distill_backward(z, idx, tl, tau, stats, w)
    masked = torch.isneginf(z.float())
    at = torch.where((idx >= 0) & (idx < z.shape[1]), idx, torch.zeros_like(idx))
    entry = torch.zeros_like(masked).scatter_(1, at, True)
    assert not back[masked & ~entry].any() and not dz[masked & ~entry].any() and torch.isfinite(back.float()).all()
    assert torch.all(back[masked & entry] <= 0)
