"""The distillation loss and its gradient on the GPU against the float64 oracle (B200 only).

Tolerances.  Exponents x = z / tau are off by one rounding, 2^-24 |x|, and ln q by that, the normaliser's and the largest x's; with
X the largest |x| of a row (finite ones), an exponential or a normaliser is off by at most e = (4 X + 32) 2^-24 of its value
(the 32: the functions' own 2 ulp and the joins of sums).  The loss is a sum of p (ln p - ln q) with p off by e and either
logarithm off by e: tau^2 ((sum p |ln p - ln q|) e + 2 e), rounded once.  The gradient is w tau (q - p): w tau (q + p) e, then
the rounding to its type, eps / 2 of its value (and half the least fp16 step).  Exponentials below the normal range are 0: an
exponential is taken relative to a largest one, whose share of the row is at most 1, in up to two factors, either of which is
0 only where it is below 2^-126 and the other at most 1; so q is off by at most 2^-126 more, and the gradient by w tau 2^-126."""
import numpy as np
import pytest

from oracle import distill as O

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


def _inputs(torch, R, V, J, t="float32", tt="float32", idx_type="int64", seed=0, spread=2.0):
    g = torch.Generator(device="cuda").manual_seed(seed + R + V + J)
    z = (torch.randn(R, V, device="cuda", generator=g) * spread).to(getattr(torch, t))
    idx = torch.stack([torch.randperm(V, device="cuda", generator=g)[:J] if V >= J else torch.randint(0, V, (J,), device="cuda", generator=g)
                       for _ in range(R)]).to(getattr(torch, idx_type))
    tl = (torch.randn(R, J, device="cuda", generator=g) * spread).to(getattr(torch, tt))
    w = torch.rand(R, device="cuda", generator=g) + 0.5
    return z, idx, tl, w


def _reference(z, idx, t, tau, w):
    z64, t64 = z.double().cpu().numpy(), t.double().cpu().numpy()
    w64 = np.ones(z.shape[0]) if w is None else w.double().cpu().numpy()
    loss, dz, p, lq = O.distill(z64, idx.cpu().numpy(), t64, tau, w64)
    # (masked and padded places apart)
    fin = np.where(np.isfinite(z64), np.abs(z64), 0).max(1) / tau
    fint = np.where(np.isfinite(t64), np.abs(t64), 0).max(1) / tau
    e = (4 * np.maximum(fin, fint) + 32) * 2.0 ** -24
    I = np.clip(idx.cpu().numpy(), 0, z.shape[1] - 1)
    with np.errstate(all="ignore"):
        term = np.where(p > 0, p * np.abs(np.log(np.where(p > 0, p, 1)) - np.take_along_axis(lq, I, 1)), 0).sum(1)
    ltol = tau * tau * (term * e + 2 * e) + 2.0 ** -23 * np.abs(loss)
    # (tau^2 times a logit next to the lowest fp32 leaves the range of the loss's type, which then holds an infinity)
    loss = np.where(loss > np.finfo(np.float32).max, np.inf, loss)
    mass = np.exp(lq)
    for r in range(p.shape[0]):
        np.add.at(mass[r], I[r], p[r])
    return loss, ltol, dz, mass * (w64 * tau * e)[:, None] + (w64 * tau * 2.0 ** -126)[:, None]


def _check(torch, got_loss, got_dz, ref):
    loss, ltol, dz, dtol = ref
    if got_loss is not None:
        x = got_loss.double().cpu().numpy()
        fine = np.isfinite(loss)
        assert np.array_equal(x[~fine], loss[~fine], equal_nan=True)
        assert np.all(np.abs(x - loss)[fine] <= ltol[fine]), np.abs(x - loss)[fine].max()
    if got_dz is not None:
        x = got_dz.double().cpu().numpy()
        tol = dtol + torch.finfo(got_dz.dtype).eps / 2 * 1.001 * np.abs(dz) + (2.0 ** -25 if got_dz.dtype == torch.float16 else 2.0 ** -133 if got_dz.dtype == torch.bfloat16 else 2.0 ** -149)
        fine = np.isfinite(dz)
        assert np.array_equal(np.isfinite(x), fine)
        bad = np.abs(x - dz)[fine] > tol[fine]
        assert not bad.any(), (int(bad.sum()), float((np.abs(x - dz)[fine] - tol[fine]).max()))


def _all_ways(torch, z, idx, t, tau, w, ref):
    from paper_2312_07759_b200 import binding as B
    loss, stats = B.distill_forward(z, idx, t, tau)
    _check(torch, loss, None, ref)
    dz = B.distill_backward(z, idx, t, tau, stats, w)
    _check(torch, None, dz, ref)
    loss2, dz2 = B.distill_step(z, idx, t, tau, w)
    _check(torch, loss2, dz2, ref)
    own = z.clone()
    loss3, dz3 = B.distill_step(own, idx, t, tau, w, out=own)          # in place
    assert dz3 is own and torch.equal(loss3.nan_to_num(-1), loss2.nan_to_num(-1)) and torch.equal(own.nan_to_num(-1), dz2.nan_to_num(-1))
    own = z.clone()
    B.distill_backward(own, idx, t, tau, stats, w, out=own)
    assert torch.equal(own.nan_to_num(-1), dz.nan_to_num(-1))
    return loss2, dz2


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("R,V,J", [(1, 1, 1), (2, 7, 3), (5, 1000, 5), (64, 1000, 8), (3, 4099, 100), (1, 50001, 64), (7, 32000, 256), (2, 151937, 50),
                                   (300, 513, 16), (9, 16384, 1), (3, 262147, 128)])
def test_loss_and_gradient(t, R, V, J):
    import torch
    z, idx, tl, w = _inputs(torch, R, V, J, t, "float32" if J % 2 else t, "int64" if R % 2 else "int32")
    for tau, weight in ((2.0, w), (1.0, None)):
        _all_ways(torch, z, idx, tl, tau, weight, _reference(z, idx, tl, tau, weight))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("R,V", [(40, 1003), (6, 60001)])
def test_padding_masks_and_repeats(t, R, V):
    """Rows without entries, entries that do not count, indices given twice and more, masked classes, the type's lowest value."""
    import torch
    z, idx, tl, w = _inputs(torch, R, V, 24, t)
    idx[0] = -1
    idx[1, 5:] = -1
    idx[2, :12] = idx[2, 12:]                   # twice
    idx[3] = idx[3, 0]                          # the same index throughout
    idx[4, ::2] = V                             # past the vocabulary
    tl[4, 1] = -float("inf")
    idx[5, 0], idx[5, 1] = V - 1, 0
    z[2, ::3] = -float("inf")                   # masked classes, a teacher's entry among them or not
    z[3, 1:200] = torch.finfo(z.dtype).min
    z[1, idx[1, 0]] = -float("inf")             # the teacher has mass where the student has none
    if R > 10:
        tl[6] = -float("inf")
        z[7, :] = 3.0                           # equal logits
        z[8, :] = -float("inf")
        z[8, 77] = 1.0                          # a single class
        idx[8, :] = 77
        idx[9] = 1 << 40                        # no entry, in 64 bits
        idx[10, 3] = -(1 << 40)
        z[11, 5] = torch.finfo(z.dtype).max if t != "float32" else 1e30
    ref = _reference(z, idx, tl, 2.0, w)
    loss, dz = _all_ways(torch, z, idx, tl, 2.0, w, ref)
    assert loss[0] == 0 and not dz[0].any() and loss[1] == float("inf") and torch.isfinite(dz[1].float()).all()
    if R > 10:
        assert loss[6] == 0 and not dz[6].any() and not dz[9].any()
        assert loss[8] < 0 and dz[8].abs().max() < 1e-5     # (one class: tau^2 times sum_j p_j ln p_j, its entries counted apart)


@pytest.mark.parametrize("t", TYPES)
def test_what_is_not_finite_stays_in_its_row(t):
    import torch
    from paper_2312_07759_b200 import binding as B
    z, idx, tl, w = _inputs(torch, 8, 3001, 16, t)
    loss, dz = B.distill_step(z, idx, tl, 1.0, w)
    z[2, 100], z[3, 5], tl[4, 3] = float("nan"), float("inf"), float("nan")
    z[5] = -float("inf")
    z[6, 9], idx[6] = float("nan"), -1          # ... of a row that has no entries: 0
    l2, d2 = B.distill_step(z, idx, tl, 1.0, w)
    for r in (0, 1, 7):
        assert l2[r] == loss[r] and torch.equal(d2[r], dz[r])
    assert torch.isnan(l2[2:6]).all() and l2[6] == 0 and not d2[6].any()
    assert torch.isnan(d2[2]).all() and torch.isnan(d2[5]).all()


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("V", [1000, 40007])
def test_strides_alignment_and_surroundings(t, V):
    import torch
    from paper_2312_07759_b200 import binding as B
    z, idx, tl, w = _inputs(torch, 6, V, 32, t)
    ref = _reference(z, idx, tl, 2.0, w)
    for at, ld in ((0, V + 24), (1, V + 24), (3, V + 7), (8, (V + 63) // 8 * 8 + 16)):
        wide = torch.full((8, ld + 16), float("nan"), device="cuda", dtype=z.dtype)
        view = wide[1:7, at:at + V]
        view.copy_(z)
        out = torch.full((8, ld + 40), 5.0, device="cuda", dtype=z.dtype)
        inner = out[1:7, 2 * at:2 * at + V]
        loss, _ = B.distill_step(view, idx, tl, 2.0, w, out=inner)
        _check(torch, loss, inner, ref)
        inner.fill_(5.0)
        assert torch.all(out == 5.0)
        loss, stats = B.distill_forward(view, idx, tl, 2.0)
        _check(torch, loss, None, ref)
        B.distill_backward(view, idx, tl, 2.0, stats, w, out=view)
        _check(torch, None, view, ref)
        view.fill_(float("nan"))
        assert torch.isnan(wide).all()
    tied = z[:1].expand(1, V)
    assert torch.equal(B.distill_step(tied, idx[:1], tl[:1], 2.0)[0], B.distill_step(z, idx, tl, 2.0)[0][:1])


@pytest.mark.parametrize("tau", [0.05, 0.7, 30.0])
def test_temperatures(tau):
    import torch
    z, idx, tl, w = _inputs(torch, 12, 2003, 10)
    _all_ways(torch, z, idx, tl, tau, w, _reference(z, idx, tl, tau, w))


def test_gradient_against_differences():
    """The loss's own differences in fp32: a step of 2^-4 has an error of its square times the third derivative (at most
    tau^2 / (4 tau^3)), and the two losses their rounding."""
    import torch
    from paper_2312_07759_b200 import binding as B
    tau, h = 1.5, 2.0 ** -4
    z, idx, tl, _ = _inputs(torch, 1, 37, 9)
    _, dz = B.distill_step(z, idx, tl, tau)
    both = torch.cat([z + h * torch.eye(37, device="cuda"), z - h * torch.eye(37, device="cuda")])
    loss, _ = B.distill_forward(both, idx.expand(74, -1).contiguous(), tl.expand(74, -1).contiguous(), tau)
    diff = (loss[:37].double() - loss[37:].double()) / (2 * h)
    tol = h * h / 6 * tau ** 2 / (4 * tau ** 3) + 2 * (float(loss.max()) + tau * tau * 4) * 60 * 2.0 ** -24 / (2 * h)
    assert (diff - dz[0].double()).abs().max() < tol


def test_streams_graphs_and_repeats():
    import torch
    from paper_2312_07759_b200 import binding as B
    z, idx, tl, w = _inputs(torch, 20, 30001, 40, "bfloat16")
    loss, dz = B.distill_step(z, idx, tl, 2.0, w)
    for _ in range(3):
        l2, d2 = B.distill_step(z, idx, tl, 2.0, w)
        assert torch.equal(l2, loss) and torch.equal(d2, dz)            # bit for bit
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    l3, d3 = B.distill_step(z, idx, tl, 2.0, w, stream=side)
    l4, d4 = B.distill_step(z, idx, tl, 2.0, w)                          # two at once
    torch.cuda.synchronize()
    assert torch.equal(l3, loss) and torch.equal(d3, dz) and torch.equal(l4, loss) and torch.equal(d4, dz)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        l5, stats = B.distill_forward(z, idx, tl, 2.0)
        d5 = B.distill_backward(z, idx, tl, 2.0, stats, w)
        l6, d6 = B.distill_step(z, idx, tl, 2.0, w)
    z.copy_(z.flip(0))
    graph.replay()
    l7, s7 = B.distill_forward(z, idx, tl, 2.0)
    assert torch.equal(l5, l7) and torch.equal(l6, B.distill_step(z, idx, tl, 2.0, w)[0]) and torch.equal(d5, B.distill_backward(z, idx, tl, 2.0, s7, w))
    assert torch.equal(d6, B.distill_step(z, idx, tl, 2.0, w)[1])


def test_refusals_of_tensors():
    import torch
    from paper_2312_07759_b200 import binding as B
    z, idx, tl, w = _inputs(torch, 4, 100, 8)
    with pytest.raises(ValueError):
        B.distill_step(z, idx, tl, 1.0, out=z[:, :99])
    with pytest.raises(ValueError):
        B.distill_step(z[:2], idx[:2], tl[:2], 1.0, out=z[1:3])         # shares rows with z without being z
    with pytest.raises(ValueError):
        B.distill_step(z, idx.cpu(), tl, 1.0)
    with pytest.raises(ValueError):
        B.distill_step(z, idx, tl, 1.0, w.double())
    with pytest.raises(B.IdkmError):
        B.distill_step(z, idx, tl, 0.0)
    with pytest.raises(B.IdkmError):
        B.distill_step(z[:0], idx[:0], tl[:0], 1.0)
    with pytest.raises(B.IdkmError):
        B.distill_step(z, idx[:, :0].contiguous(), tl[:, :0].contiguous(), 1.0)
    with pytest.raises(B.IdkmError):
        B.distill_step(z[:1].expand(4, 100), idx, tl, 1.0)              # rows on top of one another


def test_more_than_32_bits_of_offsets():
    import torch
    from paper_2312_07759_b200 import binding as B
    R, V = 70000, 65536
    z = torch.zeros(R, V, device="cuda", dtype=torch.bfloat16)
    tail, idx_tail, t_tail, _ = _inputs(torch, 3, V, 16, "bfloat16")
    z[-3:] = tail
    idx = torch.zeros(R, 16, device="cuda", dtype=torch.int64)
    idx[-3:] = idx_tail
    tl = torch.zeros(R, 16, device="cuda")
    tl[-3:] = t_tail
    ref = _reference(tail, idx_tail, t_tail, 2.0, None)
    loss, stats = B.distill_forward(z, idx, tl, 2.0)
    _check(torch, loss[-3:], None, ref)
    loss, dz = B.distill_step(z, idx, tl, 2.0, out=z)
    _check(torch, loss[-3:], dz[-3:], ref)
