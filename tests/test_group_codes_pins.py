"""Pins of the group-scale oracle, and the argument checks of the operators on group codes, without a device."""
import numpy as np
import pytest
import torch

from oracle import group_codes as O
from oracle import hard_assign as H


def test_oracle_on_hand_computed_groups():
    W = torch.tensor([[1.0, -2.0, 0.5] + [0.0] * 29 + [4.0, -1.0]])
    C = torch.tensor([-1.0, 0.0, 0.5, 1.0])
    idx, s, Wq = O.assign(W, C, 32)
    assert s.tolist() == [[2.0, 4.0]]
    # 1 = 2 * 0.5, -2 = 2 * -1, 0.5 lies between 0 and 1 (ties to the lower index), zeros, 4 = 4 * 1, -1 is nearest to 0
    assert idx[0, :4].tolist() == [2, 0, 1, 1] and idx[0, 32:].tolist() == [3, 1]
    assert Wq[0, :3].tolist() == [1.0, -2.0, 0.0] and Wq[0, 32:].tolist() == [4.0, 0.0]
    b = O.pack(idx)
    assert b.shape == (1, 32) and b[0, 0] == 0x02 and b[0, 16] == 0x13 and not b[0, 17:].any()
    assert np.array_equal(O.unpack(b, 34), idx)
    assert np.array_equal(O.weights(b, C, s, 32, 34)[0], Wq.double().numpy()[0])


def test_oracle_agrees_with_the_plain_hard_quantiser():
    """One group whose scale is 1: the indices and, for rows of a multiple of 32 weights, the bytes of the plain export."""
    g = torch.Generator().manual_seed(3)
    C = torch.rand(16, generator=g) * 2 - 1
    C[5] = 1.0
    W = (torch.rand(4, 96, generator=g) * 2 - 1) * 0.999
    W[:, 7] = 1.0
    idx, s, _ = O.assign(W, C, 96)
    assert torch.all(s == 1)
    ref = H.hard_assign(W.reshape(-1, 1).numpy(), C.reshape(-1, 1).numpy())
    assert np.array_equal(idx.reshape(-1), ref)
    assert np.array_equal(O.pack(idx).reshape(-1), H.pack_codes(ref, 16))


def test_odd_groups():
    C = torch.tensor([-1.0, float("nan"), 1.0])
    W = torch.tensor([[0.0] * 32, [float("nan")] + [1.0] * 31, [float("inf")] + [1.0] * 31])
    idx, s, _ = O.assign(W, C, 32)
    assert not idx.any() and s[0, 0] == 0 and torch.isnan(s[1, 0]) and torch.isinf(s[2, 0])


def _groups(B, W=1 << 20, wt=0, rows=4, cols=64, ld=64, C=1 << 21, k=16, t=0, g=32, codes=1 << 22, s=1 << 23, Wq=None):
    return B.lib.idkm_assign_groups(W, wt, rows, cols, ld, C, k, t, g, codes, s, Wq, None)


def _matmul(B, X=1 << 20, t=1, m=2, ldx=64, codes=1 << 21, rows=4, cols=64, pitch=32, C=1 << 22, k=16, s=1 << 23, g=32, Y=1 << 24, ldy=4):
    return B.lib.idkm_matmul_codes(X, t, m, ldx, codes, rows, cols, pitch, C, k, s, g, Y, ldy, None)


@pytest.mark.parametrize("change,status", [
    (dict(W=None), "NULL"), (dict(C=None), "NULL"), (dict(codes=None), "NULL"), (dict(s=None), "NULL"),
    (dict(k=0), "UNSUPPORTED"), (dict(k=17), "UNSUPPORTED"), (dict(wt=3), "UNSUPPORTED"), (dict(t=-1), "UNSUPPORTED"),
    (dict(g=48), "UNSUPPORTED"), (dict(cols=512, ld=512, g=192), "UNSUPPORTED"), (dict(rows=0), "SHAPE"), (dict(cols=0), "SHAPE"),
    (dict(ld=63), "SHAPE"), (dict(g=0), "SHAPE"), (dict(g=-32), "SHAPE"), (dict(rows=1 << 30, cols=1 << 30, ld=1 << 30), "SHAPE"),
    (dict(Wq=1 << 20), "PARAM"), (dict(W=(1 << 20) + 2), "ALIGN"), (dict(codes=(1 << 22) + 8), "ALIGN"), (dict(s=(1 << 23) + 1), "ALIGN")])
def test_refusals_of_assign_groups(change, status):
    from paper_2312_07759_b200 import binding as B
    assert _groups(B, **change) == getattr(B, "ERR_" + status)


@pytest.mark.parametrize("change,status", [
    (dict(X=None), "NULL"), (dict(codes=None), "NULL"), (dict(C=None), "NULL"), (dict(Y=None), "NULL"),
    (dict(t=3), "UNSUPPORTED"), (dict(k=17), "UNSUPPORTED"), (dict(g=16), "UNSUPPORTED"), (dict(cols=130, ldx=130, pitch=80, g=96), "UNSUPPORTED"),
    (dict(m=0), "SHAPE"), (dict(rows=0), "SHAPE"), (dict(ldx=63), "SHAPE"), (dict(ldy=3), "SHAPE"), (dict(pitch=16), "SHAPE"),
    (dict(g=0), "SHAPE"), (dict(cols=65, ldx=65), "SHAPE"), (dict(Y=1 << 20), "PARAM"), (dict(Y=1 << 21), "PARAM"),
    (dict(X=(1 << 20) + 1), "ALIGN"), (dict(codes=(1 << 21) + 4), "ALIGN"), (dict(pitch=40), "ALIGN"), (dict(Y=(1 << 24) + 1), "ALIGN")])
def test_refusals_of_matmul_codes(change, status):
    from paper_2312_07759_b200 import binding as B
    assert _matmul(B, **change) == getattr(B, "ERR_" + status)


def test_pitch():
    from paper_2312_07759_b200 import binding as B
    assert [B.lib.idkm_group_codes_pitch(n) for n in (-1, 0, 1, 32, 33, 512)] == [0, 0, 16, 16, 32, 256]


def test_binding_refuses_tensors_off_the_device():
    from paper_2312_07759_b200 import binding as B
    W, C = torch.zeros(4, 64), torch.linspace(-1, 1, 16)
    with pytest.raises(ValueError):
        B.assign_groups(W, C, 32)
    with pytest.raises(ValueError):
        B.matmul_codes(W, torch.zeros(4, 32, dtype=torch.uint8), C)
    with pytest.raises(ValueError):
        B.matmul_codes(W, torch.zeros(4, 16, dtype=torch.uint8), C)      # too few codes a row
    with pytest.raises(ValueError):
        B.matmul_codes(W.half(), torch.zeros(4, 32, dtype=torch.uint8), C)   # two types
    with pytest.raises(B.IdkmError):
        B.assign_groups(W.double(), C, 32)
