"""Which outputs share memory with an input: matrices whose rows lie between one another's, without a device."""
import numpy as np
import torch


def _bytes(t):
    """Every byte of a matrix's or vector's elements, one by one."""
    rows = t if t.dim() == 2 else t.reshape(1, -1)
    out = set()
    for r in range(rows.shape[0]):
        a = rows[r].data_ptr()
        out.update(range(a, a + rows.shape[1] * rows.element_size()))
    return out


def _refused(out, *inputs):
    from paper_2312_07759_b200 import binding as B
    try:
        B._apart(out, *inputs)
    except ValueError:
        return True
    return False


def test_halves_of_a_buffer():
    buf = torch.zeros(6, 200)
    assert not _refused(buf[:, 100:], buf[:, :100]) and not _refused(buf[:, :100], buf[:, 100:])
    assert _refused(buf[:, 99:], buf[:, :100]) and _refused(buf[:, :100], buf[:, 99:])
    assert not _refused(buf[:3], buf[3:]) and _refused(buf[:4], buf[3:])
    assert not _refused(buf[::2, :150], buf[1::2, 50:]) and _refused(buf[::2, :150], buf[2::2, 50:])
    assert not _refused(buf[1:, :20], buf[:-1, 180:]) and _refused(buf, buf) and not _refused(buf, None)
    assert not _refused(buf[:, 100:], buf[:, :100], None, buf[:, 50:60]) and _refused(buf[:, 100:], buf[:, :100], None, buf[:, 150:160])


def test_against_every_byte():
    rng = np.random.default_rng(5)
    flat = torch.zeros(400)
    other = flat.view(torch.uint8)
    seen = [0, 0]
    for _ in range(3000):
        made = []
        for k in range(2):
            base = flat if k == 0 or rng.random() < 0.7 else other
            cols = int(rng.integers(1, 12))
            ld = int(rng.integers(cols, 40)) if rng.random() < 0.6 else 24
            rows = int(rng.integers(1, 8))
            if ld < cols or (rows - 1) * ld + cols > 300:
                rows = 1
            at = int(rng.integers(0, base.numel() - (rows - 1) * ld - cols + 1)) if base is flat else int(rng.integers(0, 1600 - (rows - 1) * ld - cols + 1))
            made.append(base.as_strided((rows, cols), (ld, 1), at) if rng.random() < 0.8 else base[at:at + cols])
        share = bool(_bytes(made[0]) & _bytes(made[1]))
        assert _refused(made[0], made[1]) == share and _refused(made[1], made[0]) == share
        seen[share] += 1
    assert min(seen) > 300


def test_nothing_shares_with_an_empty_tensor():
    buf = torch.zeros(4, 8)
    assert not _refused(buf, buf[:0]) and not _refused(buf, buf[:, :0])
