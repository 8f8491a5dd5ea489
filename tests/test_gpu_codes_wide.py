"""Rows of more than 2^30 columns, to the largest there are (B200 only): byte offsets beyond 2^31 within a row.

X is 0 but at some columns, so that a product has few terms and the sum in float64 is known; a product's additions of zeros are
exact, and the chains of the others are no longer than their number: each rounds by at most 2^-23 of the terms' sizes."""
import numpy as np
import pytest

from oracle import group_codes as O

pytestmark = pytest.mark.gpu

MOST = 2 ** 31 - 4097


def _columns(cols):
    rng = np.random.default_rng(cols)
    near = [0, 1, 7, 8, 255, 256, 65279, 65280, 2 ** 29, 2 ** 30 - 1, 2 ** 30, 2 ** 30 + 1, 2 ** 30 + 257, cols - 65281, cols - 4096, cols - 257, cols - 2, cols - 1]
    at = np.concatenate([near, rng.integers(0, cols, 150), cols - 1 - rng.integers(0, 70000, 60)])
    return np.unique(at[(at >= 0) & (at < cols)])


@pytest.mark.parametrize("t,tokens,rows,cols,group,at", [("bfloat16", 1, 2, 2 ** 30 + 70001, 128, 0), ("float16", 2, 1, 2 ** 30 + 12, 0, 1), ("bfloat16", 1, 1, MOST, 32, 0),
                                                         ("float16", 1, 1, MOST, 1 << 40, 3), ("bfloat16", 1, 3, 2 ** 31 - 65281, 64, 5), ("float32", 1, 1, 2 ** 30 + 5, 128, 0)])
def test_products_of_wide_rows(t, tokens, rows, cols, group, at):
    import torch
    from paper_2312_07759_b200 import binding as B
    T = getattr(torch, t)
    torch.cuda.empty_cache()
    g = torch.Generator(device="cuda").manual_seed(cols % 1000)
    codes = torch.randint(0, 256, (rows, (cols + 31) // 32 * 16), device="cuda", dtype=torch.uint8, generator=g)
    C = torch.randn(16, device="cuda", generator=g).to(T)
    s = torch.exp(torch.randn(rows, -(-cols // group), device="cuda", generator=g)).to(T) if group else None
    room = torch.zeros(tokens * cols + 8, device="cuda", dtype=T)
    room[:at], room[at + tokens * cols:] = 1e4, 1e4
    X = room[at:at + tokens * cols].view(tokens, cols)
    k = torch.from_numpy(_columns(cols)).cuda()
    X[:, k] = torch.randn(tokens, k.numel(), device="cuda", generator=g).to(T)
    Y = B.matmul_codes(X, codes, C, s, group).double().cpu().numpy()
    code = (codes[:, k // 2] >> (4 * (k % 2))) & 15
    w = C.double()[code.long()]
    if s is not None:
        w = w * s.double()[:, k // min(group, cols)]
    x = X[:, k].double()
    y, size = (x @ w.T).cpu().numpy(), (x.abs() @ w.abs().T).cpu().numpy()
    tol = k.numel() * 2.0 ** -23 * size + torch.finfo(T).eps / 2 * np.abs(y) * 1.001
    assert np.all(np.abs(Y - y) <= tol), np.abs(Y - y).max()


@pytest.mark.parametrize("group", [128, 1 << 40])
def test_export_of_a_wide_row(group):
    import torch
    from paper_2312_07759_b200 import binding as B
    torch.cuda.empty_cache()
    W = torch.zeros(1, MOST, device="cuda", dtype=torch.bfloat16)
    spans = [(a, min(a + 1024, MOST)) for a in (0, 2 ** 30 - 512, 2 ** 31 - 65536, MOST // 1024 * 1024 - 1024, MOST // 1024 * 1024)]
    for a, b in spans:
        W[0, a:b] = torch.randn(b - a, device="cuda").bfloat16()
    W[0, spans[1][0] + 5] = 9.0            # (the largest of all)
    C = torch.linspace(-1, 1, 16).bfloat16()
    codes, scales, _ = B.assign_groups(W, C.cuda(), group)
    for a, b in spans:
        part = W[:, a:b].cpu()
        if group > MOST:
            assert scales.shape == (1, 1) and scales.item() == 9.0
            part = torch.cat([part, torch.full((1, 1), 9.0, dtype=torch.bfloat16)], 1)     # the scale of the whole row
        idx, s, _ = O.assign(part, C, min(group, 2048))
        want = idx[:, :b - a]
        assert np.array_equal(O.unpack(codes[:, a // 2:(b + 1) // 2].cpu().numpy(), b - a), want)
        if group < MOST:
            assert torch.equal(scales[:, a // 128:-(-b // 128)].cpu(), s)
