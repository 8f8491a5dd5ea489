"""4-bit codes with group scales on the GPU: the export against the float64 oracle bit for bit, products against it within the
rounding of fp32 sums (B200 only).

A product's terms s c x are summed in fp32, the group's sum scaled, in chains of at most 192 + cols / 128 additions (a group's
128 and the steps of one matrix instruction, the groups one after another, the joins of lanes and warps), each of which rounds or
cuts by at most 2^-23 of the sum of the terms' sizes; the result is then rounded to its type, eps / 2 of its value."""
import numpy as np
import pytest

from oracle import group_codes as O

pytestmark = pytest.mark.gpu

TYPES = ("float32", "bfloat16", "float16")


def _codebook(torch, k, dtype, seed, symmetric=False):
    g = torch.Generator().manual_seed(seed)
    c = torch.randn(k, generator=g)
    if symmetric:
        c = torch.linspace(-1, 1, k)
    return c.to(dtype)


def _check_export(torch, W, C, group):
    from paper_2312_07759_b200 import binding as B
    codes, scales, Wq = B.assign_groups(W.cuda() if not W.is_cuda else W, C.cuda(), group, want_Wq=True)
    idx, s, q = O.assign(W.cpu(), C, group)
    as_bits = lambda x: x.cpu().contiguous().view(torch.int16 if x.element_size() == 2 else torch.int32)
    same = as_bits(scales) == as_bits(s)
    assert torch.all(same | (torch.isnan(scales.cpu()) & torch.isnan(s)))
    assert np.array_equal(codes.cpu().numpy(), O.pack(idx))
    q, Wq = q.float().numpy(), Wq.float().cpu().numpy()
    assert np.array_equal(Wq, q, equal_nan=True)
    c2, s2, none = B.assign_groups(W.cuda() if not W.is_cuda else W, C.cuda(), group)
    assert none is None and torch.equal(c2, codes) and torch.equal(s2.nan_to_num(7.0), scales.nan_to_num(7.0))


@pytest.mark.parametrize("wt", TYPES)
@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,cols,group", [(1, 1, 32), (3, 31, 32), (5, 33, 64), (7, 1000, 32), (64, 512, 64), (9, 4099, 128), (4, 640, 256),
                                             (3, 1000, 384), (2, 5000, 5000), (17, 264, 4096), (1, 40, 40)])
def test_export(wt, t, rows, cols, group):
    import torch
    g = torch.Generator().manual_seed(rows * 131 + cols)
    W = (torch.randn(rows, cols, generator=g) * torch.exp(torch.randn(rows, 1, generator=g))).to(getattr(torch, wt))
    _check_export(torch, W, _codebook(torch, 16, getattr(torch, t), cols), group)


@pytest.mark.parametrize("k", [1, 2, 3, 5, 8, 15, 16])
@pytest.mark.parametrize("t", TYPES)
def test_export_ties_and_codebooks(k, t):
    """Weights on the codebook's own grid, so that ties are frequent; symmetric codebooks, equal, close and odd entries."""
    import torch
    T = getattr(torch, t)
    g = torch.Generator().manual_seed(k)
    W = torch.randint(-16, 17, (40, 512), generator=g).float() / 16
    W[:, ::64] = 1.0
    W[3] = 0.0
    for C in (_codebook(torch, k, T, k), _codebook(torch, k, T, k, symmetric=True), (torch.randint(-8, 9, (k,), generator=g) / 8.0).to(T)):
        if not C.abs().max() > 0:
            C[0] = 1.0
        _check_export(torch, W, C, 64)
        _check_export(torch, W[:, 1:].contiguous(), C, 32)
        _check_export(torch, W, C, 512)
    if k >= 3:
        C = _codebook(torch, k, torch.float32, 9)
        C[1] = C[0] * (1 + 2.0 ** -22)           # next to another
        _check_export(torch, W, C, 64)
        C[1] = 1e-30
        C[2] = 2e-30                             # not told apart next to the others
        _check_export(torch, W, C, 64)
        C[1] = float("nan")
        C[2] = float("inf")
        if k > 3:
            _check_export(torch, W, C, 64)


@pytest.mark.parametrize("scale", [1e-38, 1e-30, 1e-7, 1.0, 1e4, 1e30])
@pytest.mark.parametrize("t", TYPES)
def test_export_of_large_and_small_weights(scale, t):
    """Scales that underflow, are subnormal or overflow in their type; groups with a NaN or an infinity."""
    import torch
    g = torch.Generator().manual_seed(5)
    W = torch.randn(6, 300, generator=g) * scale
    C = _codebook(torch, 16, getattr(torch, t), 1)
    _check_export(torch, W, C, 32)
    _check_export(torch, W, (C.float() * 1e-4).to(C.dtype), 128)
    W[1, 5], W[2, 40], W[3, 299] = float("nan"), float("inf"), -float("inf")
    _check_export(torch, W, C, 32)
    _check_export(torch, W, C, 300)


def test_export_of_every_half_value():
    """All finite fp16 values as weights: every place between midpoints, subnormal ones included."""
    import torch
    W = torch.arange(0, 65536, dtype=torch.int32).to(torch.int16).view(torch.float16)
    W = W[torch.isfinite(W)].clone()
    W = W[: W.numel() // 128 * 128].view(-1, 128)
    for t in TYPES:
        _check_export(torch, W, _codebook(torch, 16, getattr(torch, t), 4), 128)
        _check_export(torch, W.reshape(4, -1), _codebook(torch, 16, getattr(torch, t), 4), 1 << 20)


def test_export_strides_and_alignment():
    import torch
    g = torch.Generator().manual_seed(6)
    big = torch.randn(20, 777, generator=g).cuda()
    C = _codebook(torch, 16, torch.bfloat16, 2)
    for view in (big[:, 3:300], big[2:9, :512], big[::3, 5:400], big[:1, 1:34], big.half()[:, 1:130]):
        _check_export(torch, view, C, 64)


def _case(torch, tokens, rows, cols, group, t, k=16, seed=0):
    T = getattr(torch, t)
    g = torch.Generator(device="cuda").manual_seed(seed + tokens * 7 + rows + cols)
    codes = torch.randint(0, 256, (rows, (cols + 31) // 32 * 16), device="cuda", dtype=torch.uint8, generator=g)   # padding is not 0
    C = torch.randn(k, device="cuda", generator=g).to(T)
    X = torch.randn(tokens, cols, device="cuda", generator=g).to(T)
    s = torch.exp(torch.randn(rows, -(-cols // group), device="cuda", generator=g)).to(T) if group else None
    return X, codes, C, s


def _check_product(torch, Y, X, codes, C, s, group):
    y, size = O.matmul(X.cpu(), codes.cpu().numpy(), C.cpu(), None if s is None else s.cpu(), group or X.shape[1])
    tol = (192 + X.shape[1] / 128) * 2.0 ** -23 * size + torch.finfo(Y.dtype).eps / 2 * np.abs(y) * 1.001 + (2.0 ** -25 if Y.dtype == torch.float16 else 0)
    err = np.abs(Y.double().cpu().numpy() - y)
    assert np.all(err <= tol), (float((err - tol).max()), np.unravel_index(int((err - tol).argmax()), err.shape))


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("group", [0, 32, 64, 128, 256, 100000])
@pytest.mark.parametrize("tokens,rows,cols", [(1, 1, 1), (1, 1000, 512), (1, 129, 4099), (2, 17, 33), (3, 300, 640), (5, 16, 1000), (8, 257, 96),
                                              (9, 130, 700), (16, 64, 2048), (17, 48, 260), (33, 200, 384), (64, 128, 128)])
def test_products(t, group, tokens, rows, cols):
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    _check_product(torch, B.matmul_codes(X, codes, C, s, group), X, codes, C, s, group)


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("group", [0, 32, 64, 128, 384])
@pytest.mark.parametrize("tokens,rows,cols", [(127, 129, 515), (128, 256, 1024), (200, 1000, 2304), (257, 300, 64), (300, 4608, 130), (1025, 513, 1088)])
def test_products_of_prompts(t, group, tokens, rows, cols):
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    _check_product(torch, B.matmul_codes(X, codes, C, s, group), X, codes, C, s, group)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("tokens", [1, 4, 40, 160])
def test_products_strides_alignment_and_small_codebooks(t, tokens):
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, 90, 421, 64, t, k=11)      # codes past the codebook stand for 0
    ref = B.matmul_codes(X, codes, C, s, 64)
    _check_product(torch, ref, X, codes, C, s, 64)
    wide = torch.zeros(tokens, 700, device="cuda", dtype=X.dtype)
    for at in (0, 1, 8):
        wide.fill_(float("nan"))                                     # what lies beside the rows is not read into a sum
        view = wide[:, at:at + 421]
        view.copy_(X)
        _check_product(torch, B.matmul_codes(view, codes, C, s, 64), X, codes, C, s, 64)
    pitched = torch.full((90, 400), 255, device="cuda", dtype=torch.uint8)
    pitched[:, :codes.shape[1]] = codes
    assert torch.equal(B.matmul_codes(X, pitched[:, :codes.shape[1]], C, s, 64), ref)
    # an output inside a larger one: what surrounds it stays
    out = torch.full((tokens + 2, 128), 7.0, device="cuda", dtype=X.dtype)
    B.matmul_codes(X, codes, C, s, 64, out=out[1:-1, 3:93])
    assert torch.equal(out[1:-1, 3:93], ref)
    out[1:-1, 3:93] = 7.0
    assert torch.all(out == 7.0)


@pytest.mark.parametrize("t", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens", [1, 7, 100])
def test_products_with_what_is_not_finite(t, tokens):
    """A NaN in one row of X, an infinite scale of one row of W: they reach what they belong to and nothing else."""
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, 50, 300, 32, t)
    ref = B.matmul_codes(X, codes, C, s, 32)
    X[tokens // 2, 17] = float("nan")
    s[11, 3] = float("inf")
    got = B.matmul_codes(X, codes, C, s, 32)
    rest = torch.ones_like(ref, dtype=torch.bool)
    rest[tokens // 2] = False
    rest[:, 11] = False
    assert torch.equal(got[rest], ref[rest])
    assert torch.isnan(got[tokens // 2]).all() and not torch.isfinite(got[:, 11]).any()


def test_codes_of_the_plain_export():
    """The bytes of `assign` for scalar weights, without scales: the product is that of the assigned centroids."""
    import torch
    from paper_2312_07759_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(8)
    W = torch.randn(200, 576, device="cuda", generator=g) * 0.05
    C = torch.linspace(-0.12, 0.12, 16, device="cuda").reshape(16, 1)
    codes, Wq = B.assign(W.reshape(-1, 1), C)
    X = torch.randn(3, 576, device="cuda", generator=g)
    Y = B.matmul_codes(X, codes.view(200, 288), C)
    _check_product(torch, Y, X, codes.view(200, 288), C, None, 0)
    assert torch.allclose(Y.double(), X.double() @ Wq.view(200, 576).double().T, atol=1e-5)


@pytest.mark.parametrize("t", ["bfloat16", "float32"])
@pytest.mark.parametrize("tokens", [1, 6, 130])
def test_streams_graphs_and_repeats(t, tokens):
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, 515, 1056, 128, t)
    ref = B.matmul_codes(X, codes, C, s, 128)
    for _ in range(3):
        assert torch.equal(B.matmul_codes(X, codes, C, s, 128), ref)      # bit for bit
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    a = B.matmul_codes(X, codes, C, s, 128, stream=side)
    b = B.matmul_codes(X, codes, C, s, 128)                               # two at once
    W = (torch.randn(64, 512, device="cuda") * 0.1)
    want = B.assign_groups(W, C, 64)
    side.wait_stream(torch.cuda.current_stream())
    got = B.assign_groups(W, C, 64, stream=side)
    torch.cuda.synchronize()
    assert torch.equal(a, ref) and torch.equal(b, ref) and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    graph, out, out2 = torch.cuda.CUDAGraph(), torch.zeros_like(ref), torch.zeros_like(ref)
    X2 = X.clone()
    with torch.cuda.graph(graph):
        B.matmul_codes(X, codes, C, s, 128, out=out)
        B.matmul_codes(X2, codes, C, s, 128, out=out2)
        captured = B.assign_groups(W, C, 64)
    X2.copy_(X.flip(0))
    graph.replay()
    assert torch.equal(out, ref) and torch.equal(out2, B.matmul_codes(X2, codes, C, s, 128)) and torch.equal(captured[0], want[0])


def test_refusals_of_tensors():
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, 2, 16, 64, 32, "float16")
    for bad in [(X, codes, C.float(), s, 32), (X, codes, C, s.float(), 32), (X, codes, C, s[:, :1], 32), (X, codes, C, s[:8], 32), (X, codes, C, s, 0),
                (X.t(), codes, C, s, 32), (X, codes.t(), C, s, 32), (X, codes.cpu(), C, s, 32), (X, codes.int(), C, s, 32), (X[0], codes, C, s, 32)]:
        with pytest.raises((ValueError, B.IdkmError)):
            B.matmul_codes(*bad)
    for out in (X, torch.empty(2, 17, device="cuda", dtype=torch.float16), torch.empty(2, 16, device="cuda"), torch.empty(2, 16, dtype=torch.float16)):
        with pytest.raises(ValueError):
            B.matmul_codes(X, codes, C, s, 32, out=out)
    with pytest.raises(ValueError):
        B.matmul_codes(X, codes, C, s, 32, out=X[:, :16])
    with pytest.raises(B.IdkmError):
        B.assign_groups(X, torch.zeros(17, device="cuda"), 32)
    with pytest.raises(B.IdkmError):
        B.matmul_codes(X[:0], codes, C, s, 32)
    with pytest.raises(B.IdkmError):
        B.matmul_codes(X.expand(2, 64)[:1].expand(4, 64), codes, C, s, 32)   # rows on top of one another


def test_more_than_32_bits_of_offsets():
    """Rows of codes beyond 4 GB, weights beyond 2^32: the last rows are right."""
    import torch
    from paper_2312_07759_b200 import binding as B
    rows, cols = (1 << 20) + 70000, 8192
    C = torch.linspace(-1, 1, 16, device="cuda").bfloat16()
    codes = torch.zeros(rows, cols // 2, device="cuda", dtype=torch.uint8)
    tail = torch.randint(0, 256, (40, cols // 2), device="cuda", dtype=torch.uint8)
    codes[-40:] = tail
    for tokens in (1, 150):
        X = torch.randn(tokens, cols, device="cuda").bfloat16()
        s = torch.full((rows, cols // 128), 0.25, device="cuda", dtype=torch.bfloat16)
        Y = B.matmul_codes(X, codes, C, s, 128)
        _check_product(torch, Y[:, -40:], X, tail, C, s[-40:], 128)
        del Y, s
    del codes
    W = torch.zeros((1 << 19) + 100, cols, device="cuda", dtype=torch.bfloat16)
    W[-20:] = torch.randn(20, cols, device="cuda").bfloat16()
    codes, scales, _ = B.assign_groups(W, C, 128)
    idx, sref, _ = O.assign(W[-20:].cpu(), C.cpu(), 128)
    assert np.array_equal(codes[-20:].cpu().numpy(), O.pack(idx)) and torch.equal(scales[-20:].cpu(), sref)


def test_the_operators_together():
    """A classifier's export, its logits from the codes, the loss against the full-precision teacher's top logits, and the gradient
    through the soft quantiser: each step against float64."""
    import torch
    from oracle import distill as OD
    from oracle import idkm_ref as R
    from paper_2312_07759_b200 import binding as B
    g = torch.Generator(device="cuda").manual_seed(11)
    V, K, M, tau_w, tau = 1000, 512, 12, 0.01, 2.0
    W = torch.randn(V, K, device="cuda", generator=g) * (1.0 / K) ** 0.5
    X = torch.randn(M, K, device="cuda", generator=g)
    t, idx = torch.topk(X @ W.T, 20, dim=1)
    ctx = B.Context()
    C0 = torch.quantile(W.flatten()[:100000], (torch.arange(16, device="cuda") + 0.5) / 16).reshape(16, 1)
    fr = ctx.forward(W.reshape(-1, 1), C0, tau_w, 0.0, 20)
    # served: codes relative to groups, one sample and all of them
    C16 = fr.C.half()
    codes, scales, _ = B.assign_groups(W, C16, 128)
    z = B.matmul_codes(X.half(), codes, C16, scales, 128)
    _check_product(torch, z, X.half(), codes, C16, scales, 128)
    assert torch.allclose(B.matmul_codes(X[:1].half(), codes, C16, scales, 128).float(), z[:1].float(), rtol=4e-3, atol=4e-3)
    # trained: the soft weights' logits, loss and gradient
    Wq = fr.Wq.view(V, K)
    zs = X @ Wq.T
    w = torch.full((M,), 1.0 / M, device="cuda")
    loss, dz = B.distill_step(zs, idx, t, tau, w)
    rl, rdz, _, _ = OD.distill(zs.cpu().numpy(), idx.cpu().numpy(), t.cpu().numpy(), tau, w.cpu().numpy())
    assert np.allclose(loss.cpu().numpy(), rl, rtol=1e-5, atol=1e-6) and np.allclose(dz.cpu().numpy(), rdz, rtol=1e-4, atol=1e-7)
    dW, dC = ctx.backward((dz.T @ X).reshape(-1, 1).contiguous(), B.IMPLICIT, 0.0, 20, 1.0)
    W64, G64 = W.double().cpu().numpy().reshape(-1, 1), (rdz.T @ X.double().cpu().numpy()).reshape(-1, 1)
    Ct = fr.C.double().cpu().numpy()
    _, _, S, F = R.final(W64, Ct, float(np.float32(tau_w)))
    rdW, rdC, _, _ = R.backward(W64, G64, Ct, float(np.float32(tau_w)), S, F, adj_max_iter=20)
    assert np.abs(dC.cpu().numpy() - rdC).max() < 2e-3 * np.abs(rdC).max()
    assert np.linalg.norm(dW.cpu().numpy() - rdW) < 3e-3 * np.linalg.norm(rdW)


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,rows,cols,group", [(1, 21, 51000, 128), (1, 5, 70000, 65536), (2, 37, 33000, 32), (8, 33, 12300, 64), (8, 50, 9000, 32),
                                                    (12, 40, 9000, 128), (16, 257, 4096, 256), (16, 30, 5200, 32), (10, 3000, 260, 0), (3, 70, 16384, 1 << 20),
                                                    (40, 513, 70, 32), (31, 2000, 1000, 640)])
def test_products_between_the_kernels(t, tokens, rows, cols, group):
    """Rows that fit into a multiprocessor's memory with the stages, with fewer of them, and not at all; groups longer than that."""
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    ref = B.matmul_codes(X, codes, C, s, group)
    _check_product(torch, ref, X, codes, C, s, group)
    wide = torch.full((tokens, cols + 3), float("nan"), device="cuda", dtype=X.dtype)
    wide[:, 3:] = X
    _check_product(torch, B.matmul_codes(wide[:, 3:], codes, C, s, group), X, codes, C, s, group)


@pytest.mark.parametrize("t", TYPES)
@pytest.mark.parametrize("rows,cols,group", [(40, 4099, 32), (17, 513, 64), (9, 1025, 128)])
def test_products_with_scales_and_rows_anywhere(t, rows, cols, group):
    """Scales, codebook and X that begin at any element of a larger tensor (odd numbers of groups a row among them)."""
    import torch
    from paper_2312_07759_b200 import binding as B
    for tokens in (1, 6, 70):
        X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
        ref = B.matmul_codes(X, codes, C, s, group)
        for at in (1, 2, 5):
            flat = torch.full((s.numel() + 8,), float("nan"), device="cuda", dtype=s.dtype)
            flat[at:at + s.numel()] = s.flatten()
            book = torch.full((24,), float("nan"), device="cuda", dtype=s.dtype)
            book[at:at + 16] = C
            got = B.matmul_codes(X, codes, book[at:at + 16], flat[at:at + s.numel()].view(s.shape), group)
            assert torch.equal(got, ref)


@pytest.mark.parametrize("t", ["bfloat16", "float32"])
def test_guard_words_around_products(t):
    """Every byte outside the result stays as it was, whichever kernel takes the product."""
    import torch
    from paper_2312_07759_b200 import binding as B
    for tokens, rows, cols in [(1, 1, 1), (1, 33, 300), (5, 1001, 640), (16, 129, 256), (18, 257, 200), (150, 131, 129)]:
        X, codes, C, s = _case(torch, tokens, rows, cols, 64, t)
        room = torch.full((tokens * rows + 4096,), 3.0, device="cuda", dtype=X.dtype)
        out = room[2048:2048 + tokens * rows].view(tokens, rows)
        B.matmul_codes(X, codes, C, s, 64, out=out)
        _check_product(torch, out, X, codes, C, s, 64)
        assert torch.all(room[:2048] == 3.0) and torch.all(room[2048 + tokens * rows:] == 3.0)


def test_guard_words_around_the_export():
    import torch
    from paper_2312_07759_b200 import binding as B
    C = torch.linspace(-1, 1, 16, device="cuda").bfloat16()
    for rows, cols, group in [(1, 1, 32), (3, 33, 32), (7, 1000, 128), (2, 5000, 384), (300, 257, 64)]:
        W = torch.randn(rows, cols, device="cuda")
        pitch, n = (cols + 31) // 32 * 16, -(-cols // group)
        codes = torch.full((rows * pitch + 512,), 0xA5, device="cuda", dtype=torch.uint8)
        scales = torch.full((rows * n + 512,), 3.0, device="cuda", dtype=torch.bfloat16)
        Wq = torch.full((rows * cols + 512,), 3.0, device="cuda")
        rc = B.lib.idkm_assign_groups(W.data_ptr(), 0, rows, cols, cols, C.data_ptr(), 16, 1, group, codes[256:].data_ptr(), scales[256:].data_ptr(),
                                      Wq[256:].data_ptr(), None)
        assert rc == B.OK
        torch.cuda.synchronize()
        want = B.assign_groups(W, C, group, want_Wq=True)
        for room, got, v in ((codes, want[0], 0xA5), (scales, want[1], 3.0), (Wq, want[2], 3.0)):
            k = got.numel()
            assert torch.equal(room[256:256 + k], got.flatten()) and torch.all(room[:256] == v) and torch.all(room[256 + k:] == v)


def test_calls_at_once_from_threads():
    """Two host threads, a stream each: every call gets its own result."""
    import threading
    import torch
    from paper_2312_07759_b200 import binding as B
    work = [_case(torch, m, 700, 1024, 128, "bfloat16", seed=i) for i, m in enumerate((1, 4, 16, 100))]
    refs = [B.matmul_codes(X, codes, C, s, 128) for X, codes, C, s in work]
    torch.cuda.synchronize()
    wrong = []

    def run(i):
        stream = torch.cuda.Stream()
        for k in range(60):
            X, codes, C, s = work[(i + k) % 4]
            Y = B.matmul_codes(X, codes, C, s, 128, stream=stream)
            stream.synchronize()
            if not torch.equal(Y, refs[(i + k) % 4]):
                wrong.append((i, k))

    threads = [threading.Thread(target=run, args=(i,)) for i in range(2)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not wrong


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("tokens,rows,cols,group", [(16, 40, 20000, 32), (9, 535, 11392, 64), (16, 300, 8197, 128), (8, 100, 28672, 0), (12, 50, 40001, 3200),
                                                    (16, 20, 140000, 65664), (3, 33, 70001, 35072), (16, 39000, 2900, 128), (5, 17, 131072, 32),
                                                    (1, 2500, 90000, 256)])
def test_products_whose_columns_come_in_parts(t, tokens, rows, cols, group):
    """X that one multiprocessor cannot hold: groups that end where a part does, in its middle, and that span several."""
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    ref = B.matmul_codes(X, codes, C, s, group)
    _check_product(torch, ref, X, codes, C, s, group)
    assert torch.equal(B.matmul_codes(X, codes, C, s, group), ref)


@pytest.mark.parametrize("t", ["bfloat16", "float16"])
@pytest.mark.parametrize("group", [0, 32, 64, 128, 384, 1280])
@pytest.mark.parametrize("tokens,rows,cols", [(17, 300, 4099), (40, 535, 11392), (64, 257, 1000), (100, 2048, 1160), (130, 200, 2312), (300, 700, 5128), (513, 256, 3200)])
def test_products_whose_columns_are_shared(t, group, tokens, rows, cols):
    """Few tiles, whose columns several pairs of blocks share: shares that begin within a group, that are shorter than others or empty."""
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    ref = B.matmul_codes(X, codes, C, s, group)
    _check_product(torch, ref, X, codes, C, s, group)
    for _ in range(3):
        assert torch.equal(B.matmul_codes(X, codes, C, s, group), ref)
