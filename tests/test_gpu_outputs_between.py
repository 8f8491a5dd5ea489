"""Outputs between the rows of an input: X and Y, or the logits and their gradient, as parts of a buffer's rows (B200 only)."""
import pytest

from test_gpu_distill import _check, _inputs, _reference

pytestmark = pytest.mark.gpu


def _codes(torch, rows, cols, dtype=None):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    dtype = dtype or torch.bfloat16
    codes = torch.randint(0, 256, (rows, cols // 2), device="cuda", dtype=torch.uint8, generator=g)
    return codes, torch.randn(16, device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("t", ["float32", "bfloat16", "float16"])
def test_outputs_between_the_rows_of_an_input(t):
    """X and Y, or the logits and their gradient, as the two halves of a buffer's rows: the results of separate tensors."""
    import torch
    from paper_2312_07759_b200 import binding as B
    T = getattr(torch, t)
    for tokens, rows, cols in [(1, 40, 256), (7, 129, 512), (16, 96, 2048), (40, 300, 1024)]:
        codes, C = _codes(torch, rows, cols, T)
        X = torch.randn(tokens, cols, device="cuda").to(T)
        want = B.matmul_codes(X, codes, C)
        for gap in (0, 3):
            buf = torch.full((tokens, cols + gap + rows + 5), 7.0, device="cuda", dtype=T)
            buf[:, :cols] = X
            Y = B.matmul_codes(buf[:, :cols], codes, C, out=buf[:, cols + gap:cols + gap + rows])
            assert torch.equal(Y, want) and torch.equal(buf[:, :cols], X)
            Y.fill_(7.0)
            assert torch.all(buf[:, cols:] == 7.0)
    for V in (64, 1003, 40007):
        z, idx, tl, w = _inputs(torch, 9, V, 6, t)
        ref = _reference(z, idx, tl, 2.0, w)
        _, stats = B.distill_forward(z, idx, tl, 2.0)
        buf = torch.full((9, 2 * V), 7.0, device="cuda", dtype=T)
        buf[:, :V] = z
        loss, dz = B.distill_step(buf[:, :V], idx, tl, 2.0, w, out=buf[:, V:])
        _check(torch, loss, dz, ref)
        dz.fill_(7.0)
        _check(torch, None, B.distill_backward(buf[:, :V], idx, tl, 2.0, stats, w, out=buf[:, V:]), ref)
        assert torch.equal(buf[:, :V], z)
    with pytest.raises(ValueError):
        B.distill_step(buf[:, :V], idx, tl, 2.0, out=buf[:, V - 1:2 * V - 1])
