"""Products with 4-bit codes of 16-bit X when a wait runs out (B200 only): copies that never arrive.
Nothing of the result may look like one.  (No GPU fault is involved: every wait ends and the kernel returns.)"""
import pytest

from test_gpu_group_codes import _case

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("t,tokens,rows,cols,group,missing", [("bfloat16", 64, 300, 512, 128, 2), ("float16", 40, 535, 11392, 32, 11), ("bfloat16", 130, 257, 4099, 64, 1),
                                                              ("bfloat16", 20, 30000, 768, 256, 3), ("float16", 200, 400, 256, 0, 1)])
def test_a_wait_that_runs_out_leaves_no_result(t, tokens, rows, cols, group, missing):
    """Blocks with the columns to themselves and shared, X copied and loaded, one tile and several, the first copy and the last."""
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    ref = B.matmul_codes(X, codes, C, s, group)
    torch.cuda.synchronize()
    try:
        B.set_codes_test_hooks(missing)
        Y = B.matmul_codes(X, codes, C, s, group)             # (some seconds)
        torch.cuda.synchronize()
        assert torch.isnan(Y).all(), (int(torch.isnan(Y).sum()), Y.numel())
        B.set_codes_test_hooks(1 << 20)                       # (a copy that there is not)
        assert torch.equal(B.matmul_codes(X, codes, C, s, group), ref)
    finally:
        B.set_codes_test_hooks(0)
    assert torch.equal(B.matmul_codes(X, codes, C, s, group), ref)


@pytest.mark.parametrize("t,tokens,rows,cols,group", [("bfloat16", 1, 5000, 1024, 128), ("float16", 7, 40, 300, 32), ("bfloat16", 3, 300, 40000, 64), ("float16", 12, 33, 256, 0)])
def test_a_wait_that_runs_out_leaves_no_result_of_a_few_rows(t, tokens, rows, cols, group):
    """X whole in shared memory and in parts."""
    import torch
    from paper_2312_07759_b200 import binding as B
    X, codes, C, s = _case(torch, tokens, rows, cols, group, t)
    ref = B.matmul_codes(X, codes, C, s, group)
    torch.cuda.synchronize()
    try:
        B.set_codes_test_hooks(1)
        Y = B.matmul_codes(X, codes, C, s, group)
        torch.cuda.synchronize()
        assert torch.isnan(Y).all(), (int(torch.isnan(Y).sum()), Y.numel())
    finally:
        B.set_codes_test_hooks(0)
    assert torch.equal(B.matmul_codes(X, codes, C, s, group), ref)


def test_refusals():
    from paper_2312_07759_b200 import binding as B
    for bad in (-1, (1 << 24) + 1):
        with pytest.raises(B.IdkmError):
            B.set_codes_test_hooks(bad)
