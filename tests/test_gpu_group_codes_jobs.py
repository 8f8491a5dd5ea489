"""The export where a block's warps have unequal work (B200 only): any number of spans, from one on, so that some warps have none."""
import numpy as np
import pytest

from oracle import group_codes as O

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("wt", ["float32", "bfloat16"])
@pytest.mark.parametrize("cols,group", [(96, 32), (700, 64), (512, 128), (1025, 256)])
def test_every_number_of_spans(wt, cols, group):
    import torch
    from paper_2312_07759_b200 import binding as B
    g = torch.Generator().manual_seed(cols)
    C = torch.randn(16, generator=g).bfloat16()
    W = torch.randn(40, cols, generator=g).to(getattr(torch, wt))
    idx, s, Wq = O.assign(W, C, group)
    packed = O.pack(idx)
    for rows in list(range(1, 19)) + [23, 40]:
        for _ in range(3):
            codes, scales, q = B.assign_groups(W[:rows].cuda(), C.cuda(), group, want_Wq=True)
            assert np.array_equal(codes.cpu().numpy(), packed[:rows]) and torch.equal(scales.cpu(), s[:rows]) and torch.equal(q.cpu(), Wq[:rows])
    # more spans than the GPU has warps for, an odd rest
    W = torch.randn(9000 + 13, cols, device="cuda").to(getattr(torch, wt))
    codes, scales, _ = B.assign_groups(W, C.cuda(), group)
    idx, s, _ = O.assign(W[-60:].cpu(), C, group)
    assert np.array_equal(codes[-60:].cpu().numpy(), O.pack(idx)) and torch.equal(scales[-60:].cpu(), s)
