"""Calls on a stream that is given (B200 only)."""
import pytest

pytestmark = pytest.mark.gpu


def _codes(torch, rows, cols, dtype=None):
    g = torch.Generator(device="cuda").manual_seed(rows + cols)
    dtype = dtype or torch.bfloat16
    codes = torch.randint(0, 256, (rows, cols // 2), device="cuda", dtype=torch.uint8, generator=g)
    return codes, torch.randn(16, device="cuda", generator=g).to(dtype)


@pytest.mark.parametrize("name", ["matmul", "groups", "forward", "backward", "step"])
def test_inputs_outlive_the_caller_s_hold_on_them(name):
    """The memory of an input that the caller lets go of right after the call is not handed out while the given stream still waits."""
    import torch
    from paper_2312_07759_b200 import binding as B
    side = torch.cuda.Stream()
    codes, C = _codes(torch, 64, 4096)
    shape = (16, 4096)
    base = torch.randn(shape, device="cuda").bfloat16()
    idx = torch.randint(0, 4096, (16, 8), device="cuda")
    t = torch.randn(16, 8, device="cuda")
    stats = B.distill_forward(base, idx, t, 2.0)[1]
    calls = {"matmul": lambda x, s: B.matmul_codes(x, codes, C, stream=s), "groups": lambda x, s: B.assign_groups(x, C, 128, stream=s)[:2],
             "forward": lambda x, s: B.distill_forward(x, idx, t, 2.0, stream=s), "step": lambda x, s: B.distill_step(x, idx, t, 2.0, stream=s),
             "backward": lambda x, s: B.distill_backward(x, idx, t, 2.0, stats, stream=s)}
    tensors = lambda r: [r] if torch.is_tensor(r) else list(r)
    want = tensors(calls[name](base, None))
    for given in (side, side.cuda_stream):
        for _ in range(5):
            torch.cuda.synchronize()
            x = base.clone()
            at = x.data_ptr()
            side.wait_stream(torch.cuda.current_stream())
            with torch.cuda.stream(side):
                torch.cuda._sleep(100_000_000)      # some 50 ms: the call below is still to run when x is let go of
            got = tensors(calls[name](x, given))
            del x
            new = [torch.empty(shape, device="cuda", dtype=torch.bfloat16) for _ in range(4)]
            waits = not side.query()                # (an allocation that went to the driver, or a kernel's first launch, waits for the device)
            assert not waits or all(n.data_ptr() != at for n in new)
            if waits:
                for n in new:
                    n.fill_(float("nan"))
            torch.cuda.synchronize()
            assert all(torch.equal(a, b) for a, b in zip(got, want))
            if waits:
                break
        else:
            raise AssertionError("the stream was past the call before the memory was asked for, five times")
