"""What bload_scan_buffers makes, on the host; and that the example's backward pass makes no second set of kept states."""
import importlib.util
import os

import pytest
import torch

import paper_2310_10879_b200 as B

HERE = os.path.dirname(os.path.abspath(__file__))


def test_states_and_scratch_are_made_as_asked():
    pos = torch.zeros((2, 5000), dtype=torch.int32)
    x, a = torch.zeros((2, 5000, 64), dtype=torch.bfloat16), torch.zeros((64, 16))
    need = [B.load().bload_scan_work_bytes(2, 5000, 64, 16, g) for g in (0, 1)]
    assert 0 < need[0] < need[1]
    for args, kept, size in (({}, True, need[1]), ({"gradient": False}, False, need[0]), ({"gradient": False, "carry": True}, True, need[0]),
                             ({"carry": False}, False, need[1]), ({"carry": True}, True, need[1])):
        carry, work = B.bload_scan_buffers(pos, x, a, **args)
        assert (carry is not None) == kept and work.numel() == size and work.dtype == torch.uint8, args
        assert not kept or (carry.shape == (2, 313, 64, 16) and carry.dtype == torch.float32)


@pytest.mark.gpu
def test_the_example_keeps_one_set_of_states():
    spec = importlib.util.spec_from_file_location("packed_state_space", os.path.join(os.path.dirname(HERE), "examples", "packed_state_space.py"))
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    b, t, c, n = 1, 512, 2048, 64
    dev = "cuda:0"
    pos = torch.arange(t, dtype=torch.int32, device=dev)[None]
    x, dt, z = (torch.randn((b, t, c), device=dev).bfloat16().requires_grad_() for _ in range(3))
    rows = [torch.randn((b, t, n), device=dev).bfloat16().requires_grad_() for _ in range(2)]
    a = (-torch.rand((c, n), device=dev)).requires_grad_()
    d, bias = (torch.randn(c, device=dev).requires_grad_() for _ in range(2))
    kept, size = b * t // 16 * c * n * 4, B.load().bload_scan_work_bytes
    inputs = (x, dt, z, *rows, a, d, bias)
    grads = sum(v.numel() * v.element_size() for v in inputs)
    room = kept // 2  # (an allocation may be served by a cached block that is up to a megabyte larger)
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    y = example.Scan.apply(*inputs, pos)
    assert torch.cuda.max_memory_allocated() - before < kept + size(b, t, c, n, 0) + x.numel() * 2 + room
    dy = torch.randn_like(y)
    before = torch.cuda.memory_allocated()
    torch.cuda.reset_peak_memory_stats()
    got = torch.autograd.grad(y, inputs, dy)
    assert torch.cuda.max_memory_allocated() - before < size(b, t, c, n, 1) + grads + room
    assert all(bool(torch.isfinite(v).all()) for v in got)
