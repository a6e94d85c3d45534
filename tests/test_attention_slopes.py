"""The slopes of PagedAttention are fp32 whatever the module around them is cast to (CPU)."""
import pytest
import torch

from paper_2607_08786_amd import attention

SLOPES = torch.tensor([0.1, 1 / 3, 2.0 ** -20, 3e5])


def module():
    m = attention.PagedAttention.__new__(attention.PagedAttention)
    torch.nn.Module.__init__(m)
    m.register_buffer("slopes", SLOPES.clone())
    return m


@pytest.mark.parametrize("cast", [lambda m: m.half(), lambda m: m.bfloat16(), lambda m: m.double(), lambda m: m.to(torch.float16),
                                  lambda m: m.to("cpu", torch.bfloat16), lambda m: m.half().float()])
def test_casts_leave_slopes(cast):
    model = torch.nn.ModuleList([module(), torch.nn.Linear(2, 2)])
    model = cast(model)
    assert model[0].slopes.dtype is torch.float32 and torch.equal(model[0].slopes, SLOPES)
    assert dict(model.named_buffers())["0.slopes"] is model[0].slopes


def test_moves_and_none():
    assert module().to("meta").slopes.device.type == "meta"
    moved = module().to("meta", torch.float16)
    assert moved.slopes.device.type == "meta" and moved.slopes.dtype is torch.float32
    none = attention.PagedAttention(4, 2, 8).half()
    assert none.slopes is None
