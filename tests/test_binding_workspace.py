"""A workspace that the kernels could not write to, or not where they think, never reaches them (no GPU: the library records its calls, and the
tensors are stand-ins that say they are on one)."""
import pytest
import torch

from paper_2509_25224_b200 import binding
from test_binding import fake  # noqa: F401  (a fixture: a library that records the calls)

GPU = torch.device("cuda", 0)


class Standin:
    """What the binding asks of a tensor."""

    def __init__(self, shape, dtype, device=GPU, contiguous=True):
        self.shape, self.dtype, self.device, self.is_cuda, self._contiguous = torch.Size(shape), dtype, device, device.type == "cuda", contiguous

    def is_contiguous(self):
        return self._contiguous

    def data_ptr(self):
        return 256

    def numel(self):
        return self.shape.numel()

    def element_size(self):
        return 1


def call(cache, workspace):
    b, i = torch.bfloat16, torch.int32
    q, table, lens = Standin((1, 1, 16, 576), b), Standin((1, 4), i), Standin((1,), i)
    out, lse = Standin((1, 1, 16, 512), b), Standin((1, 1, 16), torch.float32)
    if cache == "bf16":
        return binding.mla_decode(q, Standin((4, 64, 576), b), table, lens, 0.1, out, lse, workspace)
    if cache == "e4m3":
        return binding.mla_decode_fp8(q, Standin((4, 64, 576), torch.uint8), 1.0, table, lens, 0.1, out, lse, workspace)
    return binding.mla_decode_fp4(q, Standin((4, 20736), torch.uint8), 1.0, table, lens, 0.1, out, lse, workspace)


@pytest.mark.parametrize("cache", ["bf16", "e4m3", "fp4"])
def test_workspaces(fake, cache):  # noqa: F811
    call(cache, Standin((1 << 20,), torch.uint8))
    assert len(fake.calls) == 1
    for bad in (Standin((1 << 20,), torch.uint8, torch.device("cpu")), Standin((1 << 20,), torch.uint8, torch.device("cuda", 1)), Standin((1 << 20,), torch.uint8, contiguous=False)):
        with pytest.raises(ValueError):
            call(cache, bad)
    assert len(fake.calls) == 1
