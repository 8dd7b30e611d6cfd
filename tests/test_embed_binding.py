"""What the binding of the embedding refuses (CPU only)."""
import pytest
import torch

from paper_1901_08227_b200 import tng


@pytest.mark.parametrize("dtype", [torch.float64, torch.int8, torch.int64])
def test_an_output_type_that_no_kernel_writes_is_a_type_error(monkeypatch, dtype):
    monkeypatch.setattr(tng, "_device", lambda t=None: -1)  # what get_device() says of a CPU tensor
    with pytest.raises(TypeError):
        tng.embed(torch.zeros((7, 33)), torch.zeros(5, dtype=torch.int64), dtype=dtype)
