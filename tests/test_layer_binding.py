"""What the binding of the training-layer operators accepts and passes on (CPU only: the library is a stand-in that records its calls)."""
import subprocess
import sys
from pathlib import Path

import pytest
import torch

from paper_1901_08227_b200 import tng

ROOT = Path(__file__).resolve().parent.parent


class Recorder:
    """Stands in for the loaded library: every call is recorded and succeeds."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        def call(*args):
            self.calls.append((name, args))
            return 256 if name.endswith("_bytes") else tng.OK
        return call


@pytest.fixture
def library(monkeypatch):
    r = Recorder()
    monkeypatch.setattr(tng, "lib", lambda: r)
    monkeypatch.setattr(tng, "_device", lambda: -1)             # what get_device() says of a CPU tensor
    monkeypatch.setattr(tng, "_stream", lambda: 0)
    monkeypatch.setattr(tng, "_scratch", lambda *a: (None, None))
    return r


def stride_of(library, name):
    (args,) = [a for n, a in library.calls if n == name]
    return args[7]                                              # x, type, rows, cols, ldx, draw, q, ldq, ...


@pytest.mark.parametrize("n", [1, 20, 1001])
@pytest.mark.parametrize("make,shape", [(tng.quant8_rows, lambda n: (1, n)), (tng.quant8_cols, lambda n: (n, 1))])
def test_one_line_of_codes_inside_a_larger_buffer_is_refused(library, make, shape, n):
    # its padding up to the next multiple of 16 would be written over what follows it
    pool = torch.zeros(2048, dtype=torch.int8)
    with pytest.raises(ValueError):
        make(torch.zeros(shape(n)), q=pool[:n].view(1, n))
    assert not library.calls or all(c[0].endswith("_bytes") for c in library.calls)


@pytest.mark.parametrize("make,shape", [(tng.quant8_rows, (2, 20)), (tng.quant8_cols, (20, 2))])
def test_codes_whose_last_line_ends_with_the_buffer_are_refused(library, make, shape):
    q = torch.zeros(32 + 20, dtype=torch.int8).as_strided((2, 20), (32, 1))
    with pytest.raises(ValueError):
        make(torch.zeros(shape), q=q)
    q = torch.zeros(16 + 32 + 20, dtype=torch.int8).as_strided((2, 20), (32, 1), 16)
    with pytest.raises(ValueError):
        make(torch.zeros(shape), q=q)


@pytest.mark.parametrize("make,name,x", [(tng.quant8_rows, "tng_quant8_rows", (3, 20)), (tng.quant8_cols, "tng_quant8_cols", (20, 3))])
def test_codes_that_own_their_padding_are_accepted(library, make, name, x):
    for lines in (1, 3):
        shape = tuple(lines if n == 3 else n for n in x)
        for q, ld in [(tng.empty_codes(lines, 20, "cpu"), 32), (torch.zeros((lines, 64), dtype=torch.int8)[:, :20], 64),
                      (torch.zeros(lines * 48 + 16, dtype=torch.int8).as_strided((lines, 20), (48, 1), 16), 48), (None, 32)]:
            library.calls.clear()
            make(torch.zeros(shape), q=q)
            assert stride_of(library, name) == ld
    library.calls.clear()
    make(torch.zeros(tuple(1 if n == 3 else 32 for n in x)), q=torch.zeros((1, 32), dtype=torch.int8))      # no padding at all
    assert stride_of(library, name) == 32


def test_codes_of_nothing_are_accepted(library):
    tng.quant8_rows(torch.zeros((0, 20)), q=torch.zeros((0, 20), dtype=torch.int8))
    tng.quant8_cols(torch.zeros((0, 20)), q=torch.zeros((20, 0), dtype=torch.int8))


def test_the_package_imports_where_torch_has_no_cuda():
    """A build of torch without CUDA lacks the names that find the current device and stream."""
    code = ("import torch\n"
            "for n in ('_cuda_getDevice', '_cuda_getCurrentRawStream'):\n"
            "    delattr(torch._C, n)\n"
            "import paper_1901_08227_b200\n"
            "from paper_1901_08227_b200 import distributed, tng, workloads\n"
            "assert tng.empty_codes(2, 20, 'cpu').shape == (2, 20)\n")
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True)
    assert r.returncode == 0, r.stderr


def test_the_current_stream_is_asked_for_as_torch_does(monkeypatch):
    """CUDA is brought up first (and a forked process told that it cannot be), and torch's own call serves where the short cut is missing."""
    monkeypatch.delattr(torch._C, "_cuda_getCurrentRawStream", raising=False)
    asked = []

    class Stream:
        cuda_stream = 77

    monkeypatch.setattr(torch.cuda, "current_device", lambda: asked.append("device") or 3)
    monkeypatch.setattr(torch.cuda, "current_stream", lambda device=None: asked.append(device) or Stream)
    assert tng._stream() == 77 and asked == ["device", 3]
    assert tng._device() == 3


@pytest.mark.parametrize("default", [torch.float64, torch.bfloat16])
def test_scales_are_single_precision_whatever_the_default_type(library, default):
    before = torch.get_default_dtype()
    torch.set_default_dtype(default)
    try:
        x = torch.zeros((3, 20), dtype=torch.float32)
        assert tng.quant8_rows(x)[1].dtype == tng.quant8_cols(x)[1].dtype == torch.float32
    finally:
        torch.set_default_dtype(before)
