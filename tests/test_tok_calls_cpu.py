"""The extension module behind the Python calls of the operators over tokens refuses, with -1 and no exception, what it cannot look
at: binding.py then asks the same in Python.  (No GPU: no call reaches the library.)"""
import pytest
import torch

from paper_2303_02191_b200 import _build, binding


@pytest.fixture(scope="module")
def calls():
    _build.build()
    binding._types()
    assert binding._calls is not None
    return binding._calls


NAMES = {"quantize_rows": 5, "matmul_i8": 11, "gated_ffn_forward": 11, "gated_ffn_backward": 17, "block_norm_forward": 14, "block_norm_backward": 20}


@pytest.mark.parametrize("name", NAMES)
def test_operands_that_are_no_cuda_tensors(calls, name):
    f, n = getattr(calls, name), NAMES[name]
    m = torch.ones(4, 4)
    for operand in (None, 3, "x", m, m.to(torch.bfloat16), m.to_sparse(), torch.ones(4, 4, device="meta"), torch.nn.Parameter(m), torch.ones(0, 4), torch.ones(()), object()):
        assert f(0, 0, *[operand] * (n - 2)) == -1
        assert f(None, "device", *[operand] * (n - 2)) == -1
    assert f() == -1 and f(*[0] * (n - 1)) == -1 and f(*[0] * (n + 1)) == -1


def test_entries_takes_six_addresses(calls):
    with pytest.raises(TypeError):
        calls.entries(1)
    with pytest.raises(ValueError):
        calls.entries(0, 0, 0, 0, 0, 0)
