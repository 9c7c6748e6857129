"""The marshalling module's looks at shapes and strides, as far as they go without a GPU: which argument is at fault, what may be left out,
calls that do not fit their own description."""
import pytest
import torch

from paper_2604_02047_b200 import binding, build


@pytest.fixture(scope="module")
def marshal():
    build.build()
    return binding.load_marshal()


def test_what_may_be_left_out(marshal):
    assert marshal.shapes("iS? fSB?", "SB", 3, 4, None, None) == -1
    assert marshal.shapes("iS? fSB", "SB", 3, 4, None, None) == 1
    assert marshal.shapes("", "") == -1


def test_the_first_at_fault_is_named(marshal):
    here = torch.zeros(3, dtype=torch.int32)                   # of the right shape, on the wrong device
    assert marshal.shapes("iS? iS", "S", 3, None, here) == 1
    assert marshal.shapes("iS iS", "S", 3, here, None) == 0
    assert marshal.shapes("iS", "S", 3, object()) == 0


def test_calls_that_do_not_fit(marshal):
    for args in [(), ("iS",), ("iS", "S"), ("iS", "S", 3), ("iS", "S", "three", None), (3, "S", 3)]:
        with pytest.raises(TypeError):
            marshal.shapes(*args)
    with pytest.raises(TypeError):
        marshal.token_stride(torch.zeros(1), 1, 1)


def test_stride_of_what_is_no_such_tensor(marshal):
    assert marshal.token_stride(torch.zeros(1, 2, 3, 4, dtype=torch.bfloat16), 1, 2, 3, 4) == -1   # not on the GPU
    assert marshal.token_stride(None, 1, 2, 3, 4) == -1
