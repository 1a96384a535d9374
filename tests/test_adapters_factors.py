"""The factors of adapters by their public names.  No GPU needed."""
import torch

from paper_2605_22428_amd import binding as B


def test_the_factors_are_the_tensors_that_the_calls_read():
    a, b, scale = torch.zeros((2, 8, 16), dtype=torch.bfloat16), torch.zeros((2, 24, 8), dtype=torch.bfloat16), torch.ones(2)
    for s in (scale, None):
        adapters = B.Adapters(a, b, s)
        assert adapters.a is a and adapters.b is b and adapters.scale is s
        assert adapters.record.a_dev == a.data_ptr() and adapters.record.b_dev == b.data_ptr()
