"""CPU-only: what the binding itself works out before it calls the library."""
import ctypes as C

import pytest
import torch

import paper_2211_05953_amd as bf


# one entry, a few, both sides of a launch's table of tensors
@pytest.mark.parametrize("count", [0, 1, 2, 3, 8, 50, 219, 220, 221, 300, 441])
def test_gradient_norm_scratch_is_that_of_the_list(count):
    tensors = [torch.empty(3 + i % 5) for i in range(count)]
    sizes = (C.c_size_t * count)(*[t.numel() for t in tensors])
    want = bf.load().bf_op_grad_norm_work_bytes(count, sizes if count else None)
    assert want == max(1, -(-count // 220)) * 2048 * 8
    for _ in range(20):
        assert bf.bf_op_grad_norm_work_bytes(tensors) == want
