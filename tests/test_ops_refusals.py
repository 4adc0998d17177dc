"""CPU-only: the operators refuse bad arguments before anything reaches a device (the pointers here are made up and never
read)."""
import ctypes as C
import math

import pytest

import paper_2211_05953_amd as bf

X = 1 << 20  # an aligned address that nothing may read


def refused(name, *args):
    lib = bf.load()
    assert getattr(lib, name)(*args) == bf.BF_EINVAL, (name, args)
    assert bf.binding.last_error()


def _ptrs(*a):
    return (C.c_void_p * len(a))(*a)


def _sizes(*a):
    return (C.c_size_t * len(a))(*a)


def test_gradient_norm_refusals():
    lib = bf.load()
    need = lib.bf_op_grad_norm_work_bytes(1, _sizes(100))
    assert need > 0 and lib.bf_op_grad_norm_work_bytes(0, None) > 0
    assert lib.bf_op_grad_norm_work_bytes(1000, _sizes(*[5] * 1000)) > need
    ok = [bf.BF_FP32, 1, _ptrs(X), _sizes(100), 1.0, X, X, need, None]
    for at, bad in ((0, 7), (1, -1), (2, None), (3, None), (4, 0.0), (4, -1.0), (4, math.nan), (5, None), (6, None), (6, X + 4), (7, need - 1),
                    (2, _ptrs(None)), (2, _ptrs(X + 2))):
        refused("bf_op_grad_norm", *ok[:at], bad, *ok[at + 1:])


def test_gradient_scale_refusals():
    ok = [bf.BF_FP32, 1, _ptrs(X), _ptrs(X), _sizes(100), X, None]
    for at, bad in ((0, 7), (1, -1), (2, None), (3, None), (4, None), (5, None), (2, _ptrs(None)), (3, _ptrs(None)), (3, _ptrs(X + 2))):
        refused("bf_op_grad_scale", *ok[:at], bad, *ok[at + 1:])


def test_clipped_adam_refusals():
    entry = lambda **k: (bf.bf_adam_tensor * 1)(bf.bf_adam_tensor(**{**dict(w=X, m=X, v=X, g=X, w_lp=X, n=10), **k}))  # noqa: E731
    ok = [1, entry(), X, 1, 1e-3, 0.9, 0.99, 1e-8, 0.0, None]
    for at, bad in ((0, -1), (1, None), (2, None), (3, 0), (1, entry(w=None)), (1, entry(m=None)), (1, entry(v=None)), (1, entry(g=None)),
                    (1, entry(g=X + 2)), (1, entry(w_lp=X + 1))):
        refused("bf_op_adam_clipped", *ok[:at], bad, *ok[at + 1:])


@pytest.mark.parametrize("backward", [0, 1])
def test_vocabulary_loss_refusals(backward):
    name = "bf_op_vocab_loss_bwd" if backward else "bf_op_vocab_loss_fwd"
    for dtype in (bf.BF_FP32, bf.BF_BF16):
        need = bf.bf_op_vocab_loss_work_bytes(dtype, 10, 64, 1000, 0, backward)
        assert need > 0
        tail = [X, X, 0, X, need, None] if backward else [X, X, X, X, need, None]
        ok = [dtype, 10, 64, 1000, 0, X, X, X] + ([X, 1.0] if backward else [1.0]) + tail
        n = len(ok)
        bad = [(0, 7), (1, 0), (1, (1 << 21) + 1), (2, 0), (2, -8), (3, 0), (3, (1 << 21) + 1), (4, -1), (5, None), (6, None), (7, None), (n - 3, None),
               (n - 3, X + 128), (n - 2, need - 1)]
        bad += [(8, None), (9, math.inf), (9, math.nan), (10, None), (11, None)] if backward else [(8, math.nan), (9, None), (10, None), (11, None)]
        for at, b in bad:
            refused(name, *ok[:at], b, *ok[at + 1:])
    assert bf.bf_op_vocab_loss_work_bytes(bf.BF_BF16, 0, 64, 1000) == 0 and bf.bf_op_vocab_loss_work_bytes(9, 1, 64, 1000) == 0


@pytest.mark.parametrize("backward", [0, 1])
def test_vocabulary_loss_scratch_does_not_grow_with_the_vocabulary(backward):
    """Two pieces or twenty: the scratch is a piece's, not the logits'."""
    at = [bf.bf_op_vocab_loss_work_bytes(bf.BF_FP32, 2048, 1024, v, 8192, backward) for v in (50304, 150912, 2000000)]
    assert at[0] == at[1] == at[2] < 2048 * 50304 * 4
    at = [bf.bf_op_vocab_loss_work_bytes(bf.BF_BF16, 2048, 1024, v, 8192, 1) for v in (50304, 150912, 2000000)]
    assert at[0] == at[1] == at[2] < 2048 * 50304 * 4
