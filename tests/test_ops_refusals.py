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


def _attn(**k):
    return bf.make_attn_config(**{**dict(dtype=bf.BF_BF16, S_mb=2, S_seq=100, N_heads=4, N_kv_heads=2, S_head=64), **k})


BAD_ATTENTION = [dict(dtype=5), dict(kernels=9), dict(S_mb=0), dict(S_seq=0), dict(S_seq=(1 << 24) + 1), dict(N_heads=0), dict(N_kv_heads=0), dict(N_kv_heads=3),
                 dict(S_head=0), dict(S_head=1025), dict(S_mb=20000), dict(scale=-1.0), dict(scale=math.inf), dict(scale=math.nan), dict(cap=-1.0),
                 dict(cap=math.nan), dict(cap=math.inf), dict(ld_q=255), dict(ld_k=127), dict(ld_v=127), dict(ld_ctx=255), dict(ld_q=-256)]


def test_masked_attention_refusals():
    lib = bf.load()
    good = _attn()
    assert lib.bf_op_attention_masked_bwd_work_bytes(None) == 0
    need = bf.bf_op_attention_masked_bwd_work_bytes(good)
    assert need > 0
    fwd = [C.byref(good), X, X, X, X, None, X, X, None]
    bwd = [C.byref(good), X, X, X, X, None, X, X, X, X, X, X, X, need, None]
    for bad in BAD_ATTENTION:
        c = _attn(**bad)
        assert bf.bf_op_attention_masked_bwd_work_bytes(c) == 0, bad
        refused("bf_op_attention_masked_fwd", C.byref(c), *fwd[1:])
        refused("bf_op_attention_masked_bwd", C.byref(c), *bwd[1:])
    refused("bf_op_attention_masked_fwd", None, *fwd[1:])
    refused("bf_op_attention_masked_bwd", None, *bwd[1:])
    for at in (1, 2, 3, 4, 6):
        refused("bf_op_attention_masked_fwd", *fwd[:at], None, *fwd[at + 1:])
        refused("bf_op_attention_masked_fwd", *fwd[:at], X + 1, *fwd[at + 1:])
    for at in (1, 2, 3, 4, 6, 7, 8, 9, 10, 11, 12):
        refused("bf_op_attention_masked_bwd", *bwd[:at], None, *bwd[at + 1:])
    for at, bad in ((4, X + 8), (12, X + 128), (13, need - 1)):
        refused("bf_op_attention_masked_bwd", *bwd[:at], bad, *bwd[at + 1:])


def test_attention_span_refusals():
    assert bf.bf_op_attention_spans_elems(2, 100) > 400
    for sizes in ((0, 5), (5, 0), (1, (1 << 24) + 1), (-1, 5)):
        assert bf.bf_op_attention_spans_elems(*sizes) == 0
        refused("bf_op_attention_spans", *sizes, 1, None, None, X, None)
    refused("bf_op_attention_spans", 1, 100, 1, None, None, None, None)
    refused("bf_op_attention_spans", 1, 100, 1, None, None, X + 4, None)
    refused("bf_op_attention_spans", 70000, 10, 1, None, None, X, None)
