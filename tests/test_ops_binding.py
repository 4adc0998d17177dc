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


# attention's rows: (S_mb, S_seq, heads, S_head)
@pytest.mark.parametrize("sizes", [(2, 50, 4, 16), (1, 50, 4, 16), (2, 1, 4, 16), (3, 7, 1, 16), (2, 5, 3, 1), (1, 1, 1, 1)])
def test_attention_rows_that_the_kernels_read_as_they_are(sizes):
    B, S, H, d = sizes
    fits = lambda t, ld=0: bf.binding._token_rows(t, B, S, H, d, ld)  # noqa: E731
    n = H * d
    x = torch.zeros(B, S, n)
    assert fits(x) and fits(x, n) and fits(x.view(B * S, n)) and fits(x.view(B, S, H, d)) and fits(x.view(B * S, H, d)) and fits(x.view(-1))
    assert fits(torch.zeros(B + 1, S, n)) and fits(torch.zeros(B * S + 3, n)) and fits(torch.zeros(B * S * n + 7))
    if H % 2 == 0:  # query heads by key / value head
        assert fits(x.view(B, S, 2, H // 2, d)) and fits(x.view(B * S, H // 2, 2, d))
    wide = torch.zeros(B, S, 3 * n + 5)
    for at in (0, n, 2 * n):
        q = wide[..., at:at + n]
        assert fits(q, 3 * n + 5) and fits(q.unflatten(2, (H, d)), 3 * n + 5) and fits(wide.view(B * S, -1)[:, at:at + n], 3 * n + 5)
    assert fits(wide, 3 * n + 5) and fits(torch.zeros(B * S, 3 * n + 5), 3 * n + 5)


def test_attention_rows_that_the_kernels_would_misread():
    B, S, H, d = 2, 50, 4, 16
    n = H * d
    fits = lambda t, ld=0: bf.binding._token_rows(t, B, S, H, d, ld)  # noqa: E731
    q = torch.zeros(B, S, 3 * n).split(n, 2)[1]
    assert fits(q, 3 * n)
    # another step between the tokens than the configuration's, with all that the kernels would reach inside the storage
    for ld in (0, n, 2 * n, 3 * n - 1, 3 * n + 1):
        assert not fits(q, ld) and not fits(q.unflatten(2, (H, d)), ld) and not fits(torch.zeros(B * S, 3 * n)[:, :n], ld)
    x = torch.zeros(B, S, n)
    assert not fits(x, 2 * n)
    # tokens in front of sequences, in their order and as a view
    assert not fits(torch.zeros(S, B, n)) and not fits(torch.zeros(S, B, n).transpose(0, 1)) and not fits(torch.zeros(S, B, H, d))
    # heads in front of tokens, whole or as a view; rows that are not dense; a step of 0; too few tokens, heads or sequences
    assert not fits(torch.zeros(B, H, S, d)) and not fits(torch.zeros(B, H, S, d).transpose(1, 2)) and not fits(torch.zeros(B, S, d, H).transpose(2, 3))
    assert not fits(torch.zeros(B, 2, S, H // 2, d)) and not fits(torch.zeros(B, S, H // 2, 2, d).transpose(2, 3)) and not fits(torch.zeros(B, S, d, H))
    assert not fits(x.transpose(0, 1)) and not fits(torch.zeros(B, n, S).transpose(1, 2)) and not fits(torch.zeros(B, S, 2 * n)[..., ::2])
    assert not fits(torch.zeros(1, S, n).expand(B, S, n)) and not fits(torch.zeros(B, 1, n).expand(B, S, n))
    assert not fits(torch.zeros(B, S, 2 * H, d)[:, :, ::2]) and not fits(torch.zeros(B, S, H, 2 * d)[..., :d])
    assert not fits(torch.zeros(B, S - 1, n)) and not fits(torch.zeros(1, S, n)) and not fits(torch.zeros(B, S, n - 1))
    assert not fits(torch.zeros(B, S + 1, n)) and not fits(torch.zeros(B * S * n - 1)) and not fits(torch.zeros(B, S * n))
    assert not fits(torch.zeros(B, S, H + 1, d)) and not fits(torch.zeros(B, S, H, d + 1)) and not fits(torch.zeros(()))


@pytest.mark.parametrize("rows,h", [(2048, 8192), (2048, 1024), (2000, 1000), (33, 256), (8192, 64), (1, 8)])
def test_forward_scratch_of_the_vocabulary_loss_is_a_piece_s(rows, h):
    """bf16: asking for pieces costs no more scratch than the library's choice, less the smaller they are, and the same for any vocabulary."""
    need = lambda V, piece: bf.bf_op_vocab_loss_work_bytes(bf.BF_BF16, rows, h, V, piece, 0)  # noqa: E731
    for V in (50304, 50257, 150912):
        at = [need(V, piece) for piece in (256, 1024, 8192)] + [need(V, 0)]
        assert at == sorted(at)
    for piece in (8, 1000, 8192):
        at = [need(V, piece) for V in (50304, 50257, 150912, 2000000)]
        assert at[0] == at[1] == at[2] == at[3]
        # y and a piece of w lengthened to whole chunks, 8 bytes a row and 64 columns, and two of each row's numbers
        h8, cols = -(-h // 8) * 8, -(-piece // 8) * 8
        assert at[0] <= 2 * h8 * (rows + cols) + 8 * rows * (-(-cols // 64) + 2) + 5 * 256


X = 1 << 20  # an aligned address that nothing may read


def refused(name, *args):
    lib = bf.load()
    assert getattr(lib, name)(*args) == bf.BF_EINVAL, (name, args)
    assert bf.binding.last_error()


def test_pointers_that_are_not_aligned_to_their_elements_are_refused():
    lib = bf.load()
    one = (C.c_void_p * 1)(X), (C.c_size_t * 1)(100)
    need = lib.bf_op_grad_norm_work_bytes(1, one[1])
    refused("bf_op_grad_norm", bf.BF_FP32, 1, one[0], one[1], 1.0, X + 2, X, need, None)
    refused("bf_op_grad_scale", bf.BF_FP32, 1, one[0], one[0], one[1], X + 1, None)
    entry = (bf.bf_adam_tensor * 1)(bf.bf_adam_tensor(w=X, m=X, v=X, g=X, w_lp=X, n=10))
    refused("bf_op_adam_clipped", 1, entry, X + 2, 1, 1e-3, 0.9, 0.99, 1e-8, 0.0, None)
    for dtype, half in ((bf.BF_FP32, 2), (bf.BF_BF16, 1)):  # an address between two elements
        need = [bf.bf_op_vocab_loss_work_bytes(dtype, 10, 64, 1000, 0, k) for k in (0, 1)]
        fwd = [dtype, 10, 64, 1000, 0, X, X, X, 1.0, X, X, X, X, need[0], None]
        bwd = [dtype, 10, 64, 1000, 0, X, X, X, X, 1.0, X, X, 0, X, need[1], None]
        for at, off in ((5, half), (6, half), (7, 2), (9, 2), (10, 2), (11, 2)):
            refused("bf_op_vocab_loss_fwd", *fwd[:at], X + off, *fwd[at + 1:])
        for at, off in ((5, half), (6, half), (7, 2), (8, 2), (10, half), (11, 2)):
            refused("bf_op_vocab_loss_bwd", *bwd[:at], X + off, *bwd[at + 1:])
        cfg = bf.make_attn_config(dtype, 2, 100, 4, 2, 64)
        fwd = [C.byref(cfg), X, X, X, X, X, X, X, None]
        bwd = [C.byref(cfg), X, X, X, X, X, X, X, X, X, X, X, X, bf.bf_op_attention_masked_bwd_work_bytes(cfg), None]
        for at, off in ((1, half), (2, half), (3, half), (5, 2), (6, half), (7, 2)):
            refused("bf_op_attention_masked_fwd", *fwd[:at], X + off, *fwd[at + 1:])
        for at, off in ((5, 2), (6, half), (7, 2), (8, half), (11, half)):
            refused("bf_op_attention_masked_bwd", *bwd[:at], X + off, *bwd[at + 1:])
    refused("bf_op_attention_spans", 2, 100, 1, X + 2, None, X, None)
    refused("bf_op_attention_spans", 2, 100, 1, None, X + 1, X, None)


@pytest.mark.parametrize("dtype", [bf.BF_FP32, bf.BF_BF16])
def test_attention_that_no_launch_holds_is_refused(dtype):
    """2^32 threads along a grid: 256 to 128 queries of a head forward, 512 to 128 keys backward."""
    make = lambda seq, heads, kernels=bf.BF_KERNELS_AUTO: bf.make_attn_config(dtype, 1, seq, heads, 1, 8, kernels=kernels)  # noqa: E731
    tail = lambda n: (X,) * n  # noqa: E731
    for seq, heads in ((1 << 24, 128), ((1 << 24) - 127, 128), (1 << 20, 2048), ((1 << 15) + 1, 65535)):
        refused("bf_op_attention_masked_fwd", C.byref(make(seq, heads)), *tail(4), None, X, X, None)
    for seq, heads in ((1 << 24, 64), ((1 << 24) - 127, 64), (1 << 20, 1024), ((1 << 14) + 1, 65535)):
        cfg = make(seq, heads)
        assert bf.bf_op_attention_masked_bwd_work_bytes(cfg) == 0
        refused("bf_op_attention_masked_bwd", C.byref(cfg), *tail(4), None, *tail(7), 1 << 62, None)
        assert bf.bf_op_attention_masked_bwd_work_bytes(make(seq, heads, bf.BF_KERNELS_PLAIN)) > 0
    assert bf.bf_op_attention_masked_bwd_work_bytes(make((1 << 24) - 128, 64)) > 0


@pytest.mark.parametrize("dtype", [bf.BF_FP32, bf.BF_BF16])
def test_attention_scales_that_are_infinite_as_exponents_are_refused(dtype):
    for scale, good in ((2.0**126, True), (2.0**126 * 1.0001, False), (3e38, False), (1e-45, True)):
        cfg = bf.make_attn_config(dtype, 2, 100, 4, 2, 64, scale=scale)
        assert (bf.bf_op_attention_masked_bwd_work_bytes(cfg) > 0) == good
        if not good:
            refused("bf_op_attention_masked_fwd", C.byref(cfg), X, X, X, X, None, X, X, None)
