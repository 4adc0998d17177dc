"""CPU-only: the 8-bit operators refuse bad arguments before anything reaches a device (the pointers here are made up and never read)."""
import pytest
import torch

import paper_2211_05953_amd as bf

X = 1 << 20  # an aligned address that nothing may read
BIG = 1 << 21


def refused(name, *args):
    lib = bf.load()
    assert getattr(lib, name)(*args) == bf.BF_EINVAL, (name, args)
    assert bf.binding.last_error()


def swapped(ok, at, bad):
    return ok[:at] + [bad] + ok[at + 1:]


def test_sizes_of_a_form():
    assert [bf.bf_op_fp8_row_bytes(n) for n in (-1, 0, 1, 128, 129)] == [0, 0, 128, 128, 256]
    assert [bf.bf_op_fp8_scale_elems(r, n) for r, n in ((0, 5), (5, 0), (1, 1), (16, 128), (17, 129))] == [0, 0, 16, 16, 64]
    assert bf.bf_op_fp8_scale_elems(BIG, BIG) == 1 << 35
    assert [bf.bf_op_adam8_state_bytes(n) for n in (0, 1, 128, 129, 1 << 40)] == [0, 258, 258, 516, (1 << 33) * 258]


def test_quantize_refusals():
    ok = [bf.BF_BF16, bf.BF_E4M3, 10, 20, X, 0, X, X, X, X, None]
    for at, bad in ((0, 7), (0, -1), (1, 2), (1, -1), (2, 0), (2, -3), (2, BIG + 1), (3, 0), (3, BIG + 1), (4, None), (4, X + 1), (5, 19), (5, 1 << 41), (6, None),
                    (7, None), (8, None), (9, None), (6, X + 8), (7, X + 4), (8, X + 1), (9, X + 15)):
        refused("bf_op_fp8_quantize", *swapped(ok, at, bad))
    refused("bf_op_fp8_quantize", *ok[:6], None, None, None, None, None)
    refused("bf_op_fp8_quantize", *swapped([bf.BF_FP32] + ok[1:], 4, X + 2))


def test_product_refusals():
    ok = [bf.BF_E4M3, bf.BF_E5M2, bf.BF_BF16, 10, 20, 30, X, X, X, X, X, X, X, 0, None, 0, None]
    assert bf.bf_op_fp8_gemm_work_bytes(bf.BF_BF16, 10, 20, 30) == 0
    for at, bad in ((0, 2), (0, -1), (1, 2), (2, 7), (3, 0), (4, 0), (5, 0), (3, BIG + 1), (4, BIG + 1), (5, BIG + 1), (6, None), (7, None), (8, None), (9, None),
                    (10, None), (6, X + 8), (7, X + 4), (8, X + 8), (9, X + 2), (10, X + 1), (11, X + 2), (12, X + 1), (13, 1)):
        refused("bf_op_fp8_gemm", *swapped(ok, at, bad))
    # with a split contraction: the scratch
    need = bf.bf_op_fp8_gemm_work_bytes(bf.BF_FP32, 10, 20, 1 << 14)
    assert need > 0 and need % (10 * 20 * 4) == 0
    for work, size in ((None, need), (X + 16, need), (X, need - 1), (X, 0)):
        refused("bf_op_fp8_gemm", *swapped(swapped(ok, 2, bf.BF_FP32), 5, 1 << 14)[:14], work, size, None)
    assert [bf.bf_op_fp8_gemm_work_bytes(*s) for s in ((0, 0, 1, 1), (0, 1, -1, 1), (1, 1, 1, BIG + 1), (7, 10, 20, 1 << 14))] == [0, 0, 0, 0]


def test_adam_refusals():
    entry = lambda **k: (bf.bf_adam8_tensor * 1)(bf.bf_adam8_tensor(**{**dict(w=X, state=X, g=X, w_lp=X, n=10), **k}))  # noqa: E731
    ok = [bf.BF_FP32, 1, entry(), X, 5, 1, 1e-3, 0.9, 0.99, 1e-8, 0.0, None]
    for at, bad in ((0, 7), (1, -1), (2, None), (3, None), (3, X + 2), (5, 0), (2, entry(w=None)), (2, entry(state=None)), (2, entry(g=None)), (2, entry(w=X + 2)),
                    (2, entry(state=X + 8)), (2, entry(g=X + 2)), (2, entry(w_lp=X + 1))):
        refused("bf_op_adam8", *swapped(ok, at, bad))
    refused("bf_op_adam8", bf.BF_BF16, 1, entry(g=X + 1), *ok[3:])
    entry = lambda **k: (bf.bf_adam8_moments_tensor * 1)(bf.bf_adam8_moments_tensor(**{**dict(state=X, m=X, v=X, n=10), **k}))  # noqa: E731
    ok = [bf.BF_FP32, 1, entry(), None]
    for at, bad in ((0, 7), (1, -1), (2, None), (2, entry(state=None)), (2, entry(state=X + 8)), (2, entry(m=X + 2)), (2, entry(v=X + 1))):
        refused("bf_op_adam8_moments", *swapped(ok, at, bad))


@pytest.fixture
def on_cpu(monkeypatch):
    """The binding's checks see CPU tensors as the current device's; a call that gets past them is recorded and not made."""
    calls = []

    class Library:
        def __getattr__(self, name):
            real = getattr(bf.binding._lib, name)
            return real if name.endswith(("bytes", "elems")) else lambda *a: calls.append((name, a)) or 0

    bf.load()
    monkeypatch.setattr(bf.binding, "load", lambda: Library())
    monkeypatch.setattr(bf.binding, "_stream", lambda *a: 0)
    monkeypatch.setattr(torch._C, "_cuda_getDevice", lambda: -1, raising=False)
    return calls


def _form(rows, n):
    return torch.zeros(rows, bf.bf_op_fp8_row_bytes(n), dtype=torch.uint8), torch.zeros(bf.bf_op_fp8_scale_elems(rows, n), dtype=torch.uint8)


def test_binding_of_quantize(on_cpu):
    x, a, d = torch.zeros(6, 50, dtype=torch.bfloat16), _form(6, 50), _form(50, 6)
    go = lambda x, a=a, d=d, rows=6, cols=50, **k: bf.bf_op_fp8_quantize(bf.BF_BF16, 0, rows, cols, x, *a, *d, **k)  # noqa: E731
    go(x), go(x.view(-1)), go(torch.zeros(9, 50, dtype=torch.bfloat16))
    assert [c[1][5] for c in on_cpu] == [0, 0, 0]
    wide = torch.zeros(8, 70, dtype=torch.bfloat16)
    go(wide[1:7, 3:53]), go(wide[1:7, 3:53], ld_x=70), go(wide), go(wide, ld_x=70)
    assert [c[1][5] for c in on_cpu[3:]] == [70, 70, 70, 70] and on_cpu[3][1][4] == wide.data_ptr() + 2 * 73
    done = len(on_cpu)
    for bad in (x.float(), x[:5], x[:, :49], x.t(), wide[:, ::2][:6, :35], torch.zeros(6, 49, dtype=torch.bfloat16)):
        with pytest.raises(ValueError):
            go(bad)
    with pytest.raises(ValueError):
        go(wide[1:7, 3:53], ld_x=60)
    for a2, d2 in (((a[0].float(), a[1]), d), ((a[0][:5], a[1]), d), ((a[0], a[1][:-1]), d), (a, (d[0][:49], d[1])), (a, (d[0], d[1][1:-16]))):
        with pytest.raises(ValueError):
            go(x, a2, d2)
    assert len(on_cpu) == done


def test_binding_of_the_product(on_cpu):
    A, B, C = _form(6, 200), _form(9, 200), torch.zeros(6, 9)
    go = lambda A=A, B=B, C=C, dtype=bf.BF_FP32, **k: bf.bf_op_fp8_gemm(0, 0, dtype, 6, 9, 200, *A, *B, C, **k)  # noqa: E731
    go(), go(bias=torch.zeros(9), R=torch.zeros(54)), go((A[0].view(torch.float8_e4m3fn), A[1]))
    assert len(on_cpu) == 3
    for k in (dict(A=_form(5, 200)), dict(A=_form(6, 128)), dict(B=(B[0], B[1][1:])), dict(C=C[:5]), dict(C=C.bfloat16()), dict(C=C.t()), dict(bias=torch.zeros(8)),
              dict(bias=torch.zeros(9).bfloat16()), dict(R=torch.zeros(53)), dict(dtype=bf.BF_BF16)):
        with pytest.raises(ValueError):
            go(**k)
    assert len(on_cpu) == 3


def test_binding_of_adam(on_cpu):
    w, g, lp, s, c = torch.zeros(300), torch.zeros(300), torch.zeros(300, dtype=torch.bfloat16), torch.zeros(3 * 258, dtype=torch.uint8), torch.ones(1)
    go = lambda *t, coef=c, dtype=bf.BF_FP32: bf.bf_op_adam8(dtype, list(t), coef, 1, 1, 1e-3, 0.9, 0.95, 1e-8, 0.0)  # noqa: E731
    go((w, s, g, lp)), go((w, s, g, None), (w, s, g, lp)), go()
    assert [x[1][1] for x in on_cpu] == [1, 2, 0]
    for bad in ((w, s[:-1], g, lp), (w, s.float(), g, lp), (w, s, g[:299], lp), (w, s, g, lp[:299]), (w, s, g, lp.float()), (w.bfloat16(), s, g, lp), (w, s, lp, lp), (w[::2], s, g[::2], None)):
        with pytest.raises(ValueError):
            go(bad)
    with pytest.raises(ValueError):
        go((w, s, g, lp), coef=c.double())
    bf.bf_op_adam8_moments(bf.BF_FP32, [(s, w, g), (s, None, g), (s, w, None)])
    for bad in ((s[:-1], w, g), (s, w, g[:299]), (s, lp, g), (s.short(), w, None)):
        with pytest.raises(ValueError):
            bf.bf_op_adam8_moments(bf.BF_FP32, [bad])
    assert len(on_cpu) == 4


def test_binding_of_moments_of_which_neither_is_wanted(on_cpu):
    """Such an entry is passed over, as the library does with two null pointers; its state is looked at like the others'."""
    s, m, v = torch.zeros(2 * 258, dtype=torch.uint8), torch.zeros(200), torch.zeros(200)
    bf.bf_op_adam8_moments(bf.BF_FP32, [(s, None, None), (s, m, None), (s, None, None), (s, m, v)])
    bf.bf_op_adam8_moments(bf.BF_FP32, [(s, None, None)])
    assert [c[1][1] for c in on_cpu] == [4, 1]
    with pytest.raises(ValueError):
        bf.bf_op_adam8_moments(bf.BF_FP32, [(s.float(), None, None)])
    assert len(on_cpu) == 2
