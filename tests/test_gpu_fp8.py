"""8-bit forms and their products against the definitions in fp64.

Forms are exact: scaling is by a power of two, the one rounding is to nearest even, so codes and scales have to be equal.
Products: an fp32 result adds K / 32 partial sums one after the other, each a sum of 32 exact products, all in fp32: off by at most (K / 32 + 32)
2^-24 of the sum of the products' magnitudes, and 2 2^-24 of the terms that the epilogue adds.  A bf16 result comes from the 8-bit instructions, which
keep products of a group of neighbouring k that lie 2^13 and more under the group's largest to fewer bits: off by at most 2^-12 of
that sum (2^-13.3 was the most seen on codes of the whole range), and half a step of bf16, 2^-8, of the result."""
import pytest
import torch

import fp8_plain as P
import paper_2211_05953_amd as bf

pytestmark = pytest.mark.gpu

DT = {bf.BF_BF16: torch.bfloat16, bf.BF_FP32: torch.float32}


def _new(rows, n, fill=0xA5):
    """Buffers of a form, with guards behind that no call may touch."""
    a, b = bf.bf_op_fp8_row_bytes(n) * rows, bf.bf_op_fp8_scale_elems(rows, n)
    return torch.full((a + 64,), fill, dtype=torch.uint8, device="cuda"), torch.full((b + 64,), fill, dtype=torch.uint8, device="cuda")


def _views(buf, rows, n):
    blocks = -(-n // 128)
    return buf[0][: rows * blocks * 128].view(rows, blocks * 128), buf[1][: blocks * (-(-rows // 16) * 16)].view(blocks, -(-rows // 16) * 16)


def _guarded(buf, rows, n):
    a, b = bf.bf_op_fp8_row_bytes(n) * rows, bf.bf_op_fp8_scale_elems(rows, n)
    return bool((buf[0][a:] == 0xA5).all()) and bool((buf[1][b:] == 0xA5).all())


def _same_form(buf, x, fmt):
    rows, n = x.shape
    q, scale = P.form(x, fmt)
    got, sgot = _views(buf, rows, n)
    assert torch.equal(sgot, scale)
    nan = torch.isnan(q)
    have = got.view(P.TYPES[fmt]).double()
    assert torch.equal(torch.isnan(have), nan)
    assert torch.equal(have[~nan], q[~nan])
    assert bool((got[:, n:] == 0).all())
    assert _guarded(buf, rows, n)


def _matrix(rows, cols, dtype, seed, spread=4.0):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows, cols, generator=g, device="cuda") * torch.exp2(torch.randn(rows, cols, generator=g, device="cuda") * spread)
    return x.to(DT[dtype])


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("fmt", [bf.BF_E4M3, bf.BF_E5M2])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 128), (128, 1), (15, 17), (16, 129), (127, 127), (128, 128), (129, 131), (250, 1003), (300, 640), (1, 5000), (777, 33)])
def test_forms(rows, cols, dtype, fmt):
    x = _matrix(rows, cols, dtype, rows * 10007 + cols)
    for along, down in ((True, True), (True, False), (False, True)):
        a, d = _new(rows, cols), _new(cols, rows)
        bf.bf_op_fp8_quantize(dtype, fmt, rows, cols, x, *(a if along else (None, None)), *(d if down else (None, None)))
        if along:
            _same_form(a, x, fmt)
        if down:
            _same_form(d, x.t(), fmt)


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("fmt", [bf.BF_E4M3, bf.BF_E5M2])
def test_forms_of_values_at_the_borders(dtype, fmt):
    """Blocks of zeros, of the type's smallest and largest values, maxima on either side of a power of two's top, ties, infinities and NaN."""
    top = P.TOP[fmt][0]
    big, tiny = torch.finfo(DT[dtype]).max, torch.finfo(DT[dtype]).smallest_normal
    x = torch.zeros(40, 300)
    x[1, 5], x[2, :], x[3, 7] = big, -big, tiny
    x[4, :] = tiny / 128
    x[5, 0], x[6, 0], x[7, 0] = top, top * 1.01, top / 1.01
    x[5:8, 1:] = torch.arange(299.0) * 1.5 - 200
    x[8, :] = torch.linspace(1, 2, 300)  # ties and their neighbours
    x[9, 3], x[9, 200], x[10, 4], x[10, 5:9] = float("inf"), -3.0, float("nan"), 2.5
    x[11, :] = float("nan")
    x[12, 0], x[12, 1:] = -float("inf"), 1e-3
    x[13, 0], x[13, 1:] = 2.0**120, 1.0
    x[14, :] = 2.0**-126
    x[15, 0], x[15, 1:100] = 1.0, torch.exp2(-torch.arange(1.0, 100.0) / 4)
    x = x.to(DT[dtype]).cuda()
    a, d = _new(40, 300), _new(300, 40)
    bf.bf_op_fp8_quantize(dtype, fmt, 40, 300, x, *a, *d)
    _same_form(a, x, fmt)
    _same_form(d, x.t(), fmt)


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
def test_forms_of_views(dtype):
    """Rows of a longer row, at addresses that are aligned to an element only, with something else around them."""
    wide = _matrix(70, 400, dtype, 3)
    for at, cols in ((1, 150), (3, 256), (133, 267)):
        x = wide[3:63, at:at + cols]
        a, d = _new(60, cols), _new(cols, 60)
        bf.bf_op_fp8_quantize(dtype, bf.BF_E4M3, 60, cols, x, *a, *d)
        _same_form(a, x, 0)
        _same_form(d, x.t(), 0)
        a2 = _new(60, cols)
        bf.bf_op_fp8_quantize(dtype, bf.BF_E4M3, 60, cols, wide.view(-1)[3 * 400 + at:], *a2, ld_x=400)
        assert torch.equal(a[0], a2[0]) and torch.equal(a[1], a2[1])


def _operand(rows, n, fmt, seed, outliers=False):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows, n, generator=g, device="cuda") * torch.exp2(4 * torch.randn(rows, 1, generator=g, device="cuda"))
    if outliers:
        x = x * (1 + 30 * (torch.rand(rows, n, generator=g, device="cuda") < 0.02))
    q, scale = P.form(x, fmt)
    return (P.codes(q, fmt).contiguous(), scale), P.values(q, scale, n)


def _close(got, ref, mag, K, dtype, extra=0.0):
    if dtype == bf.BF_BF16:
        tol = 2.0**-8 * ref.abs() + (2.0**-12 + K / 128 * 2.0**-23) * mag + 2.0**-22 * extra
    else:
        tol = ((K / 32 + 32) * 2.0**-24) * mag + 2.0**-22 * extra + 2.0**-24 * ref.abs()
    worst = ((got.double() - ref).abs() - tol).max()
    assert bool(torch.isfinite(got).all()) and float(worst) <= 0, float(((got.double() - ref).abs() / (tol + 1e-300)).max())


SHAPES = [(1, 1, 1), (1, 5, 128), (3, 64, 129), (17, 33, 64), (64, 64, 300), (65, 130, 257), (128, 128, 1000), (100, 1003, 250), (1, 1000, 4096), (5, 300, 8200),
          (300, 500, 640), (2000, 1030, 384), (257, 4000, 512), (2304, 2308, 256), (3000, 6148, 260),
          (2300, 4100, 2100), (2305, 4099, 2176), (4096, 4096, 4000)]


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("M,N,K", SHAPES)
def test_products(M, N, K, dtype):
    (A, sa), a = _operand(M, K, 0, M + K)
    (B, sb), b = _operand(N, K, 0, N + K + 1)
    ref, mag = a @ b.t(), a.abs() @ b.abs().t()
    flat = torch.full((M * N + 64,), float("nan"), dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, flat[: M * N])
    _close(flat[: M * N].view(M, N), ref, mag, K, dtype)
    assert bool(torch.isnan(flat[M * N:]).all())
    first = flat.clone()
    bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, flat[: M * N])
    assert torch.equal(first[: M * N], flat[: M * N])  # the same bits again


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("fa,fb", [(0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("M,N,K", [(33, 70, 200), (100, 500, 4200), (520, 800, 300), (2100, 2200, 200), (2300, 4100, 2100)])
def test_products_of_formats(M, N, K, fa, fb, dtype):
    (A, sa), a = _operand(M, K, fa, 5, True)
    (B, sb), b = _operand(N, K, fb, 6, True)
    out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(fa, fb, dtype, M, N, K, A, sa, B, sb, out)
    _close(out, a @ b.t(), a.abs() @ b.abs().t(), K, dtype)


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("M,N,K,at", [(33, 70, 200, 0), (40, 64, 4200, 1), (40, 67, 4200, 0), (520, 800, 300, 0), (520, 801, 300, 0), (2100, 2200, 200, 1), (8190, 2044, 300, 0), (8190, 2043, 130, 0), (2300, 4100, 2050, 0), (2300, 4100, 2050, 1)])
def test_epilogues(M, N, K, at, dtype):
    """Bias, residual, both, the residual in place, accumulation; results that start at any element."""
    (A, sa), a = _operand(M, K, 0, 7)
    (B, sb), b = _operand(N, K, 0, 8)
    prod, mag = a @ b.t(), a.abs() @ b.abs().t()
    g = torch.Generator("cuda").manual_seed(1)
    size = float(prod.std())
    bias = (torch.randn(N + 1, generator=g, device="cuda") * size)[at: at + N]
    res = (torch.randn(M * N + 1, generator=g, device="cuda") * size).to(DT[dtype])[at: at + M * N]
    flat = torch.empty(M * N + 1, dtype=DT[dtype], device="cuda")
    out = flat[at: at + M * N]
    r64, b64 = res.double().view(M, N), bias.double()
    run = lambda **k: bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, out, **k)  # noqa: E731
    run(bias=bias)
    _close(out.view(M, N), prod + b64, mag, K, dtype, b64.abs() + prod.abs())
    run(R=res)
    _close(out.view(M, N), prod + r64, mag, K, dtype, r64.abs() + prod.abs())
    run(bias=bias, R=res)
    _close(out.view(M, N), prod + r64 + b64, mag, K, dtype, r64.abs() + b64.abs() + prod.abs())
    keep = out.clone()
    out.copy_(res)
    run(bias=bias, R=out)
    assert torch.equal(out, keep)
    if dtype == bf.BF_FP32:
        out.copy_(res)
        run(accumulate=1)
        _close(out.view(M, N), prod + r64, mag, K, dtype, r64.abs() + prod.abs())


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
def test_nan_codes_stay_in_their_row_and_column(dtype):
    M, N, K = 70, 90, 300
    (A, sa), a = _operand(M, K, 0, 9)
    (B, sb), b = _operand(N, K, 0, 10)
    A[3, 130], B[77, 5] = 0x7F, 0x7F
    out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, out)
    bad = torch.zeros(M, N, dtype=torch.bool, device="cuda")
    bad[3], bad[:, 77] = True, True
    assert torch.equal(torch.isnan(out), bad)
    a[3], b[77] = 0, 0
    out[bad] = 0
    _close(out, a @ b.t(), a.abs() @ b.abs().t(), K, dtype)


def _layer(T, h_in, h_out, dtype, fmt, dw_dtype):
    """A linear layer's forward and backward pass in 8 bits: (y, dx, dw), and the same from the definitions."""
    g = torch.Generator("cuda").manual_seed(T + h_in + h_out)
    x = torch.randn(T, h_in, generator=g, device="cuda").to(DT[dtype])
    w = (torch.randn(h_in, h_out, generator=g, device="cuda") * h_in**-0.5).to(DT[dtype])
    dy = (torch.randn(T, h_out, generator=g, device="cuda") * 1e-4).to(DT[dtype])
    forms = lambda t, f: _forms(t, dtype, f)  # noqa: E731
    (xa, xd), (wa, wd), (da, dd) = forms(x, 0), forms(w, 0), forms(dy, fmt)
    y, dx = torch.empty(T, h_out, dtype=DT[dtype], device="cuda"), torch.empty(T, h_in, dtype=DT[dtype], device="cuda")
    dw = torch.empty(h_in, h_out, dtype=DT[dw_dtype], device="cuda")
    bf.bf_op_fp8_gemm(0, 0, dtype, T, h_out, h_in, *xa, *wd, y)
    bf.bf_op_fp8_gemm(fmt, 0, dtype, T, h_in, h_out, *da, *wa, dx)
    bf.bf_op_fp8_gemm(0, fmt, dw_dtype, h_in, h_out, T, *xd, *dd, dw)
    return (x, w, dy), (y, dx, dw)


def _forms(t, dtype, fmt):
    rows, cols = t.shape
    a, d = _new(rows, cols), _new(cols, rows)
    bf.bf_op_fp8_quantize(dtype, fmt, rows, cols, t, *a, *d)
    return a, d


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("T,h_in,h_out", [(60, 256, 1024), (33, 250, 1003), (1, 130, 70)])
def test_a_layer_forward_and_backward(T, h_in, h_out, dtype, fmt):
    (x, w, dy), (y, dx, dw) = _layer(T, h_in, h_out, dtype, fmt, bf.BF_FP32)
    v = lambda t, f: P.values(*P.form(t, f), t.shape[1])  # noqa: E731
    for got, a, b, K, dt in ((y, v(x, 0), v(w.t(), 0), h_in, dtype), (dx, v(dy, fmt), v(w, 0), h_out, dtype), (dw, v(x.t(), 0), v(dy.t(), fmt), T, bf.BF_FP32)):
        _close(got, a @ b.t(), a.abs() @ b.abs().t(), K, dt)
    # and it is the layer's gradient: the unrounded operands' products, but for the codes' own half steps (2^-4 for e4m3, 2^-3 for e5m2, uniform
    # errors of 3^-0.5 of that at most, in both operands; held to the sum of both full half steps in 2-norm)
    for got, ref in ((y, x.double() @ w.double()), (dx, dy.double() @ w.double().t()), (dw, x.double().t() @ dy.double())):
        assert float((got.double() - ref).norm() / ref.norm()) <= 2.0**-4 + 2.0 ** -(4 - fmt)


def test_a_layer_under_capture():
    """A graph of the layer's calls, replayed with other inputs and eager work between, gives what eager calls give."""
    T, h_in, h_out = 100, 384, 520
    (x, w, dy), _ = _layer(T, h_in, h_out, bf.BF_BF16, 0, bf.BF_FP32)
    bufs = [_new(T, h_in), _new(h_in, T), _new(h_in, h_out), _new(h_out, h_in), _new(T, h_out), _new(h_out, T)]
    y, dx, dw = torch.empty(T, h_out, dtype=torch.bfloat16, device="cuda"), torch.empty(T, h_in, dtype=torch.bfloat16, device="cuda"), torch.empty(h_in, h_out, device="cuda")
    work = [torch.empty(max(256, bf.bf_op_fp8_gemm_work_bytes(*s)), dtype=torch.uint8, device="cuda") for s in ((1, T, h_out, h_in), (1, T, h_in, h_out), (0, h_in, h_out, T))]

    def step():
        bf.bf_op_fp8_quantize(1, 0, T, h_in, x, *bufs[0], *bufs[1])
        bf.bf_op_fp8_quantize(1, 0, h_in, h_out, w, *bufs[2], *bufs[3])
        bf.bf_op_fp8_quantize(1, 0, T, h_out, dy, *bufs[4], *bufs[5])
        bf.bf_op_fp8_gemm(0, 0, 1, T, h_out, h_in, *bufs[0], *bufs[3], y, work=work[0])
        bf.bf_op_fp8_gemm(0, 0, 1, T, h_in, h_out, *bufs[4], *bufs[2], dx, work=work[1])
        bf.bf_op_fp8_gemm(0, 0, 0, h_in, h_out, T, *bufs[1], *bufs[5], dw, work=work[2])

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for k in range(4):
        x.copy_(torch.randn(T, h_in, device="cuda"))
        dy.mul_(-1.5)
        y.zero_(), dx.zero_(), dw.zero_()
        graph.replay()
        torch.cuda.synchronize()
        got = [t.clone() for t in (y, dx, dw)]
        step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, (y, dx, dw))), k


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
def test_two_graphs_that_share_their_scratch(dtype):
    """Products that are cut along the contraction: graphs of two of them on the same planes, replayed in turn, with an eager call on the planes between."""
    M, N, K = 64, 512, 16384
    ops = [(_operand(M, K, 0, 20 + i)[0], _operand(N, K, 0, 30 + i)[0], torch.empty(M, N, dtype=DT[dtype], device="cuda")) for i in range(2)]
    need = bf.bf_op_fp8_gemm_work_bytes(dtype, M, N, K)
    assert need > 0
    work = torch.empty(need, dtype=torch.uint8, device="cuda")
    call = lambda i, out=None: bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, *ops[i][0], *ops[i][1], ops[i][2] if out is None else out, work=work)  # noqa: E731
    call(0), call(1)
    torch.cuda.synchronize()
    want, graphs, other = [o[2].clone() for o in ops], [], torch.empty(M, N, dtype=DT[dtype], device="cuda")
    assert not torch.equal(*want)
    for i in range(2):
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1]):
            call(i)
    for k in range(4):
        ops[0][2].zero_(), ops[1][2].zero_(), work.fill_(0xFF)
        graphs[k % 2].replay()
        call(k % 2, other)
        graphs[1 - k % 2].replay()
        torch.cuda.synchronize()
        assert torch.equal(ops[0][2], want[0]) and torch.equal(ops[1][2], want[1]) and torch.equal(other, want[k % 2]), k


def test_calls_on_two_streams_at_once():
    T, h_in, h_out = 200, 4096, 300
    want, streams, got = [], [torch.cuda.Stream() for _ in range(2)], []
    for k in range(2):
        want.append(_layer(T + k, h_in, h_out, bf.BF_BF16, 0, bf.BF_FP32)[1])
    torch.cuda.synchronize()
    for k, st in enumerate(streams):
        with torch.cuda.stream(st):
            got.append(_layer(T + k, h_in, h_out, bf.BF_BF16, 0, bf.BF_FP32)[1])
    torch.cuda.synchronize()
    for a, b in zip(want, got):
        assert all(torch.equal(x, y) for x, y in zip(a, b))


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
def test_scales_of_the_whole_range(dtype):
    """Blocks whose scales are far apart, and products of a very small by a very large one."""
    M, N, K = 80, 72, 640
    (A, sa), _ = _operand(M, K, 0, 11)
    (B, sb), _ = _operand(N, K, 0, 12)
    e = torch.tensor([-90, -30, 0, 45, 100], device="cuda")
    sa[:, :M] = (127 + e)[:, None].to(torch.uint8)
    sb[:, :N] = (127 - e + torch.arange(5, device="cuda"))[:, None].to(torch.uint8)
    a, b = P.values(A, sa, K, 0), P.values(B, sb, K, 0)
    out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, out)
    _close(out, a @ b.t(), a.abs() @ b.abs().t(), K, dtype)


@pytest.mark.parametrize("fmt,scale", [(0, 0), (0, 1), (0, 3), (1, 0), (1, 5), (1, 10)])
@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
def test_the_smallest_scales(dtype, fmt, scale):
    """Codes under the smallest normal numbers.  An fp32 result's operands are widened to bf16, whose step there is 2^-133: each is off by less than
    that, and exact from a scale of 2^-124 (e4m3, whose step is 2^-9) or 2^-117 (e5m2, 2^-16) on."""
    M, N, K = 80, 72, 250
    (A, sa), _ = _operand(M, K, fmt, 15)
    (B, sb), _ = _operand(N, K, 0, 16)
    sa[:, :M], sb[:, :N] = scale, 244 - scale
    a, b = P.values(A, sa, K, fmt), P.values(B, sb, K, 0)
    out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(fmt, 0, dtype, M, N, K, A, sa, B, sb, out)
    inexact = dtype == bf.BF_FP32 and scale < (3 if fmt == 0 else 10)
    assert out.isfinite().all()
    _close(out, a @ b.t(), a.abs() @ b.abs().t() + (2.0**-133 * b.abs().sum(1) * 2.0**24 / (K / 32 + 32) if inexact else 0.0), K, dtype)



def test_offsets_past_32_bits():
    """Operands and forms of more than 2^32 bytes, rows and results at their far ends."""
    M, K, N = (1 << 21) - 5, 2100, 6
    x = torch.empty(M, K, dtype=torch.bfloat16, device="cuda")
    torch.manual_seed(1)
    for k in range(0, M, 1 << 18):
        x[k: k + (1 << 18)] = torch.randn(min(1 << 18, M - k), K, device="cuda")
    (A, sa), (At, sat) = _new(M, K), _new(K, M)
    bf.bf_op_fp8_quantize(bf.BF_BF16, 0, M, K, x, A, sa, At, sat)
    assert A.numel() > 2**32
    for rows in (slice(0, 200), slice(M - 200, M)):
        q, s = P.form(x[rows], 0)
        got, sg = _views((A, sa), M, K)
        assert torch.equal(got[rows].view(P.TYPES[0]).double(), q) and torch.equal(sg[:, rows], s[:, : 200])
    cols, last = slice(K - 30, K), (M - 1) // 128 * 128
    q, s = P.form(x[last:, cols].t().contiguous(), 0)
    got, sg = _views((At, sat), K, M)
    assert torch.equal(got[cols, last:].view(P.TYPES[0]).double(), q) and torch.equal(sg[-1, cols], s[0, :30])
    (B, sb), b = _operand(N, K, 0, 5)
    for dtype in (bf.BF_BF16, bf.BF_FP32):
        out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
        bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A[: M * 2176], sa, B, sb, out)
        for rows in (slice(0, 300), slice(M - 300, M)):
            a = P.values(*P.form(x[rows], 0), K)
            _close(out[rows], a @ b.t(), a.abs() @ b.abs().t(), K, dtype)
    # a long contraction: x down its columns against itself, few rows and columns of it
    out = torch.empty(20, 20, device="cuda")
    T = At[: 20 * bf.bf_op_fp8_row_bytes(M)]
    st = _views((At, sat), K, M)[1]
    few = torch.full((st.shape[0], 32), 127, dtype=torch.uint8, device="cuda")
    few[:, :20] = st[:, :20]
    bf.bf_op_fp8_gemm(0, 0, bf.BF_FP32, 20, 20, M, T, few, T, few, out)
    ref = torch.zeros(20, 20, dtype=torch.float64, device="cuda")
    mag = torch.zeros_like(ref)
    for k in range(0, M, 1 << 18):
        t = P.values(*P.form(x[k: k + (1 << 18), :20].t().contiguous(), 0), min(1 << 18, M - k))
        ref += t @ t.t()
        mag += t.abs() @ t.abs().t()
    _close(out, ref, mag, M, bf.BF_FP32)


@pytest.mark.parametrize("rows,cols", [(8192, 16640), (8190, 16517), (8064, 17000)])
def test_forms_larger_than_the_caches(rows, cols):
    """Tiles in another order: whole, ragged, and where the number of tiles keeps to the first one."""
    x = _matrix(rows, cols, bf.BF_BF16, 1, 1.0)
    a, d = _new(rows, cols), _new(cols, rows)
    bf.bf_op_fp8_quantize(bf.BF_BF16, 0, rows, cols, x, *a, *d)
    _same_form(a, x, 0)
    _same_form(d, x.t(), 0)
    d2 = _new(cols, rows)
    bf.bf_op_fp8_quantize(bf.BF_BF16, 0, rows, cols, x, None, None, *d2)
    assert torch.equal(d[0], d2[0]) and torch.equal(d[1], d2[1])


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
@pytest.mark.parametrize("M,N,K", [(4100, 50004, 260), (60000, 3502, 130)])
def test_results_that_go_past_the_caches(M, N, K, dtype):
    (A, sa), a = _operand(M, K, 0, 1)
    (B, sb), b = _operand(N, K, 0, 2)
    out = torch.empty(M, N, dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, out)
    for k in range(0, M, 4100):
        rows = slice(k, min(M, k + 4100))
        for c in range(0, N, 12501):
            cols = slice(c, min(N, c + 12501))
            _close(out[rows, cols], a[rows] @ b[cols].t(), a[rows].abs() @ b[cols].abs().t(), K, dtype)


@pytest.mark.parametrize("dtype", [bf.BF_BF16, bf.BF_FP32])
def test_results_past_32_bits(dtype):
    M, N, K = 40003, 60004, 130
    (A, sa), a = _operand(M, K, 0, 17)
    (B, sb), b = _operand(N, K, 0, 18)
    out = torch.full((M, N), float("nan"), dtype=DT[dtype], device="cuda")
    bf.bf_op_fp8_gemm(0, 0, dtype, M, N, K, A, sa, B, sb, out)
    for rows in (slice(0, 100), slice(M // 2, M // 2 + 100), slice(M - 100, M)):
        _close(out[rows], a[rows] @ b.t(), a[rows].abs() @ b.abs().t(), K, dtype)
    assert not any(torch.isnan(out[i: i + 2000]).any() for i in range(0, M, 2000))
