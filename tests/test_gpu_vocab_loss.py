"""The vocabulary loss in pieces against fp64.

Bounds, element by element.  A logit is an fp32 sum of S_hidden products: off by at most eps_z = (S_hidden + 64) 2^-24 S, S the
largest sum of |y||w| (any order of additions).  exp and log add 2^-20 at most (arguments of exp up to 2^6 in fp32: 2^-24 2^6).
With A = scale (p + onehot), the sizes that dz is made of:
  dw  <= (eps_z + 2^-18 + 2^-17 for two bf16 parts + (n_rows + 64) 2^-24) A^T |y|
       and where it is added to what is there, the sum starts at that value and each of n_rows additions may round by 2^-24 of it
  dy  <= (eps_z + 2^-18 + (S_voc + 64) 2^-24) A |w| + roundings: 2^-8 of |dz| |w| and 2^-8 of |dy| in bf16"""
import math

import pytest
import torch

import paper_2211_05953_amd as bf

pytestmark = pytest.mark.gpu
TYPES = {bf.BF_FP32: torch.float32, bf.BF_BF16: torch.bfloat16}


def _guarded(x, dtype, offset):
    """A copy with NaN on both sides, `offset` elements off 16-byte alignment."""
    flat = torch.full((x.numel() + 192,), float("nan"), dtype=dtype, device="cuda")
    inner = flat[64 + offset:64 + offset + x.numel()]
    inner.copy_(x.reshape(-1))
    return flat, inner.view(x.shape)


def _inputs(dtype, T, h, V, seed=0, offset=0, ignored=True):
    g = torch.Generator("cuda").manual_seed(seed)
    t = TYPES[dtype]
    w = (torch.randn(V, h, generator=g, device="cuda") * (2 / math.sqrt(h))).to(t)
    label = torch.randint(0, V, (T,), generator=g, device="cuda")
    y = (torch.randn(T, h, generator=g, device="cuda") + 4 * torch.rand(T, 1, generator=g, device="cuda") * w[label].float()).to(t)
    label = label.int()
    if ignored and T > 2:
        label[1], label[T // 2], label[T - 1] = -1, V, -100
    return _guarded(y, t, offset)[1], _guarded(w, t, offset)[1], label


def _reference(y, w, label, scale):
    V = w.shape[0]
    y, w = y.double(), w.double()
    known = (label >= 0) & (label < V)
    at = torch.where(known, label, 0).long()
    z = y @ w.t()
    lse = torch.logsumexp(z, 1)
    p = torch.exp(z - lse[:, None])
    hot = torch.zeros_like(p)
    hot[torch.arange(len(at), device="cuda"), at] = 1
    p, hot = p * (known * scale)[:, None], hot * (known * scale)[:, None]
    rows = torch.where(known, (lse - z.gather(1, at[:, None])[:, 0]) * scale, 0.0)
    return dict(lse=lse, rows=rows, dz=p - hot, a=p + hot, known=known)


def _within(got, want, bound, what):
    over = ((got.double() - want).abs() - bound).max()
    assert bool(got.isfinite().all()) and float(over) <= 0, (what, float(over), float((got.double() - want).abs().max()))


def _check(dtype, T, h, V, piece=0, offset=0, accumulate=0, poison=False, seed=0):
    y, w, label = _inputs(dtype, T, h, V, seed, offset)
    scale = 1.7 / T
    ref = _reference(y, w, label, scale)
    if poison:  # rows without a label: nothing of them reaches a gradient
        y[~ref["known"]] = float("inf")
    flat_dy, dy = _guarded(torch.zeros(T, h), TYPES[dtype], offset)
    flat_dw, dw = _guarded(torch.ones(V, h), torch.float32, offset)
    lse, rows, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
    work = [torch.full((bf.bf_op_vocab_loss_work_bytes(dtype, T, h, V, piece, k),), 0xFF, dtype=torch.uint8, device="cuda") for k in (0, 1)]
    bf.bf_op_vocab_loss_fwd(dtype, T, h, V, y, w, label, scale, lse, rows, loss, S_piece=piece, work=work[0])
    bf.bf_op_vocab_loss_bwd(dtype, T, h, V, y, w, label, lse if not poison else torch.where(ref["known"], lse, math.nan), scale, dy, dw, accumulate,
                            S_piece=piece, work=work[1])
    torch.cuda.synchronize()
    yd = torch.where(ref["known"][:, None], y.double(), 0.0)
    wd = w.double()
    big = float((yd.abs() @ wd.abs().t()).max()) if T else 0.0
    eps_z = (h + 64) * 2.0**-24 * big + 2.0**-18
    k = ref["known"] if poison else torch.ones_like(ref["known"])
    _within(lse[k], ref["lse"][k], eps_z + 2.0**-22 * ref["lse"][k].abs(), "lse")
    _within(rows, ref["rows"], (2 * eps_z + 2.0**-21 * ref["lse"].nan_to_num(0, 0, 0).abs()) * scale, "rows")
    assert abs(float(loss) - float(rows.double().sum())) <= 2.0**-23 * abs(float(loss))
    dz, a = ref["dz"], ref["a"]
    low = dtype == bf.BF_BF16
    want = dz @ wd
    b = (eps_z + (V + 64) * 2.0**-24) * (a @ wd.abs()) + (2.0**-8 * (dz.abs() @ wd.abs()) * 1.01 + 2.0**-8 * want.abs() * 1.01 if low else 0)
    _within(dy, want, b + 1e-30, "dy")
    want = dz.t() @ yd + (1.0 if accumulate else 0.0)
    b = (eps_z + 2.0**-17 + (T + 64) * 2.0**-24) * (a.t() @ yd.abs()) + ((T + 2) * 2.0**-24 * 1.01 * want.abs() if accumulate else 0)
    _within(dw, want, b + 1e-30, "dw")
    for flat, inner in ((flat_dy, dy), (flat_dw, dw)):
        assert int(flat.isnan().sum()) == flat.numel() - inner.numel()


DTYPES = [bf.BF_FP32, bf.BF_BF16]


# rows and columns on both sides of the 64-, 128- and 256-wide tiles, odd widths and vocabularies, contractions in groups
@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,h,V", [(1, 8, 1), (1, 8, 2), (1, 256, 1003), (2, 64, 63), (33, 256, 1003), (64, 1032, 2050), (65, 72, 130), (63, 4104, 70),
                                   (130, 72, 515), (257, 128, 1000), (300, 257, 401), (128, 64, 8192), (1100, 136, 9001), (1024, 64, 16384 + 257)])
def test_sizes(dtype, T, h, V):
    _check(dtype, T, h, V)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,h,V,piece", [(70, 96, 3000, 1), (70, 96, 300, 7), (70, 96, 3000, 512), (300, 128, 5001, 2049), (33, 64, 9000, 4096),
                                         (200, 200, 4100, 4096), (1030, 64, 20000, 9999)])
def test_pieces(dtype, T, h, V, piece):
    if piece == 1:
        V = 40
    _check(dtype, T, h, V, piece)
    _check(dtype, T, h, V, piece, accumulate=1, seed=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("offset", [1, 3])
def test_rows_off_16_byte_alignment(dtype, offset):
    _check(dtype, 70, 96, 700, 0, offset)
    _check(dtype, 70, 96, 700, 256, offset, accumulate=1)


# 1001 is no multiple of a 16-byte chunk: copies, of a vocabulary long enough for two pieces of them in both directions
def test_long_vocabulary_of_rows_that_are_no_chunks():
    _check(bf.BF_BF16, 4, 1001, 70001)
    _check(bf.BF_BF16, 4, 1001, 70001, accumulate=1, seed=1)


# an unscaled plane of dz beside the scaled ones (more than 256 rows), and rows of one element
@pytest.mark.parametrize("T,h,V", [(257, 1, 3), (1, 1, 1), (300, 7, 9), (513, 4184, 70), (257, 8200, 66)])
def test_narrow_and_wide_rows(T, h, V):
    _check(bf.BF_BF16, T, h, V)
    _check(bf.BF_BF16, T, h, V, accumulate=1, seed=1)


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,h,V,piece", [(70, 96, 700, 0), (300, 257, 401, 100), (300, 128, 3000, 1024)])
def test_rows_without_a_label_leave_no_trace(dtype, T, h, V, piece):
    _check(dtype, T, h, V, piece, poison=True)


@pytest.mark.parametrize("dtype", DTYPES)
def test_no_row_has_a_label(dtype):
    y, w, label = _inputs(dtype, 40, 64, 300)
    label.fill_(-1)
    lse, rows, loss = torch.empty(40, device="cuda"), torch.empty(40, device="cuda"), torch.empty(1, device="cuda")
    bf.bf_op_vocab_loss_fwd(dtype, 40, 64, 300, y, w, label, 1.0, lse, rows, loss)
    dy, dw = torch.ones_like(y), torch.full((300, 64), 5.0, device="cuda")
    bf.bf_op_vocab_loss_bwd(dtype, 40, 64, 300, y, w, label, lse, 1.0, dy, dw, accumulate=1)
    assert float(loss) == 0 and not rows.any() and not dy.any() and bool((dw == 5).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_infinite_logits(dtype):
    """A column of -inf has no share; a row of +inf has an infinite loss and not a NaN; other rows are as without them."""
    T, h, V = 20, 64, 500
    y, w, label = _inputs(dtype, T, h, V, ignored=False)
    y[:, 0] = 1.0
    y[3, 0] = 0.0 - 1.0  # -inf times -1
    w[7, 0] = float("-inf")
    w[300:, 0] = float("-inf")
    label[label == 7] = 8
    label[label >= 300] = 9
    lse, rows, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
    for piece in (0, 128):
        bf.bf_op_vocab_loss_fwd(dtype, T, h, V, y, w, label, 1.0, lse, rows, loss, S_piece=piece)
        want = torch.logsumexp(y.double() @ w.double().t(), 1)
        keep = torch.arange(T, device="cuda") != 3
        assert float(lse[3]) == math.inf and float(rows[3]) == math.inf
        assert bool(((lse.double() - want)[keep].abs() <= 1e-4).all())


@pytest.mark.parametrize("dtype", DTYPES)
def test_gradient_against_differences_of_the_loss(dtype):
    """In fp64 on the oracle's side: the gradient that the kernels match is that of the loss they return."""
    T, h, V = 9, 24, 50
    y, w, label = _inputs(dtype, T, h, V)
    loss = lambda a, b: _reference(a, b, label, 0.3)["rows"].sum()  # noqa: E731
    lse, rows, out = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
    bf.bf_op_vocab_loss_fwd(dtype, T, h, V, y, w, label, 0.3, lse, rows, out)
    dy, dw = torch.empty_like(y), torch.empty(V, h, device="cuda")
    bf.bf_op_vocab_loss_bwd(dtype, T, h, V, y, w, label, lse, 0.3, dy, dw)
    assert abs(float(out) - float(loss(y, w))) <= 1e-5 * abs(float(out))
    g = torch.Generator("cuda").manual_seed(3)
    for x, dx in ((y, dy), (w, dw)):
        to = torch.randn(x.shape, generator=g, device="cuda", dtype=torch.float64)
        step = 1e-5
        args = [[q.double() + s * to if q is x else q.double() for q in (y, w)] for s in (step, -step)]
        slope = float(loss(*args[0]) - loss(*args[1])) / (2 * step)
        size = float(dx.double().norm() * to.norm())
        assert abs(float((dx.double() * to).sum()) - slope) <= (2.0**-7 if dtype == bf.BF_BF16 else 1e-5) * size


def test_captured_and_on_another_stream():
    dtype, T, h, V = bf.BF_BF16, 150, 128, 3000
    y, w, label = _inputs(dtype, T, h, V)
    y = y.contiguous().clone()

    def step():
        lse, rows, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
        bf.bf_op_vocab_loss_fwd(dtype, T, h, V, y, w, label, 1 / T, lse, rows, loss)
        dy, dw = torch.empty_like(y), torch.empty(V, h, device="cuda")
        bf.bf_op_vocab_loss_bwd(dtype, T, h, V, y, w, label, lse, 1 / T, dy, dw, S_piece=1024)
        return loss, lse, rows, dy, dw

    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    step()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = step()
    for k in range(3):
        y.copy_(_inputs(dtype, T, h, V, seed=k + 1)[0])
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(got, want))


def test_binding_refuses_what_a_kernel_would_misread():
    dtype, T, h, V = bf.BF_BF16, 8, 16, 30
    y, w, label = _inputs(dtype, T, h, V)
    f = lambda n: torch.empty(n, device="cuda")  # noqa: E731
    ok = [y, w, label, 1.0, f(T), f(T), f(1)]
    bf.bf_op_vocab_loss_fwd(dtype, T, h, V, *ok)
    for at, bad in ((0, y.float()), (0, y[:4]), (1, w.t()), (1, w[:5]), (2, label.long()), (2, label[:3]), (4, f(T - 1)), (5, f(2)), (6, f(0)), (0, y.cpu())):
        with pytest.raises(ValueError):
            bf.bf_op_vocab_loss_fwd(dtype, T, h, V, *ok[:at], bad, *ok[at + 1:])
    with pytest.raises(bf.BfError):
        bf.bf_op_vocab_loss_fwd(dtype, T, h, V, *ok, work=torch.empty(8, dtype=torch.uint8, device="cuda"))


@pytest.mark.parametrize("dtype", DTYPES)
@pytest.mark.parametrize("T,h,V,piece,offset", [(33, 256, 1003, 0, 0), (300, 128, 5001, 2049, 0), (300, 128, 5001, 8, 0), (70, 96, 3000, 100, 3), (257, 250, 9000, 1024, 0),
                                                (1030, 64, 20000, 9999, 0)])
def test_nothing_past_the_scratch(dtype, T, h, V, piece, offset):
    """Pieces large and small, with and without lengthened rows, in scratch of exactly the size asked for; the same call with more
    scratch gives the same bits."""
    y, w, label = _inputs(dtype, T, h, V, offset=offset)
    outs = []
    for more in (0, 4096):
        lse, rows, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
        dy, dw = torch.empty_like(y), torch.empty(V, h, device="cuda")
        need = [bf.bf_op_vocab_loss_work_bytes(dtype, T, h, V, piece, k) for k in (0, 1)]
        flat = [torch.full((n + 8192,), 0xA5, dtype=torch.uint8, device="cuda") for n in need]
        bf.bf_op_vocab_loss_fwd(dtype, T, h, V, y, w, label, 1 / T, lse, rows, loss, S_piece=piece, work=flat[0][:need[0] + more])
        bf.bf_op_vocab_loss_bwd(dtype, T, h, V, y, w, label, lse, 1 / T, dy, dw, S_piece=piece, work=flat[1][:need[1] + more])
        assert all(bool((f[n:] == 0xA5).all()) for f, n in zip(flat, need))
        outs.append((lse, rows, loss, dy, dw))
    assert all(torch.equal(a, b) for a, b in zip(*outs))


# Rows and hidden sizes of whole 256 x 256 tiles: pieces of whole rounds of them and an odd rest (logits, dw and dy with no bounds checks, sums in
# slices, shorter pieces added to the planes of longer ones); dz in three parts and two, dy's in two (up to 256 rows) and one; pieces
# as given, whole tiles too; a number of k-tiles that is no power of two
WHOLE = [(256, 256, 65536 + 1003, 0), (1024, 1024, 16384 + 1003, 0), (2048, 1024, 2 * 16384 + 77, 0), (2048, 8192, 8192 + 300, 0), (1536, 1024, 16384, 0),
         (1024, 1024, 40003, 16384), (1024, 1024, 16384, 0)]


@pytest.mark.parametrize("accumulate", [0, 1])
@pytest.mark.parametrize("T,h,V,piece", WHOLE)
def test_whole_tiles(T, h, V, piece, accumulate):
    _check(bf.BF_BF16, T, h, V, piece, accumulate=accumulate, seed=accumulate)


@pytest.mark.parametrize("T,h,V,piece", [WHOLE[0], WHOLE[2], WHOLE[5]])
def test_rows_without_a_label_leave_no_trace_on_whole_tiles(T, h, V, piece):
    _check(bf.BF_BF16, T, h, V, piece, poison=True)


def test_the_most_rows():
    """2^21 rows over a vocabulary whose tiles one launch does not hold: every 30011th row against fp64 (rows are independent)."""
    T, h, V = 1 << 21, 8, (1 << 18) + 100
    g = torch.Generator("cuda").manual_seed(5)
    y, w = torch.randn(T, h, generator=g, device="cuda").bfloat16(), torch.randn(V, h, generator=g, device="cuda").bfloat16()
    label = torch.randint(0, V, (T,), generator=g, device="cuda").int()
    some = torch.arange(0, T, 30011, device="cuda")
    label[some[0]], label[some[1]], label[some[2]] = V - 1, -1, 0
    lse, rows, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
    bf.bf_op_vocab_loss_fwd(bf.BF_BF16, T, h, V, y, w, label, 1 / T, lse, rows, loss)
    ref = _reference(y[some], w, label[some], 1 / T)
    eps_z = (h + 64) * 2.0**-24 * float((y[some].double().abs() @ w.double().abs().t()).max()) + 2.0**-18
    _within(lse[some], ref["lse"], eps_z + 2.0**-22 * ref["lse"].abs(), "lse")
    _within(rows[some], ref["rows"], (2 * eps_z + 2.0**-21 * ref["lse"].abs()) / T, "rows")
    assert abs(float(loss) - float(rows.double().sum())) <= 2.0**-23 * abs(float(loss))


def test_offsets_past_32_bits():
    """w of 4.9 GB and dw of 9.8: the loss of every row, dy, and every 7919th row of dw and its last ones, against fp64."""
    T, h, V = 5, 2048, 1200003
    g = torch.Generator("cuda").manual_seed(6)
    w = torch.empty(V, h, dtype=torch.bfloat16, device="cuda")
    for part in w.split(1 << 18):
        part.copy_(torch.randn(part.shape, generator=g, device="cuda") * (2 / math.sqrt(h)))
    label = torch.tensor([V - 1, 0, -1, 1048577, 7], device="cuda").int()
    y = torch.randn(T, h, generator=g, device="cuda").bfloat16()
    lse, rows, loss = torch.empty(T, device="cuda"), torch.empty(T, device="cuda"), torch.empty(1, device="cuda")
    dy, dw = torch.empty_like(y), torch.empty(V, h, device="cuda")
    bf.bf_op_vocab_loss_fwd(bf.BF_BF16, T, h, V, y, w, label, 0.5, lse, rows, loss)
    bf.bf_op_vocab_loss_bwd(bf.BF_BF16, T, h, V, y, w, label, lse, 0.5, dy, dw)
    yd, known = y.double(), label >= 0
    z = torch.cat([yd @ part.double().t() for part in w.split(1 << 17)], 1)
    eps_z = (h + 64) * 2.0**-24 * max(float((yd.abs() @ part.double().abs().t()).max()) for part in w.split(1 << 17)) + 2.0**-18
    want = torch.logsumexp(z, 1)
    _within(lse, want, eps_z + 2.0**-22 * want.abs(), "lse")
    at = label.long().clamp_min(0)
    row = torch.where(known, (want - z.gather(1, at[:, None])[:, 0]) * 0.5, 0.0)
    _within(rows, row, (2 * eps_z + 2.0**-21 * want.abs()) * 0.5, "rows")
    p = torch.exp(z - want[:, None]) * (0.5 * known)[:, None]
    hot = torch.zeros_like(p).scatter_(1, at[:, None], (0.5 * known.double())[:, None])
    dz, a = p - hot, p + hot
    some = torch.cat([torch.arange(0, V, 7919, device="cuda"), torch.arange(V - 300, V, device="cuda"), at])
    _within(dw[some], dz[:, some].t() @ yd, (eps_z + 2.0**-17 + (T + 64) * 2.0**-24) * (a[:, some].t() @ yd.abs()) + 1e-30, "dw")
    want = b = 0
    for i in range(0, V, 1 << 17):
        s = slice(i, i + (1 << 17))
        wd = w[s].double()
        want = want + dz[:, s] @ wd
        b = b + (eps_z + (V + 64) * 2.0**-24) * (a[:, s] @ wd.abs()) + 2.0**-8 * (dz[:, s].abs() @ wd.abs()) * 1.01
    _within(dy, want, b + 2.0**-8 * want.abs() * 1.01, "dy")
