"""The Adam step on 8-bit moments against the definition in fp64.

The step's fp32 arithmetic: m and v carry three roundings of their terms, m c1 / (sqrt(v c2) + eps) six more, w two: |w - ref| <= 2^-23 |w| + lr 2^-19 |step|
(the step's terms may cancel in m, which its magnitudes bound).  A moment's code is decided by floor(65536 y / step) + r: with y off by 2^-22 of its terms
that sum is off by 65536 2^-22 terms / step and the floor by one more, and only sums that near to a carry may go the other way."""
import pytest
import torch

import fp8_plain as P
import paper_2211_05953_amd as bf

pytestmark = pytest.mark.gpu

LR, B1, B2, EPS, WD = 1e-3, 0.9, 0.95, 1e-8, 0.1
SIZES = [1, 2, 3, 4, 5, 31, 127, 128, 129, 255, 256, 1000, 1023, 1024, 4095, 4096, 4097, 9999, 70001]
DT = {bf.BF_BF16: torch.bfloat16, bf.BF_FP32: torch.float32}


def _make(sizes, dtype, seed, odd=True, lp=True, zero=False):
    g = torch.Generator("cuda").manual_seed(seed)
    normal = lambda n: torch.randn(n, generator=g, device="cuda")  # noqa: E731
    out = []
    for i, n in enumerate(sizes):
        at = i % 3 if odd else 0
        w, grad = normal(n + 3)[at: at + n] * 0.02, (normal(n + 3) * torch.exp2(2 * normal(n + 3))).to(DT[dtype])[at: at + n]
        m, v = normal(n) * 0.1, normal(n).square() * torch.exp2(3 * normal(n)) * 0.1
        state = torch.zeros(bf.bf_op_adam8_state_bytes(n), dtype=torch.uint8, device="cuda") if zero else P.encode(m, v)
        low = torch.full((n + 3,), float("nan"), dtype=torch.bfloat16, device="cuda")[at: at + n] if lp and i % 4 != 3 else None
        full = torch.full((n + 5,), float("nan"), device="cuda")
        full[at: at + n] = w
        guarded = torch.cat([state, torch.full((32,), 0xA5, dtype=torch.uint8, device="cuda")])
        out.append((full[at: at + n], guarded[: state.numel()], grad, low, full, guarded))
    return out


def _check(tensors, before, coef, seed, t, beta2=B2):
    for i, ((w, state, g, low, full, guarded), (w0, s0)) in enumerate(zip(tensors, before)):
        n = w.numel()
        ref, m, v = P.adam(w0, s0, g, coef, t, LR, B1, beta2, EPS, WD)
        m0, v0, _, _ = P.decode(s0, n)
        gg = torch.nn.functional.pad(g.double().abs() * coef, (0, m.numel() - n)).view_as(m)
        mt, vt = B1 * m0.abs() + (1 - B1) * gg, beta2 * v0 + (1 - beta2) * gg * gg  # magnitudes of the terms
        rate = (mt / (1 - B1**t) / ((vt / (1 - beta2**t)).sqrt() + EPS)).view(-1)[:n]
        tol = 2.0**-23 * w0.double().abs() + LR * 2.0**-19 * (rate + WD * w0.double().abs())
        assert bool(((w.double() - ref).abs() <= tol).all()), (i, n)
        if low is not None:
            assert torch.equal(low, w.bfloat16())
        assert int(torch.isnan(full).sum()) == 5 and bool((guarded[state.numel():] == 0xA5).all())  # nothing beside them
        gm, gv, um, uv = P.decode(state, n)
        rm, rv = (r.view_as(m) for r in P.randoms(seed, t, i, m.numel(), "cuda"))
        for got, x, terms, unit, r, low_e, bits, top in ((gm, m, mt, um, rm, -6, 3, 448.0), (gv, v, vt, uv, rv, 0, 4, 31744.0)):
            amax = x.abs().amax(1, keepdim=True)
            some = amax > 2.0**-100
            assert bool(((amax <= top * unit * (1 + 2.0**-20)) & (amax >= top * unit / 2 * (1 - 2.0**-20)) | ~some).all())
            y = x.abs() / unit
            step = P.power((torch.frexp(y)[1] - 1).clamp(min=low_e) - bits)
            part = y / step
            near = 65536 * 2.0**-22 * terms / unit / step + 1
            want = torch.floor(part) + (torch.floor((part - torch.floor(part)) * 65536) + r >= 65536)
            have = got.abs() / unit / step
            want = torch.where((x != 0) & (want == 0) & (top == 31744.0), torch.ones_like(want), want)
            over = (torch.floor((part - torch.floor(part)) * 65536) + r - 65536).abs()
            edge = torch.minimum(part - torch.floor(part), torch.ceil(part) - part) * 65536  # y itself next to a code: floor may be the one below
            ok = (have == want) | ((have - want).abs() <= 1) & ((over <= near) | (edge <= near)) | (y > top * (1 - 2.0**-20))
            assert bool((ok | ~some).all()), (i, n, top)
            assert bool(((got >= 0) | (x < 0)).all()) and float((have != want).double().mean()) <= (1e-3 if n > 5000 else 1.0)


@pytest.mark.parametrize("dtype", [bf.BF_FP32, bf.BF_BF16])
@pytest.mark.parametrize("sizes", [[1], [130], SIZES, [33] * 150, [(1 << 20) + 5, 17]])
@pytest.mark.parametrize("zero", [False, True])
def test_step(dtype, sizes, zero):
    tensors = _make(sizes, dtype, 3, zero=zero)
    for t, seed, c in ((1, 5, 1.0), (7, 2**63 + 12345, 0.37)):
        before = [(x[0].clone(), x[1].clone()) for x in tensors]
        coef = torch.tensor([c], device="cuda")
        bf.bf_op_adam8(dtype, [x[:4] for x in tensors], coef, seed, t, LR, B1, B2, EPS, WD)
        _check(tensors, before, float(coef), seed, t)


@pytest.mark.parametrize("dtype", [bf.BF_FP32, bf.BF_BF16])
@pytest.mark.parametrize("c", [1.0, 0.37])
def test_codes_are_those_of_fp32_operations_one_by_one(dtype, c):
    """Every code and scale, over three steps: the definition in fp32, each operation rounded by itself."""
    tensors = _make([(1 << 22) + 77, 3000], dtype, 12)
    coef = torch.tensor([c], device="cuda")
    for t in (1, 2, 3):
        before = [x[1].clone() for x in tensors]
        bf.bf_op_adam8(dtype, [x[:4] for x in tensors], coef, 21, t, LR, B1, B2, EPS, WD)
        for i, ((w, state, g, *_), s0) in enumerate(zip(tensors, before)):
            n = w.numel()
            m, v, _, _ = (x.float() for x in P.decode(s0, n))
            gg = torch.nn.functional.pad(g.float() * coef, (0, m.numel() - n)).view_as(m)
            m, v = B1 * m + (1 - B1) * gg, B2 * v + (1 - B2) * gg * gg
            want = []
            for x, top, low, bits, r in zip((m, v), (448.0, 31744.0), (-6, 0), (3, 4), P.randoms(21, t, i, m.numel(), "cuda")):
                x = x.double()
                unit = P.power(P.exponent(x.abs().amax(1), top))[:, None]
                y = x.abs() / unit
                step = P.power((torch.frexp(y)[1] - 1).clamp(min=low) - bits)
                part = y / step
                code = (torch.floor(part) + (torch.floor((part - torch.floor(part)) * 65536) + r.view_as(x) >= 65536)) * step
                code = torch.where((x != 0) & (code == 0) & (low == 0), torch.full_like(code, 1 / 16), code.clamp(max=top))
                want.append(code.copysign(x) * unit)
            got = P.decode(state, n)
            assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])


def test_bits_are_a_function_of_the_call():
    first = None
    for _ in range(2):
        tensors = _make(SIZES, bf.BF_FP32, 4)
        bf.bf_op_adam8(bf.BF_FP32, [x[:4] for x in tensors], torch.ones(1, device="cuda"), 9, 2, LR, B1, B2, EPS, WD)
        now = [x[1].clone() for x in tensors]
        assert first is None or all(torch.equal(a, b) for a, b in zip(first, now))
        first = now
    for seed, t in ((10, 2), (9, 3), (9 + 2**32, 2)):
        tensors = _make(SIZES, bf.BF_FP32, 4)
        bf.bf_op_adam8(bf.BF_FP32, [x[:4] for x in tensors], torch.ones(1, device="cuda"), seed, t, LR, B1, B2, EPS, WD)
        assert not torch.equal(first[-1], tensors[-1][1])


@pytest.mark.parametrize("c", [float("nan"), float("inf"), -float("inf")])
def test_a_coefficient_that_is_not_finite_leaves_everything(c):
    tensors = _make(SIZES, bf.BF_FP32, 5)
    before = [[x.clone() for x in t[:2]] for t in tensors]
    bf.bf_op_adam8(bf.BF_FP32, [x[:4] for x in tensors], torch.tensor([c], device="cuda"), 1, 1, LR, B1, B2, EPS, WD)
    assert all(torch.equal(a, b) for t, u in zip(tensors, before) for a, b in zip(t[:2], u))
    assert all(bool(torch.isnan(t[3]).all()) for t in tensors if t[3] is not None)


def test_empty_lists_and_tensors():
    coef = torch.ones(1, device="cuda")
    bf.bf_op_adam8(bf.BF_FP32, [], coef, 1, 1, LR, B1, B2, EPS, WD)
    bf.bf_op_adam8_moments(bf.BF_FP32, [])
    none = torch.empty(0, device="cuda")
    tensors = _make([300], bf.BF_FP32, 6)
    before = [(x[0].clone(), x[1].clone()) for x in tensors]
    # an empty tensor has a place in the list all the same: the other one's random numbers are those of place 1
    bf.bf_op_adam8(bf.BF_FP32, [(none, torch.empty(0, dtype=torch.uint8, device="cuda"), none, None), tensors[0][:4]], coef, 1, 1, LR, B1, B2, EPS, WD)
    other = _make([300], bf.BF_FP32, 6)
    bf.bf_op_adam8(bf.BF_FP32, [other[0][:4]], coef, 1, 1, LR, B1, B2, EPS, WD)
    assert torch.equal(tensors[0][0], other[0][0]) and not torch.equal(tensors[0][1], other[0][1])
    _check(other, before, 1.0, 1, 1)


@pytest.mark.parametrize("dtype", [bf.BF_FP32, bf.BF_BF16])
def test_moments(dtype):
    tensors = _make(SIZES, bf.BF_FP32, 7)
    outs = []
    for i, x in enumerate(tensors):
        n = x[0].numel()
        full = [torch.full((n + 4,), float("nan"), dtype=DT[dtype], device="cuda") for _ in range(2)]
        outs.append((full, [f[i % 3: i % 3 + n] if i % 5 != k else None for k, f in enumerate(full)]))
    bf.bf_op_adam8_moments(dtype, [(x[1], *o[1]) for x, o in zip(tensors, outs)])
    for x, (full, parts) in zip(tensors, outs):
        n = x[0].numel()
        for ref, part, f in zip(P.decode(x[1], n)[:2], parts, full):
            assert int(torch.isnan(f).sum()) == (4 if part is not None else n + 4)
            if part is not None:
                assert torch.equal(part.double(), ref.reshape(-1)[:n])


def test_rounding_has_no_bias():
    """The mean of a moment over many seeds is the moment: off by under 5 standard errors of the mean, a code's step / 2 / sqrt(seeds), in every element,
    and by under 5 over all of them together."""
    n, seeds = 4096, 256
    (w, state, g, _, _, _), = _make([n], bf.BF_FP32, 8, lp=False)
    _, m, v = P.adam(w, state, g, 1.0, 5, LR, B1, B2, EPS, WD)
    coef, sums = torch.ones(1, device="cuda"), [torch.zeros(n, dtype=torch.float64, device="cuda") for _ in range(2)]
    for seed in range(seeds):
        s = state.clone()
        bf.bf_op_adam8(bf.BF_FP32, [(w.clone(), s, g, None)], coef, seed * 7919, 5, LR, B1, B2, EPS, WD)
        dm, dv, um, uv = P.decode(s, n)
        sums[0] += dm.reshape(-1)
        sums[1] += dv.reshape(-1)
    for total, x, unit, low, bits in ((sums[0], m, um, -6, 3), (sums[1], v, uv, 0, 4)):
        y = (x.abs() / unit)
        step = (P.power((torch.frexp(y)[1] - 1).clamp(min=low) - bits) * unit).reshape(-1)
        off = (total / seeds - x.reshape(-1)) / (step / 2 / seeds**0.5)
        if low == 0:
            off = off[y.reshape(-1) >= 1 / 16]  # below the smallest code v is kept at it
        assert float(off.abs().max()) <= 6  # (some 4000 of them: 5 happens)
        assert abs(float(off.mean())) * off.numel()**0.5 <= 5


def test_moments_that_move_slowly_still_move():
    """beta2 = 0.999 on gradients of zero: v falls by 0.1 % a step, far under half a code, to exp(-1) of itself in 1000 steps.  (The mean over 4096 elements of a
    walk whose steps have a standard deviation of 0.0013 to 0.04 of v: within 10 %.)"""
    n = 4096
    w, g, coef = torch.zeros(n, device="cuda"), torch.zeros(n, device="cuda"), torch.ones(1, device="cuda")
    state = P.encode(torch.zeros(n, device="cuda"), torch.rand(n, device="cuda") + 0.5)
    before = P.decode(state, n)[1].mean()
    for t in range(1, 1001):
        bf.bf_op_adam8(bf.BF_FP32, [(w, state, g, None)], coef, 77, t, LR, B1, 0.999, EPS, WD)
    ratio = float(P.decode(state, n)[1].mean() / before)
    assert abs(ratio / 0.999**1000 - 1) <= 0.1
    assert bool((w == 0).all())


def test_values_that_are_not_finite_stay_with_their_element():
    n = 256
    (w, state, g, _, _, _), = _make([n], bf.BF_FP32, 9, odd=False, lp=False)
    g = g.clone()
    g[5], g[130], g[140] = float("nan"), float("inf"), 3e38
    w1, s1 = w.clone(), state.clone()
    bf.bf_op_adam8(bf.BF_FP32, [(w1, s1, g, None)], torch.ones(1, device="cuda"), 1, 2, LR, B1, B2, EPS, WD)
    m, v, _, _ = (x.reshape(-1) if x.numel() == n else x for x in P.decode(s1, n))
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    fine[[5, 130, 140]] = False
    assert bool(torch.isnan(m[[5, 130]]).all()) and bool(torch.isfinite(m[fine]).all()) and bool(torch.isfinite(w1[fine]).all())
    ref, m64, v64 = P.adam(w, state, torch.where(fine, g, 0.0), 1.0, 2, LR, B1, B2, EPS, WD)
    first = torch.arange(n, device="cuda") < 128  # (3e38 squared is infinite in fp32: out of v's maximum, in m's)
    assert bool(((m - m64.view(-1)).abs()[fine & first] <= 2.0**-3 * m64.view(-1).abs()[fine & first] + 1e-4).all())
    assert bool(((v - v64.view(-1)).abs()[fine] <= 2.0**-4 * v64.view(-1).abs()[fine] + 2.0**-18 * v64.max()).all())


@pytest.mark.parametrize("dtype", [bf.BF_FP32, bf.BF_BF16])
@pytest.mark.parametrize("c", [1.0, 4.0])
@pytest.mark.parametrize("zero", [True, False])
def test_a_second_moment_that_overflows_stays_infinite(dtype, c, zero):
    """Gradients whose square is infinite in fp32, in the first step only: from then on their weights move by the weight decay alone, as on fp32 moments, and their
    neighbours step to the same bits as beside elements whose moments are zero.  (A resting weight is one product and one sum a step: 2^-23 of it and a little.)"""
    n, t0 = 1001, 1 if zero else 4
    places = torch.tensor([40, 43, 127, 200] + list(range(384, 512)) + [n - 1], device="cuda")  # alone, two of four neighbours, a whole block, the last
    sign = torch.where(places % 3 == 0, -1.0, 1.0)
    out = []
    for big in (1e25, 0.0):
        (w, state, g, low, full, guarded), = _make([n], dtype, 13, odd=False, zero=zero)
        m0, v0, um, uv = P.decode(state, n)
        gone = torch.zeros_like(m0).view(-1)
        gone[places] = 1
        state.copy_(P.encode(torch.where(gone > 0, 0.0, m0.view(-1))[:n], torch.where(gone > 0, 0.0, v0.view(-1))[:n]))
        g = (g * 1e-3).contiguous()
        coef, steps = torch.full((1,), c, device="cuda"), []
        kept = [w.clone(), *(x.view(-1)[:n].float().contiguous() for x in P.decode(state, n)[:2])]
        for t in range(t0, t0 + 5):
            first = g.clone()
            first[places] = (big * sign if t == t0 else 1e-3 * sign * (big > 0)).to(DT[dtype])
            bf.bf_op_adam8(dtype, [(w, state, first, low)], coef, 5, t, LR, B1, B2, EPS, WD)
            bf.bf_op_adam_clipped([(*kept, first.float(), None)], coef, t, LR, B1, B2, EPS, WD)
            m, v = (torch.empty(n, dtype=DT[dtype], device="cuda") for _ in range(2))
            bf.bf_op_adam8_moments(dtype, [(state, m, v)])
            steps.append([x.clone() for x in (w, low, state, m, v, kept[0])])
        assert bool((guarded[state.numel():] == 0xA5).all())
        out.append(steps)
    rests = torch.zeros(n, dtype=torch.bool, device="cuda")
    rests[places] = True
    codes = torch.zeros((n + 127) // 128 * 128, dtype=torch.bool, device="cuda")
    codes[:n] = rests
    codes = torch.stack([codes.view(-1, 128)] * 2, 1).view(-1)
    before = _make([n], dtype, 13, odd=False, zero=zero)[0][0].double()
    for k, (a, b) in enumerate(zip(*out)):
        w, low, state, m, v, fp32 = a
        assert all(torch.equal(x[~rests], y[~rests]) for x, y in zip((w, low, m, v), (b[0], b[1], b[3], b[4]))), k
        assert torch.equal(state[: codes.numel()][~codes], b[2][: codes.numel()][~codes]) and torch.equal(state[codes.numel():], b[2][codes.numel():]), k
        assert bool((m[rests] == 0).all()) and bool((v[rests] == float("inf")).all()), k
        ref = before[rests] * (1 - LR * WD) ** (k + 1)
        for got in (w, fp32):
            assert bool(((got[rests].double() - ref).abs() <= (k + 1) * 2.0**-22 * ref.abs()).all()), k
        assert torch.equal(low, w.bfloat16())
    # and a NaN ends it
    m, v = (torch.empty(n, device="cuda") for _ in range(2))
    w, state = out[0][-1][0], out[0][-1][2]
    bf.bf_op_adam8(dtype, [(w, state, torch.full((n,), float("nan"), dtype=DT[dtype], device="cuda"), None)], torch.ones(1, device="cuda"), 5, 9, LR, B1, B2, EPS, WD)
    bf.bf_op_adam8_moments(bf.BF_FP32, [(state, m, None)])
    assert bool(torch.isnan(m).all()) and bool(torch.isnan(w).all())


def test_captured():
    """A captured step repeats its seed and step; replays are what eager calls with them give."""
    tensors = _make(SIZES, bf.BF_FP32, 10)
    other = _make(SIZES, bf.BF_FP32, 10)
    coef = torch.ones(1, device="cuda")
    bf.bf_op_adam8(bf.BF_FP32, [x[:4] for x in other], coef, 3, 4, LR, B1, B2, EPS, WD)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        bf.bf_op_adam8(bf.BF_FP32, [x[:4] for x in tensors], coef, 3, 4, LR, B1, B2, EPS, WD)
    for k in range(3):
        graph.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for x, y in zip(tensors, other) for a, b in zip(x[:2], y[:2])), k
        bf.bf_op_adam8(bf.BF_FP32, [x[:4] for x in other], coef, 3, 4, LR, B1, B2, EPS, WD)


def test_a_training_step_in_8_bits():
    """The run of them as they are used: forms of activations, weights and gradients, forward, backward, the gradient norm, the step, and the next step's
    forms from the new weights; each against what it is given, and the whole twice, eager and captured, to the same bits."""
    T, h, f = 70, 256, 384
    g = torch.Generator("cuda").manual_seed(2)
    x = torch.randn(T, h, generator=g, device="cuda").bfloat16()
    dy = (torch.randn(T, f, generator=g, device="cuda") * 1e-2).bfloat16()
    w_start = torch.randn(h, f, generator=g, device="cuda") * h**-0.5

    def buffers():
        b = {"w": w_start.clone(), "lp": w_start.bfloat16(), "state": torch.zeros(bf.bf_op_adam8_state_bytes(h * f), dtype=torch.uint8, device="cuda"),
             "y": torch.zeros(T, f, dtype=torch.bfloat16, device="cuda"), "dx": torch.zeros(T, h, dtype=torch.bfloat16, device="cuda"), "dw": torch.zeros(h, f, device="cuda"),
             "out": torch.zeros(2, device="cuda")}
        for name, r, c in (("x", T, h), ("lp", h, f), ("dy", T, f)):
            for k, (rows, n) in (("a", (r, c)), ("d", (c, r))):
                b[name + k] = (torch.zeros(rows, bf.bf_op_fp8_row_bytes(n), dtype=torch.uint8, device="cuda"),
                               torch.zeros(bf.bf_op_fp8_scale_elems(rows, n), dtype=torch.uint8, device="cuda"))
        b["work"] = torch.empty(1 << 22, dtype=torch.uint8, device="cuda")
        return b

    def step(b, t):
        bf.bf_op_fp8_quantize(1, 0, T, h, x, *b["xa"], *b["xd"])
        bf.bf_op_fp8_quantize(1, 0, h, f, b["lp"], *b["lpa"], *b["lpd"])
        bf.bf_op_fp8_gemm(0, 0, 1, T, f, h, *b["xa"], *b["lpd"], b["y"], work=b["work"])
        bf.bf_op_fp8_quantize(1, 1, T, f, dy, *b["dya"], *b["dyd"])
        bf.bf_op_fp8_gemm(1, 0, 1, T, h, f, *b["dya"], *b["lpa"], b["dx"], work=b["work"])
        bf.bf_op_fp8_gemm(0, 1, 0, h, f, T, *b["xd"], *b["dyd"], b["dw"], work=b["work"])
        bf.bf_op_grad_norm(bf.BF_FP32, [b["dw"].view(-1)], 0.5, b["out"], work=b["work"])
        bf.bf_op_adam8(bf.BF_FP32, [(b["w"].view(-1), b["state"], b["dw"].view(-1), b["lp"].view(-1))], b["out"][1:], 11, t, LR, B1, B2, EPS, WD)

    b = buffers()
    for t in (1, 2, 3):
        w0, lp0, s0 = b["w"].clone(), b["lp"].clone(), b["state"].clone()
        step(b, t)
        v = lambda m, fmt: P.values(*P.form(m, fmt), m.shape[1])  # noqa: E731
        y, dx, dw = v(x, 0) @ v(lp0.t(), 0).t(), v(dy, 1) @ v(lp0, 0).t(), v(x.t(), 0) @ v(dy.t(), 1).t()
        for got, ref, tol in ((b["y"], y, 2.0**-8), (b["dx"], dx, 2.0**-8), (b["dw"], dw, 2.0**-20)):
            assert float((got.double() - ref).norm() / ref.norm()) <= tol
        norm = float(b["dw"].double().norm())
        assert abs(float(b["out"][0]) - norm) <= 2.0**-22 * norm and norm > 0.5
        _check([(b["w"].view(-1), b["state"], b["dw"].view(-1), b["lp"].view(-1), torch.full((5,), float("nan")), b["state"])], [(w0.view(-1), s0)], float(b["out"][1]), 11, t)
    c = buffers()
    graphs = []
    for t in (1, 2, 3):
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            step(c, t)
        graphs.append(graph)
    for graph in graphs:
        graph.replay()
        torch.cuda.synchronize()
    assert all(torch.equal(b[k], c[k]) for k in ("w", "lp", "state", "y", "dx", "dw", "out"))


def test_a_tensor_past_a_table_entry():
    """More than 2^30 elements in one tensor: the elements around the border and at the end are stepped like any others."""
    n = (1 << 30) + 777
    w, g = torch.zeros(n, device="cuda"), torch.zeros(n, dtype=torch.bfloat16, device="cuda")
    state = torch.zeros(bf.bf_op_adam8_state_bytes(n), dtype=torch.uint8, device="cuda")
    parts = [slice(0, 1280), slice((1 << 30) - 640, (1 << 30) + 640), slice((1 << 30) + 128 * 5, n)]
    for p in parts:
        w[p], g[p] = torch.randn_like(w[p]), torch.randn_like(w[p]).bfloat16()
    before = [(w[p].clone(), g[p].clone()) for p in parts]
    bf.bf_op_adam8(bf.BF_BF16, [(w, state, g, None)], torch.ones(1, device="cuda"), 5, 1, LR, B1, B2, EPS, WD)
    r = P.randoms(5, 1, 0, 1, "cuda")  # (the key's way is that of the other tests: here only places matter)
    assert len(r) == 2
    m, v = torch.empty(n, dtype=torch.bfloat16, device="cuda"), torch.empty(n, dtype=torch.bfloat16, device="cuda")
    bf.bf_op_adam8_moments(bf.BF_BF16, [(state, m, v)])
    key = 0
    for word in (5, 0, 1):
        key = P.mix(key ^ word)
    key = P.mix(key ^ 0)
    for p, (w0, g0) in zip(parts, before):
        zero = torch.zeros(-(-w0.numel() // 128) * 258, dtype=torch.uint8, device="cuda")
        ref, m64, v64 = P.adam(w0, zero, g0, 1.0, 1, LR, B1, B2, EPS, WD)
        assert bool(((w[p].double() - ref).abs() <= 2.0**-23 * w0.abs() + LR * 2.0**-18).all())
        h = P.mix((torch.arange(p.start, p.stop, device="cuda") + key) % 2**32)
        for got, x, top, low, bits, rnd in ((m[p], m64, 448.0, -6, 3, h % 65536), (v[p], v64, 31744.0, 0, 4, h // 65536)):
            x = x.view(-1)[: w0.numel()]
            blocks = torch.nn.functional.pad(x.abs(), (0, -x.numel() % 128)).view(-1, 128)
            unit = P.power(P.exponent(blocks.amax(1), top)).repeat_interleave(128)[: x.numel()]
            y = x.abs() / unit
            step = P.power((torch.frexp(y)[1] - 1).clamp(min=low) - bits)
            part = y / step
            code = torch.floor(part) + (torch.floor((part - torch.floor(part)) * 65536) + rnd >= 65536)
            code = torch.where((x != 0) & (code == 0) & (low == 0), torch.ones_like(code), code)
            off = got.double().abs() / unit != code * step
            assert float(off.double().mean()) <= 2e-3  # (moments a rounding away from the next code)
    fine = torch.ones(n, dtype=torch.bool, device="cuda")
    for p in parts:
        fine[p] = False
    assert not bool(w[fine].any()) and not bool(m[fine].any())
