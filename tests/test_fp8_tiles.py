"""Which kernel an 8-bit product's shape takes (without a device), and every such kernel against the definition in fp64: all lengths of its main loop's end, ragged edges, the formats, the
epilogues, and slices of the contraction that meet in planes.  Tolerances are those of test_gpu_fp8: a sum over s slices has s - 1 roundings more, 15 at most of the 32 allowed there."""
import ctypes

import pytest
import torch

import fp8_plain as P
import paper_2211_05953_amd as bf

DT = {bf.BF_BF16: torch.bfloat16, bf.BF_FP32: torch.float32}

# (type, M, N, K): (edge of the tile, waves, slices)
SHAPES = {
    # 8-bit instructions; 128 x 128 has four stages, so its loop runs from four blocks on and ends with none to three
    (1, 33, 70, 200): (64, 4, 1), (1, 5, 300, 8200): (64, 4, 8), (1, 2000, 1030, 384): (128, 4, 1),
    (1, 2000, 1030, 512): (128, 4, 1), (1, 1990, 1029, 600): (128, 4, 1), (1, 2000, 1030, 768): (128, 4, 1), (1, 1990, 1032, 890): (128, 4, 1), (1, 2000, 1032, 1024): (128, 4, 1),
    (1, 2000, 1029, 1150): (128, 4, 1), (1, 2048, 2048, 8192): (128, 4, 1),
    (1, 640, 2301, 16380): (128, 4, 2), (1, 200, 2304, 16384): (128, 4, 4), (1, 100, 2999, 12200): (128, 4, 8), (1, 200, 768, 20480): (128, 4, 16),
    (1, 2301, 4099, 128): (256, 8, 1), (1, 2304, 4096, 256): (256, 8, 1), (1, 2301, 4100, 300): (256, 8, 1), (1, 2304, 4096, 1920): (256, 8, 1),
    (1, 2304, 4096, 2048): (256, 8, 1), (1, 2301, 4099, 2100): (256, 8, 1), (1, 2304, 4096, 3200): (256, 4, 1), (1, 2301, 4099, 3300): (256, 4, 1),
    (1, 2000, 2301, 12200): (256, 8, 2), (1, 1000, 2304, 51200): (256, 8, 4), (1, 200, 5000, 32768): (256, 8, 8),
    # widened operands
    (0, 33, 70, 200): (64, 4, 1), (0, 5, 300, 8200): (64, 4, 8),
    (0, 2000, 2304, 128): (128, 4, 1), (0, 1990, 2301, 200): (128, 4, 1), (0, 2000, 2304, 384): (128, 4, 1), (0, 2048, 2048, 8192): (128, 4, 1),
    (0, 1000, 2301, 16380): (128, 4, 2), (0, 200, 4096, 12288): (128, 4, 4), (0, 200, 2303, 12200): (128, 4, 8), (0, 100, 2304, 20480): (128, 4, 16),
    (0, 2500, 5000, 128): (256, 8, 1), (0, 2501, 4999, 200): (256, 8, 1), (0, 2500, 5000, 384): (256, 8, 1),
    (0, 1000, 2999, 25600): (256, 8, 4), (0, 200, 8192, 40960): (256, 8, 8),
}


def test_what_a_shape_runs_on():
    for shape, want in SHAPES.items():
        assert bf.bf_op_fp8_gemm_tile(*shape) == want, (shape, bf.bf_op_fp8_gemm_tile(*shape))
    for dtype, tiles in ((1, {(64, 4), (128, 4), (256, 8), (256, 4)}), (0, {(64, 4), (128, 4), (256, 8)})):
        assert {v[:2] for k, v in SHAPES.items() if k[0] == dtype} == tiles


def test_the_scratch_is_the_slices_planes():
    cut = set()
    for dtype in (0, 1):
        for M in (1, 100, 1000, 2304, 8192):
            for N in (1, 64, 1003, 4096):
                for K in (1, 128, 300, 2048, 8192, 20000, 1 << 17):
                    edge, waves, slices = bf.bf_op_fp8_gemm_tile(dtype, M, N, K)
                    assert bf.bf_op_fp8_gemm_work_bytes(dtype, M, N, K) == (4 * slices * M * N if slices > 1 else 0)
                    assert 1 <= slices <= min(16, -(-K // 128))
                    cut.add(slices)
    assert cut >= {1, 2, 4, 8, 16}


def test_no_tile_for_what_is_refused():
    for bad in ((7, 1, 1, 1), (-1, 1, 1, 1), (1, 0, 1, 1), (1, 1, -5, 1), (0, 1, 1, 0), (0, (1 << 21) + 1, 1, 1), (0, 1, 1, (1 << 21) + 1)):
        assert bf.bf_op_fp8_gemm_tile(*bad) is None
    lib, out = bf.load(), [ctypes.c_int(5) for _ in range(3)]
    assert lib.bf_op_fp8_gemm_tile(1, 0, 1, 1, *[ctypes.byref(o) for o in out]) == 0 and [o.value for o in out] == [0, 0, 0]
    assert lib.bf_op_fp8_gemm_tile(1, 1, 1, 1, None, *[ctypes.byref(o) for o in out[1:]]) == 0


def _operand(rows, n, fmt, seed):
    g = torch.Generator("cuda").manual_seed(seed)
    x = torch.randn(rows, n, generator=g, device="cuda") * torch.exp2(2 * torch.randn(rows, 1, generator=g, device="cuda"))
    q, scale = P.form(x, fmt)
    return (P.codes(q, fmt).contiguous(), scale), P.values(q, scale, n)


@pytest.mark.gpu
@pytest.mark.parametrize("fa,fb", [(0, 0), (0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("shape", sorted(SHAPES), ids=lambda s: "-".join(map(str, s)))
def test_each_tile(shape, fa, fb):
    dtype, M, N, K = shape
    assert bf.bf_op_fp8_gemm_tile(*shape) == SHAPES[shape]
    A, a = _operand(M, K, fa, 1)
    B, b = _operand(N, K, fb, 2)
    ref, mag = a @ b.t(), a.abs() @ b.abs().t()
    del a, b
    g = torch.Generator("cuda").manual_seed(3)
    size = float(ref.std())
    bias = torch.randn(N, generator=g, device="cuda") * size
    res = (torch.randn(M, N, generator=g, device="cuda") * size).to(DT[dtype])
    flat = torch.full((M * N + 64,), float("nan"), dtype=DT[dtype], device="cuda")
    out = flat[: M * N].view(M, N)

    def run(*terms, **k):
        bf.bf_op_fp8_gemm(fa, fb, dtype, M, N, K, *A, *B, out, **k)
        want, extra = ref, 0.0
        for t in terms:
            want, extra = want + t.double(), extra + t.double().abs()
        if terms:
            extra = extra + ref.abs()
        if dtype == bf.BF_BF16:
            tol = 2.0**-8 * want.abs() + (2.0**-12 + K / 128 * 2.0**-23) * mag + 2.0**-22 * extra
        else:
            tol = (K / 32 + 32) * 2.0**-24 * mag + 2.0**-22 * extra + 2.0**-24 * want.abs()
        off = (out.double() - want).abs()
        assert bool((off <= tol).all()), float((off / tol).max())  # (NaN is not below)
        assert bool(torch.isnan(flat[M * N:]).all())

    run()
    first = out.clone()
    run()
    assert torch.equal(first, out)  # the same bits again
    run(bias, bias=bias)
    run(res, R=res)
    out.copy_(res)
    run(bias, res, bias=bias, R=out)
    if dtype == bf.BF_FP32:
        out.copy_(res)
        run(res, accumulate=1)
        out.copy_(res)
        run(res, res, bias, bias=bias, R=res, accumulate=1)
