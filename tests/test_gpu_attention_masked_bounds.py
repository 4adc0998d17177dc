"""Masked attention against fp64 at tighter bounds, element by element: any cap, and score gradients of rows with few keys.

u: the storage type's rounding (2^-8, 2^-24); u_p: that of probabilities and score gradients as they enter a product, u on the matrix
cores, none on the plain kernels, which keep them in fp32 (up to four tokens without shared heads, heads over 128, on request).
  score   eps_s = (d + 8) 2^-24 scale S (S: largest sum of |q||k|) + slope S_seq 2^-21 + the cap's: on the bf16 matrix cores up to a
          cap of 2^10, 2^-21 of the cap; else 2^-20 of the largest score (tanh to 3 ulp, three products around it)
  P       e_p = 2 eps_s + 2^-20 of itself;   a sum of n terms e_n = (n + 64) 2^-24 of the terms' sizes
  dP      e_dp = (d + 8) 2^-24 |dctx||V|
  delta   in bf16 the sum of P dP as they are, and not of dctx ctx, whose rounding would enter every score gradient of the row:
          P (|dP| (e_p + e_n) + e_dp);  in fp32 dctx ctx: |dctx| (error of ctx) + (d + 8) 2^-24 |dctx||ctx|
  dS      |dS| (u_p + e_p + 2^-22) + P slack (error of delta + e_dp) + P |dP - delta| (error of slack) where scores are capped
  slack   1 - tanh^2 x of an x that is off by at most x_e = (d + 8) 2^-24 scale S / cap + 2^-22 |x|: it falls with |x|, so it lies between its
          values at |x| - x_e (or 0) and |x| + x_e; and 2^-19 for the tanh and its square
  ctx     P |V| (u_p + e_p + e_n) + u |ctx|;   dq, dk, dv likewise from theirs"""
import math

import pytest
import torch

import paper_2211_05953_amd as bf
from test_gpu_attention_masked import BF16, FP32, Case, test_what_a_mask_hides_reaches_no_result as _hidden

pytestmark = pytest.mark.gpu


class Tight(Case):
    def __init__(self, *args, kernels=bf.BF_KERNELS_AUTO, **kw):
        super().__init__(*args, kernels=kernels, **kw)
        self.matrix = kernels == bf.BF_KERNELS_AUTO and self.d <= 128 and (self.S > 4 or self.H != self.KV)

    def want(self):
        G, S, d = self.H // self.KV, self.S, self.d
        q, dc = self.heads(self.q, self.H), self.heads(self.dctx, self.H)
        k, v = (self.heads(x, self.KV).repeat_interleave(G, 1) for x in (self.k, self.v))
        low = self.dtype == BF16
        scale, u = 1 / math.sqrt(d), 2.0**-8 if low else 2.0**-24
        u_p = u if self.matrix else 0.0
        ok = self.allowed()[:, None]
        s = q @ k.transpose(2, 3) * scale
        eps_s = (d + 8) * 2.0**-24 * scale * float((q.abs() @ k.abs().transpose(2, 3)).max())
        slack = torch.ones_like(s)
        if self.cap:
            x = (s / self.cap).abs()
            x_e = eps_s / self.cap + 2.0**-22 * x
            e_slack = torch.cosh((x - x_e).clamp(0, 300)) ** -2 - torch.cosh((x + x_e).clamp(max=300)) ** -2 + 2.0**-19
            t = torch.tanh(s / self.cap)
            slack, s = torch.cosh(x.clamp(max=300)) ** -2, self.cap * t
            eps_s += self.cap * 2.0**-21 if low and self.matrix and self.cap <= 1024 else float(s.abs().max()) * 2.0**-20
        if self.slope is not None:
            i = torch.arange(S, device="cuda")
            s = s - self.slope.double()[:, None, None] * (i[:, None] - i).abs()
            eps_s += float(self.slope.max()) * S * 2.0**-21
        s = s.masked_fill(~ok, -math.inf)
        lse = torch.logsumexp(s, 3)
        p = torch.where(ok, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
        e_p, e_n = 2 * eps_s + 2.0**-20, (S * G + 64) * 2.0**-24
        ctx = p @ v
        b_ctx = ((p @ v.abs()) * (u_p + e_p + e_n) + u * ctx.abs()) * 1.01
        dp = dc @ v.transpose(2, 3)
        e_dp = (d + 8) * 2.0**-24 * (dc.abs() @ v.abs().transpose(2, 3))
        delta = (p * dp).sum(3, keepdim=True)
        if low:
            e_delta = (p * (dp.abs() * (e_p + e_n) + e_dp)).sum(3, keepdim=True)
        else:
            e_delta = (dc.abs() * b_ctx).sum(3, keepdim=True) + (d + 8) * 2.0**-24 * (dc.abs() * ctx.abs()).sum(3, keepdim=True)
        one = ok.sum(3, keepdim=True) == 1
        raw = torch.where(one, 0.0, p * (dp - delta) * slack)
        e_raw = raw.abs() * (u_p + e_p + 2.0**-22) * 1.01 + p * slack * (e_delta + e_dp) + (p * ((dp - delta).abs() + e_delta + e_dp) * e_slack if self.cap else 0)
        e_raw = torch.where(one, 0.0, e_raw)
        kv = lambda x: x.reshape(self.B, self.KV, G, S, d).sum(2)  # noqa: E731
        dq, dk, dv = raw @ k * scale, kv(raw.transpose(2, 3) @ q * scale), kv(p.transpose(2, 3) @ dc)
        b_dq = scale * ((e_raw + e_n * raw.abs()) @ k.abs()) + u * dq.abs() * 1.01
        b_dk = kv(scale * ((e_raw + e_n * raw.abs()).transpose(2, 3) @ q.abs())) + u * dk.abs() * 1.01
        b_dv = kv((p * (u_p + e_p + e_n) * 1.01).transpose(2, 3) @ dc.abs()) + u * dv.abs() * 1.01
        whole = lambda x: x.transpose(1, 2).reshape(self.B, S, -1)  # noqa: E731
        return {"ctx": (whole(ctx), whole(b_ctx)), "lse": (lse, torch.full_like(lse, eps_s + 2.0**-20) + 2.0**-22 * lse.abs().nan_to_num(0, 0, 0)),
                "dq": (whole(dq), whole(b_dq)), "dk": (whole(dk), whole(b_dk)), "dv": (whole(dv), whole(b_dv))}


# both sides of the cap from which the tanh takes its exact form, caps that are none, caps that fp32 cannot invert
CAPS = [1e-42, 1e-39, 1e-3, 1.0, 50.0, 1000.0, 1025.0, 1e4, 1e6, 1e20, 3e38]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("B,S,H,KV,d,more", [(2, 130, 4, 2, 64, dict(docs=40, pad=1)), (1, 150, 2, 1, 128, dict(slopes=1, big=4.0)), (1, 90, 2, 2, 72, dict(offset=1, prefix=1)),
                                             (1, 60, 3, 3, 40, dict(causal=0, offset=3)), (3, 140, 72, 36, 64, dict())])
def test_any_cap(dtype, B, S, H, KV, d, more, cap):
    Tight(dtype, B, S, H, KV, d, cap=cap, **more).check()


PLAIN = dict(kernels=bf.BF_KERNELS_PLAIN)


# rows of two, three, a few keys; one, two and three chunks of 64 keys on the plain kernels; heads of more than 128
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("mask", [dict(), dict(causal=0), dict(docs=4), dict(docs=4, slopes=1, cap=5.0, big=4.0), dict(prefix=1, pad=1, cap=1e6)])
@pytest.mark.parametrize("B,S,H,KV,d,more", [(3, 2, 4, 4, 64, {}), (3, 3, 4, 4, 128, {}), (3, 4, 4, 4, 33, {}), (3, 2, 4, 2, 64, {}), (3, 4, 4, 1, 128, {}), (2, 9, 4, 4, 64, {}),
                                             (2, 40, 2, 1, 160, {}), (1, 64, 2, 2, 64, PLAIN), (1, 65, 2, 1, 64, PLAIN), (1, 130, 2, 2, 72, PLAIN), (2, 150, 4, 2, 64, {}),
                                             (1, 300, 2, 2, 128, {})])
def test_score_gradients_of_few_keys(dtype, B, S, H, KV, d, more, mask):
    Tight(dtype, B, S, H, KV, d, **mask, **more).check()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cap", CAPS)
@pytest.mark.parametrize("B,S,H,KV,d,more", [(1, 3, 2, 2, 64, {}), (1, 40, 2, 1, 160, {})])
def test_any_cap_on_the_plain_kernels(dtype, B, S, H, KV, d, more, cap):
    Tight(dtype, B, S, H, KV, d, cap=cap, **more).check()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cap", CAPS)
def test_scores_of_zero_under_any_cap(dtype, cap):
    c = Tight(dtype, 1, 70, 2, 1, 64, cap=cap)
    c.q[:, ::2] = 0.0
    c.check()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("d", [64, 128])
def test_what_a_mask_hides_under_a_large_cap(dtype, d):
    _hidden(dtype, math.nan, d, dict(causal=1, cap=1e6))
    _hidden(dtype, math.inf, d, dict(causal=0, cap=1e6, slopes=1))


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("cap", [0.0, 1.0, 1e4])
def test_scores_of_zero_under_the_largest_scale(dtype, cap):
    """2^126: no product with a score of 0 is a NaN.  Keys of zeros, so every key has the same share: ctx and dv are means, dq is 0."""
    B, S, H, KV, d = 1, 70, 2, 2, 64
    c = Case(dtype, B, S, H, KV, d, causal=0, packed=0, cap=cap)
    c.cfg.scale = 2.0**126
    c.k.zero_()
    ctx, lse, dq, dk, dv = c.run()
    torch.cuda.synchronize()
    u = 2.0**-8 if dtype == BF16 else 2.0**-22
    for got, x in ((ctx, c.v), (dv, c.dctx)):
        mean, size = x.double().mean(1, keepdim=True), x.double().abs().mean(1, keepdim=True)
        # P rounded once, and the result; sums of 70 terms
        assert float(((got.double() - mean).abs() - 2.1 * u * size - 2.0**-17 * size).max()) <= 0
    assert float((lse.double() - math.log(S)).abs().max()) <= 2.0**-20 and not dq.any()


# dozens of tiles in a row: several steps of the maximum, spans that begin and end far from their rows, prefixes longer than a workgroup's keys
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("B,S,H,KV,d,mask", [(1, 2048, 4, 2, 128, dict(docs=300, pad=1)), (1, 4100, 1, 1, 64, dict()), (1, 3001, 4, 1, 80, dict(cap=50.0, big=3.0)),
                                             (2, 1500, 2, 2, 128, dict(prefix=1, slopes=1)), (1, 2500, 2, 1, 64, dict(causal=0, docs=900, slopes=1)),
                                             (1, 1200, 1, 1, 192, dict(docs=500, cap=30.0))])
def test_long_sequences(dtype, B, S, H, KV, d, mask):
    Tight(dtype, B, S, H, KV, d, **mask).check()


@pytest.mark.parametrize("dtype,S", [(BF16, 1 << 20), (FP32, 1 << 19)])
def test_offsets_past_32_bits(dtype, S):
    """Packed rows of 5.4 GB: documents of some hundred tokens at the beginning, across 2^32 bytes and at the end against fp64, each by itself."""
    H, KV, d, t = 32, 4, 64, torch.bfloat16 if dtype == BF16 else torch.float32
    widths = (H * d, KV * d, KV * d)
    ld = sum(widths)
    g = torch.Generator("cuda").manual_seed(3)
    doc = (torch.rand(1, S, generator=g, device="cuda") < 1 / 200).int().cumsum(1).int()
    qkv, dqkv = (torch.empty(1, S, ld, dtype=t, device="cuda") for _ in range(2))
    ctx, dctx = (torch.empty(1, S, H * d, dtype=t, device="cuda") for _ in range(2))
    for x in (qkv, dctx):
        for part in x.split(1 << 17, 1):
            part.copy_(torch.randn(part.shape, generator=g, device="cuda"))
    (q, k, v), grads = qkv.split(widths, 2), dqkv.split(widths, 2)
    cfg = bf.make_attn_config(dtype, 1, S, H, KV, d, ld_q=ld, ld_k=ld, ld_v=ld)
    spans = torch.empty(bf.bf_op_attention_spans_elems(1, S), dtype=torch.int32, device="cuda")
    bf.bf_op_attention_spans(1, S, 1, doc, None, spans)
    lse = torch.empty(1, H, S, device="cuda")
    bf.bf_op_attention_masked_fwd(cfg, q, k, v, spans, None, ctx, lse)
    bf.bf_op_attention_masked_bwd(cfg, q, k, v, spans, None, ctx, lse, dctx, *grads)
    past = 2**32 // (ld * qkv.element_size())
    for at in (0, past, S - 1):
        one = (doc[0] == doc[0, at]).nonzero()[:, 0]
        a, b = int(one[0]), int(one[-1]) + 1
        c = Tight(dtype, 1, b - a, H, KV, d, packed=0)
        for mine, whole in ((c.q, q), (c.k, k), (c.v, v), (c.dctx, dctx)):
            mine.copy_(whole[:, a:b])
        want = c.want()
        for name, x in zip(("ctx", "dq", "dk", "dv"), (ctx, *grads)):
            w, bound = want[name]
            assert float(((x[:, a:b].double() - w).abs() - bound).max()) <= 1e-30, (name, a, b)
        w, bound = want["lse"]
        assert float(((lse[:, :, a:b].double() - w).abs() - bound).max()) <= 0
