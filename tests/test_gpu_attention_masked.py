"""Masked attention against fp64, element by element.

u is the storage type's largest rounding, 2^-8 for bf16 and 2^-24 for fp32; on the bf16 matrix cores probabilities and their
gradients are rounded by u too as they enter a product.  A score is off by eps_s = (S_head + 8) 2^-24 scale S (S: the largest
sum of |q||k|), plus 2^-21 of what cap and bias add (tanh and the bias in fp32, |bias| up to slope S_seq); a probability by
2 eps_s + 2^-20 of itself (exp, log-sum-exp); a sum of n terms by (n + 64) 2^-24 of the terms' sizes.  From these, with
A = |.|:
  ctx  (P A(V)) (u + e_p + e_n) + u A(ctx)
  dS   A(dS) (2 u + e_p) + P slack (error of delta + error of dP) + P A(dP - delta) 2^-19 where scores are capped
  dq   scale (error of dS) A(K) + e_n A(dS) A(K) scale + u A(dq), dk likewise;  dv (P (u + e_p + e_n))^T A(dctx) + u A(dv)
delta is the sum of dctx ctx over a head's elements, with ctx as stored."""
import math

import pytest
import torch

import paper_2211_05953_amd as bf

pytestmark = pytest.mark.gpu
TYPES = {bf.BF_FP32: torch.float32, bf.BF_BF16: torch.bfloat16}
BF16, FP32 = bf.BF_BF16, bf.BF_FP32


class Case:
    """Inputs on the device: q, k, v side by side in a token's row with gaps of NaN, or tensors of their own."""

    def __init__(self, dtype, B, S, H, KV, d, causal=1, docs=0, pad=0, prefix=0, slopes=0, cap=0.0, packed=1, offset=0, seed=0, big=1.0, kernels=bf.BF_KERNELS_AUTO):
        self.__dict__.update(dtype=dtype, B=B, S=S, H=H, KV=KV, d=d, causal=causal, cap=cap, packed=packed)
        g = torch.Generator("cuda").manual_seed(1000 + seed)
        self.t = TYPES[dtype]
        normal = lambda *s: torch.randn(s, generator=g, device="cuda")  # noqa: E731
        gap = 8 if offset == 0 else 3
        rows = (H * d, KV * d, KV * d)
        self.ld = sum(rows) + gap if packed else 0

        def hold(widths, x=None):
            """A buffer of NaN with rows of the given widths in it, as views."""
            if packed:
                flat = torch.full((B * S * (sum(widths) + gap) + 64 + offset,), math.nan, dtype=self.t, device="cuda")
                whole = flat[offset:offset + B * S * (sum(widths) + gap)].view(B, S, -1)
                parts = list(whole[..., :sum(widths)].split(widths, 2))
                return [flat], parts
            flats = [torch.full((B * S * w + 64 + offset,), math.nan, dtype=self.t, device="cuda") for w in widths]
            return flats, [f[offset:offset + B * S * w].view(B, S, w) for f, w in zip(flats, widths)]

        self.hold = hold
        self.rows = rows
        (self.q, self.k, self.v) = hold(rows)[1]
        for x, w, f in zip((self.q, self.k, self.v), rows, (big, 1.0, 1.0)):
            x.copy_(normal(B, S, w) * f)
        self.gap_o = H * d + (gap if packed else 0)
        self.flat_ctx, (self.ctx,) = hold((H * d,))
        _, (self.dctx,) = hold((H * d,))
        self.dctx.copy_(normal(B, S, H * d))
        self.doc = self.prefix = self.slope = None
        if docs or pad:
            self.doc = ((torch.rand(B, S, generator=g, device="cuda") < 1 / docs).int().cumsum(1) if docs else torch.zeros(B, S, device="cuda")).int().contiguous()
            if pad:
                self.doc[:, S - S // 5:] = -1
                self.doc[0, S // 3:S // 3 + 2] = -7
        if prefix:
            self.prefix = torch.randint(0, S + 3, (B,), generator=g, device="cuda").int()
            self.prefix[0] = -5 if B > 1 else self.prefix[0]
        if slopes:
            self.slope = 2.0 ** (-8.0 * torch.arange(1, H + 1, device="cuda") / H)
        self.cfg = bf.make_attn_config(dtype, B, S, H, KV, d, cap=cap, ld_q=self.ld, ld_k=self.ld, ld_v=self.ld, ld_ctx=self.gap_o if packed else 0,
                                       kernels=kernels)
        self.spans = torch.full((bf.bf_op_attention_spans_elems(B, S),), -1, dtype=torch.int32, device="cuda")

    def allowed(self):
        B, S = self.B, self.S
        i = torch.arange(S, device="cuda")
        ok = torch.ones(B, S, S, dtype=torch.bool, device="cuda")
        if self.causal:
            ok = (i[None, :, None] >= i[None, None, :]).expand(B, S, S)
            if self.prefix is not None:
                ok = ok | (i[None, None, :] < self.prefix[:, None, None])
        if self.doc is not None:
            run = torch.cat([torch.zeros_like(self.doc[:, :1]), (self.doc[:, 1:] != self.doc[:, :-1]).int().cumsum(1)], 1)
            ok = ok & (run[:, :, None] == run[:, None, :]) & (self.doc >= 0)[:, :, None]
        return ok

    def run(self, grads=True):
        bf.bf_op_attention_spans(self.B, self.S, self.causal, self.doc, self.prefix, self.spans)
        lse = torch.empty(self.B, self.H, self.S, device="cuda")
        bf.bf_op_attention_masked_fwd(self.cfg, self.q, self.k, self.v, self.spans, self.slope, self.ctx, lse)
        if not grads:
            return self.ctx, lse
        self.flat_grads, (dq, dk, dv) = self.hold(self.rows)
        work = torch.full((bf.bf_op_attention_masked_bwd_work_bytes(self.cfg),), 0xFF, dtype=torch.uint8, device="cuda")
        bf.bf_op_attention_masked_bwd(self.cfg, self.q, self.k, self.v, self.spans, self.slope, self.ctx, lse, self.dctx, dq, dk, dv, work=work)
        return self.ctx, lse, dq, dk, dv

    def heads(self, x, n):
        return x.double().reshape(self.B, self.S, n, self.d).transpose(1, 2)

    def want(self, clean=lambda x, n: x):
        """{name: (value, bound)}; clean(x, heads) may replace inputs (hidden infinities by zeros)."""
        G, S, d = self.H // self.KV, self.S, self.d
        q, dc = (clean(self.heads(x, self.H), self.H) for x in (self.q, self.dctx))
        k, v = (clean(self.heads(x, self.KV), self.KV).repeat_interleave(G, 1) for x in (self.k, self.v))
        scale, u = 1 / math.sqrt(d), 2.0**-8 if self.dtype == BF16 else 2.0**-24
        ok = self.allowed()[:, None]
        s = q @ k.transpose(2, 3) * scale
        eps_s = (d + 8) * 2.0**-24 * scale * float((q.abs() @ k.abs().transpose(2, 3)).max())
        slack = torch.ones_like(s)
        if self.cap:
            t = torch.tanh(s / self.cap)
            slack, s = 1 - t * t, self.cap * t
            eps_s += self.cap * 2.0**-21
        if self.slope is not None:
            i = torch.arange(S, device="cuda")
            s = s - self.slope.double()[:, None, None] * (i[:, None] - i).abs()
            eps_s += float(self.slope.max()) * S * 2.0**-21
        s = s.masked_fill(~ok, -math.inf)
        lse = torch.logsumexp(s, 3)
        p = torch.where(ok, torch.exp(s - torch.where(lse == -math.inf, 0.0, lse)[..., None]), 0.0)
        e_p, e_n = 2 * eps_s + 2.0**-20, (S * G + 64) * 2.0**-24
        ctx = p @ v
        b_ctx = (p @ v.abs()) * (u + e_p + e_n) * 1.01 + u * ctx.abs() * 1.01
        dp = dc @ v.transpose(2, 3)
        delta = (dc * ctx).sum(3, keepdim=True)
        raw = p * (dp - delta) * slack
        raw = torch.where(ok.sum(3, keepdim=True) == 1, 0.0, raw)
        e_delta = (dc.abs() * b_ctx).sum(3, keepdim=True) + (d + 8) * 2.0**-24 * (dc.abs() * ctx.abs()).sum(3, keepdim=True)
        e_dp = (d + 8) * 2.0**-24 * (dc.abs() @ v.abs().transpose(2, 3))
        e_raw = raw.abs() * (2 * u + e_p) * 1.01 + p * slack * (e_delta + e_dp) + (p * (dp - delta).abs() * 2.0**-19 if self.cap else 0)
        e_raw = torch.where(ok.sum(3, keepdim=True) == 1, 0.0, e_raw)
        dq = raw @ k * scale
        b_dq = scale * ((e_raw + e_n * raw.abs()) @ k.abs()) + u * dq.abs() * 1.01
        kv = lambda x: x.reshape(self.B, self.KV, G, S, d).sum(2)  # noqa: E731
        dk = kv(raw.transpose(2, 3) @ q * scale)
        b_dk = kv(scale * ((e_raw + e_n * raw.abs()).transpose(2, 3) @ q.abs())) + u * dk.abs() * 1.01
        dv = kv(p.transpose(2, 3) @ dc)
        b_dv = kv((p * (u + e_p + e_n) * 1.01).transpose(2, 3) @ dc.abs()) + u * dv.abs() * 1.01
        whole = lambda x: x.transpose(1, 2).reshape(self.B, S, -1)  # noqa: E731
        return {"ctx": (whole(ctx), whole(b_ctx)), "lse": (lse, torch.full_like(lse, eps_s + 2.0**-20) + 2.0**-22 * lse.abs().nan_to_num(0, 0, 0)),
                "dq": (whole(dq), whole(b_dq)), "dk": (whole(dk), whole(b_dk)), "dv": (whole(dv), whole(b_dv))}

    def check(self, grads=True, **kw):
        got = dict(zip(("ctx", "lse", "dq", "dk", "dv"), self.run(grads)))
        torch.cuda.synchronize()
        want = self.want(**kw)
        for name, x in got.items():
            w, b = want[name]
            x = x.double()
            if name == "lse":
                empty = w == -math.inf
                assert torch.equal(empty, x == -math.inf)
                x, w, b = (torch.where(empty, 0.0, y) for y in (x, w, b))
            assert bool(x.isfinite().all()), (name, "not finite", x.shape, (~x.isfinite()).nonzero()[:4].tolist())
            over = (x - w).abs() - b - 1e-30
            assert float(over.max()) <= 0, (name, float(over.max()), float((x - w).abs().max()), over.flatten().argmax().item(), over.shape)
        # what lies between the rows is as it was
        for flats, parts in [(self.flat_ctx, [got["ctx"]])] + ([(self.flat_grads, [got[n] for n in ("dq", "dk", "dv")])] if grads else []):
            assert sum(int(f.isnan().sum()) for f in flats) == sum(f.numel() for f in flats) - sum(p.numel() for p in parts)


def _spans_ref(c):
    ok = c.allowed()
    any_ = ok.any(2)
    lo = torch.where(any_, ok.int().argmax(2), 0)
    return torch.stack([lo, lo + ok.sum(2)], 2).int(), any_


@pytest.mark.parametrize("B,S", [(1, 1), (2, 3), (3, 63), (2, 64), (2, 65), (1, 1023), (2, 1024), (1, 1025), (2, 2500), (1, 6000)])
@pytest.mark.parametrize("docs,pad,prefix,causal", [(0, 0, 0, 1), (0, 0, 0, 0), (1, 0, 0, 1), (40, 1, 0, 1), (40, 1, 1, 1), (40, 0, 1, 0), (3000, 0, 0, 0), (0, 1, 1, 1)])
def test_spans(B, S, docs, pad, prefix, causal):
    c = Case(BF16, B, S, 1, 1, 8, causal, docs, pad, prefix)
    bf.bf_op_attention_spans(B, S, causal, c.doc, c.prefix, c.spans)
    want, any_ = _spans_ref(c)
    got = c.spans[:B * S * 2].view(B, S, 2)
    assert torch.equal(got[any_], want[any_])
    assert bool((got[~any_][:, 0] >= got[~any_][:, 1]).all())


SIZES = [(1, 1, 1, 1, 64), (2, 2, 2, 1, 64), (1, 63, 2, 2, 128), (2, 64, 1, 1, 64), (1, 65, 2, 1, 128), (3, 127, 2, 2, 64), (1, 129, 4, 1, 128), (2, 200, 4, 2, 80),
         (1, 257, 3, 3, 33), (2, 70, 2, 1, 8), (1, 90, 2, 2, 1), (1, 600, 2, 1, 64), (1, 520, 6, 2, 128), (1, 100, 1, 1, 200), (1, 40, 2, 1, 130)]
MASKS = [dict(causal=1), dict(causal=0), dict(causal=1, docs=30, pad=1), dict(causal=0, docs=30, pad=1, slopes=1), dict(causal=1, prefix=1, cap=20.0),
         dict(causal=1, docs=100, prefix=1, slopes=1, cap=5.0, big=4.0), dict(causal=0, docs=1), dict(causal=1, slopes=1, packed=0), dict(causal=0, pad=1, cap=30.0, packed=0)]


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("mask", MASKS)
@pytest.mark.parametrize("B,S,H,KV,d", SIZES)
def test_forward_and_backward(dtype, B, S, H, KV, d, mask):
    Case(dtype, B, S, H, KV, d, **mask).check()


# enough workgroups for the forms that share tiles between their waves
@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("mask", MASKS[:6])
@pytest.mark.parametrize("B,S,H,KV,d", [(3, 140, 72, 36, 64), (2, 140, 100, 25, 128), (2, 300, 64, 32, 72), (4, 100, 60, 60, 33)])
def test_large_launches(dtype, mask, B, S, H, KV, d):
    Case(dtype, B, S, H, KV, d, **mask).check()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("mask", MASKS[2:6])
@pytest.mark.parametrize("offset", [1, 3])
def test_rows_off_16_byte_alignment(dtype, mask, offset):
    Case(dtype, 2, 150, 4, 2, 64, offset=offset, **mask).check()
    Case(dtype, 1, 150, 2, 2, 96, offset=offset, **mask).check()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("mask", MASKS)
def test_plain_kernels(dtype, mask):
    Case(dtype, 2, 130, 4, 2, 64, kernels=bf.BF_KERNELS_PLAIN, **mask).check()


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("value", [math.nan, math.inf, -math.inf])
@pytest.mark.parametrize("d", [64, 128, 200])
@pytest.mark.parametrize("mask", [dict(causal=1), dict(causal=0), dict(causal=1, slopes=1, cap=10.0)])
def test_what_a_mask_hides_reaches_no_result(dtype, value, d, mask, H=4, KV=2):
    """Padding in the middle and at the end, and a document of its own, hold infinities or NaN in q, k, v and dctx: the other
    documents' results are those of zeros in their place."""
    c = Case(dtype, 2, 300, H, KV, d, docs=40, pad=1, **mask)
    c.doc[1, 100:130] = 5000
    bad = (c.doc < 0) | (c.doc == 5000)
    for x in (c.q, c.k, c.v, c.dctx):
        x[bad] = value
    ctx, lse, dq, dk, dv = c.run()
    torch.cuda.synchronize()
    keep = {n: torch.where(bad[:, None, :, None], 0.0, c.heads(x, h)) for n, x, h in (("q", c.q, c.H), ("k", c.k, c.KV), ("v", c.v, c.KV), ("dctx", c.dctx, c.H))}
    order = iter(("q", "dctx", "k", "v"))
    want = c.want(clean=lambda x, n: keep[next(order)])
    for name, x in (("ctx", ctx), ("dq", dq), ("dk", dk), ("dv", dv)):
        w, b = want[name]
        x, w, b = x.double()[~bad], w[~bad], b[~bad]
        assert bool(x.isfinite().all()), name
        assert float(((x - w).abs() - b).max()) <= 1e-30, name
    none = c.doc < 0
    assert not ctx[none].any() and not dq[none].any() and not dk[none].any() and not dv[none].any()
    assert bool((lse.transpose(1, 2)[none] == -math.inf).all())


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_what_a_mask_hides_in_large_launches(dtype):
    test_what_a_mask_hides_reaches_no_result(dtype, math.nan, 64, dict(causal=1), H=96, KV=96)
    test_what_a_mask_hides_reaches_no_result(dtype, math.inf, 128, dict(causal=0, cap=10.0), H=96, KV=48)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_of_scores_without_a_finite_one(dtype):
    """Keys of -inf (not masked): a row that sees nothing else has ctx 0 and lse -inf, as an empty one; rows with a finite
    score beside them are as without them."""
    for S in (40, 200):
        c = Case(dtype, 1, S, 2, 2, 64, causal=1)
        c.q.abs_()
        c.k[:, :20] = -math.inf
        ctx, lse = c.run(grads=False)
        assert not ctx[:, :20].any() and bool((lse[..., :20] == -math.inf).all())
        q, k, v = c.heads(c.q, 2), c.heads(c.k, 2), c.heads(c.v, 2)
        s = (q[:, :, 20:] @ k[:, :, 20:].transpose(2, 3)) / 8
        s = s.masked_fill(~c.allowed()[:, None, 20:, 20:], -math.inf)
        want = (torch.softmax(s, 3) @ v[:, :, 20:]).transpose(1, 2).reshape(1, S - 20, -1)
        assert float((ctx[:, 20:].double() - want).abs().max()) <= (2.0**-6 if dtype == BF16 else 1e-5)


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_rows_of_one_key_have_no_score_gradient(dtype):
    c = Case(dtype, 2, 200, 2, 1, 64, docs=1)
    _, _, dq, dk, dv = c.run()
    assert not dq.any() and not dk.any()
    want = c.heads(c.dctx, 2).reshape(2, 1, 2, 200, 64).sum(2).transpose(1, 2).reshape(2, 200, 64)
    assert float((dv.double() - want).abs().max()) <= float(want.abs().max()) * (2.0**-8 if dtype == BF16 else 2.0**-23)


@pytest.mark.parametrize("dtype", [BF16, FP32])
@pytest.mark.parametrize("mask", MASKS[3:6])
def test_gradient_against_differences(dtype, mask):
    c = Case(dtype, 1, 70, 4, 2, 64, **mask)
    _, _, dq, dk, dv = c.run()
    g = torch.Generator("cuda").manual_seed(7)
    base = [x.clone() for x in (c.q, c.k, c.v)]
    loss = lambda: float((c.want()["ctx"][0] * c.dctx.double()).sum())  # noqa: E731
    for at, dx in enumerate((dq, dk, dv)):
        to = torch.randn(dx.shape, generator=g, device="cuda", dtype=torch.float64)
        vals = []
        for sign in (1, -1):
            c.q, c.k, c.v = [x.double() + (sign * 1e-5 * to if n == at else 0) for n, x in enumerate(base)]
            vals.append(loss())
        slope = (vals[0] - vals[1]) / 2e-5
        assert abs(float((dx.double() * to).sum()) - slope) <= (2.0**-6 if dtype == BF16 else 1e-5) * float(dx.double().norm() * to.norm()) + 1e-6


@pytest.mark.parametrize("dtype", [BF16, FP32])
def test_captured_and_on_another_stream(dtype):
    c = Case(dtype, 2, 300, 4, 2, 64, docs=60, pad=1, slopes=1, cap=20.0)
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    c.run()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        got = c.run()
    got = [x.clone() if n == 0 else x for n, x in enumerate(got)][1:]  # ctx is a buffer of the case
    for seed in range(3):
        other = Case(dtype, 2, 300, 4, 2, 64, docs=60, pad=1, slopes=1, cap=20.0, seed=seed + 1)
        for a, b in ((c.q, other.q), (c.k, other.k), (c.v, other.v), (c.dctx, other.dctx), (c.doc, other.doc)):
            a.copy_(b)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            want = other.run()
        torch.cuda.synchronize()
        assert torch.equal(c.ctx, want[0]) and all(torch.equal(a, b) for a, b in zip(got, want[1:]))


def test_binding_refuses_what_a_kernel_would_misread():
    c = Case(BF16, 2, 50, 2, 1, 64, packed=0)
    c.run()
    ok = [c.q, c.k, c.v, c.spans, None, c.ctx]
    for at, bad in ((0, c.q.float()), (0, c.q[:1, :5].clone()), (1, c.k.transpose(1, 2)), (2, c.v.cpu()), (3, c.spans[:7]), (3, c.spans.long()),
                    (4, torch.ones(1, device="cuda")), (5, c.ctx[:1].clone())):
        with pytest.raises(ValueError):
            bf.bf_op_attention_masked_fwd(c.cfg, *ok[:at], bad, *ok[at + 1:])
    with pytest.raises(ValueError):
        bf.bf_op_attention_spans(2, 50, 1, torch.zeros(2, 49, dtype=torch.int32, device="cuda"), None, c.spans)


def test_binding_refuses_rows_that_are_not_where_the_configuration_says():
    """Views into packed rows without their step, heads in front of tokens: refused as inputs and as outputs, with all that the
    kernels would reach inside the storage, and nothing is written."""
    B, S, H, d = 2, 50, 2, 64
    n = H * d
    cfg, packed = (bf.make_attn_config(BF16, B, S, H, H, d, ld_q=ld, ld_k=ld, ld_v=ld) for ld in (0, 3 * n))
    qkv = torch.randn(B, S, 3 * n, device="cuda").to(torch.bfloat16)
    own = [x.contiguous() for x in qkv.split(n, 2)]
    spans = torch.zeros(bf.bf_op_attention_spans_elems(B, S), dtype=torch.int32, device="cuda")
    bf.bf_op_attention_spans(B, S, 1, None, None, spans)
    ctx, lse = torch.empty(B, S, n, dtype=torch.bfloat16, device="cuda"), torch.empty(B, H, S, device="cuda")
    bf.bf_op_attention_masked_fwd(cfg, *own, spans, None, ctx, lse)
    other = torch.empty(B, S, H, d, dtype=torch.bfloat16, device="cuda")
    bf.bf_op_attention_masked_fwd(packed, *(x.unflatten(2, (H, d)) for x in qkv.split(n, 2)), spans, None, other, lse)
    assert torch.equal(ctx, other.flatten(2))
    heads_first = own[0].unflatten(2, (H, d)).transpose(1, 2).contiguous()
    for at in range(3):
        for bad in (qkv.split(n, 2)[at], heads_first, heads_first.transpose(1, 2)):
            with pytest.raises(ValueError):
                bf.bf_op_attention_masked_fwd(cfg, *own[:at], bad, *own[at + 1:], spans, None, ctx, lse)
    with pytest.raises(ValueError):
        bf.bf_op_attention_masked_fwd(packed, *own, spans, None, ctx, lse)
    out = torch.full_like(qkv, 7.0)
    grads = [torch.full_like(x, 7.0) for x in own]
    for at, part in enumerate(out.split(n, 2)):
        with pytest.raises(ValueError):
            bf.bf_op_attention_masked_bwd(cfg, *own, spans, None, ctx, lse, ctx, *grads[:at], part, *grads[at + 1:])
    assert bool((out == 7).all()) and all(bool((x == 7).all()) for x in grads)
