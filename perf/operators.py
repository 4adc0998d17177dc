"""Operators of language model training on packed documents, as a program calls them one by one.

Three kinds: attention under a document or prefix mask (capped scores, a bias that falls with distance, shared key / value
heads), the vocabulary loss in pieces of the vocabulary, and the global gradient norm with what follows it (clipped
gradients, or the clipped Adam step).

With `own` set, run() makes the calls of paper_2211_05953_amd; without, it computes the same in elementary torch
operations in 32 bits.  exact() computes it from the definitions in 64 bits."""
import math
import random

import torch

own = False

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
LR, BETA1, BETA2, ADAM_EPS, DECAY, STEP = 1e-4, 0.9, 0.95, 1e-8, 0.1, 3
MAX_NORM = 1.0


def _attention(**more):
    case = {"kind": "attention", "dtype": "bf16", "smb": 1, "seq": 1, "heads": 1, "kv": 1, "head": 64, "causal": 1, "docs": 0,
            "pad": 0, "prefix": 0, "slopes": 0, "cap": 0.0, "grad": 1}
    case.update(more)
    return case


def listed():
    return [
        # A short sequence of three or so documents in a small model: launches and latency.
        _attention(name="attention_short", seq=60, heads=4, kv=4, docs=20),
        # One layer of the 1.3B-shaped stack on a micro-batch of packed documents, some hundred tokens each, padded at the end.
        _attention(name="attention_packed_2048", smb=2, seq=2048, heads=16, kv=16, head=128, docs=300, pad=1),
        # Long sequences, capped scores, four query heads to a key / value head.
        _attention(name="attention_capped_8192", seq=8192, heads=16, kv=4, head=128, cap=50.0),
        # Evaluation of sequences with a bidirectional prefix, of a length nobody rounded up, with a bias by distance.
        _attention(name="attention_prefix_1000", smb=4, seq=1000, heads=16, kv=16, head=64, prefix=1, slopes=1, grad=0),
        # Full precision, bidirectional, everything at once, a head size between the usual ones.
        _attention(name="attention_fp32_500", dtype="fp32", smb=2, seq=500, heads=8, kv=2, head=80, causal=0, docs=200, slopes=1, cap=30.0),
        # The head of a small model on a few tokens of a vocabulary of odd size.
        {"name": "loss_small", "kind": "loss", "dtype": "bf16", "tokens": 33, "hidden": 256, "vocab": 1003, "ignored": 0, "grad": 1},
        # One micro-batch of the 2048-wide model: loss, and the gradients of the head's input and weights.
        {"name": "loss_2048", "kind": "loss", "dtype": "bf16", "tokens": 2048, "hidden": 2048, "vocab": 50304, "ignored": 1, "grad": 1},
        # Evaluation of that model: the loss alone.
        {"name": "loss_eval_2048", "kind": "loss", "dtype": "bf16", "tokens": 8190, "hidden": 2048, "vocab": 50304, "ignored": 0, "grad": 0},
        # The head of the 8192-wide stack.
        {"name": "loss_8192", "kind": "loss", "dtype": "bf16", "tokens": 2048, "hidden": 8192, "vocab": 50304, "ignored": 0, "grad": 1},
        # Full precision.
        {"name": "loss_fp32_1000", "kind": "loss", "dtype": "fp32", "tokens": 500, "hidden": 1000, "vocab": 8003, "ignored": 1, "grad": 1},
        # The many small tensors of a small model: norm and clipped gradients.
        {"name": "clip_small", "kind": "clip", "dtype": "fp32", "tensors": 200, "low": 256, "high": 262144, "odd": 1, "adam": 0},
        # The main-grads of a rank's share: norm and clipped Adam step.
        {"name": "clip_adam_large", "kind": "clip", "dtype": "fp32", "tensors": 24, "low": 4194304, "high": 16777216, "odd": 0, "adam": 1},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind, dtype = rng.choice(["attention", "attention", "loss", "clip"]), rng.choice(["bf16", "bf16", "fp32"])
    if kind == "attention":
        seq = _log(rng, 1, 8192)
        head = rng.choice([64, 128, 128, rng.randint(1, 16) * 8, rng.randint(1, 128)])
        kv = _log(rng, 1, 16)
        heads = kv * rng.choice([1, 1, 2, 4, 8])
        smb = _log(rng, 1, 16)
        limit = 2**30 if dtype == "bf16" else 2**27
        while smb * heads * seq * max(seq, 128) > limit:
            if smb > 1:
                smb //= 2
            elif kv > 1:
                heads, kv = heads // kv * (kv // 2), kv // 2
            elif heads > 1:
                heads //= 2
            else:
                break
        return _attention(dtype=dtype, smb=smb, seq=seq, heads=heads, kv=kv, head=head, causal=rng.choice([1, 1, 0]),
                          docs=rng.choice([0, _log(rng, 1, max(2, seq))]), pad=rng.choice([0, 1]), prefix=rng.choice([0, 0, 1]),
                          slopes=rng.choice([0, 1]), cap=rng.choice([0.0, 20.0, 50.0]), grad=rng.choice([1, 1, 0]))
    if kind == "loss":
        hidden = rng.choice([_log(rng, 64, 8192) // 8 * 8, _log(rng, 64, 8192) // 64 * 64, _log(rng, 16, 1024)])
        vocab = rng.choice([50304, _log(rng, 2, 100000), _log(rng, 256, 100000) // 128 * 128])
        most = int((8e11 if dtype == "bf16" else 2e10) / hidden / vocab)
        return {"kind": kind, "dtype": dtype, "tokens": _log(rng, 1, max(1, min(8192, most))), "hidden": hidden, "vocab": vocab,
                "ignored": rng.choice([0, 1]), "grad": rng.choice([1, 1, 0])}
    tensors, adam = _log(rng, 1, 300), rng.choice([0, 1])
    high = min(_log(rng, 16, 2**25), 2**27 // tensors)
    return {"kind": kind, "dtype": "fp32" if adam else dtype, "tensors": tensors, "low": rng.randint(1, max(1, high // 4)), "high": high,
            "odd": rng.choice([0, 1]), "adam": adam}


def _sizes(case):
    """Elements of the tensors of a clipping case, the same ones for every seed, and where each starts in its arena."""
    rng = random.Random(case["tensors"] * 1000003 + case["high"])
    sizes = [_log(rng, case["low"], case["high"]) for _ in range(case["tensors"])]
    if not case["odd"]:
        sizes = [max(1, n // 64 * 64) for n in sizes]
    starts, at = [], 0
    for n in sizes:
        starts.append(at)
        at += n if case["odd"] else -(-n // 128) * 128
    return sizes, starts, at


def _distance_pairs(n, mean):
    """Expected pairs j <= i of n tokens in a row that fall into one document of geometric length."""
    if not mean:
        return n * (n + 1) / 2
    keep = 1 - 1 / max(mean, 1)
    return n + sum((n - d) * keep**d for d in range(1, min(n, 40 * mean + 1)))


def work(case):
    """Every input read once, every output written once, two operations per multiplication and addition of the products."""
    size = 2 if case["dtype"] == "bf16" else 4
    if case["kind"] == "attention":
        n = case["seq"] - (case["seq"] // 8 if case["pad"] else 0)
        lower = _distance_pairs(n, case["docs"])
        pairs = lower if case["causal"] else 2 * lower - n
        if case["causal"] and case["prefix"]:
            pairs += _distance_pairs(n // 4, case["docs"]) - n // 4
        tokens, heads, kv, d = case["smb"] * case["seq"], case["heads"], case["kv"], case["head"]
        data = tokens * d * (2 * heads + 2 * kv) * size + 4 * tokens * heads
        if case["grad"]:
            data += tokens * d * (2 * heads + 2 * kv) * size
        return {"bytes": data, "flops": (14 if case["grad"] else 4) * pairs * case["smb"] * heads * d}
    if case["kind"] == "loss":
        t, h, v = case["tokens"], case["hidden"], case["vocab"]
        data = size * (t + v) * h + 12 * t
        return {"bytes": data + (size * t * h + 4 * v * h if case["grad"] else 0), "flops": (6 if case["grad"] else 2) * t * h * v}
    n = sum(_sizes(case)[0])
    return {"bytes": n * (30 if case["adam"] else 2 * size), "flops": n * (14 if case["adam"] else 3)}


def prepare(case, seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    normal = lambda *shape: torch.randn(shape, generator=g, device=DEV)  # noqa: E731
    uniform = lambda *shape: torch.rand(shape, generator=g, device=DEV)  # noqa: E731
    dtype = TYPES[case["dtype"]]
    s = dict(case)
    if case["kind"] == "attention":
        b, n, heads, kv, d = (case[k] for k in ("smb", "seq", "heads", "kv", "head"))
        # q, k and v as the one projection in front of them leaves them: side by side in a token's row
        s["qkv"] = normal(b, n, (heads + 2 * kv) * d)
        if case["cap"]:
            s["qkv"][..., : heads * d] *= 3
        s["qkv"] = s["qkv"].to(dtype)
        s["doc"] = s["prefixes"] = s["slope"] = None
        if case["docs"] or case["pad"]:
            s["doc"] = (uniform(b, n) < 1 / max(case["docs"], 1)).int().cumsum(1).int() if case["docs"] else torch.zeros(b, n, dtype=torch.int32, device=DEV)
        if case["pad"]:
            s["doc"][:, n - n // 8:] = -1
        if case["prefix"]:
            s["prefixes"] = (uniform(b) * (n / 2)).int()
        if case["slopes"]:
            s["slope"] = 2.0 ** (-8.0 * torch.arange(1, heads + 1, device=DEV) / heads)
        s["dctx"] = normal(b, n, heads * d).to(dtype) if case["grad"] else None
    elif case["kind"] == "loss":
        t, h, v = case["tokens"], case["hidden"], case["vocab"]
        s["w"] = (normal(v, h) * (2 / math.sqrt(h))).to(dtype)
        label = (uniform(t) * v).long().clamp(max=v - 1)
        # rows that lean towards their labels, from not at all to nearly sure, as in a model under training
        s["y"] = (normal(t, h) + 4 * uniform(t, 1) * s["w"][label].float()).to(dtype)
        s["label"] = torch.where(uniform(t) < 0.2, -1, label).int() if case["ignored"] else label.int()
    else:
        sizes, starts, total = _sizes(case)
        cut = lambda x: [x[a : a + m] for a, m in zip(starts, sizes)]  # noqa: E731
        norm = 3.0 if seed % 3 else 0.5
        s["g"] = cut((normal(total) * (norm / math.sqrt(sum(sizes)))).to(dtype))
        if case["adam"]:
            w, m, v = normal(total) * 0.02, normal(total) * 1e-4, uniform(total) * 1e-8
            s["arena"] = {"w": w, "m": m, "v": v, "w_lp": w.to(torch.bfloat16)}
            s["state"] = [dict(zip(("w", "m", "v", "w_lp"), x)) for x in zip(*(cut(s["arena"][k]) for k in ("w", "m", "v", "w_lp")))]
        else:
            s["clipped"] = torch.zeros(total, dtype=dtype, device=DEV)
            s["out"] = cut(s["clipped"])
    return s


# ---- the framework's calls ------------------------------------------------------------------
def _own_attention(s):
    import paper_2211_05953_amd as bf

    b, n, heads, kv, d = (s[k] for k in ("smb", "seq", "heads", "kv", "head"))
    ld = (heads + 2 * kv) * d
    q, k, v = s["qkv"].split((heads * d, kv * d, kv * d), 2)
    cfg = bf.make_attn_config(bf.BF_BF16 if s["dtype"] == "bf16" else bf.BF_FP32, b, n, heads, kv, d, cap=s["cap"], ld_q=ld, ld_k=ld, ld_v=ld)
    spans = torch.empty(bf.bf_op_attention_spans_elems(b, n), dtype=torch.int32, device=DEV)
    bf.bf_op_attention_spans(b, n, s["causal"], s["doc"], s["prefixes"], spans)
    ctx = torch.empty(b, n, heads * d, dtype=s["qkv"].dtype, device=DEV)
    lse = torch.empty(b, heads, n, device=DEV)
    bf.bf_op_attention_masked_fwd(cfg, q, k, v, spans, s["slope"], ctx, lse)
    if not s["grad"]:
        return {"ctx": ctx, "lse": lse}
    dq, dk, dv = torch.empty_like(s["qkv"]).split((heads * d, kv * d, kv * d), 2)
    bf.bf_op_attention_masked_bwd(cfg, q, k, v, spans, s["slope"], ctx, lse, s["dctx"], dq, dk, dv)
    return {"ctx": ctx, "lse": lse, "dq": dq, "dk": dk, "dv": dv}


def _own_loss(s):
    import paper_2211_05953_amd as bf

    t, h, v = s["tokens"], s["hidden"], s["vocab"]
    dtype = bf.BF_BF16 if s["dtype"] == "bf16" else bf.BF_FP32
    lse, rows, loss = torch.empty(t, device=DEV), torch.empty(t, device=DEV), torch.empty(1, device=DEV)
    bf.bf_op_vocab_loss_fwd(dtype, t, h, v, s["y"], s["w"], s["label"], 1 / t, lse, rows, loss)
    if not s["grad"]:
        return {"loss": loss, "rows": rows, "lse": lse}
    dy, dw = torch.empty_like(s["y"]), torch.empty(v, h, device=DEV)
    bf.bf_op_vocab_loss_bwd(dtype, t, h, v, s["y"], s["w"], s["label"], lse, 1 / t, dy, dw)
    return {"loss": loss, "rows": rows, "lse": lse, "dy": dy, "dw": dw}


def _own_clip(s):
    import paper_2211_05953_amd as bf

    dtype = bf.BF_BF16 if s["dtype"] == "bf16" else bf.BF_FP32
    out = torch.empty(2, device=DEV)
    bf.bf_op_grad_norm(dtype, s["g"], MAX_NORM, out)
    if not s["adam"]:
        bf.bf_op_grad_scale(dtype, s["g"], s["out"], out[1:])
        return {"norm": out, "clipped": s["clipped"]}
    bf.bf_op_adam_clipped([(x["w"], x["m"], x["v"], g, x["w_lp"]) for x, g in zip(s["state"], s["g"])], out[1:], STEP, LR, BETA1, BETA2, ADAM_EPS, DECAY)
    return {"norm": out, **s["arena"]}


# ---- the plain form -------------------------------------------------------------------------
def _allowed(s):
    """[smb, 1, seq, seq]: which keys a token may look at."""
    n = s["seq"]
    i = torch.arange(n, device=DEV)
    ok = torch.ones(1, n, n, dtype=torch.bool, device=DEV)
    if s["causal"]:
        ok = i[None, :, None] >= i[None, None, :]
        if s["prefixes"] is not None:
            ok = ok | (i[None, None, :] < s["prefixes"][:, None, None])
    if s["doc"] is not None:
        # a document is a run of equal ids; a negative id is padding
        run = torch.cat([torch.zeros_like(s["doc"][:, :1]), (s["doc"][:, 1:] != s["doc"][:, :-1]).int().cumsum(1)], 1)
        ok = ok & (run[:, :, None] == run[:, None, :]) & (s["doc"] >= 0)[:, :, None]
    return ok[:, None]


def _plain_attention(s):
    b, n, heads, kv, d = (s[k] for k in ("smb", "seq", "heads", "kv", "head"))
    scale = 1 / math.sqrt(d)
    q, k, v = (x.reshape(b, n, -1, d).transpose(1, 2).float() for x in s["qkv"].split((heads * d, kv * d, kv * d), 2))
    k, v = (x.repeat_interleave(heads // kv, 1) for x in (k, v))
    score, capped = (q @ k.transpose(2, 3).contiguous()) * scale, None
    if s["cap"]:
        capped = torch.tanh(score / s["cap"])
        score = capped * s["cap"]
    if s["slope"] is not None:
        i = torch.arange(n, device=DEV)
        score = score - s["slope"][:, None, None] * (i[:, None] - i).abs()
    score = score.masked_fill(~_allowed(s), -math.inf)
    top = score.amax(3, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = torch.exp(score - top)
    total = p.sum(3, keepdim=True)
    lse = (top + total.log())[..., 0]
    p = p / torch.where(total == 0, 1.0, total)
    ctx = p @ v
    whole = lambda x: x.transpose(1, 2).reshape(b, n, -1).to(s["qkv"].dtype)  # noqa: E731
    if not s["grad"]:
        return {"ctx": whole(ctx), "lse": lse}
    dctx = s["dctx"].reshape(b, n, heads, d).transpose(1, 2).float()
    dv = p.transpose(2, 3).contiguous() @ dctx
    dp = dctx @ v.transpose(2, 3).contiguous()
    ds = p * (dp - (p * dp).sum(3, keepdim=True))
    if capped is not None:
        ds = ds * (1 - capped * capped)
    dq, dk = (ds @ k) * scale, (ds.transpose(2, 3).contiguous() @ q) * scale
    dk, dv = (x.reshape(b, kv, -1, n, d).sum(2) for x in (dk, dv))
    return {"ctx": whole(ctx), "lse": lse, "dq": whole(dq), "dk": whole(dk), "dv": whole(dv)}


def _plain_loss(s):
    y, w, scale = s["y"].float(), s["w"].float(), 1 / s["tokens"]
    known = (s["label"] >= 0) & (s["label"] < s["vocab"])
    label = torch.where(known, s["label"], 0).long()
    z = y @ w.t()
    top = z.amax(1)
    lse = top + torch.exp(z - top[:, None]).sum(1).log()
    rows = torch.where(known, (lse - z.gather(1, label[:, None])[:, 0]) * scale, 0.0)
    out = {"loss": rows.double().sum()[None].float(), "rows": rows, "lse": lse}
    if s["grad"]:
        dz = torch.exp(z - lse[:, None])
        dz.scatter_add_(1, label[:, None], torch.full_like(lse, -1.0)[:, None])
        dz = dz * (known * scale)[:, None]
        out |= {"dy": (dz @ w).to(s["y"].dtype), "dw": dz.t() @ y}
    return out


def _adam(x, g, coef):
    g = g * coef
    x["m"].mul_(BETA1).add_((1 - BETA1) * g)
    x["v"].mul_(BETA2).add_((1 - BETA2) * g * g)
    step = (x["m"] / (1 - BETA1**STEP)) / ((x["v"] / (1 - BETA2**STEP)).sqrt() + ADAM_EPS)
    x["w"].sub_(LR * (step + DECAY * x["w"]))
    x["w_lp"].copy_(x["w"])


def _plain_clip(s):
    norm = torch.stack([x.double().square().sum() for x in s["g"]]).sum().sqrt()
    coef = torch.where(norm > MAX_NORM, MAX_NORM / norm, 1.0).float()
    out = {"norm": torch.stack([norm.float(), coef])}
    if s["adam"]:
        _ = [_adam(x, g, coef) for x, g in zip(s["state"], s["g"])]
        return out | s["arena"]
    _ = [x.copy_(g.float() * coef) for x, g in zip(s["out"], s["g"])]
    return out | {"clipped": s["clipped"]}


def run(state):
    if own:
        return {"attention": _own_attention, "loss": _own_loss, "clip": _own_clip}[state["kind"]](state)
    return {"attention": _plain_attention, "loss": _plain_loss, "clip": _plain_clip}[state["kind"]](state)


# ---- the definitions in 64 bits ---------------------------------------------------------------
def _exact_attention(s):
    b, n, heads, kv, d = (s[k] for k in ("smb", "seq", "heads", "kv", "head"))
    f64 = {"dtype": torch.float64, "device": DEV}
    qkv = s["qkv"].double()
    out = {"ctx": torch.zeros(b, n, heads * d, **f64), "lse": torch.zeros(b, heads, n, **f64)}
    grads = torch.zeros(b, n, (heads + 2 * kv) * d, **f64)
    at = torch.arange(n, device=DEV)
    for e in range(b):
        see = torch.ones(n, n, dtype=torch.bool, device=DEV)
        if s["causal"]:
            reach = at + 1
            if s["prefixes"] is not None:
                reach = torch.maximum(reach, s["prefixes"][e].long())
            see = at[None, :] < reach[:, None]
        if s["doc"] is not None:
            ids = s["doc"][e].tolist()
            begins, begin = [], 0
            for t in range(n):
                begin = t if t and ids[t] != ids[t - 1] else begin
                begins.append(begin)
            begins = torch.tensor(begins, device=DEV)
            see = see & (begins[:, None] == begins[None, :]) & torch.tensor([x >= 0 for x in ids], device=DEV)[:, None]
        for a in range(heads):
            mine, theirs = slice(a * d, a * d + d), a // (heads // kv) * d
            cols = mine, slice(heads * d + theirs, heads * d + theirs + d), slice((heads + kv) * d + theirs, (heads + kv) * d + theirs + d)
            q, k, v = (qkv[e, :, c] for c in cols)
            x = q.mm(k.t()) / d**0.5
            slack = None
            if s["cap"]:
                slack = 1 / torch.cosh(x / s["cap"]) ** 2
                x = s["cap"] * torch.tanh(x / s["cap"])
            if s["slope"] is not None:
                x = x - s["slope"][a].double() * (at[None, :] - at[:, None]).abs()
            x = torch.where(see, x, -math.inf)
            lse = torch.logsumexp(x, 1)
            p = torch.where(see, torch.exp(x - torch.where(lse == -math.inf, 0.0, lse)[:, None]), 0.0)
            out["lse"][e, a], out["ctx"][e, :, mine] = lse, p.mm(v)
            if s["grad"]:
                do = s["dctx"][e, :, mine].double()
                into = do.mm(v.t())
                into = p * (into - (p * into).sum(1)[:, None])
                into = (into if slack is None else into * slack) / d**0.5
                grads[e, :, cols[0]] += into.mm(k)
                grads[e, :, cols[1]] += into.t().mm(q)
                grads[e, :, cols[2]] += p.t().mm(do)
    if s["grad"]:
        out["dq"], out["dk"], out["dv"] = grads.split((heads * d, kv * d, kv * d), 2)
    return out


def _exact_loss(s):
    y, w, t = s["y"].double(), s["w"].double(), s["tokens"]
    label = s["label"].long()
    keep = (label >= 0) & (label < s["vocab"])
    z = y.mm(w.t())
    lse = torch.logsumexp(z, 1)
    rows = torch.zeros(t, dtype=torch.float64, device=DEV)
    rows[keep] = (lse[keep] - z[keep, label[keep]]) / t
    out = {"loss": rows.sum()[None], "rows": rows, "lse": lse}
    if s["grad"]:
        share = torch.softmax(z, 1)
        share[keep, label[keep]] -= 1
        share[~keep] = 0
        out |= {"dy": share.mm(w) / t, "dw": share.t().mm(y) / t}
    return out


def _exact_clip(s):
    norm = math.sqrt(sum(float((g.double() ** 2).sum()) for g in s["g"]))
    coef = min(1.0, MAX_NORM / norm) if norm else 1.0
    out = {"norm": torch.tensor([norm, coef], dtype=torch.float64, device=DEV)}
    if not s["adam"]:
        arena = torch.zeros(s["clipped"].numel(), dtype=torch.float64, device=DEV)
        for (start, size), g in zip(zip(_sizes(s)[1], _sizes(s)[0]), s["g"]):
            arena[start : start + size] = g.double() * coef
        return out | {"clipped": arena}
    arenas = {k: s["arena"][k].double() for k in ("w", "m", "v")}
    low = s["arena"]["w_lp"].double()
    for start, size, g in zip(_sizes(s)[1], _sizes(s)[0], s["g"]):
        part, g = slice(start, start + size), g.double() * coef
        m = BETA1 * arenas["m"][part] + (1 - BETA1) * g
        v = BETA2 * arenas["v"][part] + (1 - BETA2) * g**2
        w = arenas["w"][part]
        w = w - LR * (m / (1 - BETA1**STEP) / (torch.sqrt(v / (1 - BETA2**STEP)) + ADAM_EPS) + DECAY * w)
        arenas["m"][part], arenas["v"][part], arenas["w"][part], low[part] = m, v, w, w
    return out | arenas | {"w_lp": low}


def exact(case, seed):
    s = prepare(case, seed)
    return {"attention": _exact_attention, "loss": _exact_loss, "clip": _exact_clip}[case["kind"]](s)
