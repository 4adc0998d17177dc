"""8-bit forms, their products and the Adam step on 8-bit moments from the definitions, in fp64."""
import torch

TOP = {0: (448.0, -6, 3), 1: (57344.0, -14, 2)}  # format: largest value, exponent of the smallest normal, bits of mantissa
TYPES = {0: torch.float8_e4m3fn, 1: torch.float8_e5m2}


def power(e):
    """2^e, exactly."""
    return ((e.long() + 1023) << 52).view(torch.float64)


def exponent(amax, top):
    """Smallest e >= -127 with amax <= top 2^e; 0 where amax is 0."""
    part, two = torch.frexp(amax.double() / top)  # in [0.5, 1)
    e = two - (part == 0.5).int()
    return torch.where(amax == 0, torch.zeros_like(e), e.clamp(min=-127))


def form(x, fmt):
    """(codes as fp64 numbers [rows, whole blocks], scale bytes [blocks, rows to 16]) of the rows of x."""
    top, low, bits = TOP[fmt]
    x = x.double()
    rows, n = x.shape
    blocks = -(-n // 128)
    y = torch.zeros(rows, blocks * 128, dtype=torch.float64, device=x.device)
    y[:, :n] = x
    y = y.view(rows, blocks, 128)
    finite = torch.isfinite(y)
    e = exponent(torch.where(finite, y.abs(), 0.0).amax(2), top)
    y = y * power(-e)[:, :, None]
    ey = (torch.frexp(y)[1] - 1).clamp(min=low)
    step = power(ey - bits)
    q = torch.where(finite, torch.round(y / step) * step, float("nan")).view(rows, blocks * 128)
    scale = torch.full((blocks, -(-rows // 16) * 16), 127, dtype=torch.uint8, device=x.device)
    scale[:, :rows] = (e.t() + 127).to(torch.uint8)
    return q, scale


def codes(q, fmt):
    """Bytes of numbers that are on the grid."""
    return q.to(torch.float32).to(TYPES[fmt]).view(torch.uint8)


def values(q, scale, n, fmt=None):
    """What a form stands for; q: numbers, or bytes of a format."""
    if fmt is not None:
        q = q.view(TYPES[fmt]).double()
    rows = q.shape[0]
    unit = power(scale[:, :rows].t().long() - 127).repeat_interleave(128, 1)
    return (q * unit)[:, :n]


def mix(x):
    for shift, factor in ((15, 0x6A09E667), (13, 0xBB67AE85), (16, 1)):
        x = ((x ^ (x >> shift)) * factor) % 2**32
    return x


def randoms(seed, t, tensor, n, device):
    """The 16 random bits of each element's m and v."""
    key = 0
    for word in (seed % 2**32, seed // 2**32, t):
        key = mix(key ^ word)
    h = mix((torch.arange(n, device=device) + mix(key ^ tensor)) % 2**32)
    return h % 65536, h // 65536


def decode(state, n):
    """(m, v, unit of m, unit of v) of a state, over whole blocks, in fp64."""
    blocks = -(-n // 128)
    c, s = state[: 256 * blocks].view(blocks, 2, 128), state[256 * blocks: 258 * blocks].view(blocks, 2).long()
    um, uv = power(s[:, :1] - 127), power(s[:, 1:] - 127)
    b = c[:, 1].long()
    v = torch.where(b < 16, b.double() / 16, (1 + b % 16 / 16.0) * power(b // 16 - 1))
    return c[:, 0].contiguous().view(torch.float8_e4m3fn).double() * um, v * uv, um, uv


def encode(m, v):
    """The state nearest to moments, for tests that need one that is not zero."""
    n = m.numel()
    blocks = -(-n // 128)
    pad = lambda x: torch.nn.functional.pad(x.double(), (0, blocks * 128 - n)).view(blocks, 128)  # noqa: E731
    q, s = form(pad(m), 0)
    y = pad(v)
    e = exponent(y.amax(1), 31744.0)
    y = y * power(-e)[:, None]
    ey = (torch.frexp(y)[1] - 1).clamp(min=0)
    b = (ey * 16 + torch.round(y * power(4 - ey))).to(torch.uint8)
    s = torch.stack([s[0, :blocks], (e + 127).to(torch.uint8)], 1)
    return torch.cat([torch.stack([codes(q, 0), b], 1).view(-1), s.view(-1)])


def adam(w, state, g, coef, t, lr, beta1, beta2, eps, wd):
    """(w, m, v) after the step, moments before they are rounded, over whole blocks."""
    n = w.numel()
    m, v, _, _ = decode(state, n)
    gg = torch.nn.functional.pad(g.double() * coef, (0, m.numel() - n)).view_as(m)
    m, v = beta1 * m + (1 - beta1) * gg, beta2 * v + (1 - beta2) * gg * gg
    step = m / (1 - beta1**t) / (torch.sqrt(v / (1 - beta2**t)) + eps)
    w = w.double()
    return w - lr * (step.view(-1)[:n] + wd * w), m, v
