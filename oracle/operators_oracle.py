"""Definitions of lnorm.h, relpos.h and adamw.h in 64 bits (torch on the CPU): test infrastructure only."""
import math

import torch


# ---- LayerNorm of rows -------------------------------------------------------------------------------------------------------

def lnorm_forward(u, gamma, beta, eps):
    """(y, xh, rstd) of rows u [rows, C]."""
    u = u.double()
    mean = u.mean(1, keepdim=True)
    rstd = 1 / torch.sqrt(((u - mean) ** 2).mean(1, keepdim=True) + eps)
    xh = (u - mean) * rstd
    y = xh if gamma is None else xh * gamma.double()
    return (y if beta is None else y + beta.double()), xh, rstd


def lnorm_backward(u, dy, gamma, dsum, eps):
    """(dx, dgamma, dbeta)."""
    _, xh, rstd = lnorm_forward(u, None, None, eps)
    dy = dy.double()
    g = dy if gamma is None else dy * gamma.double()
    dx = rstd * (g - g.mean(1, keepdim=True) - xh * (g * xh).mean(1, keepdim=True))
    return (dx if dsum is None else dx + dsum.double()), (dy * xh).sum(0), dy.sum(0)


# ---- relative position bias ----------------------------------------------------------------------------------------------------

def log_edge(buckets, max_distance, bidirectional):
    """Edges by whole numbers alone: the least r with r^n E^k >= D^k E^n."""
    side = buckets // 2 if bidirectional else buckets
    exact = side // 2
    n = side - exact
    edges = list(range(1, exact + 1))
    for k in range(1, n):
        lo, hi = 1, max_distance
        while lo < hi:
            mid = (lo + hi) // 2
            if mid ** n * exact ** k >= max_distance ** k * exact ** n:
                hi = mid
            else:
                lo = mid + 1
        edges.append(lo)
    return edges


def bucket(r, edges, bidirectional):
    """Buckets of a tensor of offsets key - query."""
    e = torch.tensor(edges, dtype=torch.int64)
    d = r.abs() if bidirectional else (-r).clamp(min=0)
    n = torch.searchsorted(e, d.contiguous(), right=True) if len(edges) else torch.zeros_like(r)
    return n + (r > 0) * (len(edges) + 1) if bidirectional else n


def sequence_bucket(q, k, start, edges, bidirectional):
    return bucket(torch.arange(k)[None, :] - torch.arange(q)[:, None] - start, edges, bidirectional)


def sequence_forward(table, q, k, start, edges, bidirectional, causal):
    """[heads, q, k] in the table's type."""
    out = table[sequence_bucket(q, k, start, edges, bidirectional)].permute(2, 0, 1).clone()
    if causal:
        out[:, torch.arange(k)[None, :] > torch.arange(q)[:, None] + start] = -math.inf
    return out


def sequence_backward(dout, start, edges, bidirectional, causal, rows):
    """[rows, heads] from dout [batch, heads, q, k]."""
    _, heads, q, k = dout.shape
    b = sequence_bucket(q, k, start, edges, bidirectional)
    keep = torch.ones(q, k, dtype=torch.bool)
    if causal:
        keep = torch.arange(k)[None, :] <= torch.arange(q)[:, None] + start
    out = torch.zeros(rows, heads, dtype=torch.float64)
    d = dout.double().sum(0) if not causal else torch.where(keep, dout.double(), torch.zeros((), dtype=torch.float64)).sum(0)
    for h in range(heads):
        out[:, h].index_add_(0, b.reshape(-1), d[h].reshape(-1))
    return out


def window_bucket(M, edges):
    """Pair of buckets of every row of a GSWA table (query - key, per axis)."""
    b = bucket(-torch.arange(1 - M, M), edges, True)
    return (b[:, None] * 2 * (len(edges) + 1) + b[None, :]).reshape(-1)


# ---- AdamW ------------------------------------------------------------------------------------------------------------------------

def adamw_update(p, g, m, v, t, lr, beta1, beta2, eps, weight_decay, clip=1.0):
    """(p', m', v') in 64 bits."""
    p, g, m, v = p.double(), g.double() * clip, m.double(), v.double()
    m = beta1 * m + (1 - beta1) * g
    v = beta2 * v + (1 - beta2) * g * g
    p = p * (1 - lr * weight_decay) - lr * (m / (1 - beta1 ** t)) / (torch.sqrt(v / (1 - beta2 ** t)) + eps)
    return p, m, v


def _mix(x):
    x = x ^ (x >> 16)
    x = x * 0x9E3779B9 & 0xFFFFFFFF
    x = x ^ (x >> 15)
    x = x * 0x6A09E667 & 0xFFFFFFFF
    return x ^ (x >> 16)


def noise(seed, t, first, n):
    """16-bit numbers for m, v and p of the elements first .. first + n of a plan (no 2^32 boundary inside)."""
    key = _mix((seed >> 32) ^ 0x510E527F)
    for part in (seed & 0xFFFFFFFF, t >> 32, t & 0xFFFFFFFF, first >> 32):
        key = _mix(key ^ part)
    h = _mix((torch.arange(n, dtype=torch.int64) + (first & 0xFFFFFFFF)) ^ key)
    return h & 0xFFFF, h >> 16, _mix(h ^ 0xBB67AE85) & 0xFFFF


def round_randomly(x, digits, noise16):
    """Magnitudes cut to `digits` bits behind the leading one, the next 16 bits against the noise."""
    f, e = torch.frexp(x.double().abs())
    step = torch.ldexp(torch.ones_like(f), e - 1 - digits)
    out = torch.sign(x.double()) * torch.floor(x.double().abs() / step + noise16.double() / 65536) * step
    return torch.where(torch.isfinite(x), out, x.double())


def hold(x, noise16, second_moment):
    """What 8 bits hold of one tensor's state (flat): blocks of 256 with a common exponent."""
    n = x.numel()
    pad = -n % 256
    y = torch.nn.functional.pad(round_randomly(x, 3, noise16), (0, pad)).view(-1, 256)
    full = torch.nn.functional.pad(x.double(), (0, pad)).view(-1, 256)
    top = full.abs().amax(1, keepdim=True)
    _, e = torch.frexp(top)
    least = 1.25 * torch.ldexp(torch.ones_like(top), e - 1 - (31 if second_moment else 15))
    small = y.abs() < least
    y = torch.where(small, least.expand_as(y) if second_moment else torch.zeros_like(y), y)
    y = torch.where(full == 0, torch.zeros_like(y), y)
    y = torch.where(torch.isfinite(top), y, torch.full_like(y, math.nan))
    return y.reshape(-1)[:n]


def held_value(codes, exponents, second_moment):
    """Values of stored codes, from the format's description."""
    c = codes.to(torch.int64)
    E = exponents.to(torch.int64).repeat_interleave(256)[: c.numel()]
    size = c if second_moment else c & 127
    T = torch.clamp(size + 8 * (E + 1) - (255 if second_moment else 127), min=1)
    value = (T << 20).to(torch.int32).view(torch.float32).double()
    value = torch.where(size > 0, value, torch.zeros_like(value))
    if not second_moment:
        value = torch.where(c > 127, -value, value)
    return torch.where(E == 255, torch.full_like(value, math.nan), value)
