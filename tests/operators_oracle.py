"""The operators around the step in 64 bits on the CPU, from their definitions, with bounds on what fp32 arithmetic may be off by."""
import math

import torch

U32 = 2.0 ** -24               # half a step of fp32, relative
FLUSH = 2.0 ** -126            # smaller results may come out as 0
E4M3 = [(-1.0) ** (b >> 7) * (math.ldexp(8 + (b & 7), ((b >> 3) & 15) - 10) if (b >> 3) & 15 else math.ldexp(b & 7, -9)) for b in range(256)]
E4M3[0x7F] = E4M3[0xFF] = math.nan
TABLE = torch.tensor(E4M3, dtype=torch.float64)


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def ld8(cols):
    return -(-cols // 32) * 32


def pow2(e):
    return ((e.long() + 1023) << 52).view(torch.float64)


# ---- checkpoints

def pack(x):
    """(codes uint8 [rows, ld8], exponents int64 [rows, ld8 / 32]) of a matrix."""
    rows, cols = x.shape
    x = torch.cat([x.double(), torch.zeros(rows, ld8(cols) - cols, dtype=torch.float64)], 1).view(rows, ld8(cols) // 32, 32)
    finite = torch.isfinite(x)
    x = torch.where(finite & (x.abs() >= 1.9375 * 2.0 ** 127), torch.sign(x) * 1.875 * 2.0 ** 127, x)      # 2^128 would be no number
    largest = torch.where(finite, x.abs(), 0.0).amax(2, keepdim=True)
    e = torch.full_like(largest, -100, dtype=torch.int64)
    while True:                                            # the smallest e >= -100 with largest <= 448 * 2^e
        more = largest > 448 * pow2(e)
        if not more.any():
            break
        e = e + more.long()
    y = torch.where(finite, x, 0.0) * pow2(-e)
    # the nearest of the positive codes 0 .. 0x7E, whose values rise; of two equally near the even one
    values = TABLE[:0x7F]
    hi = torch.searchsorted(values, y.abs()).clamp(max=0x7E)
    lo = (hi - 1).clamp(min=0)
    up, down = values[hi] - y.abs(), y.abs() - values[lo]
    code = torch.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    code = torch.where(torch.signbit(x) & finite, code + 128, code)
    return torch.where(finite, code, 0x7F).to(torch.uint8).view(rows, -1), e[:, :, 0]


def pack_bytes(x):
    codes, e = pack(x)
    return torch.cat([codes.reshape(-1), (e + 127).to(torch.uint8).reshape(-1)])


def values(ckpt, rows, cols):
    """What a checkpoint's bytes stand for, [rows, cols]."""
    ld = ld8(cols)
    x = TABLE[ckpt[:rows * ld].long()].view(rows, ld // 32, 32)
    return (x * pow2(ckpt[rows * ld:].long() - 127).view(rows, ld // 32, 1)).view(rows, ld)[:, :cols]


# ---- token log-probabilities

def logprobs(logits, targets, scale):
    """dict of 64-bit results and, as *_off, what they may be off by in fp32: for a row of V values summed by at most V / 256 + 24
    additions one after another, of exponentials whose argument is rounded twice and counts up to 30 (exp(-30) V is nothing)."""
    z = logits.double()
    vocab = z.shape[1]
    most = z.amax(1)
    none = most == -math.inf
    safe = torch.where(none, 0.0, most)
    d = scale * (z - safe[:, None])
    log_sum = torch.where(none, 0.0, torch.logsumexp(d, 1))
    logp = torch.where(none[:, None], -math.inf, d - log_sum[:, None])
    p = logp.exp()
    entropy = -torch.where(p == 0, 0.0, p * logp).sum(1)
    has = (targets >= 0) & (targets < vocab)
    at = torch.where(has, targets, 0)[:, None]
    out = {"most": most, "log_sum": log_sum, "logp": logp, "entropy": torch.where(none, 0.0, entropy),
           "logprob": torch.where(has, logp.gather(1, at)[:, 0], 0.0)}
    steps = vocab / 256 + 24 + 3 * 30 + 8
    out["log_sum_off"] = U32 * (steps + 2 * log_sum.abs())
    weighted = torch.where(p == 0, 0.0, p * d.abs()).sum(1)
    out["entropy_off"] = U32 * (2 * steps * (1 + weighted) + 4 * log_sum.abs())
    out["logp_off"] = out["log_sum_off"][:, None] + U32 * torch.where(logp == -math.inf, 0.0, 3 * d.abs() + logp.abs())
    out["logprob_off"] = torch.where(has, out["logp_off"].gather(1, at)[:, 0], 0.0)
    return out


def top(logits, k):
    """Indices of the k largest of each row; equal ones in order, NaN first."""
    return torch.sort(logits.double(), dim=1, descending=True, stable=True).indices[:, :k]


def logprobs_backward(logits, targets, scale, d_logprob, d_entropy):
    """(gradient, what it may be off by before it is rounded to its type)."""
    f = logprobs(logits, targets, scale)
    logp, p = f["logp"], f["logp"].exp()
    has = (targets >= 0) & (targets < logits.shape[1])
    one = torch.zeros_like(p)
    one[has.nonzero()[:, 0], targets[has]] = 1.0
    one[f["most"] == -math.inf] = 0.0
    dl = torch.where(has, d_logprob.double(), 0.0)[:, None]
    dh = d_entropy.double()[:, None]
    h = f["entropy"][:, None]
    lp = torch.where(p == 0, 0.0, logp)
    grad = scale * (dl * (one - p) - dh * p * (lp + h))
    size = scale * (dl.abs() * (one + p) + dh.abs() * p * (lp.abs() + h))
    off = size * (f["logp_off"] + 16 * U32) + scale * dh.abs() * p * (f["logp_off"] + f["entropy_off"][:, None])
    return grad, torch.where(torch.isnan(off), 0.0, off) + FLUSH


# ---- gated activation

def _sigmoid_off(g):
    """Relative: the exponential's argument is rounded, then it, the sum and the reciprocal (at most a step each)."""
    return U32 * (3 * g.abs() + 10)


def swiglu(gate, up):
    g, u = gate.double(), up.double()
    out = g * torch.sigmoid(g) * u
    return out, out.abs() * (_sigmoid_off(g) + 4 * U32) + (g * u).abs() * FLUSH + FLUSH


def swiglu_backward(d_out, g, u):
    """((d_gate, off), (d_up, off), (out, off)) at the 64-bit values g, u."""
    d = d_out.double()
    t = torch.sigmoid(g)
    silu, r = g * t, _sigmoid_off(g)
    slope = t + silu * (1 - t)
    slope_off = r * (t + silu.abs() * (1 - t) + silu.abs() * t) + 8 * U32 * (t + silu.abs()) + (1 + g.abs()) * FLUSH
    d_gate = d * u * slope
    d_up = d * silu
    return ((d_gate, (d * u).abs() * (slope_off + 4 * U32 * slope.abs()) + FLUSH),
            (d_up, d_up.abs() * (r + 4 * U32) + (d * g).abs() * FLUSH + FLUSH), swiglu(g, u))


# ---- weight gradient

def wgrad(d_out, x):
    """(d_out^T x, off): sums of exact products, every addition rounded (twice the half step covers other roundings than to nearest)."""
    y = d_out.double()
    return y.t() @ x, (d_out.shape[0] + 8) * 2 * U32 * (y.abs().t() @ x.abs()) + FLUSH
