"""The operators that keep nothing between the passes in 64 bits, from their definitions, with bounds on what fp32 arithmetic and the roundings
that the operators document may be off by.  Works on the device that its inputs are on.

A sum of K products in fp32 is off by at most (K + 1) half steps of the sum of their magnitudes: K - 1 additions, in any order, and, with
fp32 data, a rounding of each product; the matrix cores add in no wider steps than that.  One more for what a split adds.
"""
import math

import torch

U32 = 2.0 ** -24               # half a step of fp32, relative
FLUSH = 2.0 ** -125            # smaller numbers may come out as 0 on the way


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def product(a, b_t):
    """a b_t^T and what fp32 sums may be off by."""
    a, b = a.double(), b_t.double()
    return a @ b.t(), (a.shape[1] + 2) * U32 * (a.abs() @ b.abs().t())


# ---- log-probabilities from the head's input

def linear_logprobs(x, weight, targets, scale):
    z, z_off = product(x, weight)
    rows, vocab = z.shape
    most = z.amax(1)
    none = most == -math.inf
    safe = torch.where(none, 0.0, most)
    d = scale * (z - safe[:, None])
    log_sum = torch.where(none, 0.0, torch.logsumexp(d, 1))
    logp = torch.where(none[:, None], -math.inf, d - log_sum[:, None])
    # an exponent is off by what z and the maximum are off by and by two roundings of itself, of which 30 count (exp(-30) V is nothing); the sums
    # are at most V / 256 + 24 additions one after another
    finite = torch.where(torch.isfinite(z_off), z_off, 0.0).amax(1)
    log_sum_off = 2 * scale * finite + (60 + vocab / 256 + 130) * U32 + U32 * log_sum.abs()
    has = (targets >= 0) & (targets < vocab)
    at = torch.where(has, targets, 0)[:, None]
    logprob = torch.where(has, logp.gather(1, at)[:, 0], 0.0)
    logprob_off = 2 * scale * finite + log_sum_off + 4 * U32 * torch.where(torch.isfinite(logprob), logprob.abs() + log_sum.abs(), 0.0)
    return {"z": z, "most": most, "most_off": finite, "log_sum": log_sum, "log_sum_off": log_sum_off, "logp": logp, "has": has, "at": at,
            "logprob": logprob, "logprob_off": torch.where(has, logprob_off, 0.0)}


def linear_logprobs_backward(x, weight, targets, scale, d_logprob, dtype):
    """(d_x, off, d_weight, off): dtype is the operands', to which d_z is rounded."""
    f = linear_logprobs(x, weight, targets, scale)
    d = torch.where(f["has"], d_logprob.double(), 0.0)[:, None]
    p = f["logp"].exp()
    one = torch.zeros_like(p).scatter_(1, f["at"], 1.0)
    d_z = torch.where(d == 0, 0.0, scale * d * (one - p))
    logp = torch.where(p > 0, f["logp"], 0.0)
    p_off = p * (2 * scale * f["most_off"][:, None] + f["log_sum_off"][:, None] + (5 * logp.abs() + 10) * U32) + FLUSH
    off = (scale * d).abs() * p_off + d_z.abs() * (half_step(dtype) + 3 * U32)
    x, w = x.double(), weight.double()
    d_x, d_w = d_z @ w, d_z.t() @ x
    big = d_z.abs() + off
    d_x_off = off @ w.abs() + (d_z.shape[1] + 66) * U32 * (big @ w.abs())             # up to 64 parts and pieces
    d_w_off = off.t() @ x.abs() + (d_z.shape[0] + 66) * U32 * (big.t() @ x.abs())
    return d_x, d_x_off, d_w, d_w_off


# ---- gated projections

def gated_linear(x, w_gate, w_up):
    g, g_off = product(x, w_gate)
    u, u_off = product(x, w_up)
    t = torch.sigmoid(g)
    silu = g * t
    # |silu'| < 1.1; the exponential's argument is rounded: relative 3 |g| half steps, and a dozen roundings
    off = 1.1 * g_off * (u.abs() + u_off) + silu.abs() * u_off + (silu * u).abs() * (14 + 3 * g.abs()) * U32 + FLUSH * u.abs()
    return {"g": g, "g_off": g_off, "u": u, "u_off": u_off, "out": silu * u, "out_off": off}


def gated_gradients(g, g_off, u, u_off, d_out, dtype):
    """(d_g, off, d_u, off) for g and u that are off by so much."""
    d, t = d_out.double(), torch.sigmoid(g)
    slope = t * (1 + g * torch.sigmoid(-g))                 # |slope| < 1.1, its own slope at most 0.5
    d_g, d_u = d * u * slope, d * g * t
    few = (24 + 3 * g.abs()) * U32
    g_part = d.abs() * (u.abs() * 0.5 * g_off + 1.1 * u_off) + (d * u).abs() * t * (1 + g.abs()) * few + FLUSH
    u_part = d.abs() * 1.1 * g_off + d_u.abs() * few + FLUSH
    return (d_g, g_part + (d_g.abs() + g_part) * half_step(dtype), d_u, u_part + (d_u.abs() + u_part) * half_step(dtype))


def gated_linear_backward(g, g_off, u, u_off, x, w_gate, w_up, d_out, dtype):
    d_g, d_g_off, d_u, d_u_off = gated_gradients(g, g_off, u, u_off, d_out, dtype)
    x, wg, wu = x.double(), w_gate.double(), w_up.double()

    def both(a, a_off, b):
        n = a.shape[1]
        return a @ b, a_off @ b.abs() + (n + 66) * U32 * ((a.abs() + a_off) @ b.abs())

    gx, gx_off = both(d_g, d_g_off, wg)
    ux, ux_off = both(d_u, d_u_off, wu)
    wgs, wgs_off = both(d_g.t(), d_g_off.t(), x)
    wus, wus_off = both(d_u.t(), d_u_off.t(), x)
    return {"d_x": gx + ux, "d_x_off": gx_off + ux_off + 2 * U32 * (gx.abs() + ux.abs()), "d_w_gate": wgs, "d_w_gate_off": wgs_off,
            "d_w_up": wus, "d_w_up_off": wus_off}


# ---- dropout

def philox(counter, key):
    """Philox4x32-10: four words from four words of counter and two of key, Python's whole numbers."""
    c, k = list(counter), list(key)
    for _ in range(10):
        a, b = 0xD2511F53 * c[0], 0xCD9E8D57 * c[2]
        c = [(b >> 32) ^ c[1] ^ k[0], b & 0xFFFFFFFF, (a >> 32) ^ c[3] ^ k[1], a & 0xFFFFFFFF]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def keep(rows, cols, p, seed, offset):
    """Truth values [rows, cols]."""
    blocks = -(-cols // 4)
    least = round(p * 2 ** 32)
    out = torch.zeros(rows, blocks * 4, dtype=torch.bool)
    for i in range(rows):
        for b in range(blocks):
            n = (offset + i * blocks + b) % 2 ** 64
            words = philox((n & 0xFFFFFFFF, n >> 32, 0, 0), (seed & 0xFFFFFFFF, seed >> 32))
            out[i, 4 * b:4 * b + 4] = torch.tensor([w >= least for w in words])
    return out[:, :cols]


def dropout(x, p, seed, offset, residual=None):
    factor = float(torch.tensor(1 / (1 - p) if p < 1 else 0.0, dtype=torch.float32))
    y = torch.where(keep(x.shape[0], x.shape[1], p, seed, offset), x.double() * factor, 0.0)
    return y if residual is None else y + residual.double()
