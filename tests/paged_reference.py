"""Plain forms in 64 bits of the calls on paged caches and of the log probabilities, with the error each may be off by."""
import math
import struct

import torch

E4M3_MAX = 448.0
# a3_paged_rows, a3_paged_queries and a3_logit_rows as bytes, for calls of the library that the binding would not make
PAGED_ROWS = struct.Struct("@8P4Q4i")
PAGED_QUERIES = struct.Struct("@6P2Q2ifi")
LOGIT_ROWS = struct.Struct("@6PQ4i")


def turned(x, pos, theta, layout):
    """Rows x [M][heads][D] rotated to positions pos [M]; also the sum of the magnitudes that go into each element."""
    x, d = x.double(), x.shape[-1]
    angle = pos.double()[:, None] * theta ** (-torch.arange(0, d, 2, device=x.device, dtype=torch.float64) / d)
    c, s = angle.cos()[:, None], angle.sin()[:, None]
    a, b = (x[..., : d // 2], x[..., d // 2:]) if layout == 0 else (x[..., 0::2], x[..., 1::2])
    lo, hi, mag = a * c - b * s, a * s + b * c, a.abs() + b.abs()
    if layout == 0:
        return torch.cat([lo, hi], -1), torch.cat([mag, mag], -1)
    return torch.stack([lo, hi], -1).flatten(-2), torch.stack([mag, mag], -1).flatten(-2)


def gathered(pool, scale, table, n):
    """Slots 0..n-1 of a sequence, [n][heads][D] in 64 bits."""
    size = pool.shape[1]
    t = torch.arange(n, device=pool.device)
    x = pool.view(torch.uint8)[table.long()[t // size], t % size].view(pool.dtype).double()
    return x if scale is None else x * scale.double()[:, None]


def attention(q, k, v, scale, packed, q_heads):
    """One sequence: q [Hq][D], k and v [n][Hkv][D]; returns (out, lse, bounds of their errors).

    A logit is a sum of D products in fp32, off by D 2^-24 of the sum of their magnitudes at most, then scaled (2^-23 of itself) and
    raised by an exponential that is off by 2^-22: a weight is off by a relative delta of those together, the output by 2 delta of
    sum p |v| (in the products and in the sum that divides).  A weight enters the product with two bf16 terms (2^-17 of itself)
    or, with 8-bit values, as fp16 (2^-11 of itself, 2^-25 where it is small); sums of n terms in fp32 add n 2^-24.  The output is rounded to
    bf16: 2^-8 of itself."""
    n, hkv, d = k.shape
    q = q.double().view(hkv, q_heads // hkv, d)
    x = torch.einsum("hgd,nhd->hgn", q, k) * scale
    size = torch.einsum("hgd,nhd->hgn", q.abs(), k.abs()) * abs(scale)
    delta = (size.amax(-1) * d * 2.0 ** -24 + x.abs().amax(-1) * 2.0 ** -22 + 2.0 ** -22 + n * 2.0 ** -24)[..., None]
    p = torch.softmax(x, -1)
    out, mass = torch.einsum("hgn,nhd->hgd", p, v), torch.einsum("hgn,nhd->hgd", p, v.abs())
    bound = out.abs() * 2.0 ** -8 + mass * (2 * delta + (2.0 ** -11 if packed else 2.0 ** -16))
    if packed:
        bound = bound + n * 2.0 ** -25 * v.abs().amax()
    lse = torch.logsumexp(x, -1)
    return out.reshape(q_heads, d), lse.flatten(), bound.reshape(q_heads, d), (delta[..., 0] + lse.abs() * 2.0 ** -22).flatten()


def logprobs(logits):
    """(log softmax, entropy, bounds of both).  Sums of V terms in fp32, each term's exponential off by 2^-21 in all where it counts
    (the argument |d| <= 20 rounded once, 2^-24 |d| log2 e): r relative; log of it r absolute, entropy's second term 2 r of itself."""
    x = logits.double()
    lp = torch.log_softmax(x, 1)
    p = lp.exp()
    h = -torch.where(p > 0, p * lp, torch.zeros_like(p)).sum(1)
    r = 2.0 ** -19 + (x.shape[1] / 512 + 64) * 2.0 ** -24
    lse = torch.logsumexp(x, 1)
    top = x.amax(1)
    # |x - M| and log s are rounded once each
    return lp, h, r + (lp.abs() + (lse - top).abs()[:, None] * 2) * 2.0 ** -23, r * (1 + 3 * (h + (lse - top).abs()))


def ranked(logits, n):
    """Ids of the n largest, ties to the lower id, NaN last."""
    x = torch.nan_to_num(logits.double(), nan=-math.inf, posinf=math.inf, neginf=-1e300) + 0.0
    return torch.argsort(x, dim=1, descending=True, stable=True)[:, :n]
