"""Attention of one token in 64 bits, with the magnitudes that meet in every element of its result, and the interval that they leave for a
result in bf16.

A score is off by ds = (K / 4 + 8) 2^-24 A, A = scale sum |q_i k_i| (the largest of the row's), a weight e^(s - m) by a factor of 1 +- (2 ds + 2^-21).
For the product with the values a weight is the sum of two bf16 numbers: the first is within 2^-7 of it, the second the rest rounded,
together within 2^-16.  The sum of the weights is at most n / 4 + 64 additions deep (a lane has a quarter of a wavefront's tokens), each 2^-24; the
products with the values go through at most n / 16 + 32 sums, each 2^-23 (the matrix cores' own may be cut off).  The division adds 2^-21.
So an element is sum p_j v_j / l before it is rounded, off by at most
    e = (4 ds + 2^-19 + 2^-16 + (n / 4 + 64) 2^-24 + (n / 16 + 32) 2^-23) sum p_j |v_j| / l
and, as rounding keeps the order, the result lies between the roundings of the exact value less e and plus e."""
import torch


def attention(q, k, v, scale):
    """(o, e) of one query q [K] over k, v [n,K], all in 64 bits."""
    n, K = k.shape
    s = scale * (k @ q)
    p = torch.exp(s - s.max())
    p = p / p.sum()
    ds = (K / 4 + 8) * 2.0 ** -24 * abs(scale) * float((k.abs() @ q.abs()).max())
    return p @ v, (4 * ds + 2.0 ** -19 + 2.0 ** -16 + (n / 4 + 64) * 2.0 ** -24 + (n / 16 + 32) * 2.0 ** -23) * (p @ v.abs())


def outside(got, want, e):
    """Which elements of a bf16 result (as float64) lie outside the interval."""
    lo, hi = ((want + x).float().bfloat16().double() for x in (-e, e))
    return ~((got >= lo) & (got <= hi))


def paged(q, k_cache, v_cache, table, lengths, seq, scale, window):
    """(o, e) [B,Hq,K] over a paged cache; rows that see nothing are zero."""
    B, Hq, K = q.shape
    page, Hk = k_cache.shape[1], k_cache.shape[2]
    o, e = torch.zeros(B, Hq, K, dtype=torch.float64), torch.zeros(B, Hq, K, dtype=torch.float64)
    for b in range(B):
        n = int(lengths[b])
        if n <= 0:
            continue
        j = torch.arange(max(0, n - window) if window else 0, n)
        at = table[int(seq[b])][j // page].long(), j % page
        k, v = k_cache[at], v_cache[at]
        for h in range(Hq):
            kv = h * Hk // Hq
            o[b, h], e[b, h] = attention(q[b, h], k[:, kv], v[:, kv], scale)
    return o, e
