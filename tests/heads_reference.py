"""The operators around the recurrence, plainly, in 64 bits on the CPU: norm and rotation of rows, the append to a paged cache and
attention over it, token by token and page by page."""
import math

import torch


def f64(t):
    return None if t is None else t.detach().double().cpu()


def turn(y, table, pos, interleaved, sign=1.0):
    """Pairs of y [..., K] turned by the angles of pos [...] (broadcast over the heads axis before the last)."""
    if table is None:
        return y
    R = table.shape[1]
    cos, sin = table[pos][..., : R // 2].unsqueeze(-2), sign * table[pos][..., R // 2:].unsqueeze(-2)
    z = y.clone()
    for i in range(R // 2):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + R // 2)
        z[..., a] = y[..., a] * cos[..., i] - y[..., b] * sin[..., i]
        z[..., b] = y[..., a] * sin[..., i] + y[..., b] * cos[..., i]
    return z


def norm_rows(x, w, table, pos, norm, eps, interleaved):
    """x [B,T,H,K] in 64 bits; pos [B,T]; tokens of a negative position are zero.  Differentiable."""
    y = x
    if norm != "none":
        m = 1.0 if norm == "l2" else 1.0 / x.shape[-1]
        y = x * (m * (x * x).sum(-1, keepdim=True) + eps) ** -0.5
    if w is not None:
        y = y * w
    y = turn(y, table, pos.clamp(min=0), interleaved)
    return torch.where((pos < 0)[..., None, None], torch.zeros_like(y), y)


def decode(q, k_cache, v_cache, table, lengths, seq, scale, window):
    """(o [B,Hq,K], lse [B,Hq]) in 64 bits, and per query head the largest sum of |q_i k_i| scale over the tokens seen."""
    B, Hq, K = q.shape
    page, Hk = k_cache.shape[1], k_cache.shape[2]
    o, lse = torch.zeros(B, Hq, K, dtype=torch.float64), torch.full((B, Hq), -math.inf, dtype=torch.float64)
    size = torch.zeros(B, Hq, dtype=torch.float64)
    for b in range(B):
        n = int(lengths[b])
        lo = max(0, n - window) if window else 0
        if n <= 0:
            continue
        j = torch.arange(lo, n)
        g = table[int(seq[b])][j // page].long()
        k, v = k_cache[g, j % page], v_cache[g, j % page]                 # [n, Hk, K]
        for h in range(Hq):
            kv = h * Hk // Hq
            s = scale * (k[:, kv] @ q[b, h])
            size[b, h] = abs(scale) * (k[:, kv].abs() @ q[b, h].abs()).max()
            m = s.max()
            p = torch.exp(s - m)
            o[b, h] = (p @ v[:, kv]) / p.sum()
            lse[b, h] = m + torch.log(p.sum())
    return o, lse, size
