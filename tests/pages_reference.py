"""The pages of a cache, the 4-bit rows and the selection of pages, plainly on the CPU: requests one by one, elements one by one, whole numbers and 64 bits."""
import math

import torch

GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def plan(table, cached, fresh, seq, free, n_free, page, tokens, n_pages):
    """(lengths, starts, positions, rows, slots, n_free); the table is written in place."""
    n_seqs, max_pages = table.shape
    n_free = max(0, min(int(n_free), free.numel()))
    names = [int(s) for s, f in zip(seq, fresh) if int(f) > 0 and 0 <= int(s) < n_seqs]
    have, asked, wanted = n_free, 0, 0
    lengths, starts, pos, rows, slots = [], [0], [], [], []
    for s, c, f in zip(seq.tolist(), cached.tolist(), fresh.tolist()):
        known = 0 <= s < n_seqs
        valid = known and c >= 0 and f >= 0 and c + f <= min(max_pages * page, 2 ** 31 - 1) and not (f > 0 and names.count(s) > 1)
        c = c if known and c >= 0 else 0
        f = f if valid else 0
        first = -(-c // page)
        need = -(-(c + f) // page) - first if valid else 0
        asked, wanted = asked + need, wanted + f
        if (need and asked > have) or (f and wanted > tokens):
            need = f = 0
        for i in range(need):
            n_free -= 1
            table[s, first + i] = free[n_free]
        for i in range(c, c + f):
            g = int(table[s, i // page])
            pos.append(i)
            rows.append(s)
            slots.append(g * page + i % page if 0 <= g < n_pages else -1)
        lengths.append(c + f)
        starts.append(len(pos))
    fill = [-1] * (tokens - len(pos))
    return lengths, starts, pos + fill, rows + fill, slots + fill, n_free


def release(table, lengths, seq, free, n_free, page, n_pages):
    """How many pages the list holds then; the table and the list are written in place."""
    n_seqs, max_pages = table.shape
    n_free = max(0, min(int(n_free), free.numel()))
    names = [int(s) for s, n in zip(seq, lengths) if int(n) > 0 and 0 <= int(s) < n_seqs]
    back = []
    for s, n in zip(seq.tolist(), lengths.tolist()):
        if n <= 0 or not 0 <= s < n_seqs or names.count(s) > 1:
            continue
        for i in range(min(max_pages, -(-n // page))):
            if 0 <= int(table[s, i]) < n_pages:
                back.append(int(table[s, i]))
            table[s, i] = -1
    for i, g in enumerate(reversed(back)):
        if n_free + i < free.numel():
            free[n_free + i] = g
    return min(free.numel(), n_free + len(back))


def pack(x):
    """Rows [.., K] in 64 bits to (codes [.., K / 2], scales [.., K / 32]): by the distance to each value, a tie to the even code."""
    y = x.double().unflatten(-1, (-1, 32))
    top = y.abs().amax(-1)
    scale = torch.empty(top.shape, dtype=torch.uint8)
    for i in torch.cartesian_prod(*(torch.arange(n) for n in top.shape)).reshape(-1, top.dim()).tolist():
        t = float(top[tuple(i)])
        if not math.isfinite(t):
            scale[tuple(i)] = 255
            continue
        e = -120
        while e < 125 and t > 7.0 * 2.0 ** e:
            e += 1
        scale[tuple(i)] = e + 127
    z = y.abs() / torch.ldexp(torch.ones(1, dtype=torch.float64), scale.int() - 127).unsqueeze(-1)
    grid = torch.tensor(GRID, dtype=torch.float64)
    d = (z.unsqueeze(-1) - grid).abs()
    least = d.amin(-1, keepdim=True)
    odd = torch.arange(8) % 2
    code = torch.where(d == least, odd * 8 + torch.arange(8), 99).amin(-1) % 8             # of the nearest, the even code's
    code = code + 8 * torch.signbit(y)
    code = torch.where((scale == 255).unsqueeze(-1), torch.zeros_like(code), code).flatten(-2)
    return (code[..., 0::2] | (code[..., 1::2] << 4)).to(torch.uint8), scale


def values(codes, scales):
    """The values in 64 bits; a scale of 255: NaN."""
    grid = torch.tensor(GRID + tuple(-g for g in GRID), dtype=torch.float64)
    x = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], dim=-1).flatten(-2).unflatten(-1, (-1, 32))
    s = torch.ldexp(torch.ones(1, dtype=torch.float64), scales.int() - 127)
    return torch.where(scales == 255, torch.full_like(s, math.nan), s).unsqueeze(-1).mul(x).flatten(-2)


def bounds(keys, table, cached, lengths, seq, old):
    """keys [n_pages, page, Hk, K], old [n_pages, Hk, 2, K], both in 64 bits: the bounds with the new tokens."""
    new, page = old.clone(), keys.shape[1]
    for s, c, n in zip(seq.tolist(), cached.tolist(), lengths.tolist()):
        c = max(c, 0)
        if not 0 <= s < table.shape[0]:
            continue
        for i in range(c // page, -(-n // page) if n > c else 0):
            if i >= table.shape[1] or not 0 <= int(table[s, i]) < keys.shape[0]:
                continue
            g, a, b = int(table[s, i]), max(c - i * page, 0), min(n - i * page, page)
            lo, hi = keys[g, a:b].amin(0), keys[g, a:b].amax(0)
            if a > 0:
                lo, hi = torch.minimum(lo, new[g, :, 0]), torch.maximum(hi, new[g, :, 1])
            new[g] = torch.stack([lo, hi], dim=1)
    return new


def select(q, bounds, table, lengths, seq, page, pages, first, last, max_length):
    """(chosen [B,Hk,pages], tokens [B,Hk]); q and bounds in 64 bits."""
    B, Hq, K = q.shape
    n_pages, Hk = bounds.shape[:2]
    G = Hq // Hk
    chosen, tokens = torch.full((B, Hk, pages), -1, dtype=torch.int32), torch.zeros(B, Hk, dtype=torch.int32)
    for b, (n, s) in enumerate(zip(lengths.tolist(), seq.tolist())):
        if n <= 0:
            continue
        have = -(-n // page)
        if not 0 <= s < table.shape[0] or n > max_length or have > table.shape[1]:
            tokens[b] = 2 ** 31 - 1
            continue
        at = table[s, :have].tolist()
        for h in range(Hk):
            score = []
            for g in at:
                if not 0 <= g < n_pages:
                    score.append(math.inf)
                    continue
                qh = q[b, h * G:(h + 1) * G]
                x = float(torch.maximum(qh * bounds[g, h, 0], qh * bounds[g, h, 1]).sum())
                score.append(1e400 if math.isnan(x) else x)
            always = set(range(min(first, have))) | set(range(max(0, have - last), have))
            rest = sorted((i for i in range(have) if i not in always), key=lambda i: (-score[i], i))
            take = range(have) if have <= pages else sorted(list(always) + rest[: pages - first - last])
            for j, i in enumerate(take):
                chosen[b, h, j] = at[i] if 0 <= at[i] < n_pages else -1
            tokens[b, h] = (len(take) - 1) * page + (n - 1) % page + 1
    return chosen, tokens
