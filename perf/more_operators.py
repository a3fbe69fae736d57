"""What serving adds to the paged cache, as cases to be timed: the page table and the places of new tokens from the
lengths of the requests, a cache of 4-bit keys and values (append, attention of one token over it), and attention over a few
pages that a cheap score selects for each query, over a cache of either kind.

``listed()`` names the cases, ``draw(rng)`` makes one more of the same ranges, ``prepare`` builds
what the program holds before the call, ``run`` makes one pass, ``work`` says what a pass cannot do
without, and ``exact`` is the definition in 64 bits.  With ``own`` false ``run`` computes the operators with
elementary torch operations, with ``own`` true through ``paper_2605_13473_amd.binding``.

Fields of a case
  kind        plan      B requests, a token or a prompt each: pages from the list of free ones, lengths, places of the tokens
              turnover  B sequences end and give their pages back, B prompts take their rows
              append    T new tokens of each of B sequences into a 4-bit cache, queries made ready in the same pass, and read back
              packed    the same of prompts packed on one token axis of T tokens
              decode    one new token for each of B sequences over a 4-bit cache of up to T tokens
              sparse    the same over the pages that are selected: bounds of the newest page, selection, attention
  B T Hq Hk K sizes (K: width of a head); io "bf16" or "f32": queries and results (sparse: and the cache, unless it is in 4 bits)
  page        tokens of a page; order "head" (a page holds its tokens head after head) or "token"
  prompts     plan: some requests are whole prompts (T: tokens in all, at most)
  short       plan: the list of free pages does not do for all
  ragged      decode, sparse: lengths spread from 1 to T, some sequences empty
  window      decode: only the last so many tokens are seen (0: all)
  pages       sparse: pages selected, at most
  mx          sparse: the cache is in 4 bits
  norm rotary append: as by the append to a cache of whole numbers of bytes ("rms" with learned weights, "l2" or "none"; elements that turn)

A row of the 4-bit cache: blocks of 32 adjacent elements share a scale 2^e, kept as the byte e + 127, and every element is a sign
and one of 0, 1/2, 1, 3/2, 2, 3, 4, 6 times the scale, the nearest (ties to the even code); e is the smallest, from -120 to 125, with the
largest element no more than 7 * 2^e.
"""
import math

import numpy as np
import torch

own = False

THETA, EPS = 10000.0, 1e-6
GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _attend(kind, B, T, Hq, Hk, K=128, io="bf16", page=64, order="head", ragged=False, window=0, pages=0, mx=True, name=None):
    c = dict(kind=kind, B=B, T=T, Hq=Hq, Hk=Hk, K=K, io=io, page=page, order=order, ragged=ragged)
    c.update(dict(window=window) if kind == "decode" else dict(pages=pages, mx=mx))
    return c if name is None else dict(c, name=name)


def _append(kind, B, T, Hq, Hk, K=128, io="bf16", page=64, order="head", norm="rms", rotary=128, name=None):
    c = dict(kind=kind, B=B, T=T, Hq=Hq, Hk=Hk, K=K, io=io, page=page, order=order, norm=norm, rotary=rotary)
    return c if name is None else dict(c, name=name)


def _plan(kind, B, T, page=64, prompts=False, short=False, name=None):
    c = dict(kind=kind, B=B, T=T, page=page)
    if kind == "plan":
        c.update(prompts=prompts, short=short)
    return c if name is None else dict(c, name=name)


def listed():
    return [
        # a serving batch of conversations, one token each: a page now and then
        _plan("plan", 256, 256, page=16, name="plan_256_tokens"),
        # prompts and conversations in one batch, more than the free pages hold
        _plan("plan", 96, 65536, prompts=True, short=True, name="plan_prompts_65536"),
        # a batch of prompts takes the place of one that is through
        _plan("turnover", 64, 1531, name="turnover_64"),
        # one user, one token: all latency
        _append("append", 1, 1, 16, 4, page=16, name="append_mx_one_sequence"),
        # a serving batch, one token per sequence
        _append("append", 512, 1, 16, 4, name="append_mx_512"),
        # prompts packed on one token axis go into the cache
        _append("packed", 1, 65536, 16, 4, name="append_mx_packed_65536"),
        # one user, one token, a context of some pages and a bit
        _attend("decode", 1, 1531, 16, 4, page=16, name="decode_mx_one_sequence"),
        # one long context
        _attend("decode", 1, 131072, 32, 8, name="decode_mx_long_context"),
        # the full serving batch
        _attend("decode", 512, 4096, 16, 4, ragged=True, name="decode_mx_512_ragged"),
        # one long context of which 64 pages are read
        _attend("sparse", 1, 131072, 32, 8, page=32, pages=64, mx=False, name="sparse_long_context"),
        # a batch of long conversations in 4 bits, a page order that comes with the projection
        _attend("sparse", 48, 32768, 32, 8, order="token", ragged=True, pages=32, name="sparse_mx_48_ragged"),
        # fp32, every query head with its own keys (debugging, ablations)
        _attend("sparse", 8, 4096, 8, 8, K=64, io="f32", page=16, pages=40, mx=False, name="sparse_fp32"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "turnover", "append", "packed", "decode", "decode", "sparse", "sparse"])
    page = rng.choice([8, 16, 32, 64, 128])
    if kind == "plan":
        prompts = rng.random() < 0.5
        B = _log_int(rng, 1, 2048)
        return _plan(kind, B, _log_int(rng, max(B, 100), 65536) if prompts else B, page, prompts, rng.random() < 0.4)
    if kind == "turnover":
        B = _log_int(rng, 1, 256)
        return _plan(kind, B, _log_int(rng, 1, min(8192, 65536 // B)), page)
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    es = 2 if io == "bf16" else 4
    K = rng.choice([64, 128, 128, 256])
    Hk = rng.choice([1, 2, 4, 8, 16])
    Hq = Hk * rng.choice([1, 2, 4, 5, 7, 8, 16])
    if Hq > 64:
        Hq = Hk * 2
    order = rng.choice(["head", "token"])
    if kind in ("append", "packed"):
        c = dict(norm=rng.choice(["l2", "rms", "rms", "none"]), rotary=rng.choice([0, K, K, K // 2]), page=page, order=order)
        most = (1 << 28) // ((Hq + 2 * Hk) * K * es)
        if kind == "packed":
            return _append(kind, 1, _log_int(rng, 100, min(65536, most)), Hq, Hk, K, io, **c)
        T = rng.choice([1, 1, _log_int(rng, 2, 64)])
        return _append(kind, _log_int(rng, 1, min(512, most // T)), T, Hq, Hk, K, io, **c)
    # at most a quarter of the tokens of the largest listed case (uneven lengths halve it there)
    most = (1 << 28) // (Hk * K * 2)
    T = _log_int(rng, 1, min(131072, most))
    B = _log_int(rng, 1, max(1, min(512, most // T)))
    ragged = rng.random() < 0.6
    if kind == "decode":
        return _attend(kind, B, T, Hq, Hk, K, io, page, order, ragged, window=rng.choice([0, 0, 0, _log_int(rng, 1, T)]))
    return _attend(kind, B, T, Hq, Hk, K, io, page, order, ragged, pages=_log_int(rng, 2, 256), mx=rng.random() < 0.5)


# ------------------------------------------------------------------------------------ inputs ----
def _shape_rng(case):
    return np.random.Generator(np.random.Philox(case["B"] * 1000003 + case["T"]))


def _lengths(case):
    """Lengths of the cached sequences (part of the case's shape: the same for every seed)."""
    B, T = case["B"], case["T"]
    if not case["ragged"]:
        return [T] * B
    rng = _shape_rng(case)
    n = [1 + int(x * (T - 1)) for x in rng.random(B)]
    n[0] = T
    for b in range(1, B):
        if rng.random() < 1 / 16:
            n[b] = 0                    # a slot of the batch that nobody uses
    return n


def _visible(case):
    """Tokens that attention reads, over all sequences."""
    return sum(min(n, case["window"]) if case["window"] else n for n in _lengths(case))


def _append_places(case):
    """(sequence, position) of every new token, and how many tokens each sequence then has."""
    B, T = case["B"], case["T"]
    rng = _shape_rng(case)
    if case["kind"] == "append":        # T tokens each, behind what the cache holds already
        before = [int(x) for x in rng.integers(0, 4096, B)]
        seq = np.repeat(np.arange(B), T)
        pos = (np.array(before)[:, None] + np.arange(T)[None, :]).reshape(-1)
        return seq, pos, [n + T for n in before]
    cu = [0]
    while cu[-1] < T:                   # prompts of the lengths of packed documents
        cu.append(min(T, cu[-1] + min(4096, 1 + int(rng.exponential(1200.0)))))
    lens = [b - a for a, b in zip(cu, cu[1:])]
    return np.repeat(np.arange(len(lens)), lens), np.concatenate([np.arange(n) for n in lens]), lens


def _table(lens, page, rng):
    """A page table whose pages lie in any order, and the number of pages."""
    need = [max(1, -(-n // page)) for n in lens]
    order = rng.permutation(sum(need))
    table = np.full((len(lens), max(need)), -1, dtype=np.int32)
    at = 0
    for b, n in enumerate(need):
        table[b, :n] = order[at:at + n]
        at += n
    return table, int(sum(need))


def _requests(case):
    """Tokens that the sequences have, tokens that are new, and free pages (part of the case's shape)."""
    c, rng = case, _shape_rng(case)
    B, T, page = c["B"], c["T"], c["page"]
    if c["kind"] == "turnover":
        cached, fresh = [0] * B, [1 + int(x * (T - 1)) for x in rng.random(B)]
    else:
        cached, fresh = [int(x) for x in rng.integers(0, 4096, B)], [1] * B
        if c["prompts"]:
            left = T - B
            for b in range(B):
                if rng.random() < 0.7 and left > 0:
                    fresh[b] += min(left, int(rng.exponential(1.4 * T / B)))
                    left -= fresh[b] - 1
                    cached[b] = cached[b] if rng.random() < 0.3 else 0
                elif rng.random() < 0.1:
                    fresh[b] = 0
    need = [-(-(n + m) // page) - -(-n // page) for n, m in zip(cached, fresh)]
    spare = 5 if c["kind"] == "turnover" else sum(need) // 2 if c["short"] else sum(need) + 7
    return cached, fresh, need, spare


def _rotary_table(rows, width, dev):
    """[rows, width]: the cosines of a position's angles, then their sines."""
    angle = torch.arange(rows, dtype=torch.float64, device=dev)[:, None] * THETA ** (
        -2.0 * torch.arange(width // 2, dtype=torch.float64, device=dev) / width)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _stored(rows, c):
    """[pages, heads, slots, *] put into the case's order: [pages, slots, heads, *]."""
    t = rows.transpose(1, 2)
    return t if c["order"] == "head" else t.contiguous()


def _cache(n_pages, c, rnd, dt):
    return _stored(rnd(n_pages, c["Hk"], c["page"], c["K"]).to(dt), c)


def _cache_mx(n_pages, c, rnd):
    """Codes [pages, slots, heads, K / 2] and scales [pages, slots, heads, K / 32] of rows of that distribution."""
    codes, scales = [], []
    step = max(1, (1 << 26) // (c["Hk"] * c["page"] * c["K"]))
    for at in range(0, n_pages, step):
        q, e = _pack(rnd(min(step, n_pages - at), c["Hk"], c["page"], c["K"]))
        codes.append(q)
        scales.append(e)
    return _stored(torch.cat(codes), c), _stored(torch.cat(scales), c)


def _bounds_of(values, count):
    """Smallest and largest of the first `count` [pages] tokens of every page, for each head and element: [pages, heads, 2, K]."""
    page = values.shape[1]
    out = []
    step = max(1, (1 << 26) // (page * values.shape[2] * values.shape[3]))
    for at in range(0, values.shape[0], step):
        x, n = values[at:at + step], count[at:at + step]
        there = (torch.arange(page, device=x.device)[None] < n[:, None])[:, :, None, None]
        two = torch.stack([x.masked_fill(~there, math.inf).amin(1), x.masked_fill(~there, -math.inf).amax(1)], dim=2)
        out.append(two.masked_fill((n == 0)[:, None, None, None], 0.0))
    return torch.cat(out)


def prepare(case, seed):
    c = case
    B, T = c["B"], c["T"]
    dev = "cuda"
    host = np.random.Generator(np.random.Philox(seed))
    i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=dev)
    s = dict(case=c)
    if c["kind"] in ("plan", "turnover"):
        cached, fresh, need, spare = _requests(c)
        held = need if c["kind"] == "turnover" else [-(-n // c["page"]) for n in cached]
        n_pages, rows = sum(held) + spare, 2 * B + 3
        order, row = host.permutation(n_pages), host.permutation(rows)[:B]
        table = np.full((rows, max(h + n for h, n in zip(held, need)) + 1), -1, dtype=np.int32)
        at = 0
        for b, n in enumerate(held):
            table[row[b], :n] = order[at:at + n]
            at += n
        free = np.full(n_pages, -1, dtype=np.int32)
        free[:spare] = order[at:]
        s.update(table=i32(table), free=i32(free), n_free=i32([spare]), seq=i32(row), cached=i32(cached), fresh=i32(fresh), lengths=i32(fresh),
                 tokens=T if c["kind"] == "plan" else sum(fresh))
        return s
    Hq, Hk, K = c["Hq"], c["Hk"], c["K"]
    dt = torch.bfloat16 if c["io"] == "bf16" else torch.float32
    g = torch.Generator(device=dev).manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device=dev, generator=g)
    if c["kind"] in ("append", "packed"):
        x = rnd(B, T, (Hq + 2 * Hk) * K).to(dt)             # slices of one projection
        s["q"], s["k"], s["v"] = (y.unflatten(2, (-1, K)) for y in x.split([Hq * K, Hk * K, Hk * K], dim=2))
        s["wq"], s["wk"] = ((1.0 + 0.1 * rnd(K)) if c["norm"] == "rms" else None for _ in range(2))
        seq, pos, lens = _append_places(c)
        table, n_pages = _table(lens, c["page"], host)
        empty = lambda n: _stored(torch.zeros(n_pages, Hk, c["page"], n, dtype=torch.uint8, device=dev), c)
        s.update(cache=(empty(K // 2), empty(K // 2), empty(K // 32), empty(K // 32)), table=i32(table), seq=i32(seq).view(B, T), positions=i32(pos).view(B, T))
        s["rotary"] = _rotary_table(max(lens), c["rotary"], dev) if c["rotary"] else None
        return s
    lens = _lengths(c)
    table, n_pages = _table(lens, c["page"], host)
    s.update(q=(2.0 * rnd(B, Hq, K)).to(dt), table=i32(table), lengths=i32(lens), longest=max(lens))
    if c["kind"] == "decode" or c["mx"]:
        (k, ks), (v, vs) = (_cache_mx(n_pages, c, rnd) for _ in range(2))
        s["cache"] = (k, v, ks, vs)
    else:
        s["cache"] = tuple(_cache(n_pages, c, rnd, dt) for _ in range(2))
    if c["kind"] == "sparse":
        s["cached"] = (s["lengths"] - 1).clamp(min=0)
        count = torch.zeros(n_pages, dtype=torch.int32, device=dev)
        at = torch.arange(table.shape[1], device=dev)[None] * c["page"]
        there = s["table"] >= 0
        count[s["table"][there].long()] = (s["cached"][:, None] - at).clamp(0, c["page"])[there].int()
        s["bounds"] = _bounds_of(_values(s["cache"][0], s["cache"][2], dt) if c["mx"] else s["cache"][0], count)
    return s


# ------------------------------------------------------------------------- plain forms ----
def _pack(x):
    """Rows in 32 or 64 bits to codes and scales."""
    y = x.unflatten(-1, (-1, 32))
    m, k = torch.frexp(y.abs().amax(-1))                                       # largest = m 2^k, 1/2 <= m < 1; 7 = 7/8 * 2^3
    e = (k - torch.where(m <= 0.875, 3, 2)).clamp(-120, 125)
    e = torch.where(m == 0, torch.full_like(e, -120), e)
    y = y * ((127 - e) << 23).int().view(torch.float32)[..., None].to(x.dtype)
    a = y.abs()
    code = (a > 0.25).to(torch.uint8)
    for border, even in ((0.75, True), (1.25, False), (1.75, True), (2.5, False), (3.5, True), (5.0, False)):
        code += (a >= border) if even else (a > border)
    code += 8 * torch.signbit(y).to(torch.uint8)
    code = code.flatten(-2)
    return code[..., 0::2] | (code[..., 1::2] << 4), (e + 127).to(torch.uint8)


def _values(codes, scales, dt=torch.float32):
    """The values that codes and scales stand for."""
    grid = torch.tensor(GRID + tuple(-x for x in GRID), dtype=torch.float32, device=codes.device)
    x = torch.stack([grid[(codes & 15).long()], grid[(codes >> 4).long()]], dim=-1).flatten(-2)
    scale = (scales.int() << 23).view(torch.float32)
    return (x.unflatten(-1, (-1, 32)) * scale[..., None]).flatten(-2).to(dt)


def _ready(x, w, s, dt):
    """Rows normed, weighted and turned by their positions."""
    c = s["case"]
    y = x.to(dt)
    if c["norm"] != "none":
        y = y * ((1.0 if c["norm"] == "l2" else 1.0 / c["K"]) * (y * y).sum(-1, keepdim=True) + EPS).rsqrt()
    if w is not None:
        y = y * w
    R = c["rotary"]
    if not R:
        return y
    t = s["rotary"][s["positions"].long()]
    cos, sin = t[..., None, : R // 2], t[..., None, R // 2:]
    z = y.clone()
    z[..., : R // 2] = y[..., : R // 2] * cos - y[..., R // 2: R] * sin
    z[..., R // 2: R] = y[..., : R // 2] * sin + y[..., R // 2: R] * cos
    return z


def _plain_append(s):
    c = s["case"]
    dt = s["q"].dtype
    seq, pos = s["seq"].reshape(-1).long(), s["positions"].reshape(-1).long()
    at = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    k, v, ks, vs = s["cache"]
    # (a key next to the border of two codes: 64 bits)
    for rows, codes, scales in ((_ready(s["k"], s["wk"], s, torch.float64), k, ks), (s["v"].float(), v, vs)):
        codes[at], scales[at] = _pack(rows.flatten(0, 1))
    back = [_values(codes[at], scales[at], dt).view(c["B"], c["T"], c["Hk"], c["K"]) for codes, scales in ((k, ks), (v, vs))]
    return _ready(s["q"], s["wq"], s, torch.float32).to(dt), back[0], back[1]


def _softmax_rows(q, k, v, seen):
    """o and lse of q [.., G, K] over k, v [.., n, K], of which those that are `seen` count."""
    score = torch.matmul(q, k.transpose(-1, -2)) * q.shape[-1] ** -0.5
    top = score.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.where(seen, torch.exp(score - top), torch.zeros_like(score))
    total = p.sum(-1, keepdim=True)
    return torch.matmul(p, v) / torch.where(total == 0, torch.ones_like(total), total), (top + torch.log(total)).squeeze(-1)


def _plain_decode(s):
    c = s["case"]
    B, Hq, Hk, K, n = c["B"], c["Hq"], c["Hk"], c["K"], s["longest"]
    at = s["table"][:, : -(-n // c["page"])].clamp(min=0).long()
    k, v, ks, vs = s["cache"]
    rows = lambda codes, scales: _values(codes[at], scales[at]).flatten(1, 2)[:, :n].permute(0, 2, 1, 3)      # [B, Hk, n, K]
    j, lens = torch.arange(n, device=at.device)[None], s["lengths"][:, None]
    seen = j < lens
    if c["window"]:
        seen = seen & (j >= lens - c["window"])
    o, lse = _softmax_rows(s["q"].float().view(B, Hk, Hq // Hk, K), rows(k, ks), rows(v, vs), seen[:, None, None])
    return o.view(B, Hq, K).to(s["q"].dtype), lse.view(B, Hq)


def _plain_sparse(s):
    c = s["case"]
    B, Hq, Hk, K, page, n = c["B"], c["Hq"], c["Hk"], c["K"], c["page"], c["pages"]
    dt, dev = s["q"].dtype, s["q"].device
    lens = s["lengths"].long()
    last = (lens - 1).clamp(min=0)
    # the newest token joins its page's bounds
    g, slot, live = s["table"].gather(1, (last // page)[:, None])[:, 0].long(), last % page, lens > 0
    k_new = _values(s["cache"][0][g, slot], s["cache"][2][g, slot], dt) if c["mx"] else s["cache"][0][g, slot]
    old, both = s["bounds"][g], torch.stack([k_new, k_new], dim=2)
    joined = torch.stack([torch.minimum(old[:, :, 0], k_new), torch.maximum(old[:, :, 1], k_new)], dim=2)
    s["bounds"][g[live]] = torch.where((slot == 0)[:, None, None, None], both, joined)[live]
    # an upper bound of every score within a page, summed over the query heads that share its keys: 64 bits, as places are at stake
    q = s["q"].double().view(B, Hk, Hq // Hk, K)
    weight = torch.cat([q.clamp(max=0.0).sum(2), q.clamp(min=0.0).sum(2)], dim=-1)                             # [B, Hk, 2 K]
    P = s["table"].shape[1]
    score = torch.empty(B, Hk, P, dtype=torch.float64, device=dev)
    for b in range(B):                  # (one by one: the bounds in 64 bits)
        of = s["bounds"][s["table"][b].clamp(min=0).long()].double()                                          # [P, Hk, 2, K]
        score[b] = (of.flatten(2) * weight[b][None]).sum(-1).T
    have = (lens + page - 1) // page
    i = torch.arange(P, device=dev)[None]
    there = (i < have[:, None])[:, None].expand(B, Hk, P)
    always = ((i == 0) | (i == have[:, None] - 1))[:, None].expand(B, Hk, P) & there
    score = score.masked_fill(always, math.inf).masked_fill(~there, -math.inf)
    rank = score.sort(dim=-1, descending=True, stable=True).indices[..., :n]                                  # (ties: the first)
    take = torch.zeros(B, Hk, P, dtype=torch.bool, device=dev).scatter_(2, rank, True) & there
    # the selected pages in their order, then none
    place = torch.where(take, i[:, None].expand_as(take), P).sort(dim=-1).values[..., :n]
    place = torch.nn.functional.pad(place, (0, n - place.shape[-1]), value=P)
    here = place < P
    chosen = torch.where(here, s["table"].long()[:, None].expand(B, Hk, P).gather(2, place.clamp(max=P - 1)), -1).int()
    tokens = torch.where(lens[:, None] > 0, (take.sum(-1) - 1) * page + (last % page + 1)[:, None], 0).int()
    rows = chosen.clamp(min=0).long()
    head = torch.arange(Hk, device=dev)[None, :, None]
    at = (rows, slice(None), head)
    take_rows = lambda i: (_values(s["cache"][i][at], s["cache"][i + 2][at]) if c["mx"] else s["cache"][i][at].float()).flatten(2, 3)
    seen = torch.arange(n * page, device=dev)[None, None] < tokens[..., None]
    o, lse = _softmax_rows(s["q"].float().view(B, Hk, Hq // Hk, K), take_rows(0), take_rows(1), seen[:, :, None])
    return o.view(B, Hq, K).to(dt), lse.view(B, Hq), chosen, tokens, s["bounds"]


def _plain_release(s):
    """The pages of the sequences go onto the list, so that they are taken again in the same order."""
    c = s["case"]
    held = (s["lengths"].long() + c["page"] - 1) // c["page"]
    i = torch.arange(s["table"].shape[1], device=held.device)[None]
    rows = s["table"][s["seq"].long()]
    there = (i < held[:, None]) & (rows >= 0) & (rows < s["free"].shape[0])
    pages = rows[there]
    n = s["n_free"].long()
    s["free"][n + torch.arange(pages.numel() - 1, -1, -1, device=held.device)] = pages
    s["table"][s["seq"].long()] = torch.where(i < held[:, None], -1, rows)
    return s["n_free"] + pages.numel()


def _plain_plan(s, n_free):
    c = s["case"]
    page, N, dev = c["page"], s["tokens"], s["table"].device
    cached, fresh = s["cached"].long(), s["fresh"].long()
    first = (cached + page - 1) // page
    need = (cached + fresh + page - 1) // page - first
    served = ((need == 0) | (need.cumsum(0) <= n_free)) & ((fresh == 0) | (fresh.cumsum(0) <= N))
    need, fresh = torch.where(served, need, 0), torch.where(served, fresh, 0)
    ends = need.cumsum(0)
    i = torch.arange(int(ends[-1]), device=dev)
    b = torch.searchsorted(ends, i, right=True)
    s["table"][s["seq"][b].long(), first[b] + i - (ends - need)[b]] = s["free"][n_free.long() - 1 - i]
    starts = torch.cat([torch.zeros(1, dtype=torch.long, device=dev), fresh.cumsum(0)])
    j = torch.arange(N, device=dev)
    b = torch.searchsorted(starts[1:], j, right=True).clamp(max=c["B"] - 1)
    there = j < starts[-1]
    pos = torch.where(there, cached[b] + j - starts[b], -1)
    row = torch.where(there, s["seq"][b].long(), -1)
    slots = torch.where(there, s["table"][row.clamp(min=0), pos.clamp(min=0) // page].long() * page + pos.clamp(min=0) % page, -1)
    return ((cached + fresh).int(), starts.int(), pos.int(), row.int(), slots, (n_free - ends[-1]).int())


def run(s):
    c = s["case"]
    kind = c["kind"]
    if own:
        from paper_2605_13473_amd import binding as ob
        if kind in ("plan", "turnover"):
            n_free = s["n_free"]
            if kind == "turnover":
                n_free = ob.paged_release(s["table"], s["lengths"], s["free"], n_free, c["page"], seq=s["seq"])
            p = ob.paged_plan(s["table"], s["cached"], s["fresh"], s["free"], n_free, c["page"], s["tokens"], seq=s["seq"], want_slots=True)
            return p["lengths"], p["starts"], p["positions"].view(-1), p["seq"].view(-1), p["slots"], p["n_free"], s["table"], s["free"]
        if kind in ("append", "packed"):
            hp = ob.NormHyper(norm=c["norm"], eps=EPS)
            q = ob.paged_append_mx(s["k"], s["v"], s["cache"], s["table"], s["positions"], s["seq"], q=s["q"], weight_q=s["wq"], weight_k=s["wk"],
                                   rotary=s["rotary"], hp=hp)
            k, v = ob.paged_read_mx(s["cache"], s["table"], s["positions"], s["seq"], dtype=q.dtype)
            return q, k, v
        if kind == "decode":
            return ob.paged_decode_mx(s["q"], s["cache"], s["table"], s["lengths"], window=c["window"], max_length=s["longest"], want_lse=True)
        keys = (s["cache"][0], s["cache"][2]) if c["mx"] else s["cache"][0]
        ob.page_bounds(keys, s["table"], s["cached"], s["lengths"], s["bounds"], max_new=1)
        chosen, tokens = ob.page_select(s["q"], s["bounds"], s["table"], s["lengths"], c["page"], c["pages"], max_length=s["longest"])
        if c["mx"]:
            o, lse = ob.paged_decode_pages_mx(s["q"], s["cache"], chosen, tokens, want_lse=True)
        else:
            o, lse = ob.paged_decode_pages(s["q"], *s["cache"], chosen, tokens, want_lse=True)
        return o, lse, chosen, tokens, s["bounds"]
    if kind in ("plan", "turnover"):
        return _plain_plan(s, _plain_release(s) if kind == "turnover" else s["n_free"]) + (s["table"], s["free"])
    if kind in ("append", "packed"):
        return _plain_append(s)
    return _plain_decode(s) if kind == "decode" else _plain_sparse(s)


# ------------------------------------------------------------ the definition, in 64 bits ----
def _nearest(x):
    """What rows x [.., K] in 64 bits are kept as, by distance: of the two nearest values the even code's where they are as near."""
    y = x.unflatten(-1, (-1, 32))
    top = y.abs().amax(-1, keepdim=True)
    e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 7.0))
    e = torch.where(top <= 7.0 * torch.exp2(e - 1), e - 1, torch.where(top <= 7.0 * torch.exp2(e), e, e + 1)).clamp(-120, 125)
    scale = torch.where(top > 0, torch.exp2(e), 1.0)
    z = y.abs() / scale
    # odd codes lose their ties: they stand a little farther off, less than any distance that is not a tie's
    best, kept = torch.full_like(z, math.inf), torch.zeros_like(z)
    for values in (GRID[0::2], GRID[1::2]):
        for value in values:
            d = (z - value).abs()
            nearer = d < best
            best, kept = torch.where(nearer, d, best), torch.where(nearer, torch.full_like(z, value), kept)
    return (kept * scale * torch.sign(y)).flatten(-2)


def _exact_rows(x, w, s):
    """R(position) (x / |x| * w) of every row: the pairs as complex numbers."""
    c = s["case"]
    y = x.double()
    if c["norm"] == "l2":
        y = y / torch.sqrt(torch.linalg.vecdot(y, y)[..., None] + EPS)
    elif c["norm"] == "rms":
        y = y / torch.sqrt(y.square().mean(-1, keepdim=True) + EPS)
    if w is not None:
        y = y * w.double()
    R = c["rotary"]
    if R:
        t = s["rotary"].double()[s["positions"].long()]
        z = torch.complex(t[..., : R // 2], t[..., R // 2:]).unsqueeze(2)
        turned = torch.complex(y[..., : R // 2].contiguous(), y[..., R // 2: R].contiguous()) * z
        y = torch.cat([turned.real, turned.imag, y[..., R:]], dim=-1)
    return y


def _exact_attention(q, k, v):
    """q [G, K] over k, v [n, K]."""
    score = q @ k.T / math.sqrt(q.shape[-1])
    return torch.softmax(score, -1) @ v, torch.logsumexp(score, -1)


def _exact_cache(s, i):
    """Rows of the cache at (page, slot, head) in 64 bits."""
    c = s["case"]
    if c["kind"] == "sparse" and not c["mx"]:
        return lambda *at: s["cache"][i][at].double()
    signed = torch.tensor([x for x in GRID] + [-x for x in GRID], dtype=torch.float64, device="cuda")

    def rows(*at):
        b, e = s["cache"][i][at].int(), s["cache"][i + 2][at].double() - 127.0
        x = torch.empty(*b.shape[:-1], 2 * b.shape[-1], dtype=torch.float64, device="cuda")
        x[..., 0::2], x[..., 1::2] = signed[b % 16], signed[b // 16]
        return x * torch.repeat_interleave(torch.exp2(e), 32, dim=-1)
    return rows


def _exact_plan(s):
    c = s["case"]
    page, N = c["page"], s["tokens"]
    table, free, seq = s["table"].cpu().numpy().copy(), s["free"].cpu().numpy().copy(), s["seq"].cpu().numpy()
    cached, fresh, n_free = s["cached"].cpu().numpy(), s["fresh"].cpu().numpy(), int(s["n_free"][0])
    if c["kind"] == "turnover":
        back = []
        for b, n in enumerate(s["lengths"].cpu().numpy()):
            for i in range(-(-int(n) // page)):
                back.append(table[seq[b], i])
                table[seq[b], i] = -1
        for x in reversed(back):
            free[n_free] = x
            n_free += 1
    at, asked, tokens = 0, 0, 0
    have = n_free
    lengths, starts = [], [0]
    pos, row, slots = (np.full(N, -1, dtype=np.int64) for _ in range(3))
    for b in range(c["B"]):
        n, m = int(cached[b]), int(fresh[b])
        held = [i for i in range(-(-n // page), -(-(n + m) // page))]
        asked, tokens = asked + len(held), tokens + m
        if (held and asked > have) or (m and tokens > N):
            m = 0
        else:
            for i in held:
                n_free -= 1
                table[seq[b], i] = free[n_free]
        for i in range(n, n + m):
            pos[at], row[at], slots[at] = i, seq[b], int(table[seq[b], i // page]) * page + i % page
            at += 1
        lengths.append(n + m)
        starts.append(at)
    t = lambda x: torch.as_tensor(np.array(x, dtype=np.int64), device="cuda")
    return t(lengths), t(starts), t(pos), t(row), t(slots), t([n_free]), t(table), t(free)


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] in ("plan", "turnover"):
        return _exact_plan(s)
    if c["kind"] in ("append", "packed"):
        return _exact_rows(s["q"], s["wq"], s), _nearest(_exact_rows(s["k"], s["wk"], s)), _nearest(s["v"].double())
    B, Hq, Hk, K, page = c["B"], c["Hq"], c["Hk"], c["K"], c["page"]
    G = Hq // Hk
    o = torch.zeros(B, Hq, K, dtype=torch.float64, device="cuda")
    lse = torch.full((B, Hq), -math.inf, dtype=torch.float64, device="cuda")
    keys, values = _exact_cache(s, 0), _exact_cache(s, 1)
    if c["kind"] == "decode":
        for b, n in enumerate(_lengths(c)):
            lo = max(0, n - c["window"]) if c["window"] else 0
            if n == 0:
                continue
            j = torch.arange(lo, n, device="cuda")
            at = s["table"][b, j // page].long(), j % page
            k, v = keys(*at), values(*at)
            for h in range(Hk):
                of = slice(h * G, (h + 1) * G)
                o[b, of], lse[b, of] = _exact_attention(s["q"][b, of].double(), k[:, h], v[:, h])
        return o, lse
    n_sel = c["pages"]
    chosen, tokens = torch.full((B, Hk, n_sel), -1), torch.zeros(B, Hk, dtype=torch.long)
    bounds = s["bounds"].double()
    for b, n in enumerate(_lengths(c)):
        if n == 0:
            continue
        have = -(-n // page)
        pages = s["table"][b, :have].long()
        g = int(pages[-1])
        new = keys(g, torch.arange(n - n % page if n % page else n - page, n, device="cuda") % page)        # the last page, whole: [tokens, Hk, K]
        bounds[g, :, 0], bounds[g, :, 1] = new.amin(0), new.amax(0)
        for h in range(Hk):
            of = slice(h * G, (h + 1) * G)
            q = s["q"][b, of].double()
            best = torch.maximum(q[:, None] * bounds[pages, h, 0][None], q[:, None] * bounds[pages, h, 1][None]).sum((0, 2)).cpu().numpy()
            by_score = sorted(range(1, have - 1), key=lambda i: (-best[i], i))
            kept = sorted(([0, have - 1] if have > 1 else [0]) + by_score[: max(0, n_sel - 2)])
            chosen[b, h, : len(kept)] = pages.cpu()[kept]
            tokens[b, h] = (len(kept) - 1) * page + (n - 1) % page + 1
            j = torch.cat([torch.arange(i * page, min(n, (i + 1) * page)) for i in kept]).cuda()
            at = s["table"][b, j // page].long(), j % page, torch.full_like(j, h)
            o[b, of], lse[b, of] = _exact_attention(q, keys(*at), values(*at))
    return o, lse, chosen.cuda(), tokens.cuda(), bounds


# ------------------------------------------------------------------------------------- work ----
def work(case):
    """Every input read once and every output written once; the products of attention and of the bounds."""
    c = case
    if c["kind"] in ("plan", "turnover"):
        cached, fresh, need, spare = _requests(c)
        tokens = c["T"] if c["kind"] == "plan" else sum(fresh)
        pages = sum(need)
        # pages off the list into the table (turnover: and back), requests and lengths, three arrays of tokens
        return {"bytes": 8 * pages * (2 if c["kind"] == "turnover" else 1) + 20 * c["B"] + 16 * tokens, "flops": 4 * (c["B"] + tokens)}
    B, T, Hq, Hk, K = c["B"], c["T"], c["Hq"], c["Hk"], c["K"]
    es = 2 if c["io"] == "bf16" else 4
    mx = K / 2 + K / 32
    if c["kind"] in ("append", "packed"):
        rows = B * T
        table = 0 if not c["rotary"] else 4 * c["rotary"] * min(rows, T if c["kind"] != "append" else rows)
        flops = rows * (Hq + Hk) * (4 * K + 3 * c["rotary"]) + 4 * rows * Hk * K
        # rows in, queries out; keys and values into the cache, out of it and as rows
        return {"bytes": int(rows * ((2 * Hq + 4 * Hk) * K * es + 4 * Hk * mx)) + table + 8 * rows, "flops": flops}
    rows_qo = 2 * B * Hq * K * es + 4 * B * Hq
    if c["kind"] == "decode":
        n = _visible(c)
        return {"bytes": int(2 * n * Hk * mx) + rows_qo + 4 * (n // c["page"] + B) + 4 * B, "flops": 4 * n * Hq * K}
    width = mx if c["mx"] else K * es
    lens = _lengths(c)
    have = [-(-n // c["page"]) for n in lens]
    read = sum(min(h, c["pages"]) * c["page"] - (-n % c["page"]) for n, h in zip(lens, have))
    scored = sum(h for h in have if h > c["pages"])                    # (where all pages are taken none needs a score)
    return {"bytes": int(2 * read * Hk * width) + rows_qo + scored * Hk * 2 * K * es + sum(1 for n in lens if n) * Hk * (int(width) + 4 * K * es) + 4 * sum(have),
            "flops": 4 * read * Hq * K + 4 * scored * Hk * K}
