"""The operators around the recurrence, as cases to be timed: the norms of queries and keys with the position
rotation (forward and training step), the append of keys and values to a paged cache, and the attention of
one new token over such a cache.  Together they are what a stack of OSDN and softmax-attention layers does next to
the recurrence: the first makes the keys of unit length that OSDN asks its caller for, the other two
are the serving form of an attention layer.

``listed()`` names the cases, ``draw(rng)`` makes one more of the same ranges, ``prepare`` builds
what the program holds before the call, ``run`` makes one pass, ``work`` says what a pass cannot do
without, and ``exact`` is the definition in 64 bits.  With ``own`` false ``run`` computes the operators with
elementary torch operations in 32 bits, with ``own`` true through ``paper_2605_13473_amd.binding``.

Fields of a case
  kind        norm    queries and keys of whole sequences, forward
              train   the same, forward and backward
              append  T new tokens of each of B sequences into the pages of a cache, queries made ready in the same pass
              packed  append of prompts packed on one token axis of T tokens
              decode  one new token for each of B sequences over a cache of up to T tokens
  B T Hq Hk K sizes (K: width of a head); io "bf16" or "f32"
  norm        "l2", "rms" or "none"; weighted: with learned weights
  rotary      width of the rotated part (0: none); interleaved: pairs (2i, 2i+1), else (i, i + rotary/2)
  fused       queries, keys and values are slices of one projection's output
  page        tokens of a page; order "head" (a page holds its tokens head after head) or "token"
  ragged      decode: lengths spread from 1 to T, some sequences empty
  window      decode: only the last so many tokens are seen (0: all)
"""
import math

import numpy as np
import torch

own = False

THETA, EPS = 10000.0, 1e-6


def _case(kind, B, T, Hq, Hk, K=128, io="bf16", norm="rms", weighted=True, rotary=128, interleaved=False, fused=False,
          page=64, order="head", ragged=False, window=0, name=None):
    c = dict(kind=kind, B=B, T=T, Hq=Hq, Hk=Hk, K=K, io=io)
    if kind == "decode":
        c.update(page=page, order=order, ragged=ragged, window=window)
    else:
        c.update(norm=norm, weighted=weighted, rotary=rotary, interleaved=interleaved, fused=fused)
        if kind in ("append", "packed"):
            c.update(page=page, order=order)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # one prompt of an odd length: unit queries and keys for the recurrence
        _case("norm", 1, 1531, 16, 16, norm="l2", weighted=False, rotary=0, name="norm_prefill_odd_length"),
        # the 1.3B-shaped training step: unit queries and keys, forward and backward
        _case("train", 4, 4096, 16, 16, norm="l2", weighted=False, rotary=0, name="norm_train_1p3B"),
        # an attention layer with shared key heads in training: slices of one projection, learned weights, rotation
        _case("train", 2, 8192, 32, 8, fused=True, name="norm_train_rotary_fused"),
        # a small fp32 layer, half of a head rotated in adjacent pairs (debugging, ablations)
        _case("train", 2, 1000, 4, 4, K=64, io="f32", rotary=32, interleaved=True, name="norm_train_fp32"),
        # one user, one token: all latency
        _case("append", 1, 1, 16, 4, page=16, name="append_one_sequence"),
        # a serving batch, one token per sequence
        _case("append", 512, 1, 16, 4, name="append_512_sequences"),
        # prompts packed on one token axis go into the cache
        _case("packed", 1, 65536, 16, 4, name="append_packed_65536"),
        # one user, one token, a context of some pages and a bit
        _case("decode", 1, 1531, 16, 4, page=16, name="decode_one_sequence"),
        # a batch of conversations of very different lengths, a page order that comes with the projection
        _case("decode", 64, 8192, 32, 8, order="token", ragged=True, name="decode_64_ragged"),
        # one long context
        _case("decode", 1, 131072, 32, 8, name="decode_long_context"),
        # fp32, every query head with its own keys, the last 1000 tokens
        _case("decode", 8, 4096, 8, 8, K=64, io="f32", window=1000, page=32, name="decode_fp32_window"),
        # the full serving batch
        _case("decode", 512, 4096, 16, 4, ragged=True, name="decode_512_ragged"),
    ]


def _log_int(rng, lo, hi):
    n = max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))
    return n + 1 if n == 3072 else n


def draw(rng):
    kind = rng.choice(["norm", "train", "train", "append", "packed", "decode", "decode", "decode"])
    io = rng.choice(["bf16", "bf16", "bf16", "f32"])
    es = 2 if io == "bf16" else 4
    K = rng.choice([64, 128, 128, 256])
    Hk = rng.choice([1, 2, 4, 8, 16])
    Hq = Hk * rng.choice([1, 2, 4, 5, 7, 8, 16])
    if Hq > 64:
        Hq = Hk * 2
    while Hq * K == 3072 or (Hq + 2 * Hk) * K == 3072:
        Hq += Hk
    page, order = rng.choice([8, 16, 32, 64, 128]), rng.choice(["head", "token"])
    if kind == "decode":
        # at most a quarter of the tokens of the largest listed case in each form (uneven lengths halve it there)
        most = (1 << 28) // (Hk * K * es)
        T = _log_int(rng, 1, min(131072, most))
        B = _log_int(rng, 1, max(1, min(512, most // T)))
        window = rng.choice([0, 0, 0, _log_int(rng, 1, T)])
        return _case(kind, B, T, Hq, Hk, K, io, page=page, order=order, ragged=rng.random() < 0.6, window=window)
    norm = rng.choice(["l2", "rms", "rms", "none"])
    rotary = rng.choice([0, K, K, K // 2])
    c = dict(norm=norm, weighted=rng.random() < 0.6, rotary=rotary, interleaved=rng.random() < 0.3, fused=rng.random() < 0.5)
    most = (1 << 28) // ((Hq + 2 * Hk) * K * es)
    if kind in ("norm", "train"):
        T = _log_int(rng, 1, min(32768, most))
        return _case(kind, _log_int(rng, 1, max(1, min(16, most // T))), T, Hq, Hk, K, io, **c)
    c.update(page=page, order=order)
    if kind == "packed":
        return _case(kind, 1, _log_int(rng, 100, min(65536, most)), Hq, Hk, K, io, **c)
    T = rng.choice([1, 1, _log_int(rng, 2, 64)])
    return _case(kind, _log_int(rng, 1, min(512, most // T)), T, Hq, Hk, K, io, **c)


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


def _rotary_table(rows, width, dev):
    """[rows, width]: the cosines of a position's angles, then their sines."""
    angle = torch.arange(rows, dtype=torch.float64, device=dev)[:, None] * THETA ** (
        -2.0 * torch.arange(width // 2, dtype=torch.float64, device=dev) / width)
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


def _cache(n_pages, c, rnd, dt):
    """[pages, tokens of a page, heads, width], stored in the case's order."""
    if c["order"] == "head":
        return rnd(n_pages, c["Hk"], c["page"], c["K"]).to(dt).permute(0, 2, 1, 3)
    return rnd(n_pages, c["page"], c["Hk"], c["K"]).to(dt)


def prepare(case, seed):
    c = case
    B, T, Hq, Hk, K = c["B"], c["T"], c["Hq"], c["Hk"], c["K"]
    dev, dt = "cuda", torch.bfloat16 if c["io"] == "bf16" else torch.float32
    g = torch.Generator(device=dev).manual_seed(seed)
    rnd = lambda *shape: torch.randn(*shape, device=dev, generator=g)
    host = np.random.Generator(np.random.Philox(seed))
    i32 = lambda a: torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=dev)
    s = dict(case=c)
    if c["kind"] == "decode":
        lens = _lengths(c)
        table, n_pages = _table(lens, c["page"], host)
        s.update(q=(2.0 * rnd(B, Hq, K)).to(dt), k_cache=_cache(n_pages, c, rnd, dt), v_cache=_cache(n_pages, c, rnd, dt), table=i32(table),
                 lengths=i32(lens), longest=max(lens))
        return s
    if c["fused"]:
        x = rnd(B, T, (Hq + 2 * Hk) * K).to(dt)
        s["q"], s["k"], s["v"] = (y.unflatten(2, (-1, K)) for y in x.split([Hq * K, Hk * K, Hk * K], dim=2))
    else:
        s["q"], s["k"], s["v"] = (rnd(B, T, H, K).to(dt) for H in (Hq, Hk, Hk))
    s["wq"], s["wk"] = ((1.0 + 0.1 * rnd(K)) if c["weighted"] else None for _ in range(2))
    s["positions"] = None
    if c["kind"] in ("append", "packed"):
        seq, pos, lens = _append_places(c)
        table, n_pages = _table(lens, c["page"], host)
        s.update(k_cache=_cache(n_pages, c, rnd, dt), v_cache=_cache(n_pages, c, rnd, dt), table=i32(table), seq=i32(seq).view(B, T),
                 positions=i32(pos).view(B, T))
        rows = max(lens)
    else:
        rows = T
    s["rotary"] = _rotary_table(rows, c["rotary"], dev) if c["rotary"] else None
    if c["kind"] == "train":
        s["dq"], s["dk"] = rnd(B, T, Hq, K).to(dt), rnd(B, T, Hk, K).to(dt)
    return s


# --------------------------------------------------------------- plain forms, in 32 bits ----
def _factor(x, c):
    """1 over the norm of every row, and what one squared element counts for in it."""
    if c["norm"] == "none":
        return None, 0.0
    m = 1.0 if c["norm"] == "l2" else 1.0 / c["K"]
    return (m * (x * x).sum(-1, keepdim=True) + EPS).rsqrt(), m


def _turn(x, s, back=False):
    """The pairs of a row turned by the angles of its position (back: by their negatives)."""
    c, R = s["case"], s["case"]["rotary"]
    if not R:
        return x
    t = s["rotary"][: c["T"]][None] if s["positions"] is None else s["rotary"][s["positions"].long()]
    cos, sin = t[..., None, : R // 2], t[..., None, R // 2:]
    if back:
        sin = -sin
    y = x.clone()
    a, b = (slice(0, R, 2), slice(1, R, 2)) if c["interleaved"] else (slice(0, R // 2), slice(R // 2, R))
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., a] * sin + x[..., b] * cos
    return y


def _plain_norm(x, w, s):
    y = x.float()
    r, _ = _factor(y, s["case"])
    if r is not None:
        y = y * r
    if w is not None:
        y = y * w
    return _turn(y, s).to(x.dtype)


def _plain_norm_backward(x, w, dz, s):
    x32, dy = x.float(), _turn(dz.float(), s, back=True)
    r, m = _factor(x32, s["case"])
    xr = x32 if r is None else x32 * r
    dw = None if w is None else (dy * xr).sum((0, 1, 2))
    gr = dy if w is None else dy * w
    if r is not None:
        gr = r * (gr - xr * (m * (gr * xr).sum(-1, keepdim=True)))
    return gr.to(x.dtype), dw


def _plain_append(s):
    c = s["case"]
    seq, pos = s["seq"].reshape(-1).long(), s["positions"].reshape(-1).long()
    at = s["table"][seq, pos // c["page"]].long(), pos % c["page"]
    s["k_cache"][at] = _plain_norm(s["k"], s["wk"], s).reshape(-1, c["Hk"], c["K"])
    s["v_cache"][at] = s["v"].reshape(-1, c["Hk"], c["K"])
    return _plain_norm(s["q"], s["wq"], s), s["k_cache"], s["v_cache"]


def _plain_decode(s):
    c = s["case"]
    B, Hq, Hk, K, n = c["B"], c["Hq"], c["Hk"], c["K"], s["longest"]
    at = s["table"][:, : -(-n // c["page"])].clamp(min=0).long()
    rows = lambda cache: cache[at].flatten(1, 2)[:, :n].permute(0, 2, 1, 3).float()          # [B, Hk, n, K]
    q = s["q"].float().view(B, Hk, Hq // Hk, K)
    score = torch.matmul(q, rows(s["k_cache"]).transpose(2, 3)) * K ** -0.5
    j, lens = torch.arange(n, device=q.device)[None], s["lengths"][:, None]
    seen = j < lens
    if c["window"]:
        seen = seen & (j >= lens - c["window"])
    seen = seen[:, None, None]
    top = score.masked_fill(~seen, -math.inf).amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, torch.zeros_like(top), top)
    p = torch.where(seen, torch.exp(score - top), torch.zeros_like(score))
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p, rows(s["v_cache"])) / torch.where(total == 0, torch.ones_like(total), total)
    return o.view(B, Hq, K).to(s["q"].dtype), (top + torch.log(total)).view(B, Hq)


def run(s):
    c = s["case"]
    if own:
        from paper_2605_13473_amd import binding as ob
        if c["kind"] == "decode":
            return ob.paged_decode(s["q"], s["k_cache"], s["v_cache"], s["table"], s["lengths"], window=c["window"],
                                   max_length=s["longest"], want_lse=True)
        hp = ob.NormHyper(norm=c["norm"], eps=EPS, interleaved=c["interleaved"])
        if c["kind"] in ("append", "packed"):
            q = ob.paged_append(s["k"], s["v"], s["k_cache"], s["v_cache"], s["table"], s["positions"], s["seq"], q=s["q"],
                                weight_q=s["wq"], weight_k=s["wk"], rotary=s["rotary"], hp=hp)
            return q, s["k_cache"], s["v_cache"]
        q, k = ob.qk_norm(s["q"], s["k"], s["wq"], s["wk"], s["rotary"], s["positions"], hp)
        if c["kind"] == "norm":
            return q, k
        g = ob.qk_norm_backward(s["q"], s["k"], s["dq"], s["dk"], s["wq"], s["wk"], s["rotary"], s["positions"], hp)
        return (q, k, g["dq"], g["dk"]) + ((g["dweight_q"], g["dweight_k"]) if c["weighted"] else ())
    if c["kind"] == "decode":
        return _plain_decode(s)
    if c["kind"] in ("append", "packed"):
        return _plain_append(s)
    q, k = _plain_norm(s["q"], s["wq"], s), _plain_norm(s["k"], s["wk"], s)
    if c["kind"] == "norm":
        return q, k
    (dq, dwq), (dk, dwk) = _plain_norm_backward(s["q"], s["wq"], s["dq"], s), _plain_norm_backward(s["k"], s["wk"], s["dk"], s)
    return (q, k, dq, dk) + ((dwq, dwk) if c["weighted"] else ())


# ------------------------------------------------------------ the definition, in 64 bits ----
def _exact_rows(x, w, s):
    """R(position) (x / |x| * w) of every row: the pairs as complex numbers."""
    c = s["case"]
    y = x
    if c["norm"] == "l2":
        y = x / torch.sqrt(torch.linalg.vecdot(x, x)[..., None] + EPS)
    elif c["norm"] == "rms":
        y = x / torch.sqrt(x.square().mean(-1, keepdim=True) + EPS)
    if w is not None:
        y = y * w
    R = c["rotary"]
    if R:
        p = torch.arange(c["T"], device=x.device).expand(c["B"], -1) if s["positions"] is None else s["positions"].long()
        t = s["rotary"].double()[p]
        z = torch.complex(t[..., : R // 2], t[..., R // 2:]).unsqueeze(2)
        pairs = y[..., :R].unflatten(-1, (R // 2, 2) if c["interleaved"] else (2, R // 2))
        if not c["interleaved"]:
            pairs = pairs.transpose(-1, -2)
        turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * z)
        if not c["interleaved"]:
            turned = turned.transpose(-1, -2)
        y = torch.cat([turned.flatten(-2), y[..., R:]], dim=-1)
    return y


def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["kind"] == "decode":
        o = torch.zeros(c["B"], c["Hq"], c["K"], dtype=torch.float64, device="cuda")
        lse = torch.full((c["B"], c["Hq"]), -math.inf, dtype=torch.float64, device="cuda")
        for b, n in enumerate(_lengths(c)):
            lo = max(0, n - c["window"]) if c["window"] else 0
            if n == 0:
                continue
            j = torch.arange(lo, n, device="cuda")
            at = s["table"][b, j // c["page"]].long(), j % c["page"]
            k, v = s["k_cache"][at].double(), s["v_cache"][at].double()
            for h in range(c["Hk"]):
                of = slice(h * c["Hq"] // c["Hk"], (h + 1) * c["Hq"] // c["Hk"])
                score = s["q"][b, of].double() @ k[:, h].T / math.sqrt(c["K"])
                lse[b, of] = torch.logsumexp(score, -1)
                o[b, of] = torch.softmax(score, -1) @ v[:, h]
        return o, lse
    w = [None if s[n] is None else s[n].double().requires_grad_(c["kind"] == "train") for n in ("wq", "wk")]
    x = [s[n].double().requires_grad_(c["kind"] == "train") for n in ("q", "k")]
    y = [_exact_rows(a, b, s) for a, b in zip(x, w)]
    if c["kind"] == "norm":
        return tuple(y)
    if c["kind"] == "train":
        leaves = x + [a for a in w if a is not None]
        grads = torch.autograd.grad(y, leaves, [s["dq"].double(), s["dk"].double()])
        return tuple(a.detach() for a in y) + tuple(grads)
    kc, vc = s["k_cache"].double(), s["v_cache"].double()
    table, seq, pos = s["table"].cpu().numpy(), s["seq"].cpu().numpy().reshape(-1), s["positions"].cpu().numpy().reshape(-1)
    at = torch.as_tensor(table[seq, pos // c["page"]], device="cuda").long(), torch.as_tensor(pos % c["page"], device="cuda").long()
    kc.index_put_(at, y[1].flatten(0, 1))
    vc.index_put_(at, s["v"].double().flatten(0, 1))
    return y[0], kc, vc


# ------------------------------------------------------------------------------------- work ----
def work(case):
    """Every input read once and every output written once; the products of attention."""
    c = case
    B, T, Hq, Hk, K = c["B"], c["T"], c["Hq"], c["Hk"], c["K"]
    es = 2 if c["io"] == "bf16" else 4
    if c["kind"] == "decode":
        n = _visible(c)
        pages = -(-n // c["page"]) + B
        return {"bytes": 2 * n * Hk * K * es + 2 * B * Hq * K * es + 4 * B * Hq + 4 * pages + 4 * B, "flops": 4 * n * Hq * K}
    rows = B * T
    table = 0 if not c["rotary"] else 4 * c["rotary"] * min(rows, T if c["kind"] != "append" else rows)
    weights = 8 * K if c["weighted"] else 0
    turn = 3 * c["rotary"]
    flops = rows * (Hq + Hk) * (4 * K + turn)
    if c["kind"] in ("append", "packed"):
        return {"bytes": 2 * rows * (Hq + 2 * Hk) * K * es + table + weights + 8 * rows + 4 * rows // c["page"], "flops": flops}
    if c["kind"] == "norm":
        return {"bytes": 2 * rows * (Hq + Hk) * K * es + table + weights, "flops": flops}
    return {"bytes": 5 * rows * (Hq + Hk) * K * es + 2 * table + 3 * weights, "flops": 4 * flops}
