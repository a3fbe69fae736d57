"""A stack of two token-mixing layers on one GPU: an OSDN recurrence and an attention layer with a paged cache.

    python examples/hybrid_stack.py --sequences 4 --prompt 300 --new 64

Prompts of different lengths go through both layers, then tokens one by one: the recurrence keeps its state (``step``), the
attention layer its pages (``paged_append``, ``paged_decode``).  Queries and keys of both come out of ``qk_norm``'s arithmetic: unit length
for the recurrence, unit mean square with learned weights and rotation for attention.  Weights are random; what is printed is the
time of a token and how far the outputs lie from those of the whole text at once.  ``mixer_step`` is the training side: forward and
backward of the recurrence with the norm in front of it.
"""
import argparse
import os
import sys
import time
from dataclasses import dataclass

import torch

if __package__ in (None, ""):
    sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
from paper_2605_13473_amd import binding as ob  # noqa: E402

UNIT = ob.NormHyper(norm="l2")
ROTATED = ob.NormHyper(norm="rms")


@dataclass
class Config:
    width: int = 512
    heads: int = 4               # of the recurrence
    query_heads: int = 8         # of attention
    key_heads: int = 2
    head_width: int = 128
    page: int = 16
    longest: int = 4096


def make_weights(c: Config, seed=0, device="cuda"):
    g = torch.Generator(device=device).manual_seed(seed)
    lin = lambda i, o: (torch.randn(i, o, device=device, generator=g) * i ** -0.5).bfloat16()
    n = c.heads * c.head_width
    return dict(mix_in=lin(c.width, 3 * n), mix_gates=lin(c.width, 2 * c.heads), mix_out=lin(n, c.width),
                att_in=lin(c.width, (c.query_heads + 2 * c.key_heads) * c.head_width), att_out=lin(c.query_heads * c.head_width, c.width),
                wq=1 + 0.1 * torch.randn(c.head_width, device=device, generator=g), wk=1 + 0.1 * torch.randn(c.head_width, device=device, generator=g),
                rotary=ob.rotary_table(c.longest, c.head_width, device=device))


def split(x, *heads):
    """Slices of a projection's output as rows [B,T,heads,K]; nothing is copied."""
    K = x.shape[-1] // sum(heads)
    return [y.unflatten(2, (h, K)) for y, h in zip(x.split([h * K for h in heads], dim=2), heads)]


class Serving:
    """What a batch of sequences keeps between calls."""

    def __init__(self, c: Config, w, sequences, device="cuda"):
        self.c, self.w = c, w
        pages = -(-c.longest // c.page)
        self.k, self.v = ob.alloc_paged_cache(sequences * pages, c.page, c.key_heads, c.head_width, device=device)
        self.table = torch.randperm(sequences * pages, device=device).int().view(sequences, pages)
        self.lengths = torch.zeros(sequences, dtype=torch.int32, device=device)
        self.S = torch.zeros(sequences, c.heads, c.head_width, c.head_width, device=device)
        self.d = torch.ones(sequences, c.heads, c.head_width, device=device)

    def mix(self, x, row=None):
        """The recurrence over x [1,T,width] of sequence `row`, or over one token x [B,1,width] of each sequence."""
        c, w = self.c, self.w
        q, k, v = split(x @ w["mix_in"], c.heads, c.heads, c.heads)
        gates = (x @ w["mix_gates"]).float()
        beta, log_alpha = torch.sigmoid(gates[..., : c.heads]).contiguous(), -torch.nn.functional.softplus(gates[..., c.heads:] - 2).contiguous()
        q, k = ob.qk_norm(q, k, hp=UNIT)
        if row is None:
            o, self.S, self.d = ob.step(q, k, v.contiguous(), beta, log_alpha, None, self.d, self.S, in_place=True)
        else:
            o, self.S[row], self.d[row], _ = ob.forward(q, k, v.contiguous(), beta, log_alpha, None, self.d[row:row + 1], self.S[row:row + 1])
        return x + o.flatten(2) @ w["mix_out"]

    def attend(self, x, positions, seq, longest):
        """Attention of the tokens x [B,T,width] at `positions` of the sequences `seq` (both [B,T]): every token is appended, then every
        token sees its own past.  longest: no position is above longest - 1."""
        c, w = self.c, self.w
        q, k, v = split(x @ w["att_in"], c.query_heads, c.key_heads, c.key_heads)
        q = ob.paged_append(k, v, self.k, self.v, self.table, positions, seq, q=q, weight_q=w["wq"], weight_k=w["wk"], rotary=w["rotary"], hp=ROTATED)
        o = ob.paged_decode(q.flatten(0, 1), self.k, self.v, self.table, positions.flatten() + 1, seq.flatten(), max_length=longest)
        return x + o.view(*x.shape[:2], -1) @ w["att_out"]

    def prompt(self, row, x):
        """A prompt x [T,width] of one sequence; returns the outputs [T,width]."""
        T, at = x.shape[0], int(self.lengths[row])
        positions = torch.arange(at, at + T, dtype=torch.int32, device=x.device)[None]
        y = self.attend(self.mix(x[None], row), positions, torch.full_like(positions, row), at + T)
        self.lengths[row] += T
        return y[0]

    def token(self, x, longest):
        """One new token x [B,width] of every sequence; returns the outputs [B,width].  longest: no sequence is longer afterwards."""
        positions, seq = self.lengths[:, None].contiguous(), torch.arange(x.shape[0], dtype=torch.int32, device=x.device)[:, None]
        y = self.attend(self.mix(x[:, None]), positions, seq, longest)
        self.lengths += 1
        return y[:, 0]


def mixer_step(q, k, v, beta, log_alpha, dO, hp=ob.Hyper()):
    """A training step of the recurrence with the norm of its queries and keys: (o, gradients by name)."""
    qn, kn = ob.qk_norm(q, k, hp=UNIT)
    o, _, _, ctx = ob.forward(qn, kn, v, beta, log_alpha, hp=hp, for_backward=True)
    g = ob.backward(ctx, dO)
    n = ob.qk_norm_backward(q, k, g["dq"], g["dk"], hp=UNIT)
    return o, {"dq": n["dq"], "dk": n["dk"], "dv": g["dv"], "dbeta": g["dbeta"], "dlog_alpha": g["dlog_alpha"]}


def run(sequences=4, prompt=300, new=64, c=Config(), seed=0):
    """(outputs of prompts and tokens, the same from whole texts at once) per sequence, and seconds for a token."""
    w = make_weights(c, seed)
    g = torch.Generator(device="cuda").manual_seed(seed + 1)
    lens = [max(1, prompt - 37 * i) for i in range(sequences)]
    text = [torch.randn(n + new, c.width, device="cuda", generator=g).bfloat16() for n in lens]
    s = Serving(c, w, sequences)
    out = [[s.prompt(i, t[:n])] for i, (t, n) in enumerate(zip(text, lens))]
    torch.cuda.synchronize()
    began = time.perf_counter()
    for j in range(new):
        y = s.token(torch.stack([t[n + j] for t, n in zip(text, lens)]), max(lens) + j + 1)
        for i in range(sequences):
            out[i].append(y[i:i + 1])
    torch.cuda.synchronize()
    seconds = (time.perf_counter() - began) / max(1, new)
    whole = Serving(c, w, sequences)
    return [(torch.cat(o), whole.prompt(i, t)) for i, (o, t) in enumerate(zip(out, text))], seconds


if __name__ == "__main__":
    a = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    for name, value in (("sequences", 4), ("prompt", 300), ("new", 64), ("seed", 0)):
        a.add_argument("--" + name, type=int, default=value)
    a = a.parse_args()
    pairs, seconds = run(a.sequences, a.prompt, a.new, seed=a.seed)
    worst = max(float((x.float() - y.float()).abs().max()) for x, y in pairs)
    print(f"{a.sequences} sequences, {a.new} tokens each after prompts of up to {a.prompt}: {seconds * 1e6:.0f} us a token, "
          f"outputs within {worst:.3g} of the whole texts at once")
