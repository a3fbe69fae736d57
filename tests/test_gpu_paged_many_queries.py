"""More queries than a launch of attention takes, as a packed prompt brings them: handed on in one call of the binding."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob

pytestmark = pytest.mark.gpu


def _exact(q, k, v, lengths):
    """q [B,K], rows [B,n,K], 64 bits on the CPU."""
    s = (k @ q[:, :, None])[..., 0] * q.shape[1] ** -0.5
    s = s.masked_fill(torch.arange(k.shape[1])[None] >= lengths[:, None], -float("inf"))
    return (torch.softmax(s, -1)[:, None] @ v)[:, 0], torch.logsumexp(s, -1)


@pytest.mark.parametrize("B,Hq,named", [(65536, 1, True), (70001, 1, False), (40000, 64, True)])
def test_more_queries_than_a_launch_takes(B, Hq, named):
    """fp32: a score is off by ds = (K / 4 + 8) 2^-24 sum |q k| / 8, the sum below 128 for rows of this width: ds < 2^-15, which is lse's error, too.  o is off by
    4 ds of the values, which are below 6."""
    K, page = 64, 16
    g = torch.Generator(device="cuda").manual_seed(B)
    rnd = lambda *s: torch.randn(*s, device="cuda", generator=g)
    seqs = 40 if named else B
    kc, vc = (rnd(seqs if named else 500, page, 1, K).clamp(-6, 6) for _ in range(2))
    table = (torch.arange(seqs, dtype=torch.int32, device="cuda") % kc.shape[0])[:, None].contiguous()
    lengths = torch.randint(1, page + 1, (B,), device="cuda", generator=g, dtype=torch.int32)
    seq = torch.randint(0, seqs, (B,), device="cuda", generator=g, dtype=torch.int32) if named else None
    q = rnd(B, Hq, K)
    o, lse = ob.paged_decode(q, kc, vc, table, lengths, seq, want_lse=True)
    assert torch.equal(ob.paged_decode(q, kc, vc, table, lengths, seq), o)
    at = table[torch.arange(B, device="cuda") if seq is None else seq.long(), 0].long()
    for b in (slice(0, 300), slice(B // 2 - 150, B // 2 + 150), slice(B - 300, B)):
        k, v = (c[at[b], :, 0].double().cpu() for c in (kc, vc))
        want, wlse = _exact(q[b, 0].double().cpu(), k, v, lengths[b].cpu())
        assert ((o[b, 0].double().cpu() - want).abs() <= 6 * 2.0 ** -13).all() and ((lse[b, 0].double().cpu() - wlse).abs() <= 2.0 ** -15).all()
    if Hq > 1:                          # every head of every query, against itself one by one
        for h in (1, Hq - 1):
            one = torch.cat([ob.paged_decode(q[i:i + 20000, h:h + 1], kc, vc, table, lengths[i:i + 20000], seq[i:i + 20000]) for i in range(0, B, 20000)])
            assert torch.allclose(o[:, h:h + 1], one, rtol=0, atol=6 * 2.0 ** -13)


def test_what_does_not_fit_is_refused_as_before():
    B = 65536
    kc = torch.randn(4, 16, 1, 64, device="cuda")
    table, lengths = torch.zeros(1, 1, dtype=torch.int32, device="cuda"), torch.ones(B, dtype=torch.int32, device="cuda")
    q, seq = torch.randn(B, 1, 64, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    for kw, error in ((dict(lengths=lengths[:-1]), ValueError), (dict(lengths=torch.cat([lengths, lengths])), ValueError), (dict(seq=seq[:5]), ValueError),
                      (dict(seq=seq.long()), TypeError), (dict(lengths=None), (TypeError, ob.OsdnError)), (dict(window=-1), ob.OsdnError), (dict(q=q.cpu()), TypeError)):
        with pytest.raises(error):
            ob.paged_decode(**{**dict(q=q, k_cache=kc, v_cache=kc, page_table=table, lengths=lengths, seq=seq), **kw})
    p = ob.make_decode_params(B, 1, 1, 64, False, 16)                       # the entry point itself
    with pytest.raises(ob.OsdnError):
        ob.osdn_paged_decode(p, q, kc, kc, table, lengths, seq, torch.empty_like(q), None)
