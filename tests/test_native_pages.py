"""The way through the extension module of the operators on pages against their way through Python: the same bits for what the module takes, everything else left to the
Python code with the errors it gives."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob


def _args(dev, bf16=True, seq=False):
    g = torch.Generator(device=dev).manual_seed(5)
    rnd = lambda *s: torch.randn(*s, device=dev, generator=g)
    dt, i32 = torch.bfloat16 if bf16 else torch.float32, dict(dtype=torch.int32, device=dev)
    x = rnd(1, 21, 10 * 64).to(dt)
    q, k, v = (y.unflatten(2, (-1, 64)) for y in x.split([6 * 64, 2 * 64, 2 * 64], dim=2))
    return dict(q=q, k=k, v=v, w=1 + rnd(64) / 8, rotary=rnd(40, 64), table=torch.full((3, 6), -1, **i32), free=torch.tensor([4, 0, 7, 3, 8, 1, 6, 2, 5], **i32), n_free=torch.tensor([9], **i32),
                cached=torch.zeros(3, **i32), fresh=torch.tensor([9, 11, 1], **i32), seq=torch.tensor([2, 0, 1], **i32) if seq else None, cache=ob.alloc_paged_cache_mx(9, 4, 2, 64, device=dev),
                rows=tuple(c.to(dt) for c in (rnd(9, 4, 2, 64), rnd(9, 4, 2, 64))), dt=dt)


def _calls(a):
    """Every operator once; what is written in place comes with the results."""
    table, free, cache, dt = a["table"].clone(), a["free"].clone(), tuple(t.clone().zero_() for t in a["cache"]), a["dt"]
    p = ob.paged_plan(table, a["cached"], a["fresh"], free, a["n_free"], 4, 23, seq=a["seq"], want_slots=True)
    pos, of = p["positions"][:, :21].contiguous(), p["seq"][:, :21].contiguous()
    ready = ob.paged_append_mx(a["k"], a["v"], cache, table, pos, of, a["q"], a["w"], a["w"], a["rotary"])
    read = [x for t in (torch.bfloat16, torch.float32) for x in ob.paged_read_mx(cache, table, pos, of, t)]
    bounds = [torch.zeros(9, 2, 2, 64, dtype=t, device=table.device) for t in (dt, dt)]
    ob.page_bounds((cache[0], cache[2]), table, a["cached"], p["lengths"], bounds[0], seq=a["seq"], max_new=11)
    ob.page_bounds(a["rows"][0], table, a["cached"], p["lengths"], bounds[1], seq=a["seq"])
    q, at = ready[0], (pos[0] + 1).contiguous()
    o, lse = ob.paged_decode_mx(q, cache, table, at, of[0], window=7, max_length=11, want_lse=True)
    plain = ob.paged_decode_mx(q, cache, table, at, of[0], scale=0.25)
    chosen, tokens = ob.page_select(q, bounds[0], table, at, 4, 2, seq=of[0], max_length=12)
    few = ob.paged_decode_pages_mx(q, cache, chosen, tokens, want_lse=True)
    rows = ob.paged_decode_pages(q, *a["rows"], chosen, tokens, max_length=8, scale=0.5)
    left = ob.paged_release(table, p["lengths"], free, p["n_free"], 4, seq=a["seq"], n_pages=9)
    return [p[n] for n in ("lengths", "starts", "positions", "seq", "n_free", "slots")] + [ready, *read, *bounds, o, lse, plain, chosen, tokens, *few, rows, left, table, free, *cache]


def test_the_module_leaves_tensors_of_the_host_alone():
    a = _args("cpu")
    ob.lib()
    n = ob._rows_native
    assert n is not None
    c, t, pos = a["cache"], a["table"], torch.zeros(1, 21, dtype=torch.int32)
    assert n.paged_plan(t, a["cached"], a["fresh"], a["free"], a["n_free"], None, 4, 23, None, False, 0, 0) is None
    assert n.paged_release(t, a["cached"], a["free"], a["n_free"], None, 4, None, 0, 0) is None
    assert n.paged_append_mx(a["k"], a["v"], *c, t, pos, None, a["q"], None, None, None, ob.NormHyper(), 0, 0) is None
    assert n.paged_read_mx(*c, t, pos, None, True, False, 0, 0) is None
    assert n.paged_decode_mx(a["q"][0], *c, t, pos[0], None, None, None, 0, None, False, 0, 0) is None
    b, chosen = torch.zeros(9, 2, 2, 64, dtype=a["dt"]), torch.zeros(21, 2, 2, dtype=torch.int32)
    assert n.paged_decode_pages(a["q"][0], *a["rows"], None, None, chosen, chosen[..., 0].contiguous(), None, None, None, False, 0, 0) is None
    assert n.page_bounds(c[0], c[2], t, a["cached"], a["fresh"], None, b, None, 0, 0) is None
    assert n.page_select(a["q"][0], b, t, pos[0], None, None, 4, 2, 1, 1, None, 0, 0) is None


def test_structs_of_another_size_are_refused():
    from paper_2605_13473_amd import _native
    ob.lib()
    sizes = [ob.ctypes.sizeof(c) for c in (ob.OsdnPages, ob.OsdnCacheMx, ob.OsdnSelectParams)]
    for i in range(3):
        with pytest.raises(ImportError, match="built for"):
            _native.bind_pages((0,) * 14, *(s + 8 * (i == j) for j, s in enumerate(sizes)))
    with pytest.raises(TypeError, match="14"):
        _native.bind_pages((0,) * 13, *sizes)


@pytest.mark.gpu
@pytest.mark.parametrize("case", [dict(), dict(bf16=False), dict(seq=True)], ids=str)
def test_same_bits_as_the_python_way(case, monkeypatch):
    a = _args("cuda", **case)
    ob.lib()
    dev, st = torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream
    assert type(ob._rows_native.paged_plan(a["table"].clone(), a["cached"], a["fresh"], a["free"], a["n_free"], a["seq"], 4, 23, None, False, dev, st)) is tuple
    got = _calls(a)
    with monkeypatch.context() as m:
        m.setattr(ob, "_rows_native", None)
        want = _calls(a)
    for x, y in zip(got, want):
        assert x.dtype == y.dtype and x.stride() == y.stride() and torch.equal(x, y)


@pytest.mark.gpu
def test_what_is_out_of_the_ordinary_goes_through_python():
    a = _args("cuda")
    want = _calls(a)
    lists = dict(a, cache=list(a["cache"]))
    assert all(torch.equal(x, y) for x, y in zip(_calls(lists), want))

    class Sub(torch.Tensor):
        pass

    assert all(torch.equal(x, y) for x, y in zip(_calls(dict(a, cached=a["cached"].as_subclass(Sub), q=a["q"].as_subclass(Sub))), want))
    t, i32 = a["table"].clone(), dict(dtype=torch.int32, device="cuda")
    plan = lambda **kw: ob.paged_plan(**{**dict(page_table=t, cached=a["cached"], fresh=a["fresh"], free_pages=a["free"], n_free=a["n_free"], page_size=4, tokens=23), **kw})
    for kw, error in [(dict(cached=a["cached"].long()), TypeError), (dict(fresh=a["fresh"][:2]), ValueError), (dict(page_table=t.long()), TypeError), (dict(page_table=t.t()), ValueError),
                      (dict(page_table=t[0]), ValueError), (dict(page_table=t.cpu()), TypeError), (dict(n_free=a["n_free"].repeat(2)), ValueError), (dict(free_pages=a["free"][::2]), ValueError),
                      (dict(seq=a["fresh"].float()), TypeError), (dict(page_size=3), ob.OsdnError), (dict(tokens=0), ob.OsdnError), (dict(tokens=2 ** 31), ob.OsdnError), (dict(tokens=2 ** 30 + 1), ob.OsdnError), (dict(tokens=-1), ob.OsdnError),
                      (dict(n_pages=0), ob.OsdnError), (dict(page_table=t[:1].expand(3, 6)), ob.OsdnError), (dict(cached=a["cached"][:0], fresh=a["fresh"][:0]), ob.OsdnError)]:
        with pytest.raises(error):
            plan(**kw)
    b, q, at = torch.zeros(9, 2, 2, 64, dtype=a["dt"], device="cuda"), a["q"][0], torch.ones(21, **i32)
    table, seq = torch.zeros(3, 6, **i32), torch.zeros(21, **i32)
    select = lambda **kw: ob.page_select(**{**dict(q=q, bounds=b, page_table=table, lengths=at, page_size=4, pages=3, seq=seq), **kw})
    assert select()[0].shape == (21, 2, 3)
    for kw, error in [(dict(q=q.float()), TypeError), (dict(bounds=b[:, :1]), ValueError), (dict(bounds=b[:, :, :1]), ValueError), (dict(lengths=at[:3]), ValueError), (dict(pages=0), ob.OsdnError), (dict(pages=1), ob.OsdnError),
                      (dict(first=-1), ob.OsdnError), (dict(last=0), ob.OsdnError), (dict(page_size=5), ob.OsdnError), (dict(seq=seq.long()), TypeError), (dict(q=q[:, :5]), ob.OsdnError), (dict(pages=2 ** 40), ob.OsdnError),
                      (dict(max_length=2 ** 40), ob.OsdnError)]:
        with pytest.raises(error):
            select(**kw)
    chosen, tokens = select()
    few = lambda **kw: ob.paged_decode_pages_mx(**{**dict(q=q, cache=a["cache"], chosen=chosen, tokens=tokens), **kw})
    for kw, error in [(dict(chosen=chosen[:, :1]), ValueError), (dict(tokens=tokens[:, :1]), ValueError), (dict(chosen=chosen[..., ::2]), ValueError), (dict(tokens=tokens.long()), TypeError), (dict(cache=a["cache"][:3]), TypeError),
                      (dict(cache=(a["cache"][0].int(), *a["cache"][1:])), TypeError), (dict(cache=(a["cache"][0][:5], *a["cache"][1:])), ValueError), (dict(chosen=chosen[..., :0]), ob.OsdnError),
                      (dict(workspace=torch.zeros(4, device="cuda")), TypeError)]:
        with pytest.raises(error):
            few(**kw)
    few(max_length=0)
    with pytest.raises(ob.OsdnError):
        few(max_length=2 ** 40)
