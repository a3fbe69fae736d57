"""The way through the extension module of the operators around the recurrence against their way through Python: the same bits
for what the module takes, everything else left to the Python code with the errors it gives."""
import pytest
import torch

from paper_2605_13473_amd import binding as ob


def _args(dev, bf16=True, rotary=64, weighted=True, seq=False):
    g = torch.Generator(device=dev).manual_seed(5)
    rnd = lambda *s: torch.randn(*s, device=dev, generator=g)
    dt = torch.bfloat16 if bf16 else torch.float32
    B, T, Hq, Hk, K, page = 2, 5, 6, 2, 64, 8
    x = rnd(B, T, (Hq + 2 * Hk) * K).to(dt)
    q, k, v = (y.unflatten(2, (-1, K)) for y in x.split([Hq * K, Hk * K, Hk * K], dim=2))
    cache = [rnd(6, Hk, page, K).to(dt).transpose(1, 2) for _ in range(2)]
    i32 = dict(dtype=torch.int32, device=dev)
    return dict(q=q, k=k, v=v, w=(1 + rnd(K) / 8) if weighted else None, rotary=rnd(30, rotary) if rotary else None, cache=cache,
                table=torch.tensor([[0, 3, 5], [2, 1, 4]], **i32), pos=(torch.arange(T, **i32)[None] + torch.tensor([[3], [11]], **i32)),
                seq=torch.tensor([[1] * T, [0] * T], **i32) if seq else None, lengths=torch.tensor([8, 16], **i32), dq=rnd(B, T, Hq, K).to(dt), dk=rnd(B, T, Hk, K).to(dt),
                hp=ob.NormHyper(norm="rms"))


def _calls(a):
    """Every operator once; the cache it leaves comes with the results."""
    kc, vc = (c.clone() for c in a["cache"])
    q, k = ob.qk_norm(a["q"], a["k"], a["w"], a["w"], a["rotary"], a["pos"], a["hp"])
    g = ob.qk_norm_backward(a["q"], a["k"], a["dq"], a["dk"], a["w"], a["w"], a["rotary"], a["pos"], a["hp"])
    ready = ob.paged_append(a["k"], a["v"], kc, vc, a["table"], a["pos"], a["seq"], a["q"], a["w"], a["w"], a["rotary"], a["hp"])
    o, lse = ob.paged_decode(ready[:, -1], kc, vc, a["table"], a["lengths"], None if a["seq"] is None else a["seq"][:, 0].contiguous(), window=9, max_length=20, want_lse=True)
    plain = ob.paged_decode(ready[:, 0], kc, vc, a["table"], a["lengths"], scale=0.25)
    return [q, k, g["dq"], g["dk"], g["dweight_q"], g["dweight_k"], ready, kc, vc, o, lse, plain]


def test_the_module_leaves_tensors_of_the_host_alone():
    a = _args("cpu")
    ob.lib()
    assert ob._rows_native is not None
    n = ob._rows_native
    assert n.qk_norm(a["q"], a["k"], None, None, None, None, a["hp"], 0, 0) is None
    assert n.qk_norm_backward(a["q"], a["k"], a["dq"], a["dk"], None, None, None, None, a["hp"], 0, 0) is None
    assert n.paged_append(a["k"], a["v"], *a["cache"], a["table"], a["pos"], None, a["q"], None, None, None, a["hp"], 0, 0) is None
    assert n.paged_decode(a["q"][:, 0], *a["cache"], a["table"], a["lengths"], None, None, None, 0, None, False, 0, 0) is None


def test_structs_of_another_size_are_refused():
    from paper_2605_13473_amd import _native
    ob.lib()
    sizes = [ob.ctypes.sizeof(c) for c in (ob.OsdnRows, ob.OsdnNormParams, ob.OsdnCache, ob.OsdnDecodeParams)]
    for i in range(4):
        with pytest.raises(ImportError, match="built for"):
            _native.bind_rows(0, 0, 0, 0, 0, 0, *(s + 8 * (i == j) for j, s in enumerate(sizes)))


@pytest.mark.gpu
@pytest.mark.parametrize("case", [dict(), dict(bf16=False), dict(rotary=0, weighted=False), dict(seq=True)])
def test_same_bits_as_the_python_way(case, monkeypatch):
    a = _args("cuda", **case)
    ob.lib()
    dev, st = torch.cuda.current_device(), torch.cuda.current_stream().cuda_stream
    assert type(ob._rows_native.qk_norm(a["q"], a["k"], a["w"], a["w"], a["rotary"], a["pos"], a["hp"], dev, st)) is tuple
    got = _calls(a)
    with monkeypatch.context() as m:
        m.setattr(ob, "_rows_native", None)
        want = _calls(a)
    for x, y in zip(got, want):
        assert (x is None and y is None) or (x.dtype == y.dtype and x.stride() == y.stride() and torch.equal(x, y))


@pytest.mark.gpu
def test_what_is_out_of_the_ordinary_goes_through_python():
    a = _args("cuda")
    ob.lib()
    want = ob.qk_norm(a["q"], a["k"], a["w"], a["w"], a["rotary"], a["pos"], a["hp"])
    norm = lambda **kw: ob.qk_norm(*[dict(a, **kw)[n] for n in ("q", "k", "w", "w", "rotary", "pos", "hp")])
    for kw, error in [(dict(q=a["q"].float()), TypeError), (dict(w=a["w"][:32]), ValueError), (dict(k=a["k"][:, :4]), ValueError), (dict(q=a["q"].transpose(2, 3)), ValueError),
                      (dict(pos=a["pos"].long()), TypeError), (dict(rotary=a["rotary"].double()), TypeError), (dict(k=a["k"].cpu()), TypeError), (dict(w=a["w"].cpu()), TypeError),
                      (dict(hp=ob.NormHyper(norm="none of these")), ValueError), (dict(hp=ob.NormHyper(eps=-1.0)), ob.OsdnError), (dict(q=a["q"][..., ::2]), ValueError)]:
        with pytest.raises(error):
            norm(**kw)
    with torch.device("cuda"):                                                      # (a torch function mode)
        assert torch.equal(norm()[0], want[0])
    assert torch.equal(norm(hp=ob.NormHyper(norm="rms", eps=1e-6, interleaved=0))[0], want[0])

    class Sub(torch.Tensor):
        pass

    assert torch.equal(norm(q=a["q"].as_subclass(Sub))[0], want[0])
    kc, vc = a["cache"]
    append = lambda **kw: ob.paged_append(**{**dict(k=a["k"], v=a["v"], k_cache=kc, v_cache=vc, page_table=a["table"], positions=a["pos"]), **kw})
    for kw, error in [(dict(v=a["v"][:, :, :1]), ValueError), (dict(k_cache=kc.float()), TypeError), (dict(v_cache=vc[:5]), ValueError), (dict(page_table=a["table"].long()), TypeError),
                      (dict(page_table=a["table"].t()), ValueError), (dict(positions=None), ob.OsdnError), (dict(k_cache=kc[:, :7]), ValueError), (dict(k_cache=kc[:, :7], v_cache=vc[:, :7]), ob.OsdnError),
                      (dict(seq=a["pos"][0]), ValueError), (dict(k_cache=kc.expand(6, 8, 2, 64)[..., 1:], v_cache=vc), ValueError)]:
        with pytest.raises(error):
            append(**kw)
    decode = lambda **kw: ob.paged_decode(**{**dict(q=a["q"][:, 0], k_cache=kc, v_cache=vc, page_table=a["table"], lengths=a["lengths"]), **kw})
    for kw, error in [(dict(q=a["q"]), TypeError), (dict(q=a["q"][:, 0, :5]), ob.OsdnError), (dict(lengths=a["lengths"][:1]), ValueError), (dict(lengths=a["lengths"].long()), TypeError),
                      (dict(window=-1), ob.OsdnError), (dict(max_length=-1), ob.OsdnError), (dict(workspace=torch.empty(3, dtype=torch.uint8, device="cuda"), max_length=4096), ob.OsdnError),
                      (dict(seq=a["lengths"].cpu()), TypeError), (dict(k_cache=kc[..., :32], v_cache=vc[..., :32]), ValueError), (dict(scale=float("nan")), ob.OsdnError)]:
        with pytest.raises(error):
            decode(**kw)
