"""The native form of the calls of relative-bias attention, dropout and norm against the general one: the same results bit for bit, the
same errors, for plain arguments and for those that only the general form takes."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(params=["native", "general"])
def hdt(request, monkeypatch):
    import paper_2407_08330_amd as hdt
    from paper_2407_08330_amd import binding
    binding.load_library()
    if request.param == "general":
        monkeypatch.setattr(binding, "_calls", binding._NoCalls)
    else:
        assert binding._calls is not binding._NoCalls
    return hdt


def tensors(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    return dict(q=n(2, 4, 50, 64), k=n(2, 2, 60, 64), v=n(2, 2, 60, 64), bias=n(32, 4), d_o=n(2, 4, 50, 64), x=n(5, 6, 40), y=n(5, 6, 40),
                w=n(40), b=n(40), dn=n(5, 6, 40), rng=torch.tensor([3, 4], device="cuda"))


def everything(hdt, t, **kw):
    import torch
    table = hdt.hdt_rel_table(32, 128)
    ints = dict(lengths=torch.tensor([60, 41], dtype=torch.int32, device="cuda"), q_start=torch.tensor([10, -3], dtype=torch.int32, device="cuda"))
    out = []
    for more in ({}, ints, dict(causal=False, lengths=ints["lengths"])):
        o, lse = hdt.hdt_rel_attn_fwd(t["q"], t["k"], t["v"], t["bias"], table, 0.125, **more, **kw)
        out += [o, lse, *hdt.hdt_rel_attn_bwd(t["q"], t["k"], t["v"], t["bias"], table, o, lse, t["d_o"], 0.125, **more, **kw)]
    for p in (0.0, 0.25):
        out.append(hdt.hdt_dropout_add(t["y"], p, t["rng"], 7, x=t["x"], **kw))
        out.append(hdt.hdt_dropout_add(t["y"], p, t["rng"], **kw))
        n, h, mean, rstd = hdt.hdt_add_norm_fwd(t["x"], t["w"], t["b"], y=t["y"], p=p, rng=t["rng"], site=1, **kw)
        out += [n, h, mean, rstd, *hdt.hdt_add_norm_bwd(t["dn"], h, t["w"], mean, rstd, dh=t["y"], p=p, rng=t["rng"], site=1, **kw)]
    return out


@pytest.fixture(scope="module")
def first():
    return {}


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("other_stream", [False, True])
def test_both_give_the_same_bits(hdt, first, name, other_stream):
    import torch
    t = tensors({"bf16": torch.bfloat16, "f32": torch.float32}[name])
    torch.cuda.synchronize()
    got = everything(hdt, t, **(dict(stream=torch.cuda.Stream()) if other_stream else {}))
    torch.cuda.synchronize()
    want = first.setdefault(name, got)
    assert len(got) == len(want) and all(a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(got, want))


def test_results_are_the_callers_tensors(hdt):
    import torch
    t = tensors(torch.float32)
    table, o = hdt.hdt_rel_table(32, 128), torch.empty(2, 50, 4, 64, device="cuda").transpose(1, 2)
    lse = torch.empty(2, 4, 50, device="cuda")
    got = hdt.hdt_rel_attn_fwd(t["q"], t["k"], t["v"], t["bias"], table, 0.125, o=o, lse=lse)
    assert got[0] is o and got[1] is lse
    out = torch.empty_like(t["y"])
    assert hdt.hdt_dropout_add(t["y"], 0.1, t["rng"], out=out) is out
    n, h = torch.empty_like(t["x"]), torch.empty_like(t["x"])
    got = hdt.hdt_add_norm_fwd(t["x"], t["w"], y=t["y"], n=n, h=h)
    assert got[0] is n and got[1] is h


def test_refusals(hdt):
    import torch
    t = tensors(torch.float32)
    table = hdt.hdt_rel_table(32, 128)
    good = dict(q=t["q"], k=t["k"], v=t["v"], bias=t["bias"], table=table, softmax_scale=0.125)
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    for bad in (dict(k=t["k"][:, :, :, :32]), dict(v=t["v"][:, :, :5]), dict(k=t["k"].bfloat16()), dict(q=t["q"].half()), dict(q=t["q"][0]),
                dict(bias=t["bias"][:, :3]), dict(bias=t["bias"].t()), dict(bias=t["bias"].double()), dict(table=table.long()), dict(table=table[1:]),
                dict(table=table[::2]), dict(lengths=i32(1)), dict(lengths=i32(1, 2).long()), dict(q_start=i32(1, 2, 3)), dict(k=t["k"][:, [0, 1, 1]], v=t["v"][:, [0, 1, 1]]),
                dict(softmax_scale=0.0), dict(q=t["q"].transpose(2, 3).contiguous().transpose(2, 3)), dict(k=t["k"].cpu()), dict(lengths=i32(1, 2).cpu()),
                dict(o=torch.empty(2, 4, 50, 64, device="cuda").bfloat16()), dict(o=torch.empty(2, 4, 49, 64, device="cuda")), dict(o=t["q"]),
                dict(o=torch.empty(2, 1, 50, 64, device="cuda").expand(2, 4, 50, 64)), dict(lse=torch.empty(2, 4, 49, device="cuda")),
                dict(lse=torch.empty(2, 4, 50, device="cuda").double())):
        with pytest.raises((ValueError, TypeError, hdt.HdtError)):
            hdt.hdt_rel_attn_fwd(**{**good, **bad})
    o, lse = hdt.hdt_rel_attn_fwd(**good)
    good.update(o=o, lse=lse, d_o=t["d_o"])
    for bad in (dict(d_o=t["d_o"][:, :, :9]), dict(lse=lse[:, :3]), dict(dq=t["q"]), dict(dk=torch.empty_like(t["q"])), dict(dbias=torch.empty(32, 4, device="cuda").bfloat16()),
                dict(dbias=torch.empty(31, 4, device="cuda")), dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, hdt.HdtError)):
            hdt.hdt_rel_attn_bwd(**{**good, **bad})
    for bad in (dict(p=1.0), dict(p=-0.5), dict(p=float("nan")), dict(rng=None), dict(rng=t["rng"].int()), dict(rng=t["rng"][:1]), dict(rng=t["rng"].cpu()), dict(x=t["x"][1:]),
                dict(x=t["x"].bfloat16()), dict(y=t["y"].transpose(0, 1)), dict(y=t["y"].half()), dict(out=t["x"][:3]), dict(y=t["y"].reshape(-1)[1:], x=None)):
        with pytest.raises((ValueError, TypeError, hdt.HdtError)):
            hdt.hdt_dropout_add(**{**dict(y=t["y"], p=0.1, rng=t["rng"], x=t["x"]), **bad})
    norm = dict(x=t["x"], weight=t["w"], bias=t["b"], y=t["y"], p=0.1, rng=t["rng"])
    for bad in (dict(weight=t["w"][:39]), dict(bias=t["b"].bfloat16()), dict(y=t["y"][1:]), dict(rng=None), dict(eps=-1.0), dict(p=2.0), dict(n=t["x"]), dict(h=t["y"]),
                dict(mean=torch.empty(5, device="cuda")), dict(rstd=torch.empty(30, device="cuda").double()), dict(x=t["x"].transpose(0, 1), y=t["y"].transpose(0, 1))):
        with pytest.raises((ValueError, TypeError, hdt.HdtError)):
            hdt.hdt_add_norm_fwd(**{**norm, **bad})
    n, h, mean, rstd = hdt.hdt_add_norm_fwd(**norm)
    back = dict(dn=t["dn"], h=h, weight=t["w"], mean=mean, rstd=rstd, p=0.1, rng=t["rng"])
    for bad in (dict(dn=t["dn"][1:]), dict(mean=mean[1:]), dict(rng=None), dict(dx=h), dict(dy=t["dn"]), dict(dweight=t["w"].bfloat16()), dict(p=1.0),
                dict(workspace=torch.empty(16, dtype=torch.uint8, device="cuda"))):
        with pytest.raises((ValueError, TypeError, hdt.HdtError)):
            hdt.hdt_add_norm_bwd(**{**back, **bad})


def test_numbers_that_are_not_plain(hdt):
    """numpy scalars and whole numbers where a float is meant."""
    import torch
    t = tensors(torch.float32)
    table = hdt.hdt_rel_table(32, 128)
    a = hdt.hdt_rel_attn_fwd(t["q"], t["k"], t["v"], t["bias"], table, np.float64(1.0), causal=1)
    b = hdt.hdt_rel_attn_fwd(t["q"], t["k"], t["v"], t["bias"], table, 1, causal=True)
    assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert torch.equal(hdt.hdt_dropout_add(t["y"], np.float32(0.25), t["rng"], np.int64(3)), hdt.hdt_dropout_add(t["y"], 0.25, t["rng"], 3))
    assert torch.equal(hdt.hdt_add_norm_fwd(t["x"], t["w"], y=t["y"], p=0)[0], hdt.hdt_add_norm_fwd(t["x"], t["w"], y=t["y"])[0])
