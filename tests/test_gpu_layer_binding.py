"""The native form of the calls of embeddings, the feed-forward block and the norms around a block against the general one: the same results
bit for bit, the same errors."""
import numpy as np
import pytest

from test_gpu_operator_binding import hdt  # noqa: F401  (a fixture, both forms)

pytestmark = pytest.mark.gpu


def tensors(dtype):
    import torch
    gen = torch.Generator(device="cuda").manual_seed(1)
    n = lambda *s: torch.randn(s, generator=gen, device="cuda").to(dtype)  # noqa: E731
    return dict(ids=torch.randint(-1, 9, (5, 6), generator=gen, device="cuda", dtype=torch.int32), table=n(9, 40), x=n(5, 6, 40), y=n(5, 6, 40), d=n(5, 6, 40), w=n(40), v=n(40),
                wg=n(56, 40), wu=n(56, 40), wd=n(40, 56))


def everything(hdt, t, **kw):  # noqa: F811
    import torch
    out = []
    for dtype in (None, torch.bfloat16, torch.float32):
        out.append(hdt.hdt_embed_fwd(t["ids"], t["table"], 2.0, dtype=dtype, **kw))
        out.append(hdt.hdt_embed_bwd(t["d"], t["ids"], 9, 2.0, dtype=dtype, **kw))
    out.append(hdt.hdt_embed_bwd(t["d"], t["ids"], 9, 0.5, grad=t["table"].clone(), accumulate=True, **kw))
    for act in ("silu", "gelu", "gelu_tanh"):
        y, *kept = hdt.hdt_ffn_fwd(t["x"], t["wg"], t["wu"], t["wd"], act, **kw)
        out += [y, *kept, hdt.hdt_ffn_fwd(t["x"], t["wg"], t["wu"], t["wd"], act, train=False, **kw)[0]]
        out += hdt.hdt_ffn_bwd(t["d"], t["x"], t["wg"], t["wu"], t["wd"], *kept, **kw)
    for more in ({}, dict(gate=t["v"]), dict(gate=t["v"], post_bias=t["w"], bias=t["v"]), dict(post_bias=t["w"])):
        for rms in (False, True):
            n, h, s = hdt.hdt_gate_norm_fwd(t["x"], t["y"], t["w"], t["v"], **more, scale=0.5, rms=rms, **kw)
            back = {k: v for k, v in more.items() if k != "bias"}
            got = hdt.hdt_gate_norm_bwd(t["d"], h, t["y"], s, t["w"], t["v"], **back, bias="bias" in more, dh=t["x"], scale=0.5, rms=rms, **kw)
            assert [g is not None for g in got[4:]] == ["gate" in more, "post_bias" in more, "bias" in more]
            out += [n, h, s, *(g for g in got if g is not None)]
    return out


@pytest.fixture(scope="module")
def first():
    return {}


@pytest.mark.parametrize("name", ["bf16", "f32"])
@pytest.mark.parametrize("other_stream", [False, True])
def test_both_give_the_same_bits(hdt, first, name, other_stream):  # noqa: F811
    import torch
    t = tensors({"bf16": torch.bfloat16, "f32": torch.float32}[name])
    torch.cuda.synchronize()
    got = everything(hdt, t, **(dict(stream=torch.cuda.Stream()) if other_stream else {}))
    torch.cuda.synchronize()
    want = first.setdefault(name, got)
    assert len(got) == len(want) and all(a.shape == b.shape and a.dtype == b.dtype and torch.equal(a, b) for a, b in zip(got, want))


def test_results_are_the_callers_tensors(hdt):  # noqa: F811
    import torch
    t = tensors(torch.float32)
    e = {k: torch.empty_like(v) for k, v in t.items()}
    assert hdt.hdt_embed_fwd(t["ids"], t["table"], out=e["x"]) is e["x"]
    assert hdt.hdt_embed_bwd(t["d"], t["ids"], 9, grad=e["table"]) is e["table"]
    kept = [torch.empty(5, 6, 56, device="cuda") for _ in range(3)]
    got = hdt.hdt_ffn_fwd(t["x"], t["wg"], t["wu"], t["wd"], y=e["y"], by_gate=kept[0], by_up=kept[1], hidden=kept[2])
    assert all(a is b for a, b in zip(got, (e["y"], *kept)))
    grads = dict(dx=e["x"], dw_gate=e["wg"], dw_up=e["wu"], dw_down=e["wd"])
    assert all(a is b for a, b in zip(hdt.hdt_ffn_bwd(t["d"], t["x"], t["wg"], t["wu"], t["wd"], *kept, **grads), grads.values()))
    stats = torch.empty(4, 5, 6, device="cuda")
    got = hdt.hdt_gate_norm_fwd(t["x"], t["y"], t["w"], t["v"], h=e["x"], n=e["y"], stats=stats)
    assert got[0] is e["y"] and got[1] is e["x"] and got[2] is stats
    grads = dict(dx=e["d"], dy=torch.empty_like(t["x"]), dpost_weight=e["w"], dweight=e["v"])
    assert all(a is b for a, b in zip(hdt.hdt_gate_norm_bwd(t["d"], e["x"], t["y"], stats, t["w"], t["v"], **grads), grads.values()))


def refused(hdt, call, good, bads):  # noqa: F811
    for bad in bads:
        with pytest.raises((ValueError, TypeError, hdt.HdtError)):
            call(**{**good, **bad})


def test_refusals(hdt):  # noqa: F811
    import torch
    t = tensors(torch.float32)
    ws = [torch.empty(8, dtype=torch.uint8, device="cuda"), torch.zeros(1, dtype=torch.uint8, device="cuda").expand(1 << 30), torch.zeros(1 << 26, dtype=torch.uint8, device="cuda")[::2]]
    refused(hdt, hdt.hdt_embed_fwd, dict(ids=t["ids"], table=t["table"]), [
        dict(ids=t["ids"].long()), dict(ids=t["ids"].t()), dict(ids=t["ids"].cpu()), dict(table=t["table"][0]), dict(table=t["table"].t()), dict(table=t["table"].half()),
        dict(table=t["table"].cpu()), dict(dtype=torch.float16), dict(out=torch.empty(5, 6, 39, device="cuda")), dict(out=torch.empty(5, 40, device="cuda")),
        dict(out=torch.empty(5, 6, 40, device="cuda"), dtype=torch.bfloat16), dict(out=torch.empty(5, 6, 80, device="cuda")[:, :, ::2]), dict(scale=float("nan")),
        dict(table=torch.empty(0, 40, device="cuda")), dict(table=t["table"].view(-1)[1:321].view(8, 40))])
    refused(hdt, hdt.hdt_embed_bwd, dict(d_out=t["d"], ids=t["ids"], vocab=9), [
        dict(d_out=t["d"][:, :5]), dict(d_out=t["d"].transpose(0, 1)), dict(d_out=t["d"].half()), dict(ids=t["ids"].long()), dict(vocab=-1), dict(vocab=0), dict(vocab=2 ** 32 + 9),
        dict(accumulate=True), dict(grad=torch.empty(8, 40, device="cuda")), dict(grad=torch.empty(9, 41, device="cuda")), dict(grad=torch.empty(9, 40, device="cuda").half()),
        dict(grad=torch.empty(9, 40, device="cuda"), dtype=torch.bfloat16), dict(grad=torch.empty(40, 9, device="cuda").t()), dict(scale=float("inf")), *(dict(workspace=w) for w in ws)])
    ffn = dict(x=t["x"], w_gate=t["wg"], w_up=t["wu"], w_down=t["wd"])
    refused(hdt, hdt.hdt_ffn_fwd, ffn, [
        dict(x=t["x"][:, :, :39]), dict(x=t["x"].transpose(0, 1)), dict(x=t["x"].bfloat16()), dict(x=t["x"].half()), dict(w_gate=t["wg"][:55]), dict(w_up=t["wu"].bfloat16()), dict(w_down=t["wu"]),
        dict(w_gate=t["wd"].t(), w_up=t["wd"].t()), dict(w_gate=t["wg"].cpu()), dict(act="relu"), dict(act=None), dict(act=0), dict(y=t["x"]), dict(y=torch.empty(5, 6, 41, device="cuda")),
        dict(hidden=torch.empty(5, 6, 55, device="cuda")), dict(hidden=torch.empty(5, 6, 56, device="cuda"), train=False), dict(by_up=torch.empty(5, 6, 56, device="cuda").bfloat16()),
        dict(train=False, workspace=ws[0]), dict(workspace=ws[1]), dict(workspace=ws[2]), dict(x=t["x"].view(-1)[1:1 + 40].view(1, 40))])
    y, a, b, c = hdt.hdt_ffn_fwd(**ffn)
    refused(hdt, hdt.hdt_ffn_bwd, dict(ffn, dy=t["d"], by_gate=a, by_up=b, hidden=c), [
        dict(dy=t["d"][:4]), dict(dy=t["d"].bfloat16()), dict(by_gate=a[:, :, :55]), dict(hidden=None), dict(dx=t["x"]), dict(dw_gate=torch.empty(56, 41, device="cuda")),
        dict(dw_down=torch.empty(56, 40, device="cuda").t()), dict(dw_up=t["wu"]), *(dict(workspace=w) for w in ws)])
    norm = dict(x=t["x"], y=t["y"], post_weight=t["w"], weight=t["v"], gate=t["w"], post_bias=t["v"], bias=t["v"])
    refused(hdt, hdt.hdt_gate_norm_fwd, norm, [
        dict(y=t["y"][1:]), dict(y=t["y"].bfloat16()), dict(x=t["x"].transpose(0, 1), y=t["y"].transpose(0, 1)), dict(weight=t["w"][:39]), dict(gate=t["w"].bfloat16()), dict(bias=t["w"].cpu()),
        dict(post_weight=None), dict(eps=-1.0), dict(scale=float("inf")), dict(h=t["x"]), dict(n=t["y"]), dict(stats=torch.empty(4, 30, device="cuda")), dict(stats=torch.empty(2, 5, 6, device="cuda")),
        dict(stats=torch.empty(4, 5, 6, device="cuda").double()), dict(x=t["x"].half(), y=t["y"].half())])
    n, h, s = hdt.hdt_gate_norm_fwd(**norm)
    back = dict(dn=t["d"], h=h, y=t["y"], stats=s, post_weight=t["w"], weight=t["v"], gate=t["w"], post_bias=t["v"], bias=True)
    refused(hdt, hdt.hdt_gate_norm_bwd, back, [
        dict(dn=t["d"][1:]), dict(dh=t["d"].bfloat16()), dict(stats=s[:3]), dict(dx=h), dict(dy=t["d"]), dict(dgate=torch.empty(39, device="cuda")), dict(gate=None, dgate=torch.empty(40, device="cuda")),
        dict(bias=False, dbias=torch.empty(40, device="cuda")), dict(post_bias=None, dpost_bias=torch.empty(40, device="cuda")), dict(dweight=torch.empty(40, device="cuda").bfloat16()),
        dict(scale=float("nan")), *(dict(workspace=w) for w in ws)])


def test_numbers_that_are_not_plain(hdt):  # noqa: F811
    """numpy scalars, and whole numbers where a float is meant."""
    import torch
    t = tensors(torch.float32)
    assert torch.equal(hdt.hdt_embed_fwd(t["ids"], t["table"], np.float64(2)), hdt.hdt_embed_fwd(t["ids"], t["table"], 2))
    assert torch.equal(hdt.hdt_embed_bwd(t["d"], t["ids"], np.int64(9), np.float32(2)), hdt.hdt_embed_bwd(t["d"], t["ids"], 9, 2.0))
    a, b = (hdt.hdt_gate_norm_fwd(t["x"], t["y"], t["w"], t["v"], scale=s, rms=r)[0] for s, r in ((np.float64(2), 1), (2.0, True)))
    assert torch.equal(a, b)
    a, b = (hdt.hdt_ffn_fwd(t["x"], t["wg"], t["wu"], t["wd"], train=r)[0] for r in (0, False))
    assert torch.equal(a, b)
