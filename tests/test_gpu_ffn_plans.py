"""GPU tests of the feed-forward block at sizes that meet every form of its kernels (tests/ffn_cases.py, whose forms test_ffn_plan.py checks), bit for bit: on whole
numbers, and G a multiple of 128, where each activation is G or 0 and its slope 1, 0 or (at 0) a half, every sum is exact in fp32 in any order, and a result is
the exact one rounded once.  So one wrong element, part or tile is seen."""
import pytest

import ffn_cases
from gpu_common import GuardedWorkspace, say

pytestmark = pytest.mark.gpu


class Given:
    """A tensor of NaN that a call fills, with a guard behind it."""

    def __init__(self, shape, dtype):
        import torch
        n = shape[0] * shape[1]
        self.room = torch.full((n + 64,), float("nan"), dtype=dtype, device="cuda")
        self.room[n:] = 7
        self.t = self.room[:n].view(shape)

    def check(self, want, name):
        import torch
        assert bool((self.room[-64:] == 7).all()), f"{name}: written behind its end"
        want = want.to(self.t.dtype)
        if not torch.equal(self.t, want):
            wrong = ~(self.t == want)
            at = wrong.nonzero()[0].tolist()
            raise AssertionError(f"{name}: {int(wrong.sum())} of {wrong.numel()} wrong, the first at {at}: {float(self.t[tuple(at)])}, not {float(want[tuple(at)])}")


def scratch(nbytes):
    ws = GuardedWorkspace(nbytes)
    ws.buf[:ws.nbytes] = 0xFF
    return ws


def exact_in_32_bits(*sizes):
    """sums of magnitudes, of values that are multiples of 1: below 2^24 every partial sum is exact"""
    assert all(float(s.max()) < 2 ** 24 for s in sizes)


def check(rows, width, inner, dtype):
    import torch
    import paper_2407_08330_amd as hdt
    lib, code = hdt.load_library(), 0 if dtype == torch.bfloat16 else 1
    act = "silu" if (rows + inner) % 2 else "gelu_tanh"
    gen = torch.Generator(device="cuda").manual_seed(rows + width + inner)

    def whole(*shape, k):
        """-1, 0 and 1, so many of them that a sum of k products has a variance of 16 at most"""
        p = min(1.0, 4 / k ** 0.5)
        u = torch.rand(shape, generator=gen, device="cuda")
        return ((u < p / 2).to(torch.int8) - (u > 1 - p / 2).to(torch.int8)).to(dtype)

    x, wg, wu, wd = whole(rows, width, k=width), whole(inner, width, k=width) * 128, whole(inner, width, k=width), whole(width, inner, k=inner)
    y = Given((rows, width), dtype)
    kept = [Given((rows, inner), dtype) for _ in range(3)]
    ws = scratch(lib.hdt_ffn_fwd_workspace_bytes(rows, width, inner, 1, code))
    hdt.hdt_ffn_fwd(x, wg, wu, wd, act, y=y.t, by_gate=kept[0].t, by_up=kept[1].t, hidden=kept[2].t, workspace=ws.view)
    ws.check()
    g, u = x.double() @ wg.double().t(), x.double() @ wu.double().t()
    for t, (name, want) in zip(kept, (("by_gate", u * torch.where(g > 0, 1.0, torch.where(g < 0, 0.0, 0.5))), ("by_up", g.clamp_min(0)), ("hidden", g.clamp_min(0) * u))):
        t.check(want, name)
    exact_in_32_bits((kept[2].t.double().abs() / 128) @ wd.double().abs().t())
    y.check(kept[2].t.double() @ wd.double().t(), "y")
    only = Given((rows, width), dtype)
    ws = scratch(lib.hdt_ffn_fwd_workspace_bytes(rows, width, inner, 0, code))
    hdt.hdt_ffn_fwd(x, wg, wu, wd, act, train=False, y=only.t, workspace=ws.view)
    ws.check()
    only.check(y.t, "y alone")
    del g, u, y, only, kept

    dy, by_gate, by_up, hidden = whole(rows, width, k=width), whole(rows, inner, k=16), whole(rows, inner, k=16), whole(rows, inner, k=16)
    wd = whole(width, inner, k=width)
    out = [Given((rows, width), dtype), Given((inner, width), dtype), Given((inner, width), dtype), Given((width, inner), dtype)]
    ws = scratch(lib.hdt_ffn_bwd_workspace_bytes(rows, width, inner, code))
    hdt.hdt_ffn_bwd(dy, x, wg, wu, wd, by_gate, by_up, hidden, **{k: t.t for k, t in zip(("dx", "dw_gate", "dw_up", "dw_down"), out)}, workspace=ws.view)
    ws.check()
    dh = dy.double() @ wd.double()
    assert float(dh.abs().max()) <= 256  # (dG and dU are exact in bf16)
    dg, du = dh * by_gate.double(), dh * by_up.double()
    x, wg, wu, dy, hidden = (t.double() for t in (x, wg, wu, dy, hidden))
    exact_in_32_bits(dg.abs() @ wg.abs() + du.abs() @ wu.abs(), dg.abs().t() @ x.abs(), du.abs().t() @ x.abs(), dy.abs().t() @ hidden.abs())
    for t, (name, want) in zip(out, (("dx", dg @ wg + du @ wu), ("dw_gate", dg.t() @ x), ("dw_up", du.t() @ x), ("dw_down", dy.t() @ hidden))):
        t.check(want, name)


@pytest.mark.parametrize("rows,width,inner,forms", ffn_cases.BF16)
def test_bf16(rows, width, inner, forms):
    import torch
    say(f"[ffn plans] bf16 {rows} x {width} x {inner}: {forms}")
    check(rows, width, inner, torch.bfloat16)


@pytest.mark.parametrize("rows,width,inner,forms", ffn_cases.F32)
def test_f32(rows, width, inner, forms):
    import torch
    say(f"[ffn plans] f32 {rows} x {width} x {inner}: {forms}")
    check(rows, width, inner, torch.float32)
