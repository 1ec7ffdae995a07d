"""CPU checks of what embeddings, the feed-forward block and the norms around a block refuse: argument errors answer without a GPU."""
import os

import pytest

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 4
NAN, INF = float("nan"), float("inf")


@pytest.fixture(scope="module")
def lib():
    from paper_2407_08330_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2407_08330_amd import build
        build.build()
    return binding.load_library()


# every call below is refused before anything is enqueued: the addresses are never used
def call(lib, name, defaults, **kw):
    assert set(kw) <= set(defaults)
    return getattr(lib, name)(*{**defaults, **kw}.values())


EMBED = dict(ids=4, tokens=3, table=16, vocab=5, width=8, scale=1.0, out=32, table_dt=0, dt=0, stream=None)
EMBED_BWD = dict(d_out=16, ids=4, tokens=3, vocab=5, width=8, scale=1.0, accumulate=0, grad=32, table_dt=0, dt=0, workspace=48, nbytes=1 << 30, stream=None)
FFN = dict(x=16, wg=32, wu=48, wd=64, rows=3, width=8, inner=16, act=0, y=80, by_gate=96, by_up=112, hidden=128, dt=0, workspace=None, nbytes=0, stream=None)
FFN_BWD = dict(dy=16, x=32, wg=48, wu=64, wd=80, by_gate=96, by_up=112, hidden=128, rows=3, width=8, inner=16, dx=144, dwg=160, dwu=176, dwd=192, dt=0, workspace=208,
               nbytes=1 << 40, stream=None)
NORM = dict(x=16, y=32, wp=48, bp=64, gate=80, w=96, b=112, rows=3, width=8, eps=1e-5, scale=1.0, rms=0, h=128, n=144, stats=160, dt=0, wdt=0, stream=None)
NORM_BWD = dict(dn=16, dh=32, h=48, y=64, stats=80, wp=96, bp=112, gate=128, w=144, rows=3, width=8, scale=1.0, rms=0, dx=160, dy=176, dwp=192, dbp=208, dgate=224, dw=240, db=256,
                dt=0, wdt=0, workspace=272, nbytes=1 << 30, stream=None)

SIZES = [(INVALID, dict(width=-1)), (SHAPE, dict(width=0)), (UNSUPPORTED, dict(dt=2))]
REFUSED = {
    "hdt_embed_fwd": (EMBED, [*SIZES, (INVALID, dict(tokens=-1)), (INVALID, dict(vocab=-1)), (SHAPE, dict(vocab=0)), (SHAPE, dict(vocab=(1 << 24) + 1)), (SHAPE, dict(width=32769)),
                              (SHAPE, dict(tokens=(1 << 28) + 1)), (SHAPE, dict(tokens=1 << 28, width=136)), (UNSUPPORTED, dict(table_dt=-1)), (INVALID, dict(scale=NAN)),
                              (INVALID, dict(scale=INF)), (INVALID, dict(out=16)), (INVALID, dict(ids=6))]),
    "hdt_embed_bwd": (EMBED_BWD, [*SIZES, (INVALID, dict(tokens=-1)), (SHAPE, dict(vocab=0)), (SHAPE, dict(vocab=1 << 24, width=4096)), (UNSUPPORTED, dict(table_dt=9)),
                                  (INVALID, dict(scale=-INF)), (INVALID, dict(grad=16)), (INVALID, dict(nbytes=100)), (INVALID, dict(workspace=40)), (INVALID, dict(ids=2)),
                                  (INVALID, dict(grad=None, tokens=0, d_out=None, ids=None, workspace=None))]),
    "hdt_ffn_fwd": (FFN, [*SIZES, (INVALID, dict(rows=-1)), (INVALID, dict(inner=-1)), (SHAPE, dict(inner=0)), (SHAPE, dict(inner=65537)), (SHAPE, dict(rows=(1 << 28) + 1)),
                          (SHAPE, dict(rows=1 << 28, inner=256)), (UNSUPPORTED, dict(act=3)), (UNSUPPORTED, dict(act=-1)), (INVALID, dict(y=16)), (INVALID, dict(by_gate=48)),
                          (INVALID, dict(by_up=128)), (INVALID, dict(by_gate=None)), (INVALID, dict(hidden=None)), (INVALID, dict(by_up=None, by_gate=None, hidden=None))]),
    "hdt_ffn_bwd": (FFN_BWD, [*SIZES, (INVALID, dict(rows=-1)), (SHAPE, dict(inner=0)), (INVALID, dict(dx=16)), (INVALID, dict(dwg=176)), (INVALID, dict(nbytes=64)),
                              (INVALID, dict(rows=0, dwd=None)), (INVALID, dict(workspace=None))]),
    "hdt_gate_norm_fwd": (NORM, [*SIZES, (INVALID, dict(rows=-1)), (SHAPE, dict(width=32769)), (SHAPE, dict(rows=1 << 31)), (UNSUPPORTED, dict(wdt=3)), (INVALID, dict(eps=-1.0)),
                                 (INVALID, dict(eps=NAN)), (INVALID, dict(scale=INF)), (INVALID, dict(h=16)), (INVALID, dict(n=128)), (INVALID, dict(stats=144)), (INVALID, dict(stats=162)),
                                 (INVALID, dict(n=112))]),
    "hdt_gate_norm_bwd": (NORM_BWD, [*SIZES, (INVALID, dict(rows=-1)), (UNSUPPORTED, dict(wdt=3)), (INVALID, dict(scale=NAN)), (INVALID, dict(dx=16)), (INVALID, dict(dy=160)),
                                     (INVALID, dict(dw=192)), (INVALID, dict(dgate=128)), (INVALID, dict(gate=None)), (INVALID, dict(nbytes=64)), (INVALID, dict(workspace=None)),
                                     (INVALID, dict(db=257)), (INVALID, dict(rows=0, dw=None))]),
}
OPTIONAL = {"workspace", "bp", "gate", "b", "dh", "dbp", "dgate", "db", "stream"}
VALUES = {"tokens", "vocab", "width", "scale", "accumulate", "table_dt", "dt", "nbytes", "rows", "inner", "act", "eps", "rms", "wdt"}


@pytest.mark.parametrize("name", REFUSED)
def test_refused(lib, name):
    defaults, bad = REFUSED[name]
    for status, kw in bad:
        assert call(lib, name, defaults, **kw) == status, kw
        assert len(lib.hdt_last_error()) > 10
    for p in set(defaults) - VALUES - OPTIONAL - {"by_gate", "by_up", "hidden"}:
        assert call(lib, name, defaults, **{p: None}) == INVALID, p
        assert call(lib, name, defaults, **{p: 16 * 30 + (1 if p in ("ids", "stats", "dwp", "dbp", "dgate", "dw", "db") else 8)}) == INVALID, p


def test_nothing_to_do(lib):
    none = lambda d, *keep: {k: None for k in set(d) - VALUES - set(keep)}  # noqa: E731
    assert call(lib, "hdt_embed_fwd", EMBED, tokens=0, **none(EMBED)) == OK
    assert call(lib, "hdt_embed_bwd", EMBED_BWD, tokens=0, accumulate=1, **none(EMBED_BWD, "grad")) == OK
    assert call(lib, "hdt_ffn_fwd", FFN, rows=0, **none(FFN)) == OK
    assert call(lib, "hdt_gate_norm_fwd", NORM, rows=0, **none(NORM)) == OK


def test_workspace_sizes(lib):
    assert lib.hdt_embed_bwd_workspace_bytes(0, 8) == 0 and lib.hdt_embed_bwd_workspace_bytes(5, 0) == 0 and lib.hdt_embed_bwd_workspace_bytes(1 << 31, 8) == 0
    assert lib.hdt_embed_bwd_workspace_bytes(1 << 28, 32) > (1 << 31)
    assert lib.hdt_ffn_bwd_workspace_bytes(0, 8, 8, 0) == 0 and lib.hdt_ffn_bwd_workspace_bytes(5, 8, 8, 7) == 0 and lib.hdt_ffn_bwd_workspace_bytes(5, -8, 8, 0) == 0
    assert lib.hdt_ffn_fwd_workspace_bytes(100, 8, 24, 0, 0) >= 4800 and lib.hdt_ffn_fwd_workspace_bytes(-1, 8, 24, 0, 0) == 0
    assert lib.hdt_ffn_bwd_workspace_bytes(1 << 20, 8, 32768, 0) >= 1 << 37
    assert lib.hdt_gate_norm_bwd_workspace_bytes(0, 8) == 0 and lib.hdt_gate_norm_bwd_workspace_bytes(3, 40000) == 0 and lib.hdt_gate_norm_bwd_workspace_bytes(1 << 31, 8) == 0
