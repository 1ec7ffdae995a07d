"""CPU checks of what the relative-bias attention, the dropout and the norm refuse: argument errors answer without a GPU."""
import ctypes

import pytest

OK, INVALID, SHAPE, UNSUPPORTED = 0, 1, 2, 4


@pytest.fixture(scope="module")
def lib():
    import os
    from paper_2407_08330_amd import binding
    if not os.path.exists(binding.library_path()):
        from paper_2407_08330_amd import build
        build.build()
    return binding.load_library()


def call(**kw):
    from paper_2407_08330_amd.binding import _RelAttn
    c = _RelAttn(2, 4, 2, 8, 8, 64, 1, 32, 128, 0, 0, 0.125, 16, 16, None, None)
    for name, value in kw.items():
        if isinstance(value, tuple):
            s = getattr(c, name)
            s.batch, s.head, s.row = value
        else:
            setattr(c, name, value)
    return c


def fwd(lib, c, ptrs=None, lse=4096):
    p = ptrs or [16 * (i + 1) for i in range(4)]
    return lib.hdt_rel_attn_fwd(ctypes.byref(c), *p, lse, None, 0, None)


# every call below is refused before anything is enqueued: the addresses are never used
@pytest.mark.parametrize("status,kw", [
    (INVALID, dict(batch=-1)), (INVALID, dict(heads=-4)), (INVALID, dict(n_q=-1)), (INVALID, dict(n_kv=-1)),
    (SHAPE, dict(kv_heads=3)), (SHAPE, dict(kv_heads=0)), (SHAPE, dict(kv_heads=-2)), (UNSUPPORTED, dict(head_dim=96)),
    (UNSUPPORTED, dict(head_dim=0)), (UNSUPPORTED, dict(dtype=2)), (UNSUPPORTED, dict(bias_dtype=7)), (INVALID, dict(softmax_scale=0.0)),
    (INVALID, dict(softmax_scale=-1.0)), (INVALID, dict(softmax_scale=float("nan"))), (INVALID, dict(softmax_scale=float("inf"))),
    (INVALID, dict(softmax_scale=1e-39)), (INVALID, dict(softmax_scale=1e20)), (SHAPE, dict(max_distance=0)), (SHAPE, dict(max_distance=1025)), (SHAPE, dict(n_buckets=0)),
    (SHAPE, dict(n_buckets=4097)), (SHAPE, dict(n_kv=(1 << 24) + 1)), (SHAPE, dict(batch=1 << 20, heads=1 << 10, kv_heads=1 << 10)), (SHAPE, dict(n_kv=1 << 24, heads=8, kv_heads=1)),
    (SHAPE, dict(batch=2 ** 31 - 1, heads=2 ** 30, kv_heads=2 ** 30, n_q=1 << 24)),
    (INVALID, dict(d_bias=None)), (INVALID, dict(d_table=None)),
    (INVALID, dict(q=(4096, 512, 65))), (INVALID, dict(q=(4096, 513, 64))), (INVALID, dict(k=(-4096, 512, 64))), (INVALID, dict(v=(4096, 512, 32))),
    (INVALID, dict(q=(1 << 30, 1 << 28, 1 << 21))), (INVALID, dict(o=(0, 512, 64))), (INVALID, dict(o=(2048, 0, 64))),
    (INVALID, dict(o=(2048, 256, 64))), (INVALID, dict(o=(2048, 64, 128))),
])
def test_forward_refuses(lib, status, kw):
    assert fwd(lib, call(**kw)) == status
    assert len(lib.hdt_last_error()) > 10


def test_forward_refuses_pointers(lib):
    c = call()
    assert lib.hdt_rel_attn_fwd(None, 16, 32, 48, 64, 80, None, 0, None) == INVALID
    for i in range(4):
        p = [16, 32, 48, 64]
        p[i] = None
        assert fwd(lib, c, p) == INVALID
        p[i] = 24 + 16 * i
        assert fwd(lib, c, p) == INVALID
    assert fwd(lib, c, lse=None) == INVALID and fwd(lib, c, lse=4098) == INVALID
    for i in range(3):
        assert fwd(lib, c, [16, 32, 48, 16 * (i + 1)]) == INVALID  # o is an input
    assert lib.hdt_rel_attn_fwd(ctypes.byref(c), 16, 32, 48, 64, 80, 100, 4096, None) == INVALID  # workspace misaligned


def test_empty_forwards_do_nothing(lib):
    for kw in (dict(batch=0), dict(heads=0), dict(n_q=0)):
        assert fwd(lib, call(**kw), [None] * 4, None) == OK
        assert lib.hdt_rel_attn_fwd_workspace_bytes(ctypes.byref(call(**kw))) == 0
    assert lib.hdt_rel_attn_bwd_workspace_bytes(ctypes.byref(call(head_dim=80))) == 0


def bwd(lib, c, change=(), workspace=4096, nbytes=1 << 40):
    p = [16 * (i + 1) for i in range(10)]
    for i, v in change:
        p[i] = v
    return lib.hdt_rel_attn_bwd(ctypes.byref(c), *p, workspace, nbytes, None)


def test_backward_refuses(lib):
    c = call()
    for i in range(10):
        assert bwd(lib, c, [(i, None)]) == INVALID
        if i not in (4, 9):
            assert bwd(lib, c, [(i, 8)]) == INVALID
    assert bwd(lib, c, [(4, 82)]) == INVALID
    for out in (6, 7, 8):
        for inp in (0, 1, 2, 3, 5):
            assert bwd(lib, c, [(out, 16 * (inp + 1))]) == INVALID
    assert bwd(lib, c, [(7, 112)]) == INVALID  # dk is dq
    assert bwd(lib, c, workspace=None) == INVALID and bwd(lib, c, workspace=4104) == INVALID
    need = lib.hdt_rel_attn_bwd_workspace_bytes(ctypes.byref(c))
    assert need > 0 and bwd(lib, c, nbytes=need - 1) == INVALID
    for name in ("dq", "dk", "dv"):
        assert bwd(lib, call(**{name: (0, 512, 64)})) == INVALID
    assert bwd(lib, call(heads=0, n_kv=0), [(i, None) for i in range(10)], None) == OK


def test_table_refuses(lib):
    for args, status in (((1, 128, 0), SHAPE), ((3, 128, 1), SHAPE), ((2, 128, 1), SHAPE), ((32, 16, 0), SHAPE), ((32, 8, 1), SHAPE),
                         ((32, 1025, 0), SHAPE), ((4097, 1024, 0), SHAPE), ((-1, 128, 0), INVALID), ((32, -1, 0), INVALID)):
        assert lib.hdt_rel_table(*args, 16, None) == status, args
    assert lib.hdt_rel_table(32, 128, 0, None, None) == INVALID


def test_dropout_refuses(lib):
    def go(y=16, x=None, out=32, n=8, p=0.1, rng=64, dt=0):
        return lib.hdt_dropout_add(y, x, out, n, p, rng, 0, dt, None)
    assert go(y=None) == INVALID and go(out=None) == INVALID and go(rng=None) == INVALID
    assert go(n=-1) == INVALID and go(n=(1 << 35) + 1) == SHAPE and go(dt=3) == UNSUPPORTED
    assert go(y=18) == INVALID and go(x=20) == INVALID and go(out=40) == INVALID and go(rng=68) == INVALID
    for p in (-0.1, 1.0, 1.5, float("nan"), 0.999999):
        assert go(p=p) == INVALID
    assert go(y=None, out=None, rng=None, n=0) == OK


def test_norm_refuses(lib):
    def f(x=16, y=32, w=48, b=64, rows=4, width=8, eps=1e-5, p=0.1, rng=80, h=96, n=112, mean=128, rstd=144, dt=0, wdt=0):
        return lib.hdt_add_norm_fwd(x, y, w, b, rows, width, eps, p, rng, 0, h, n, mean, rstd, dt, wdt, None)
    for kw in (dict(x=None), dict(w=None), dict(n=None), dict(mean=None), dict(rstd=None), dict(h=None), dict(rng=None), dict(rows=-1), dict(eps=-1.0),
               dict(eps=float("nan")), dict(eps=float("inf")), dict(p=1.0), dict(p=-1.0), dict(x=24), dict(y=24), dict(w=24), dict(b=24), dict(h=24),
               dict(n=24), dict(n=16), dict(n=32), dict(h=16), dict(h=32), dict(h=112), dict(rng=84)):
        assert f(**kw) == INVALID, kw
    for kw in (dict(width=0), dict(width=32769), dict(rows=1 << 31), dict(rows=1 << 30, width=64)):
        assert f(**kw) == SHAPE, kw
    assert f(dt=2) == UNSUPPORTED and f(wdt=-1) == UNSUPPORTED
    assert f(rows=0, x=None, y=None, w=None, n=None, rng=None, h=None) == OK

    def g(dn=16, dh=32, h=48, w=64, mean=80, rstd=96, rows=4, width=8, p=0.1, rng=112, dx=128, dy=144, dw=160, db=176, dt=0, wdt=0, ws=4096, nb=1 << 30):
        return lib.hdt_add_norm_bwd(dn, dh, h, w, mean, rstd, rows, width, p, rng, 0, dx, dy, dw, db, dt, wdt, ws, nb, None)
    need = lib.hdt_add_norm_bwd_workspace_bytes(4, 8)
    assert need > 0 and lib.hdt_add_norm_bwd_workspace_bytes(0, 8) == 0 and lib.hdt_add_norm_bwd_workspace_bytes(4, 0) == 0
    for kw in (dict(dn=None), dict(h=None), dict(w=None), dict(mean=None), dict(rstd=None), dict(dx=None), dict(dy=None), dict(dw=None), dict(rng=None),
               dict(ws=None), dict(ws=4104), dict(nb=need - 1), dict(dx=16), dict(dx=32), dict(dx=48), dict(dy=16), dict(dy=128), dict(dn=24), dict(dh=40),
               dict(dx=136), dict(rows=-1)):
        assert g(**kw) == INVALID, kw
    assert g(width=0) == SHAPE and g(dt=4) == UNSUPPORTED


def test_binding_refuses_host_tensors():
    """What would hand a host address to a kernel is an error before the call."""
    import torch
    import paper_2407_08330_amd as hdt
    with pytest.raises(ValueError):
        hdt.hdt_rel_table(32, 128, device="cpu")
    q, table, bias = torch.zeros(1, 1, 4, 64), torch.zeros(257, dtype=torch.int32), torch.zeros(32, 1)
    with pytest.raises(ValueError):
        hdt.hdt_rel_attn_fwd(q, q, q, bias, table, 1.0)
    with pytest.raises(ValueError):
        hdt.hdt_rel_attn_bwd(q, q, q, bias, table, q, torch.zeros(1, 1, 4), q, 1.0)
    x, w, rng = torch.zeros(2, 8), torch.zeros(8), torch.zeros(2, dtype=torch.int64)
    for call in (lambda: hdt.hdt_dropout_add(x, 0.1, rng), lambda: hdt.hdt_add_norm_fwd(x, w, w),
                 lambda: hdt.hdt_add_norm_bwd(x, x, w, torch.zeros(2), torch.zeros(2))):
        with pytest.raises(ValueError):
            call()
