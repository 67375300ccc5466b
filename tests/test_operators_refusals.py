"""Calls of the operators around the exchange that are refused before anything is launched: through the C ABI with pointers that are never
followed, and by the binding on tensors of the host.  No GPU is needed."""
import ctypes

import pytest
import torch

from paper_1806_04090_b200 import api

INVALID, CAPACITY = 1, 3
GOOD = 1 << 20            # stands for a device address: 16-byte aligned, never read here


@pytest.fixture(scope="module")
def ctx():
    from paper_1806_04090_b200 import build
    build.build()
    lib = api.load_library()
    h = ctypes.c_void_p()
    lib.atomo_create(ctypes.byref(h), 0)                 # without a GPU the context exists all the same
    yield lib, h
    lib.atomo_destroy(h)


def test_grad_norm(ctx):
    lib, h = ctx
    size = lib.atomo_grad_norm_workspace_bytes
    one = lambda n, kind=0: (api._Tensor * 1)((GOOD, n, kind, 0))
    assert size(one(4), 1) == 0 and size(one(1 << 30), 1) > 0 and size(one(0), 1) >= 0
    assert size(one(-1), 1) == size(one(4, 3), 1) == size(one(4), 0) == size(None, 1) == -1
    need = size(one(1 << 24), 1)

    def call(data=GOOD, n=1 << 24, kind=0, count=1, max_norm=1.0, out=GOOD, ws=GOOD, size=need):
        return lib.atomo_grad_norm(h, (api._Tensor * 1)((data, n, kind, 0)), count, max_norm, out, ws, size, None)

    for bad in (dict(data=None), dict(data=GOOD + 2), dict(data=GOOD + 1, kind=1), dict(n=-1), dict(kind=3), dict(kind=-1), dict(count=0), dict(count=-1), dict(count=2 ** 20 + 1),
                dict(max_norm=0.0), dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(out=None), dict(out=GOOD + 2), dict(ws=None), dict(ws=GOOD + 4)):
        assert call(**bad) == INVALID, bad
    assert call(size=need - 1) == CAPACITY
    many = lambda n: (api._Tensor * 2)((GOOD, n, 0, 0), (GOOD, n, 0, 0))              # 2^40 values in all, at most
    assert size(many(1 << 39), 2) > 0 and size(many((1 << 39) + 1), 2) == -1
    assert lib.atomo_grad_norm(h, many((1 << 39) + 1), 2, 1.0, GOOD, GOOD, 1 << 20, None) == INVALID
    assert lib.atomo_grad_norm(None, (api._Tensor * 1)((GOOD, 4, 0, 0)), 1, 1.0, GOOD, GOOD, need, None) == INVALID


def test_adamw(ctx):
    lib, h = ctx

    def call(param=GOOD, m=GOOD, v=GOOD, ms=None, vs=None, master=None, n=4, decay=0.0, kind=0, grad=GOOD, count=1, lr=1e-3, b1=0.9, b2=0.999, eps=1e-8, step=1, scale=None, bits=32,
             gkind=0):
        args = api._AdamWArgs(lr, b1, b2, eps, step, 0, scale, bits, gkind)
        return lib.atomo_adamw(h, (api._AdamWTensor * 1)((param, m, v, ms, vs, master, n, decay, kind)), (ctypes.c_void_p * 1)(grad), count, ctypes.byref(args), None)

    inf, nan = float("inf"), float("nan")
    for bad in (dict(param=None), dict(param=GOOD + 2), dict(param=GOOD + 1, kind=1), dict(m=None), dict(v=None), dict(m=GOOD + 2), dict(grad=None), dict(grad=GOOD + 2),
                dict(master=GOOD + 2), dict(n=-1), dict(n=1 << 41), dict(decay=-0.1), dict(decay=nan), dict(decay=inf), dict(kind=3), dict(gkind=3), dict(count=0), dict(lr=-1.0), dict(lr=nan),
                dict(lr=inf), dict(b1=1.0), dict(b1=-0.1), dict(b2=1.0), dict(b2=nan), dict(eps=-1e-8), dict(eps=inf), dict(step=0), dict(step=-3), dict(scale=GOOD + 2), dict(bits=16),
                dict(bits=8), dict(bits=8, ms=GOOD), dict(bits=8, vs=GOOD), dict(bits=8, ms=GOOD, vs=GOOD, n=1 << 34)):
        assert call(**bad) == INVALID, bad


def test_embedding(ctx):
    lib, h = ctx

    def look(table=GOOD, kind=0, rows=8, cols=4, ld=4, ids=GOOD, width=8, n=3, scale=1.0, out=GOOD, ld_out=4, status=None):
        return lib.atomo_embedding(h, table, kind, rows, cols, ld, ids, width, n, scale, out, ld_out, status, None)

    for bad in (dict(table=None), dict(table=GOOD + 2), dict(kind=5), dict(rows=0), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 22) + 1, ld=1 << 25, ld_out=1 << 25), dict(ld=3),
                dict(ids=None), dict(ids=GOOD + 4), dict(width=2), dict(n=-1), dict(n=1 << 31), dict(scale=float("nan")), dict(out=None), dict(ld_out=3), dict(status=GOOD + 1)):
        assert look(**bad) == INVALID, bad

    size = lib.atomo_embedding_workspace_bytes
    assert size(3, 8, 4) == size(0, 8, 4) == 0 and size(100000, 8, 4) > 0
    assert size(-1, 8, 4) == size(3, 0, 4) == size(3, 8, 0) == size(1 << 31, 8, 4) == size(3, 1 << 31, 4) == -1

    def back(ids=GOOD, width=8, n=3, grad=GOOD, kind=0, ld=4, rows=8, cols=4, scale=1.0, padding=-1, out=GOOD, ld_out=4, status=None, ws=GOOD, nbytes=1 << 30):
        return lib.atomo_embedding_backward(h, ids, width, n, grad, kind, ld, rows, cols, scale, padding, out, ld_out, 0, status, ws, nbytes, None)

    for bad in (dict(ids=None), dict(ids=GOOD + 4), dict(width=1), dict(n=-1), dict(grad=None), dict(grad=GOOD + 2), dict(kind=-1), dict(ld=3), dict(rows=0), dict(cols=0), dict(scale=float("inf")),
                dict(padding=-2), dict(padding=8), dict(out=None), dict(out=GOOD + 2), dict(ld_out=3), dict(status=GOOD + 2), dict(n=100000, ws=None), dict(n=100000, ws=GOOD + 8)):
        assert back(**bad) == INVALID, bad
    assert back(n=100000, nbytes=size(100000, 8, 4) - 1) == CAPACITY


def test_layer_norm(ctx):
    lib, h = ctx

    def forward(x=GOOD, kind=0, rows=3, cols=4, ld=4, w=GOOD, b=GOOD, wkind=0, eps=1e-5, y=GOOD, ld_y=4, mean=GOOD, rstd=GOOD):
        return lib.atomo_layer_norm(h, x, kind, rows, cols, ld, w, b, wkind, eps, y, ld_y, mean, rstd, None)

    for bad in (dict(x=None), dict(x=GOOD + 2), dict(kind=3), dict(rows=-1), dict(rows=1 << 31), dict(cols=0), dict(cols=(1 << 22) + 1, ld=1 << 25, ld_y=1 << 25), dict(ld=3), dict(w=GOOD + 2),
                dict(b=GOOD + 1), dict(wkind=7), dict(eps=-1.0), dict(eps=float("nan")), dict(y=None), dict(ld_y=3), dict(mean=None), dict(rstd=None)):
        assert forward(**bad) == INVALID, bad

    size = lib.atomo_layer_norm_workspace_bytes
    assert size(3, 4) == size(256, 4) == 0 and size(257, 4) > 0 and size(1000, 4) > 0 and size(3, 100000) > 0 and size(-1, 4) == size(3, 0) == size((1 << 30) + 1, 4) == -1

    def backward(dy=GOOD, ld_dy=4, x=GOOD, ld_x=4, kind=0, rows=3, cols=4, w=GOOD, wkind=0, mean=GOOD, rstd=GOOD, dx=GOOD, ld_dx=4, dw=GOOD, db=GOOD, ws=GOOD, nbytes=1 << 30):
        return lib.atomo_layer_norm_backward(h, dy, ld_dy, x, ld_x, kind, rows, cols, w, wkind, mean, rstd, dx, ld_dx, dw, db, ws, nbytes, None)

    for bad in (dict(dy=None), dict(ld_dy=3), dict(x=None), dict(x=GOOD + 2), dict(ld_x=3), dict(kind=4), dict(rows=-1), dict(cols=0), dict(w=GOOD + 2), dict(wkind=-1), dict(mean=None),
                dict(rstd=GOOD + 2), dict(dx=None), dict(ld_dx=2), dict(dw=GOOD + 2), dict(db=GOOD + 1), dict(rows=1000, ws=None), dict(rows=1000, ws=GOOD + 4)):
        assert backward(**bad) == INVALID, bad
    assert backward(rows=1000, nbytes=size(1000, 4) - 1) == CAPACITY


def test_adamw_state_checks_its_tensors():
    p = [torch.zeros(40)]
    with pytest.raises(ValueError, match="CUDA"):
        api.AdamWState(p, [torch.zeros(40)], [torch.zeros(40)])
    with pytest.raises(ValueError, match="at least one"):
        api.AdamWState([], [], [])
    with pytest.raises(ValueError, match="both states"):
        api.AdamWState(p, p, p, exp_avg_scale=p)
    with pytest.raises(ValueError, match="per parameter"):
        api.AdamWState(p, [], p)
    with pytest.raises(ValueError, match="per parameter"):
        api.AdamWState(p, p, p, weight_decay=[0.0, 0.0])
    with pytest.raises(ValueError, match="not negative"):
        api.AdamWState(p, p, p, weight_decay=-1.0)
    with pytest.raises(ValueError, match="8 or 32"):
        api.AdamWState.zeros(p, bits=16)


def test_rows_of_a_tensor():
    x = torch.zeros(4, 5, 6)
    assert api._rows(x, 6, "x") == (20, 6)
    assert api._rows(x[:, :, :3], 3, "x") == (20, 6)
    assert api._rows(torch.zeros(6), 6, "x") == (1, 6)
    assert api._rows(x[:, 2], 6, "x") == (4, 30)
    assert api._rows(x[1:2, :, :2], 2, "x") == (5, 6)
    assert api._rows(torch.zeros(7, 1)[:, :1], 1, "x") == (7, 1)
    assert api._rows(torch.zeros(7, 3)[:, 1:2], 1, "x") == (7, 3)
    assert api._rows(torch.zeros(1, 9)[:, :4], 4, "x")[0] == 1
    for bad in (x[:, ::2, :3], x.transpose(0, 1), x[:, :, ::2], torch.zeros(1, 6).expand(3, 6), x.transpose(1, 2)):
        cols = bad.shape[-1]
        if bad is not x and bad.is_contiguous():
            continue
        with pytest.raises(ValueError):
            api._rows(bad, cols, "x")
    with pytest.raises(ValueError):
        api._rows(x, 5, "x")


def test_host_numbers_beyond_fp32(ctx):
    """Finite in 64 bits, Inf in the kernels' arithmetic."""
    lib, h = ctx
    step = lambda lr, eps, step=1, b1=0.9: lib.atomo_adamw(h, (api._AdamWTensor * 1)((GOOD, GOOD, GOOD, None, None, None, 0, 0.0, 0)), (ctypes.c_void_p * 1)(GOOD), 1,  # noqa: E731
                                                           ctypes.byref(api._AdamWArgs(lr, b1, 0.999, eps, step, 0, None, 32, 0)), None)
    assert step(1e39, 1e-8) == step(1e-3, 1e39) == step(1e38, 1e-8) == INVALID          # (1e38 / (1 - 0.9) is beyond it too)
    for s in (1e39, -1e300):
        assert lib.atomo_embedding(h, GOOD, 0, 8, 4, 4, GOOD, 8, 3, s, GOOD, 4, None, None) == INVALID
        assert lib.atomo_embedding_backward(h, GOOD, 8, 3, GOOD, 0, 4, 8, 4, s, -1, GOOD, 4, 0, None, GOOD, 1 << 30, None) == INVALID
    assert lib.atomo_layer_norm(h, GOOD, 0, 3, 4, 4, GOOD, GOOD, 0, 1e39, GOOD, 4, GOOD, GOOD, None) == INVALID


def test_layer_norm_workspace_of_long_rows(ctx):
    """Of rows that several CTAs read again, a partial sum of the weight's and the bias's gradient for each 32 rows: never a multiple of the operands."""
    lib, _ = ctx
    size = lib.atomo_layer_norm_workspace_bytes
    for rows, cols in ((1, 8193), (32, 1 << 20), (592, 1 << 22), (100000, 16384)):
        assert size(rows, cols) == min(-(-rows // 32), 592) * 2 * cols * 4
        assert size(rows, cols) <= max(rows // 16, 2) * cols * 4 + 8 * cols
