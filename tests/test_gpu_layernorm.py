"""GPU: layer norm and its backward pass, against 64 bits."""
import numpy as np
import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def atomo():
    from paper_1806_04090_b200 import api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    a = api.Atomo(0)
    yield a
    a.close()


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _np(t):
    return t.double().cpu().numpy()


def _input(rows, cols, dtype, gen):
    x = torch.randn(rows, cols, generator=gen, device="cuda") * 2.0
    x[:, ::13] *= 6.0
    x += torch.randn(rows, 1, generator=gen, device="cuda") * 3.0
    return x.to(dtype)


def _check(atomo, x, dy, weight, bias, eps=1e-5):
    """Both passes of tensors that are seen as matrices."""
    cols = x.shape[-1]
    y, mean, rstd = atomo.atomo_layer_norm(x, weight, bias, eps=eps)
    assert y.shape == x.shape and y.dtype == x.dtype and mean.shape == rstd.shape == x.shape[:-1]
    w = np.ones(cols) if weight is None else _np(weight)
    b = np.zeros(cols) if bias is None else _np(bias)
    xs, dys = _np(x).reshape(-1, cols), _np(dy).reshape(-1, cols)
    (wy, wm, wr), (oy, om, orr) = ref.layer_norm(xs, w, b, eps)
    ref.near(mean, wm, om)
    ref.near(rstd, wr, orr)
    ref.near(y, wy, ref.rounded(oy, wy, x.dtype))
    dx, dw, db = atomo.atomo_layer_norm_backward(dy, x, weight, mean, rstd)
    assert dx.shape == x.shape and dx.dtype == x.dtype and dw.dtype == db.dtype == torch.float32
    (wx, ww, wb), (ox, ow, ob) = ref.layer_norm_backward(dys, xs, w, _np(mean).reshape(-1), _np(rstd).reshape(-1))
    ref.near(dx, wx, ref.rounded(ox, wx, x.dtype))
    ref.near(dw, ww, ow)
    ref.near(db, wb, ob)


COLS = [1, 2, 7, 16, 33, 64, 127, 128, 256, 257, 511, 512, 513, 1000, 1023, 1024, 2047, 2048, 2056, 4096, 4100, 8191, 8192, 8193, 10000, 16384]


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("cols", COLS)
def test_widths(atomo, dtype, cols):
    gen = _gen(1)
    for rows in (1, 5, 37):
        x, dy = _input(rows, cols, dtype, gen), torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
        weight, bias = torch.randn(cols, generator=gen, device="cuda") + 1.0, torch.randn(cols, generator=gen, device="cuda")
        if rows == 5:
            weight, bias = weight.to(dtype), bias.to(dtype)
        _check(atomo, x, dy, weight, bias)


@pytest.mark.parametrize("rows", [0, 1, 2, 15, 16, 17, 300, 1184, 1185, 2369, 5000, 40000])
@pytest.mark.parametrize("cols,dtype", [(48, torch.bfloat16), (260, torch.float32), (770, torch.float16)])
def test_heights(atomo, rows, cols, dtype):
    gen = _gen(2)
    x, dy = _input(rows, cols, dtype, gen), torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    if rows == 0:
        y, mean, rstd = atomo.atomo_layer_norm(x)
        dx, dw, db = atomo.atomo_layer_norm_backward(dy, x, None, mean, rstd)
        assert y.shape == dx.shape == (0, cols) and mean.shape == (0,) and bool((dw == 0).all()) and bool((db == 0).all())
        return
    _check(atomo, x, dy, torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda"))


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("cols,limit", [(3, 256), (128, 256), (129, 64), (512, 64), (513, 32), (1023, 32), (1536, 16), (2048, 16), (4095, 8), (8192, 8)])
def test_rows_that_one_launch_takes(atomo, cols, limit, dtype):
    """Up to `limit` rows the weight's gradient is added inside one launch, without a workspace; a result that is not asked for is left out."""
    size = atomo.lib.atomo_layer_norm_workspace_bytes
    assert size(limit, cols) == 0 and size(limit + 1, cols) > 0
    gen = _gen(6)
    w = torch.randn(cols, generator=gen, device="cuda")
    for rows in (limit // 8, limit // 2 + 1, limit, limit + 1):
        x, dy = _input(rows, cols, dtype, gen), torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
        _check(atomo, x, dy, w, w)
    x, dy = x[:limit], dy[:limit]
    _, mean, rstd = atomo.atomo_layer_norm(x, w, w)
    dx, dw, db = atomo.atomo_layer_norm_backward(dy, x, w, mean, rstd)
    kind = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}[dtype]
    for want_w in (True, False):
        got, room = torch.empty_like(dx), torch.full((2, cols), 7.0, device="cuda")
        args = (dy.data_ptr(), cols, x.data_ptr(), cols, kind, limit, cols, w.data_ptr(), 0, mean.data_ptr(), rstd.data_ptr(), got.data_ptr(), cols)
        assert atomo.lib.atomo_layer_norm_backward(atomo._h, *args, room[0].data_ptr() if want_w else None, None if want_w else room[1].data_ptr(), None, 0, None) == 0
        torch.cuda.synchronize()
        assert torch.equal(got, dx) and torch.equal(room[0], dw if want_w else torch.full_like(dw, 7.0)) and torch.equal(room[1], torch.full_like(db, 7.0) if want_w else db)


def test_without_weight_or_bias(atomo):
    gen = _gen(3)
    for cols in (40, 3000, 9000):
        x, dy = _input(9, cols, torch.float32, gen), torch.randn(9, cols, generator=gen, device="cuda")
        w = torch.randn(cols, generator=gen, device="cuda")
        _check(atomo, x, dy, None, None)
        _check(atomo, x, dy, w, None)
        _check(atomo, x, dy, None, w)


@pytest.mark.parametrize("dtype", ref.TYPES)
def test_strided_and_unaligned_rows(atomo, dtype):
    gen = _gen(4)
    big, grad = _input(30, 1300, dtype, gen), torch.randn(30, 1300, generator=gen, device="cuda").to(dtype)
    w = torch.randn(1300, generator=gen, device="cuda")
    for c0, c1 in ((0, 1024), (1, 1025), (8, 264), (3, 40), (16, 1300)):
        _check(atomo, big[:, c0:c1], grad[:, c0:c1], w[c0:c1].clone(), w[c0:c1].clone())
        _check(atomo, big[::3, c0:c1], grad[:10, c0:c1], w[c0:c1].clone(), None)
    _check(atomo, big.view(5, 6, 1300), grad.view(5, 6, 1300), w, w)
    _check(atomo, big.view(5, 6, 1300)[:, 2], grad.view(5, 6, 1300)[:, 3], w, w)
    # the results in rows of a larger matrix, whose other columns stay
    room = torch.full((30, 1300), 5.0, device="cuda", dtype=dtype)
    y, mean, rstd = atomo.atomo_layer_norm(big[:, 8:520], w[:512].clone(), None)
    got, _, _ = atomo.atomo_layer_norm(big[:, 8:520], w[:512].clone(), None, out=room[:, 16:528])
    assert torch.equal(got, y)
    dx, _, _ = atomo.atomo_layer_norm_backward(grad[:, 8:520], big[:, 8:520], w[:512].clone(), mean, rstd)
    got, _, _ = atomo.atomo_layer_norm_backward(grad[:, 8:520], big[:, 8:520], w[:512].clone(), mean, rstd, out=room[:, 16:528])
    assert torch.equal(got, dx)
    room[:, 16:528] = 5.0
    assert bool((room == 5.0).all())


@pytest.mark.parametrize("cols", [96, 1001, 2048, 12000])
def test_in_place(atomo, cols):
    gen = _gen(5)
    x, dy = _input(50, cols, torch.bfloat16, gen), torch.randn(50, cols, generator=gen, device="cuda").bfloat16()
    w = torch.randn(cols, generator=gen, device="cuda")
    y, mean, rstd = atomo.atomo_layer_norm(x, w, w)
    dx, dw, db = atomo.atomo_layer_norm_backward(dy, x, w, mean, rstd)
    for over in ("dy", "x"):
        a, b = dy.clone(), x.clone()
        got = atomo.atomo_layer_norm_backward(a, b, w, mean, rstd, out=a if over == "dy" else b)
        assert all(torch.equal(p, q) for p, q in zip(got, (dx, dw, db)))
    z = x.clone()
    got = atomo.atomo_layer_norm(z, w, w, out=z)
    assert all(torch.equal(p, q) for p, q in zip(got, (y, mean, rstd))) and torch.equal(z, y)


def test_rows_that_do_not_vary(atomo):
    x = torch.full((4, 300), 3.0, device="cuda")
    x[1] = 0.0
    w, b = torch.randn(300, device="cuda", generator=_gen(6)), torch.randn(300, device="cuda", generator=_gen(7))
    y, mean, rstd = atomo.atomo_layer_norm(x, w, b, eps=1e-5)
    assert torch.equal(y, b.expand(4, 300)) and mean.tolist() == [3.0, 0.0, 3.0, 3.0]
    # 1 / sqrt(eps): eps in fp32, the root and the quotient round once each
    assert np.all(np.abs(_np(rstd) - 1e-5 ** -0.5) <= 4 * ref.U32 * 1e-5 ** -0.5)


def test_values_that_are_not_finite_stay_in_their_rows(atomo):
    gen = _gen(8)
    for cols in (100, 2048, 9000):
        x = _input(40, cols, torch.float32, gen)
        clean, _, _ = atomo.atomo_layer_norm(x)
        x[7, 3], x[21, 50] = float("nan"), float("inf")
        y, _, _ = atomo.atomo_layer_norm(x)
        rest = [i for i in range(40) if i not in (7, 21)]
        assert torch.equal(y[rest], clean[rest]) and bool(torch.isnan(y[7]).all()) and bool(torch.isnan(y[21]).all())


def test_a_large_offset_costs_no_precision(atomo):
    """Variance from centred values: an offset far above the deviation leaves what fp32 has of the deviations themselves."""
    x = torch.randn(20, 1024, generator=_gen(9), device="cuda") + 4096.0
    _check(atomo, x, torch.ones(20, 1024, device="cuda"), None, None)


def test_gradient_against_differences(atomo):
    """<dx, d> against the central difference of <dy, y(x + h d)> in 64 bits.  Its error is h^2 / 6 of the third derivative: y is smooth on the
    scale of a row's deviation (about 2 here), so with |d| <= 5 and h = 1e-4 it is below 1e-6 of the sum of sizes; the rest are the kernel's roundings."""
    gen = _gen(10)
    rows, cols = 12, 200
    x, dy = _input(rows, cols, torch.float32, gen), torch.randn(rows, cols, generator=gen, device="cuda")
    w, b = torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    _, mean, rstd = atomo.atomo_layer_norm(x, w, b)
    dx, dw, db = atomo.atomo_layer_norm_backward(dy, x, w, mean, rstd)
    X, DY, W, B = _np(x), _np(dy), _np(w), _np(b)
    rng = np.random.default_rng(1)
    h = 1e-4

    def loss(x, w, b):
        return float((DY * ref.layer_norm(x, w, b, 1e-5)[0][0]).sum())

    (_, _, _), (ox, ow, ob) = ref.layer_norm_backward(DY, X, W, _np(mean), _np(rstd))
    for _ in range(3):
        d = rng.standard_normal((rows, cols)).clip(-5, 5)
        slope = (loss(X + h * d, W, B) - loss(X - h * d, W, B)) / (2 * h)
        # the statistics are fp32 roundings of those in 64 bits: dx moves by as much, relatively
        allowed = float((np.abs(d) * (ox + 8 * ref.U32 * np.abs(_np(dx)))).sum()) + 1e-6 * float(np.abs(_np(dx) * d).sum())
        assert abs(float((_np(dx) * d).sum()) - slope) <= allowed
        e = rng.standard_normal(cols)
        for got, off, at in ((dw, ow, (X, W + h * e, B)), (db, ob, (X, W, B + h * e))):
            back = (X, W - h * e, B) if at[1] is not W else (X, W, B - h * e)
            slope = (loss(*at) - loss(*back)) / (2 * h)
            allowed = float((np.abs(e) * (off + 8 * ref.U32 * np.abs(_np(got)))).sum()) + 1e-6 * float(np.abs(_np(got) * e).sum())
            assert abs(float((_np(got) * e).sum()) - slope) <= allowed


def test_repeats_bit_for_bit_on_streams_and_in_graphs(atomo):
    gen = _gen(11)
    x, dy = _input(3000, 300, torch.bfloat16, gen), torch.randn(3000, 300, generator=gen, device="cuda").bfloat16()
    w, b = torch.randn(300, generator=gen, device="cuda"), torch.randn(300, generator=gen, device="cuda")

    def both(stream=None):
        y, mean, rstd = atomo.atomo_layer_norm(x, w, b, stream=stream)
        return (y, mean, rstd, *atomo.atomo_layer_norm_backward(dy, x, w, mean, rstd, stream=stream))

    want = both()
    torch.cuda.synchronize()
    graphs = []
    for _ in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = both()
        graphs.append((g, out, torch.cuda.Stream()))
    for _ in range(3):
        for g, _, stream in graphs:
            with torch.cuda.stream(stream):
                g.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = both(side)
    side.synchronize()
    for out in [got] + [o for _, o, _ in graphs]:
        assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_refused_tensors(atomo):
    x = torch.zeros(6, 8, device="cuda")
    w = torch.ones(8, device="cuda")
    for bad in (dict(x=x.cpu()), dict(x=x.double()), dict(x=x.t()), dict(x=torch.zeros(6, 16, device="cuda")[:, ::2]), dict(weight=torch.ones(7, device="cuda")), dict(weight=w.cpu()),
                dict(bias=torch.ones(16, device="cuda")[::2]), dict(weight=w, bias=w.half()), dict(out=torch.zeros(5, 8, device="cuda")), dict(out=x.half())):
        with pytest.raises(ValueError):
            atomo.atomo_layer_norm(**{"x": x, **bad})
    from paper_1806_04090_b200 import api
    with pytest.raises(api.AtomoError):
        atomo.atomo_layer_norm(x, eps=-1.0)
    with pytest.raises(api.AtomoError):
        atomo.atomo_layer_norm(torch.zeros(3, 0, device="cuda"))
    s = torch.zeros(6, device="cuda")
    for bad in (dict(dy=x[:5]), dict(dy=x.half()), dict(mean=s[:5]), dict(rstd=s.half()), dict(rstd=torch.zeros(12, device="cuda")[::2]), dict(weight=torch.ones(9, device="cuda"))):
        with pytest.raises(ValueError):
            atomo.atomo_layer_norm_backward(**{"dy": x, "x": x, "weight": w, "mean": s, "rstd": s, **bad})


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (5, 64), (9, 1023), (40, 2048), (3, 8192), (2, 8200), (4, 16384)])
def test_rows_without_variance_and_no_eps(atomo, rows, cols, dtype):
    """rstd is 1 / sqrt(0), and y a zero times that; the rows beside are as they are alone."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(41)
    x = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype) if cols > 1 else torch.zeros(rows, cols, device="cuda", dtype=dtype)
    want = atomo.atomo_layer_norm(x, eps=0.0)
    x[rows // 2] = 3.0 if cols & (cols - 1) == 0 else 0.0          # (sums of which the mean is exact)
    y, mean, rstd = atomo.atomo_layer_norm(x, eps=0.0)
    assert float(rstd[rows // 2]) == float("inf") and float(mean[rows // 2]) == float(x[rows // 2, 0]) and bool(y[rows // 2].isnan().all())
    others = torch.arange(rows, device="cuda") != rows // 2
    for a, b in zip((y, mean, rstd), want):
        assert torch.equal(a[others], b[others])


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 96), (31, 1023), (64, 4096), (333, 770), (9, 8192), (40000, 48), (40000, 260), (5000, 1023), (700, 8200), (33, 16385)])
def test_sums_over_rows_of_whole_numbers(atomo, rows, cols, dtype):
    """With a mean of 0 and an rstd of 1, dweight and dbias are sums of whole numbers below 2^24, exact in fp32 in whatever order: not one row may be lost."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(42)
    x, dy = (torch.randint(-8, 9, (rows, cols), generator=gen, device="cuda") for _ in range(2))
    zeros, ones = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    _, dweight, dbias = atomo.atomo_layer_norm_backward(dy.to(dtype), x.to(dtype), torch.ones(cols, device="cuda"), zeros, ones)
    assert int((dy * x).sum(0).abs().max()) < 1 << 24
    assert torch.equal(dweight, (dy * x).sum(0).float()) and torch.equal(dbias, dy.sum(0).float())
