"""GPU: operands of more than 2^31 elements: what lies behind 32-bit offsets is read and written like the rest.  Compared on whole numbers, whose sums are exact, or
with the same rows in a call of their own."""
import pytest
import torch

pytestmark = pytest.mark.gpu

PAST = (1 << 31) + 4099          # elements


@pytest.fixture(scope="module")
def atomo():
    from paper_1806_04090_b200 import api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    a = api.Atomo(0)
    yield a
    a.close()
    torch.cuda.empty_cache()


@pytest.fixture(autouse=True)
def room():
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("60 GB of device memory are needed")
    yield
    torch.cuda.empty_cache()


def _noise(n, dtype, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    return torch.randint(-8, 9, (n,), generator=gen, device="cuda", dtype=torch.int8).to(dtype)


def test_norm(atomo):
    g = torch.zeros(PAST, dtype=torch.bfloat16, device="cuda")
    g[5], g[-3], g[1 << 31] = 3.0, 4.0, 12.0
    assert float(atomo.atomo_grad_norm([g])[0]) == 13.0
    # the sum 178 is exact; its root is rounded in 64 bits, then to fp32
    assert abs(float(atomo.atomo_grad_norm([g[1:], g[:7]])[0]) - 178.0 ** 0.5) <= 2.0 ** -20


@pytest.mark.parametrize("bits", [32, 8])
def test_adamw(atomo, bits):
    """The last elements are those of a short tensor with the same values (in 32 bits; in 8 the rounding's words differ, so that only their magnitude is held)."""
    from paper_1806_04090_b200 import api
    tail = 5000
    p, g = _noise(PAST, torch.bfloat16, 1), _noise(PAST, torch.bfloat16, 2)
    q, h = p[-tail:].clone(), g[-tail:].clone()
    first = p[:tail].clone()
    state, short = api.AdamWState.zeros([p], bits=bits), api.AdamWState.zeros([q], bits=bits)
    atomo.atomo_adamw(state, [g], lr=0.5, step=1, seed=3)
    atomo.atomo_adamw(short, [h], lr=0.5, step=1, seed=3)
    assert torch.equal(p[-tail:], q) and not torch.equal(p[:tail], first)
    for a, b in ((state.exp_avg[0], short.exp_avg[0]), (state.exp_avg_sq[0], short.exp_avg_sq[0])):
        a = a[-tail:]
        if bits == 32:
            assert torch.equal(a, b)
        else:
            assert bool(((a.float() != 0) | (h == 0)).all())
    if bits == 8:
        assert int(state.exp_avg_sq_scale[0].view(torch.uint8)[-1]) > 0


@pytest.mark.parametrize("cols", [2048, 2047])
def test_layer_norm(atomo, cols):
    rows, last = PAST // cols + 40, 50
    x, dy = _noise(rows * cols, torch.bfloat16, 4).view(rows, cols), _noise(rows * cols, torch.bfloat16, 5).view(rows, cols)
    w = _noise(cols, torch.float32, 6)
    y, mean, rstd = atomo.atomo_layer_norm(x, w)
    # (whole rows in a buffer that starts as the big one's last rows do, so that the same form takes them)
    shift = (rows - last) * cols % 8

    def cut(t):
        return torch.cat([torch.zeros(shift, dtype=t.dtype, device="cuda"), t[-last:].reshape(-1)])[shift:].view(last, cols)
    ys, means, rstds = atomo.atomo_layer_norm(cut(x), w)
    assert torch.equal(y[-last:], ys) and torch.equal(mean[-last:], means) and torch.equal(rstd[-last:], rstds)
    dx, _, _ = atomo.atomo_layer_norm_backward(dy, x, w, mean, rstd)
    dxs, _, _ = atomo.atomo_layer_norm_backward(cut(dy), cut(x), w, means, rstds)
    assert torch.equal(dx[-last:], dxs)
    del y, dx
    zeros, ones = torch.zeros(rows, device="cuda"), torch.ones(rows, device="cuda")
    dy *= torch.rand(rows, 1, device="cuda") < 0.2             # sums below 2^24
    _, dweight, dbias = atomo.atomo_layer_norm_backward(dy, x, None, zeros, ones)
    want_w, want_b = torch.zeros(cols, device="cuda"), torch.zeros(cols, device="cuda")
    for i in range(0, rows, 65536):
        want_w += (dy[i:i + 65536].float() * x[i:i + 65536].float()).sum(0)
        want_b += dy[i:i + 65536].float().sum(0)
    assert float(want_w.abs().max()) < 1 << 24 and torch.equal(dweight, want_w) and torch.equal(dbias, want_b)


@pytest.mark.parametrize("cols", [2048, 2047])
def test_embedding(atomo, cols):
    rows = PAST // cols + 40
    table = _noise(rows * cols, torch.bfloat16, 7).view(rows, cols)
    ids = torch.tensor([0, rows - 1, rows // 2, rows - 2, 1], device="cuda")
    assert torch.equal(atomo.atomo_embedding(table, ids), table[ids])
    many = torch.arange(rows, device="cuda").flip(0)
    out = atomo.atomo_embedding(table, many)
    assert torch.equal(out[:100], table[-100:].flip(0)) and torch.equal(out[-100:], table[:100].flip(0))
    del out
    # the gradient of a table past 2^31 elements (fp32), of few tokens and of many; then of as many token rows into a small table
    for ids in (torch.tensor([rows - 1, 3, rows - 1, rows // 2], device="cuda"), torch.cat([torch.arange(5000, device="cuda") % 7 + rows - 7, torch.tensor([0], device="cuda")])):
        grad = _noise(len(ids) * cols, torch.bfloat16, 8).view(len(ids), cols)
        got = atomo.atomo_embedding_backward(ids, grad, rows)
        where, at = ids.unique(return_inverse=True)
        want = torch.zeros(len(where), cols, device="cuda").index_add_(0, at, grad.float())
        assert torch.equal(got[where], want)
        got[where] = 0
        assert not bool(got.any())
        del got
    del grad
    small = torch.arange(rows, device="cuda") % 97
    got = atomo.atomo_embedding_backward(small, table, 97)
    want = torch.zeros(97, cols, device="cuda")
    for i in range(0, rows, 65536):
        want.index_add_(0, small[i:i + 65536], table[i:i + 65536].float())
    assert torch.equal(got, want)
