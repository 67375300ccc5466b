"""GPU: the operators around the exchange beside autograd: they record no graph, and refuse to end one without a word; as an autograd Function they have one."""
import pytest
import torch

pytestmark = pytest.mark.gpu

ROWS, COLS, TOKENS = 50, 96, 300


@pytest.fixture(scope="module")
def atomo():
    from paper_1806_04090_b200 import api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    a = api.Atomo(0)
    yield a
    a.close()


@pytest.fixture
def data():
    gen = torch.Generator(device="cuda")
    gen.manual_seed(51)
    rand = lambda *s: torch.randn(*s, generator=gen, device="cuda")  # noqa: E731
    return {"table": rand(ROWS, COLS), "weight": rand(COLS), "bias": rand(COLS), "ids": torch.randint(0, ROWS, (TOKENS,), generator=gen, device="cuda"), "dy": rand(TOKENS, COLS)}


def _calls(atomo, d):
    """Each call, and the tensors of it that may require a gradient."""
    x = d["table"][d["ids"]]
    _, mean, rstd = atomo.atomo_layer_norm(x, d["weight"], d["bias"])
    return [(lambda table, out: atomo.atomo_embedding(table, d["ids"], out=out), [d["table"], torch.empty_like(x)]),
            (lambda grad, out: atomo.atomo_embedding_backward(d["ids"], grad, ROWS, out=out), [d["dy"], torch.empty_like(d["table"])]),
            (lambda x, w, b, out: atomo.atomo_layer_norm(x, w, b, out=out), [x, d["weight"], d["bias"], torch.empty_like(x)]),
            (lambda dy, x, w, out: atomo.atomo_layer_norm_backward(dy, x, w, mean, rstd, out=out), [d["dy"], x, d["weight"], torch.empty_like(x)])]


def test_no_gradient_is_cut_without_a_word(atomo, data):
    side = torch.cuda.Stream()
    for call, tensors in _calls(atomo, data):
        call(*tensors)
        for i in range(len(tensors)):
            leaf = [t.clone().requires_grad_(i == k) for k, t in enumerate(tensors)]
            with pytest.raises(RuntimeError, match="no autograd graph"):
                call(*leaf)
            inner = [t * 1.0 if t.requires_grad else t for t in leaf]
            with pytest.raises(RuntimeError, match="no autograd graph"):
                call(*inner)
            with torch.no_grad():
                call(*leaf)
            with torch.inference_mode():
                call(*leaf)
    with pytest.raises(RuntimeError, match="no autograd graph"):
        atomo.atomo_embedding(data["table"].clone().requires_grad_(True), data["ids"], stream=side)


def test_inside_an_autograd_function(atomo, data):
    class Embedding(torch.autograd.Function):
        @staticmethod
        def forward(ctx, table, ids):
            ctx.save_for_backward(ids)
            return atomo.atomo_embedding(table, ids, scale=0.5)

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dout):
            return atomo.atomo_embedding_backward(ctx.saved_tensors[0], dout, ROWS, scale=0.5), None

    class LayerNorm(torch.autograd.Function):
        @staticmethod
        def forward(ctx, x, weight, bias):
            y, mean, rstd = atomo.atomo_layer_norm(x, weight, bias)
            ctx.save_for_backward(x, weight, mean, rstd)
            return y

        @staticmethod
        @torch.autograd.function.once_differentiable
        def backward(ctx, dy):
            return atomo.atomo_layer_norm_backward(dy, *ctx.saved_tensors)

    leaves = [data[k].clone().requires_grad_(True) for k in ("table", "weight", "bias")]
    y = LayerNorm.apply(Embedding.apply(leaves[0], data["ids"]), leaves[1], leaves[2])
    got = torch.autograd.grad(y, leaves, data["dy"])
    t, w, b = (data[k].double().requires_grad_(True) for k in ("table", "weight", "bias"))
    x = t[data["ids"]] * 0.5
    rstd = 1 / (x.var(1, keepdim=True, correction=0) + 1e-5).sqrt()
    hat = (x - x.mean(1, keepdim=True)) * rstd
    exact = torch.autograd.grad(hat * w + b, (t, w, b), data["dy"].double())
    # the magnitudes of all that is added up; each sum has at most 300 terms, each term at most 20 roundings (those of mean and rstd among them)
    with torch.no_grad():
        dy = data["dy"].double().abs()
        u, hat = dy * w.abs(), hat.abs()
        dx = rstd * (u + u.mean(1, keepdim=True) + hat * (u * hat).mean(1, keepdim=True))
        sizes = [torch.zeros_like(t).index_add_(0, data["ids"], dx * 0.5), (dy * hat).sum(0), dy.sum(0)]
    for g, e, size in zip(got, exact, sizes):
        assert bool(((g.double() - e).abs() <= 320 * 2.0 ** -24 * size).all())


def test_what_a_call_writes_counts_as_changed(atomo, data):
    """A tensor that autograd has saved and a call has written over is found out by the backward pass."""
    from paper_1806_04090_b200 import api
    p = data["table"].clone().requires_grad_(True)
    state = api.AdamWState.zeros([p], bits=8)
    loss = (p * p).sum()
    atomo.atomo_adamw(state, [torch.ones_like(p)], lr=0.1, step=1)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    for call, tensors in _calls(atomo, data):
        out = tensors[-1]
        w = torch.ones_like(out).requires_grad_(True)
        loss = (w * out).sum()
        call(*tensors)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
    out = torch.zeros(2, device="cuda")
    w = torch.ones(2, device="cuda", requires_grad=True)
    loss = (w * out).sum()
    atomo.atomo_grad_norm([data["dy"]], out=out)
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        loss.backward()
    with torch.inference_mode():                         # tensors without a version
        q = torch.zeros(64, device="cuda")
        atomo.atomo_adamw(api.AdamWState.zeros([q]), [torch.ones(64, device="cuda")], lr=0.1, step=1)
        assert float(q.max()) < 0.0
