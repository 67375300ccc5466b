"""GPU: a training step from the tokens to the weights as it is used: embedding, layer norm and their gradients, both workers' gradients encoded,
the payloads averaged, norm and clipping, AdamW."""
import dataclasses
import os
import re
import threading

import numpy as np
import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu

ROWS, COLS, TOKENS = 120, 64, 500
SCALE = COLS ** 0.5


@pytest.fixture(scope="module")
def atomo():
    from paper_1806_04090_b200 import api
    assert torch.cuda.is_available(), "GPU tests need a CUDA device"
    a = api.Atomo(0)
    yield a
    a.close()


def _np(t):
    return t.double().cpu().numpy()


def _backward(atomo, table, weight, bias, ids, target):
    """Gradients of sum((layer_norm(embedding) - target)^2) / 2, in fp32."""
    x = atomo.atomo_embedding(table, ids, scale=SCALE)
    y, mean, rstd = atomo.atomo_layer_norm(x, weight, bias)
    dx, dweight, dbias = atomo.atomo_layer_norm_backward(y - target, x, weight, mean, rstd)
    return atomo.atomo_embedding_backward(ids, dx, ROWS, scale=SCALE), dweight, dbias


@pytest.mark.parametrize("spectral", [False, True])
@pytest.mark.parametrize("bits", [32, 8])
def test_step(atomo, spectral, bits):
    from paper_1806_04090_b200 import api
    gen = torch.Generator(device="cuda")
    gen.manual_seed(31)
    table = torch.randn(ROWS, COLS, generator=gen, device="cuda") * 0.3
    weight, bias = torch.ones(COLS, device="cuda"), torch.zeros(COLS, device="cuda")
    params = [table, weight, bias]
    old = [_np(p) for p in params]
    state = api.AdamWState.zeros(params, bits=bits, weight_decay=[0.1, 0.0, 0.0])
    payloads, small, wanted = [], [], []
    for worker in range(2):
        ids = torch.randint(0, ROWS, (TOKENS,), generator=gen, device="cuda")
        target = torch.randn(TOKENS, COLS, generator=gen, device="cuda")
        grads = _backward(atomo, table, weight, bias, ids, target)
        # against autograd in 64 bits; the chain's roundings are below 1e-5 of the gradients' sizes (500 terms of about eight roundings each: 4e-6)
        t, w, b = (p.double().requires_grad_(True) for p in params)
        h = t[ids] * SCALE
        h = (h - h.mean(1, keepdim=True)) / (h.var(1, keepdim=True, correction=0) + 1e-5).sqrt() * w + b
        exact = torch.autograd.grad(((h - target) ** 2).sum() / 2, (t, w, b))
        for g, e in zip(grads, exact):
            assert float((g.double() - e).abs().max()) <= 1e-5 * float(e.abs().max())
        # the table is encoded; a budget that keeps every atom makes the payload's decode the gradient
        if spectral:
            pay, _ = atomo.atomo_encode_spectral([grads[0]], float(COLS), seed=worker, step=1, k_cap=COLS)
        else:
            pay, _ = atomo.atomo_encode_entrywise([grads[0].view(-1)], float(ROWS * COLS), seed=worker, step=1, k_cap=ROWS * COLS)
        payloads.append(pay)
        small.append(grads[1:])
        wanted.append([_np(e) for e in exact])
    mean = [atomo.atomo_decode_average(payloads)[0]] + [(a + b) / 2 for a, b in zip(*small)]
    for m, a, b in zip(mean, *wanted):
        want = (a + b) / 2
        assert np.abs(_np(m).reshape(want.shape) - want).max() <= (2e-3 if spectral else 1e-5) * np.abs(want).max()   # spectral: vectors of an fp32 Gram matrix
    scale = atomo.atomo_grad_norm(mean, max_norm=1.0)
    norm = np.sqrt(sum((_np(m) ** 2).sum() for m in mean))
    assert norm > 1.0 and abs(float(scale[0]) / norm - 1) <= 18 * ref.U32 and abs(float(scale[1]) * (norm + 1e-6) - 1) <= 20 * ref.U32
    atomo.atomo_adamw(state, mean, lr=1e-2, step=1, seed=9, scale=scale)
    for p, g, before, decay in zip(params, mean, old, state.weight_decay):
        (want, _, _), (off, _, _) = ref.adamw(before.reshape(-1), _np(g).reshape(-1), np.zeros(g.numel()), np.zeros(g.numel()), 1e-2, 1, 0.9, 0.999, 1e-8, decay, float(scale[1]))
        ref.near(p, want.reshape(p.shape), off.reshape(p.shape))


def test_a_sparse_table_gradient_keeps_its_zero_rows_through_the_exchange(atomo):
    """Rows without tokens are exact zeros, so no atom of theirs is ever kept."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(32)
    ids = torch.randint(0, ROWS // 4, (TOKENS,), generator=gen, device="cuda") * 4
    grad = atomo.atomo_embedding_backward(ids, torch.randn(TOKENS, COLS, generator=gen, device="cuda"), ROWS)
    for s in (50.0, 1000.0):
        pay, _ = atomo.atomo_encode_entrywise([grad.view(-1)], s, seed=3, step=2)
        out = atomo.atomo_decode(pay)[0].view(ROWS, COLS)
        assert atomo.payload_status(pay)[0] == 0 and bool((out[grad == 0] == 0).all()) and int((out != 0).sum()) > 0


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("rows,cols,tokens,dtype", [(ROWS, COLS, TOKENS, torch.float32), (700, 520, 6000, torch.bfloat16), (90, 33, 2500, torch.float16)])
def test_step_as_a_captured_graph(atomo, rows, cols, tokens, dtype, bits):
    """Forward, backward and update of one worker in one graph: replayed on two batches, bit for bit what the calls give one by one."""
    from paper_1806_04090_b200 import api
    gen = torch.Generator(device="cuda")
    gen.manual_seed(33)
    start = [torch.randn(rows, cols, generator=gen, device="cuda").to(dtype), torch.ones(cols, device="cuda").to(dtype), torch.zeros(cols, device="cuda").to(dtype)]
    batches = [(torch.randint(0, rows, (tokens,), generator=gen, device="cuda"), torch.randn(tokens, cols, generator=gen, device="cuda").to(dtype)) for _ in range(2)]

    def step(params, state, ids, dy):
        x = atomo.atomo_embedding(params[0], ids, scale=0.5)
        y, mean, rstd = atomo.atomo_layer_norm(x, params[1], params[2])
        dx, dweight, dbias = atomo.atomo_layer_norm_backward(dy, x, params[1], mean, rstd)
        grads = [atomo.atomo_embedding_backward(ids, dx, rows, scale=0.5), dweight, dbias]
        atomo.atomo_adamw(state, grads, lr=1e-2, step=3, seed=4, scale=atomo.atomo_grad_norm(grads, max_norm=1.0))

    def run():
        params = [p.clone() for p in start]
        return params, api.AdamWState.zeros(params, bits=bits, master=dtype != torch.float32)

    eager, eager_state = run()
    for ids, dy in batches:
        step(eager, eager_state, ids, dy)
    params, state = run()
    ids, dy = batches[0][0].clone(), batches[0][1].clone()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step(params, state, ids, dy)
    for batch in batches:
        ids.copy_(batch[0]); dy.copy_(batch[1])
        graph.replay()
    torch.cuda.synchronize()
    for a, b in zip(eager + eager_state.exp_avg + eager_state.exp_avg_sq, params + state.exp_avg + state.exp_avg_sq):
        assert torch.equal(a.view(torch.uint8), b.view(torch.uint8))


def _readme_step():
    """The lines of the README that show a step."""
    with open(os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "README.md")) as f:
        blocks = re.findall(r"```python\n(.*?)```", f.read(), re.S)
    found = [b for b in blocks if "atomo_adamw" in b]
    assert len(found) == 1
    return found[0]


def test_workers_that_step_as_the_readme_says_stay_alike():
    """Two workers, a thread each, on batches of their own: after every step their weights and states are the same bit for bit, and the vectors' gradients the
    mean of both.  (Nothing on the GPU waits for the other worker: the threads meet on the host, between calls.)"""
    from paper_1806_04090_b200 import api
    code = compile(_readme_step(), "README.md", "exec")
    steps, meet = 3, threading.Barrier(2, timeout=120)
    slots, own, results, errors = [None, None], [None, None], [None, None], []

    class Exchange:
        def __init__(self, rank):
            self.rank = rank

        def all_gather_bytes(self, buf):
            torch.cuda.synchronize()
            slots[self.rank] = buf
            meet.wait()
            both = list(slots)
            meet.wait()
            return both

    def worker(rank):
        try:
            ctx = api.Atomo(0)
            gen = torch.Generator(device="cuda")
            gen.manual_seed(71)
            params = [torch.randn(ROWS, COLS, generator=gen, device="cuda") * 0.3, torch.ones(COLS, device="cuda"), torch.zeros(COLS, device="cuda")]
            state = api.AdamWState.zeros(params, bits=8)
            gen.manual_seed(72 + rank)
            after = []
            for step in range(1, steps + 1):
                ids = torch.randint(0, ROWS, (TOKENS,), generator=gen, device="cuda")
                dy = torch.randn(TOKENS, COLS, generator=gen, device="cuda")
                x = ctx.atomo_embedding(params[0], ids)
                _, mean, rstd = ctx.atomo_layer_norm(x, params[1], params[2])
                own[rank] = ctx.atomo_layer_norm_backward(dy, x, params[1], mean, rstd)[1:]
                names = dict(atomo=ctx, dataclasses=dataclasses, dist=Exchange(rank), table=params[0], weight=params[1], bias=params[2], ids=ids, dy=dy, state=state, rank=rank, step=step)
                exec(code, names)
                torch.cuda.synchronize()
                meet.wait()
                for got, a, b in zip((names["dweight"], names["dbias"]), *own):
                    want = (a.double() + b.double()) / 2
                    # a kept atom is rescaled by 1 / p, p = 1 or the next number to it; the mean's sum and quotient round once each
                    assert bool(((got.double() - want).abs() <= 4 * ref.U32 * (a.abs() + b.abs()).double()).all())
                meet.wait()
                after.append([t.view(torch.uint8).clone() for t in params + state.exp_avg + state.exp_avg_sq + state.exp_avg_scale + state.exp_avg_sq_scale])
            results[rank] = after
            torch.cuda.synchronize()
            ctx.close()
        except BaseException as e:                       # noqa: B036  (told by the test's own thread)
            errors.append(e)
            meet.abort()

    threads = [threading.Thread(target=worker, args=(r,)) for r in range(2)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    if errors:
        raise errors[0]
    for a, b in zip(*results):
        assert all(torch.equal(x, y) for x, y in zip(a, b))
    assert not torch.equal(results[0][0][0], results[0][-1][0])
