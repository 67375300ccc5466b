"""GPU: embedding lookup with scaling, and the gradient of the table by sorted tokens, against 64 bits."""
import math

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


def _ids(kind, n, rows, gen):
    if kind == "same":
        return torch.full((n,), rows - 1, device="cuda", dtype=torch.int64)
    if kind == "ascending":
        return torch.arange(n, device="cuda") % rows
    if kind == "few":                                   # long runs beside single tokens
        x = torch.randint(0, rows, (n,), generator=gen, device="cuda")
        x[torch.rand(n, generator=gen, device="cuda") < 0.6] = rows // 2
        x[torch.rand(n, generator=gen, device="cuda") < 0.2] = 0
        return x
    return torch.randint(0, rows, (n,), generator=gen, device="cuda")


def _want(ids, grad, rows, scale, padding=-1):
    """(sum, how far fp32 sums may be off): each addition rounds once, the scale once."""
    ids, g = ids.cpu().numpy().reshape(-1), grad.double().cpu().numpy()
    g = g.reshape(-1, g.shape[-1])
    want, size, count = np.zeros((rows, g.shape[1])), np.zeros((rows, g.shape[1])), np.zeros(rows)
    ok = (ids >= 0) & (ids < rows) & (ids != padding)
    np.add.at(want, ids[ok], g[ok]); np.add.at(size, ids[ok], np.abs(g[ok])); np.add.at(count, ids[ok], 1)
    return want * scale, (count[:, None] + 3) * ref.U32 * size * abs(scale)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,cols,n", [(1, 1, 1), (7, 3, 5), (100, 16, 33), (33, 515, 70), (50, 1024, 1), (9, 98, 1000), (20, 4097, 6), (300, 40, 0), (5, 2048, 70001)])
def test_lookup(atomo, dtype, rows, cols, n):
    gen = _gen(1)
    table = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    for id_type in (torch.int64, torch.int32):
        ids = torch.randint(0, rows, (n,), generator=gen, device="cuda").to(id_type)
        out = atomo.atomo_embedding(table, ids, scale=1.7)
        # one product, rounded to fp32 and then to the type
        assert torch.equal(out, (table[ids.long()].float() * torch.tensor(1.7, device="cuda")).to(dtype))
        assert torch.equal(atomo.atomo_embedding(table, ids), table[ids.long()])


def test_lookup_shapes_strides_and_views(atomo):
    gen = _gen(2)
    flat = torch.randn(50, 200, generator=gen, device="cuda").bfloat16()
    ids = torch.randint(0, 50, (3, 4, 5), generator=gen, device="cuda")
    for c0, c1 in ((0, 64), (1, 65), (2, 100), (8, 136), (0, 1)):
        table = flat[:, c0:c1]
        assert torch.equal(atomo.atomo_embedding(table, ids), table[ids])
        room = torch.full((60, 200), 9.0, device="cuda", dtype=torch.bfloat16)
        out = atomo.atomo_embedding(table, ids.view(-1), out=room[:, c0:c1])
        assert torch.equal(out, table[ids.view(-1)])
        room[:, c0:c1] = 9.0
        assert bool((room == 9.0).all())


def test_lookup_of_ids_without_a_row(atomo):
    table = torch.ones(10, 24, device="cuda")
    for bad in (-1, 10, 2 ** 31 - 1, -2 ** 31, 2 ** 32, 2 ** 32 + 3, -2 ** 63):
        ids = torch.tensor([3, bad, 4], device="cuda", dtype=torch.int64 if abs(bad) >= 2 ** 31 else torch.int32)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        out = atomo.atomo_embedding(table, ids, status=status)
        assert out.sum(1).tolist() == [24.0, 0.0, 24.0] and int(status) == 1
        status.zero_()
        grad = atomo.atomo_embedding_backward(ids, torch.ones(3, 24, device="cuda"), 10, status=status)
        assert grad.sum(1).tolist() == [0, 0, 0, 24, 24, 0, 0, 0, 0, 0] and int(status) == 1
        status.zero_()
        atomo.atomo_embedding(table, ids[::2].contiguous(), status=status)
        atomo.atomo_embedding_backward(ids[::2].contiguous(), torch.ones(2, 24, device="cuda"), 10, status=status)
        assert int(status) == 0


@pytest.mark.parametrize("kind", ["same", "ascending", "few", "random"])
@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 64, 65, 1000, 1024, 1025, 9001, 66000])
def test_gradient_lengths(atomo, kind, n):
    gen = _gen(3)
    for rows, cols, dtype in ((257, 20, torch.float32), (40, 33, torch.bfloat16)):
        ids = _ids(kind, n, rows, gen)
        grad = torch.randn(n, cols, generator=gen, device="cuda").to(dtype)
        want, off = _want(ids, grad, rows, 0.5)
        ref.near(atomo.atomo_embedding_backward(ids, grad, rows, scale=0.5), want, off)


@pytest.mark.parametrize("rows", [1, 2, 255, 256, 65535, 65536, 70001])
def test_gradient_table_sizes(atomo, rows):
    """Among them the largest numbers of a number of bits."""
    gen = _gen(4)
    ids = _ids("random", 3000, rows, gen)
    ids[::7] = rows - 1
    grad = torch.randn(3000, 8, generator=gen, device="cuda")
    want, off = _want(ids, grad, rows, 1.0)
    ref.near(atomo.atomo_embedding_backward(ids.int(), grad, rows), want, off)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("cols", [1, 2, 7, 98, 128, 515, 1023, 1025, 2048, 4104])
def test_gradient_widths(atomo, dtype, cols):
    gen = _gen(5)
    ids = _ids("few", 300, 19, gen)
    grad = torch.randn(300, cols, generator=gen, device="cuda").to(dtype)
    want, off = _want(ids, grad, 19, -3.0)
    ref.near(atomo.atomo_embedding_backward(ids, grad, 19, scale=-3.0), want, off)


def test_gradient_of_no_tokens(atomo):
    ids = torch.zeros(0, dtype=torch.int64, device="cuda")
    grad = torch.zeros(0, 12, device="cuda")
    assert bool((atomo.atomo_embedding_backward(ids, grad, 100) == 0).all())
    kept = torch.ones(100, 12, device="cuda")
    atomo.atomo_embedding_backward(ids, grad, 100, out=kept, accumulate=True)
    assert bool((kept == 1).all())
    # all of them padding, or without a row
    ids = torch.full((70,), 3, device="cuda")
    assert bool((atomo.atomo_embedding_backward(ids, torch.ones(70, 12, device="cuda"), 100, padding_idx=3) == 0).all())
    assert bool((atomo.atomo_embedding_backward(ids + 97, torch.ones(70, 12, device="cuda"), 100) == 0).all())


def test_gradient_padding(atomo):
    gen = _gen(6)
    ids = _ids("few", 2000, 50, gen)
    ids[5] = 50
    grad = torch.randn(2000, 36, generator=gen, device="cuda")
    for padding in (0, 25, 49):
        want, off = _want(ids, grad, 50, 2.0, padding)
        got = atomo.atomo_embedding_backward(ids, grad, 50, scale=2.0, padding_idx=padding)
        ref.near(got, want, off)
        assert bool((got[padding] == 0).all())


def test_gradient_accumulates_in_strided_rows(atomo):
    gen = _gen(7)
    room = torch.randn(60, 300, generator=gen, device="cuda")
    wide = torch.randn(900, 300, generator=gen, device="cuda").half()
    ids = _ids("few", 900, 60, gen)
    for c0, c1 in ((0, 256), (1, 130), (4, 100)):
        old = room.clone()
        want, off = _want(ids, wide[:, c0:c1], 60, 1.5)
        before = old[:, c0:c1].double().cpu().numpy()
        atomo.atomo_embedding_backward(ids, wide[:, c0:c1], 60, scale=1.5, out=room[:, c0:c1], accumulate=True)
        ref.near(room[:, c0:c1], want + before, off + 2 * ref.U32 * (np.abs(want) + np.abs(before)))
        atomo.atomo_embedding_backward(ids, wide[:, c0:c1], 60, scale=1.5, out=room[:, c0:c1])
        ref.near(room[:, c0:c1], want, off)
        keep = torch.ones(300, dtype=torch.bool, device="cuda")
        keep[c0:c1] = False
        assert torch.equal(room[:, keep], old[:, keep])


def test_gradient_repeats_bit_for_bit(atomo):
    gen = _gen(8)
    ids = _ids("few", 40000, 500, gen)
    grad = torch.randn(40000, 64, generator=gen, device="cuda")
    first = atomo.atomo_embedding_backward(ids, grad, 500)
    for _ in range(10):
        torch.empty(1 << 24, dtype=torch.uint8, device="cuda").random_()      # other work of the allocator in between
        assert torch.equal(atomo.atomo_embedding_backward(ids, grad, 500), first)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("rows,cols,n", [(255, 130, 5000), (256, 8, 4097), (65535, 3, 8193), (70001, 12, 6000), (1, 33, 4500), ((1 << 24) + 5, 1, 5001), (900, 1025, 2600),
                                         (300, 2048, 2049), (900, 7, 131073), (65536, 2, 150001), ((1 << 24) + 5, 1, 140000), (17, 4104, 4200)])
def test_gradient_of_long_lists(atomo, rows, cols, n, dtype):
    """Lists that are sorted by a kernel of their own: keys of one to four passes, several tiles per CTA, ids that are not 16 bytes aligned, padding, ids without a row."""
    gen = _gen(11)
    ids = torch.cat([torch.randint(0, rows, (n // 2,), generator=gen, device="cuda"), torch.randint(0, min(rows, 5), (n - n // 2,), generator=gen, device="cuda") * (rows // 5)])
    ids = ids.clamp(max=rows - 1)[torch.randperm(n, generator=gen, device="cuda")]
    ids[n // 3], ids[n // 2], ids[-1] = rows, -1, rows - 1
    padding = rows // 5 if rows > 1 else -1
    grad = torch.randn(n, cols, generator=gen, device="cuda").to(dtype)
    want, off = _want(ids, grad, rows, 1.5, padding)
    for shifted in (torch.empty(n + 1, dtype=torch.int64, device="cuda")[1:], torch.empty(n + 1, dtype=torch.int32, device="cuda")[1:]):
        shifted.copy_(ids)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        got = atomo.atomo_embedding_backward(shifted, grad, rows, scale=1.5, padding_idx=padding, status=status)
        ref.near(got, want, off)
        assert int(status) == 1
    room = torch.full((rows, cols + 3), 0.25, device="cuda")
    atomo.atomo_embedding_backward(ids, grad, rows, scale=1.5, padding_idx=padding, out=room[:, 1:cols + 1], accumulate=True)
    ref.near(room[:, 1:cols + 1], want + 0.25, off + 2 * ref.U32 * (np.abs(want) + 0.25))
    room[:, 1:cols + 1] = 0.25
    assert bool((room == 0.25).all())


def test_gradient_is_the_lookups_derivative(atomo):
    """<dout, lookup(table)> is linear in the table: its difference along any direction is <gradient, direction>, to the roundings of both."""
    gen = _gen(9)
    ids = _ids("few", 700, 30, gen)
    dout = torch.randn(700, 48, generator=gen, device="cuda")
    direction = torch.randn(30, 48, generator=gen, device="cuda")
    grad = atomo.atomo_embedding_backward(ids, dout, 30, scale=1.25)
    moved = atomo.atomo_embedding(direction, ids, scale=1.25)
    a, b = float((grad.double() * direction.double()).sum()), float((moved.double() * dout.double()).sum())
    _, off = _want(ids, dout, 30, 1.25)
    allowed = float((torch.from_numpy(off).cuda() * direction.double().abs()).sum()) + ref.U32 * float((moved.double() * dout.double()).abs().sum())
    assert abs(a - b) <= allowed


def test_gradients_on_streams_and_in_graphs(atomo):
    gen = _gen(10)
    ids = [_ids("few", 5000, 200, gen) for _ in range(2)]
    dout = [torch.randn(5000, 40, generator=gen, device="cuda") for _ in range(2)]
    want = [atomo.atomo_embedding_backward(i, d, 200) for i, d in zip(ids, dout)]
    graphs = []
    torch.cuda.synchronize()
    for i, d in zip(ids, dout):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = atomo.atomo_embedding_backward(i, d, 200)
        graphs.append((g, out, torch.cuda.Stream()))
    for _ in range(3):
        for g, out, stream in graphs:
            with torch.cuda.stream(stream):
                out.fill_(7.0)
                g.replay()
    torch.cuda.synchronize()
    for (_, out, _), w in zip(graphs, want):
        assert torch.equal(out, w)
    side = torch.cuda.Stream()
    got = atomo.atomo_embedding_backward(ids[0], dout[0], 200, stream=side)
    looked = atomo.atomo_embedding(want[0], ids[0], stream=side)
    side.synchronize()
    assert torch.equal(got, want[0]) and torch.equal(looked, want[0][ids[0]])


def test_refused_tensors(atomo):
    table, ids = torch.zeros(10, 8, device="cuda"), torch.zeros(4, dtype=torch.int64, device="cuda")
    for bad in (dict(table=table.cpu()), dict(table=table.double()), dict(table=table.t()[:8, ::2]), dict(table=table[0]), dict(ids=ids.cpu()), dict(ids=ids.float()), dict(ids=ids[::2]),
                dict(out=torch.zeros(3, 8, device="cuda")), dict(out=torch.zeros(4, 8, device="cuda").half()), dict(status=torch.zeros(1, device="cuda"))):
        with pytest.raises(ValueError):
            atomo.atomo_embedding(**{"table": table, "ids": ids, **bad})
    grad = torch.zeros(4, 8, device="cuda")
    for bad in (dict(grad=grad[:3]), dict(grad=grad.cpu()), dict(grad=grad.double()), dict(accumulate=True), dict(out=torch.zeros(9, 8, device="cuda")),
                dict(out=torch.zeros(10, 8, device="cuda").bfloat16()), dict(grad=torch.zeros(1, 8, device="cuda").expand(4, 8))):
        with pytest.raises(ValueError):
            atomo.atomo_embedding_backward(**{"ids": ids, "grad": grad, "rows": 10, **bad})
    from paper_1806_04090_b200 import api
    with pytest.raises(api.AtomoError):
        atomo.atomo_embedding_backward(ids, grad, 10, padding_idx=10)
    with pytest.raises(api.AtomoError):
        atomo.atomo_embedding(table, ids, scale=math.inf)


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("kind", ["same", "ascending", "few", "random"])
@pytest.mark.parametrize("n", [1000, 4096, 9001, 66000, 150001])
def test_gradient_of_whole_numbers(atomo, kind, n, dtype):
    """Sums of whole numbers below 2^24 are exact in fp32 in whatever order: not one token may be lost or taken twice, however long its run."""
    gen = _gen(12)
    for rows, cols in ((257, 20), (40, 33), (3, 260)):
        ids = _ids(kind, n, rows, gen)
        grad = torch.randint(-8, 9, (n, cols), generator=gen, device="cuda")
        want = torch.zeros(rows, cols, dtype=torch.int64, device="cuda").index_add_(0, ids, grad)
        assert int(want.abs().max()) < 1 << 24
        got = atomo.atomo_embedding_backward(ids, grad.to(dtype), rows, scale=0.5)
        assert torch.equal(got, want.float() * 0.5)
        atomo.atomo_embedding_backward(ids, grad.to(dtype), rows, scale=0.5, out=got, accumulate=True)
        assert torch.equal(got, want.float())


@pytest.mark.parametrize("dtype,cols", [(torch.float32, 260), (torch.float32, 384), (torch.float32, 257), (torch.float32, 383), (torch.bfloat16, 528), (torch.bfloat16, 768),
                                        (torch.float16, 522), (torch.float16, 766), (torch.bfloat16, 261), (torch.float16, 383)])
def test_rows_of_65_to_96_packs(atomo, dtype, cols):
    """Rows that a block of 96 x 2 threads takes, in all three widths of a pack."""
    gen = _gen(13)
    rows, n = 61, 6001
    ids = _ids("few", n, rows, gen)
    table = torch.randn(rows, cols, generator=gen, device="cuda").to(dtype)
    assert torch.equal(atomo.atomo_embedding(table, ids), table[ids])
    grad = torch.randn(n, cols, generator=gen, device="cuda").to(dtype)
    want, off = _want(ids, grad, rows, 1.0)
    ref.near(atomo.atomo_embedding_backward(ids, grad, rows), want, off)
    whole = torch.randint(-8, 9, (n, cols), generator=gen, device="cuda")
    assert torch.equal(atomo.atomo_embedding_backward(ids, whole.to(dtype), rows), torch.zeros(rows, cols, device="cuda").index_add_(0, ids, whole.float()))


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("cols,ld,first", [(33, 34, 1), (33, 35, 0), (257, 259, 2), (300, 304, 1), (300, 304, 4), (64, 72, 8), (1, 3, 1), (513, 515, 1)])
def test_gradient_of_long_lists_in_strided_and_shifted_rows(atomo, dtype, cols, ld, first):
    """Gradient rows that start anywhere and lie apart, of lists that are sorted by a kernel of their own; the buffer ends with the last row's last value."""
    gen = _gen(14)
    rows, n = 50, 5003
    ids = _ids("few", n, rows, gen)
    buffer = torch.randint(-8, 9, ((n - 1) * ld + first + cols,), generator=gen, device="cuda").to(dtype)
    grad = buffer.as_strided((n, cols), (ld, 1), first)
    want = torch.zeros(rows, cols, device="cuda").index_add_(0, ids, grad.float())
    assert torch.equal(atomo.atomo_embedding_backward(ids, grad, rows), want)
    room = torch.full((rows * (ld + 1) + 8,), 7.0, device="cuda")
    out = room.as_strided((rows, cols), (ld + 1, 1), 3)
    atomo.atomo_embedding_backward(ids.int(), grad, rows, out=out)
    assert torch.equal(out, want)
    out.fill_(7.0)
    assert bool((room == 7.0).all())
