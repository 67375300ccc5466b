"""GPU: global gradient norm and AdamW over lists of tensors, against the formulas in 64 bits."""
import math

import numpy as np
import pytest
import torch

from tests import operator_reference as ref

pytestmark = pytest.mark.gpu

HYPER = dict(lr=2e-3, beta1=0.9, beta2=0.995, eps=1e-8)


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


def _odd(flat, n, shift):
    """n elements of a buffer that start `shift` elements behind an aligned address."""
    return flat[shift:shift + n]


def _norm_check(atomo, grads, max_norm):
    out = atomo.atomo_grad_norm(grads, max_norm=max_norm)
    want = math.sqrt(sum(float((g.double() ** 2).sum()) for g in grads))
    # up to 32 squares are added in fp32, the root halves that; then one rounding (and that of the subnormal result)
    off = 18 * ref.U32 * want + 2.0 ** -150
    assert abs(float(out[0]) - want) <= off
    factor = min(1.0, max_norm / (want + 1e-6))
    assert abs(float(out[1]) - factor) <= 20 * ref.U32 * factor


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("lengths", [[1], [3], [4096], [16384 * 8 + 5], [2000001], [0, 7, 0, 1023, 4097, 0], [5] * 300, [9] * 1500, [70000] * 40])
def test_norm(atomo, dtype, lengths):
    gen = _gen(1)
    grads = [torch.randn(n, generator=gen, device="cuda").to(dtype) for n in lengths]
    _norm_check(atomo, grads, 1.0)
    _norm_check(atomo, grads, float("inf"))


@pytest.mark.parametrize("dtype", ref.TYPES)
@pytest.mark.parametrize("shift", [1, 2, 3, 5, 7])
def test_norm_of_unaligned_views(atomo, dtype, shift):
    flat = torch.randn(100100, generator=_gen(2), device="cuda").to(dtype)
    for n in (1, 2, 6, 8, 15, 16, 17, 33, 4099, 100000):
        _norm_check(atomo, [_odd(flat, n, shift)], 0.5)


@pytest.mark.parametrize("n", [5, 300001])
@pytest.mark.parametrize("size", [1e-44, 1e-30, 1e-19, 1e15, 1e19, 1e30, 3e38])
def test_norm_of_extreme_values(atomo, n, size):
    g = torch.full((n,), size, dtype=torch.float32, device="cuda")
    g[n // 2] = 0.0
    want = math.sqrt(float((g.double() ** 2).sum()))
    got = float(atomo.atomo_grad_norm([g], max_norm=1.0)[0])
    if want > 3.4e38:
        assert got == math.inf
    else:
        assert abs(got - want) <= 18 * ref.U32 * want + 2.0 ** -150


def test_norm_zero_and_not_finite(atomo):
    z = atomo.atomo_grad_norm([torch.zeros(1000, device="cuda")], max_norm=1.0).tolist()
    assert z == [0.0, 1.0]
    assert atomo.atomo_grad_norm([torch.zeros(0, device="cuda")], max_norm=1.0).tolist() == [0.0, 1.0]
    for n in (10, 500000):
        for bad in (math.nan, math.inf, -math.inf):
            g = torch.ones(n, device="cuda")
            g[n - 3] = bad
            out = atomo.atomo_grad_norm([torch.ones(3, device="cuda"), g]).tolist()
            assert not math.isfinite(out[0]) and math.isnan(out[1])


def test_norm_repeats_bit_for_bit(atomo):
    grads = [torch.randn(n, generator=_gen(3), device="cuda") for n in (1 << 20, 333333, 17)]
    first = atomo.atomo_grad_norm(grads, max_norm=1.0)
    for _ in range(5):
        assert torch.equal(atomo.atomo_grad_norm(grads, max_norm=1.0), first)


# ---- AdamW ----------------------------------------------------------------------------------------
def _case(lengths, param, grad, bits, master, seed, shift=0):
    """Tensors of a list of parameters in buffers with a margin of canaries behind each."""
    from paper_1806_04090_b200 import api
    gen = _gen(seed)
    rand = lambda n, s: torch.randn(n + 40, generator=gen, device="cuda") * s  # noqa: E731
    flats = {"param": [], "grad": [], "m": [], "v": [], "ms": [], "vs": [], "master": []}
    for n in lengths:
        p = rand(n, 0.1)
        flats["param"].append(p.to(param))
        flats["grad"].append(rand(n, 0.01).to(grad))
        flats["master"].append((p.to(param).float() + rand(n, 1e-5)) if master else None)
        m, v = rand(n, 0.005), rand(n, 0.01).square()
        if bits == 32:
            flats["m"].append(m); flats["v"].append(v)
        else:
            blocks = -(-n // 32) + 40
            for name, x, scale in (("m", m, "ms"), ("v", v, "vs")):
                flats[name].append((x / x.abs().max() * 300).to(torch.float8_e4m3fn))
                byte = torch.randint(100, 118, (blocks,), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
                byte[::5] = 0 if name == "m" else 104
                flats[scale].append(byte.view(torch.float8_e8m0fnu))
    view = lambda name: [_odd(f, n, shift) for f, n in zip(flats[name], lengths)]  # noqa: E731
    blocks = lambda name: [_odd(f, -(-n // 32), shift) for f, n in zip(flats[name], lengths)] if bits == 8 else None  # noqa: E731
    decay = [0.1 if i % 2 == 0 else 0.0 for i in range(len(lengths))]
    state = api.AdamWState(view("param"), view("m"), view("v"), blocks("ms"), blocks("vs"), view("master") if master else None, decay)
    return state, view("grad"), flats


def _np(t):
    return t.double().cpu().numpy().reshape(-1)


def _snapshot(flats):
    return {k: [None if t is None else t.clone() for t in v] for k, v in flats.items()}


def _check_step(atomo, lengths, param, grad, bits, master, seed, scale=None, shift=0, step=3):
    state, grads, flats = _case(lengths, param, grad, bits, master, seed, shift)
    before = _snapshot(flats)
    c = 1.0 if scale is None else float(scale[1])
    rounding_seed = 0x123456789ABCDEF
    atomo.atomo_adamw(state, grads, step=step, seed=rounding_seed, scale=scale, **HYPER)
    torch.cuda.synchronize()
    for i, n in enumerate(lengths):
        at = slice(shift, shift + n)
        ab = slice(shift, shift + -(-n // 32))
        g = _np(before["grad"][i][at])
        p = _np((before["master"] if master else before["param"])[i][at])
        if bits == 8:
            m = ref.decode_state(before["m"][i][at], before["ms"][i][ab])
            v = ref.decode_state(before["v"][i][at], before["vs"][i][ab])
        else:
            m, v = _np(before["m"][i][at]), _np(before["v"][i][at])
        (p1, m1, v1), (po, mo, vo) = ref.adamw(p, g, m, v, HYPER["lr"], step, HYPER["beta1"], HYPER["beta2"], HYPER["eps"], state.weight_decay[i], c)
        if master:
            ref.near(state.master[i], p1, po)
        ref.near(state.params[i], p1, ref.rounded(po, p1, param) if param != torch.float32 else po)
        if bits == 32:
            ref.near(state.exp_avg[i], m1, mo)
            ref.near(state.exp_avg_sq[i], v1, vo)
        elif n:
            words = ref.philox_words(n, i, step, rounding_seed)
            for x, off, codes, scales, r, keep in ((m1, mo, state.exp_avg[i], state.exp_avg_scale[i], words & 0xFFFF, False),
                                                   (v1, vo, state.exp_avg_sq[i], state.exp_avg_sq_scale[i], words >> 16, True)):
                want, quantum, apart = ref.encode_state(x, r.astype(np.float64), keep)
                got = ref.decode_state(codes, scales)
                # the value that is rounded is off by what fp32 arithmetic is, and by the cut at 2^-20 of a quantum; where that reaches
                # the next whole number, either neighbour is right
                unsure = apart <= off / quantum + 2.0 ** -19
                assert np.all((got == want) | (unsure & (np.abs(got - want) <= quantum * (1 + 1e-9))))
                assert unsure.mean() < 0.01 or n < 1000
    # nothing around the tensors was written
    for name, tensors in flats.items():
        for i, t in enumerate(tensors):
            if t is None:
                continue
            n = lengths[i] if name not in ("ms", "vs") else -(-lengths[i] // 32)
            old = before[name][i]
            assert torch.equal(t[:shift].view(torch.uint8), old[:shift].view(torch.uint8)) and torch.equal(t[shift + n:].view(torch.uint8), old[shift + n:].view(torch.uint8)), name


LISTS = [[1], [3], [31], [32], [33], [4095], [4096], [4097], [0, 5, 0, 12289, 64, 0], [100003, 17]]


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("lengths", LISTS)
def test_step_lengths(atomo, bits, lengths):
    _check_step(atomo, lengths, torch.float32, torch.float32, bits, False, 11)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("param,grad,master", [(torch.float32, torch.bfloat16, False), (torch.bfloat16, torch.float32, False), (torch.bfloat16, torch.bfloat16, True),
                                               (torch.float16, torch.float16, False), (torch.float16, torch.float32, True), (torch.float32, torch.float16, False)])
def test_step_types(atomo, bits, param, grad, master):
    _check_step(atomo, [5000, 1, 8192, 333], param, grad, bits, master, 12, scale=torch.tensor([4.0, 0.25], device="cuda"))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [1, 2, 3, 4, 6])
@pytest.mark.parametrize("param,grad,master", [(torch.float32, torch.float32, False), (torch.bfloat16, torch.float32, True)])
def test_step_unaligned(atomo, bits, shift, param, grad, master):
    _check_step(atomo, [4099, 70, 1], param, grad, bits, master, 13, shift=shift)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("count", [9, 65, 381, 900])
def test_step_many_tensors(atomo, bits, count):
    _check_step(atomo, [(37 * i) % 211 for i in range(count)], torch.float32, torch.float32, bits, False, 14)


@pytest.mark.parametrize("step", [1, 2, 1000000, 2 ** 31 + 5])
def test_step_numbers(atomo, step):
    _check_step(atomo, [1000], torch.float32, torch.float32, 8, False, 15, step=step)


@pytest.mark.parametrize("bits", [32, 8])
def test_first_step_from_zero(atomo, bits):
    """The first step from states of zero moves every parameter by about lr against the sign of its gradient."""
    from paper_1806_04090_b200 import api
    p = torch.zeros(5000, device="cuda")
    g = torch.randn(5000, generator=_gen(16), device="cuda")
    state = api.AdamWState.zeros([p], bits=bits, weight_decay=0.0)
    atomo.atomo_adamw(state, [g], lr=0.1, step=1, eps=0.0)
    # m / sqrt(v) = g / |g|; its roundings: those of m (4 units), of v (6, halved), of the quotient (16)
    ref.near(p, -0.1 * np.sign(_np(g)), np.full(5000, 0.1 * 32 * ref.U32))


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("beta2,step", [(0.999, 1), (0.999999, 1), (0.999, 5000)])
@pytest.mark.parametrize("eps", [1e-13, 1e-12, 4e-12, 1.2e-10, 4e-9])
def test_small_eps_beside_smaller_moments(atomo, eps, beta2, step, bits):
    """Second moments on both sides of the smallest normal number, whose roots count beside an eps of this size where the bias is corrected for by a large factor."""
    from paper_1806_04090_b200 import api
    n = 6000
    gen = _gen(25)
    g = torch.randn(n, generator=gen, device="cuda") * 10.0 ** torch.linspace(-18.0, -14.0, n, device="cuda")
    if beta2 == 0.999999:
        g *= 30.0
    p = torch.zeros(n, device="cuda")
    state = api.AdamWState.zeros([p], bits=bits, weight_decay=0.0)
    atomo.atomo_adamw(state, [g], lr=0.1, step=step, beta1=0.9, beta2=beta2, eps=eps, seed=1)
    (want, _, v), (off, _, _) = ref.adamw(np.zeros(n), _np(g), np.zeros(n), np.zeros(n), 0.1, step, 0.9, beta2, eps, 0.0, 1.0)
    assert (v < 2.0 ** -126).any() and (v > 2.0 ** -126).any()
    ref.near(p, want, off)


def test_mixed_types_in_one_call(atomo):
    from paper_1806_04090_b200 import api
    gen = _gen(17)
    params = [torch.randn(n, generator=gen, device="cuda").to(t) for n, t in ((100, torch.float32), (4097, torch.bfloat16), (64, torch.float16))]
    old = [p.clone() for p in params]
    grads = [torch.randn(p.numel(), generator=gen, device="cuda") for p in params]
    state = api.AdamWState.zeros(params, bits=32, master=True, weight_decay=[0.0, 0.1, 0.0])
    assert state.master[0] is None and state.master[1].dtype == torch.float32
    atomo.atomo_adamw(state, grads, step=1, **HYPER)
    for i, p in enumerate(params):
        (p1, _, _), (po, _, _) = ref.adamw(_np(old[i]), _np(grads[i]), np.zeros(p.numel()), np.zeros(p.numel()), HYPER["lr"], 1, HYPER["beta1"], HYPER["beta2"], HYPER["eps"],
                                           state.weight_decay[i], 1.0)
        ref.near(p, p1, ref.rounded(po, p1, p.dtype) if i else po)


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("bad", [math.nan, math.inf, -math.inf])
def test_no_step_where_the_norm_is_not_finite(atomo, bits, bad):
    state, grads, flats = _case([5000, 33], torch.bfloat16, torch.float32, bits, True, 18)
    grads[1][7] = bad
    before = _snapshot(flats)
    scale = atomo.atomo_grad_norm(grads, max_norm=1.0)
    atomo.atomo_adamw(state, grads, step=4, scale=scale, **HYPER)
    for name in ("param", "m", "v", "ms", "vs", "master"):
        for t, old in zip(flats[name], before[name]):
            assert torch.equal(t.view(torch.uint8), old.view(torch.uint8))


def test_state_in_8_bits_of_values_that_are_not_finite(atomo):
    """A gradient that is not finite makes NaN of its own states, and leaves the others of its block as they should be."""
    from paper_1806_04090_b200 import api
    g = torch.randn(96, generator=_gen(19), device="cuda")
    g[40], g[41], g[70] = math.nan, math.inf, 1e30
    p = torch.zeros(96, device="cuda")
    state = api.AdamWState.zeros([p], bits=8)
    atomo.atomo_adamw(state, [g], step=1, seed=5, **HYPER)
    m = ref.decode_state(state.exp_avg[0], state.exp_avg_scale[0])
    v = ref.decode_state(state.exp_avg_sq[0], state.exp_avg_sq_scale[0])
    assert np.flatnonzero(np.isnan(m)).tolist() == [40, 41] and np.flatnonzero(np.isnan(v)).tolist() == [40, 41, 70]
    fine = np.ones(96, bool)
    fine[[40, 41, 70]] = False
    fine[64:96] = False                                  # beside 1e30 the others' first moments are below its block's range
    want = 0.1 * _np(g)
    # rounded up or down by less than one of e4m3's steps, 2^-3 of the value at most above its smallest normal number
    assert np.all(np.abs(m - want)[fine] <= 2.0 ** -3 * np.abs(want)[fine] * (1 + 1e-5) + np.abs(want[fine]).max() * 2.0 ** -16)


@pytest.mark.parametrize("shift", [0, 3])
def test_state_in_8_bits_of_large_values(atomo, shift):
    """Blocks with finite moments of 2^13 to 2^15, 1e10 and beyond, of one size or beside small ones, from states with exponent bytes up to 220."""
    from paper_1806_04090_b200 import api
    n, step, seed = 8192 + 40, 9, 1234567
    blocks = -(-n // 32)
    gen = _gen(24)
    rand = lambda k: torch.randn(k + 40, generator=gen, device="cuda")  # noqa: E731
    size = torch.tensor([1e-3, 1.0, 2.0 ** 14, 3e5, 1e7, 1e10, 1e15], device="cuda")[torch.arange(n + 40, device="cuda") // 32 % 7]
    g = rand(n) * size
    g[::64 * 3] = 1e15                                    # one large value in a block of another size
    codes, scales = [], []
    for top in (220, 190):                                # the second moment's next value stays finite: 448 * 2^63, and 1e30 / 200
        codes.append((rand(n) * 60).clamp(-448, 448).abs().to(torch.float8_e4m3fn))
        scales.append(torch.randint(90, top + 1, (blocks + 40,), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8))
        scales[-1][::3] = torch.randint(134, 146, (scales[-1][::3].numel(),), generator=gen, device="cuda", dtype=torch.int32).to(torch.uint8)
        scales[-1][::7] = 0
    codes[0] = (codes[0].float() * torch.sign(rand(n))).to(torch.float8_e4m3fn)
    codes, scales = [_odd(c, n, shift) for c in codes], [_odd(c.view(torch.float8_e8m0fnu), blocks, shift) for c in scales]
    m, v = (ref.decode_state(c, e) for c, e in zip(codes, scales))
    grads = [_odd(g, n, shift)]
    state = api.AdamWState([torch.zeros(n, device="cuda")], [codes[0]], [codes[1]], [scales[0]], [scales[1]])
    atomo.atomo_adamw(state, grads, step=step, seed=seed, **HYPER)
    m, v = _moments_in_fp32(m, v, grads[0].cpu().numpy(), 1.0, HYPER["beta1"], HYPER["beta2"])
    assert np.isfinite(m).all() and np.isfinite(v).all() and np.abs(m).max() > 1e29 and (np.abs(m) < 1e-3).any()
    words = ref.philox_words(n, 0, step, seed)
    for x, got, random, keep in ((m, ref.decode_state(codes[0], scales[0]), words & 0xFFFF, False), (v, ref.decode_state(codes[1], scales[1]), words >> 16, True)):
        x, random = x.astype(np.float64), random.astype(np.float64)
        _, quantum, _ = ref.encode_state(x, random, keep)
        cut = np.round(x / quantum * 2.0 ** 20) / 2.0 ** 20 * quantum           # what of a value far below its block's largest is looked at
        want, _, _ = ref.encode_state(np.where(cut == 0, x, cut), random, keep)
        assert np.array_equal(got, want)


def test_8_bit_states_are_unbiased(atomo):
    """The mean over many seeds of a rounded state is the state: within five standard deviations of the mean of so many roundings of one quantum."""
    from paper_1806_04090_b200 import api
    n, runs = 2048, 400
    g = torch.randn(n, generator=_gen(20), device="cuda")
    total_m, total_v = np.zeros(n), np.zeros(n)
    for seed in range(runs):
        state = api.AdamWState.zeros([torch.zeros(n, device="cuda")], bits=8)
        atomo.atomo_adamw(state, [g], step=1, seed=seed, **HYPER)
        total_m += ref.decode_state(state.exp_avg[0], state.exp_avg_scale[0])
        total_v += ref.decode_state(state.exp_avg_sq[0], state.exp_avg_sq_scale[0])
    for total, want in ((total_m, 0.1 * _np(g)), (total_v, 0.005 * _np(g) ** 2)):
        _, quantum, _ = ref.encode_state(want, np.zeros(n), False)
        # a rounding's variance is at most quantum^2 / 4; values kept above zero are biased by less than a quantum of their block: leave them out
        big = np.abs(want) >= quantum
        assert big.mean() > 0.5
        off = np.abs(total / runs - want)[big] / (quantum[big] * 0.5 / math.sqrt(runs))
        assert off.max() < 6.0 and np.sqrt((off ** 2).mean()) < 1.1


def test_8_bit_states_follow_a_decaying_average(atomo):
    """An average that shrinks by 0.5 % a step, far less than half a quantum, still shrinks."""
    from paper_1806_04090_b200 import api
    n = 4096
    state = api.AdamWState.zeros([torch.zeros(n, device="cuda")], bits=8, weight_decay=0.0)
    g = torch.ones(n, device="cuda")
    atomo.atomo_adamw(state, [g], step=1, seed=1, **HYPER)
    zero = torch.zeros(n, device="cuda")
    for t in range(2, 302):
        atomo.atomo_adamw(state, [zero], step=t, seed=1, **HYPER)
    v = ref.decode_state(state.exp_avg_sq[0], state.exp_avg_sq_scale[0])
    want = 0.005 * 0.995 ** 300
    # each step's rounding changes a value by a quantum of at most v / 8 with a variance of at most quantum * change = v^2 0.005 / 8; the mean
    # over 4096 values of 300 such steps has a relative deviation of about sqrt(300 * 0.005 / 8 / 4096) * (0.995^-300 at most)
    assert abs(v.mean() / want - 1) < 5 * math.sqrt(300 * 0.005 / 8 / n) * 2


def _moments_in_fp32(m, v, g, c, beta1, beta2):
    """The moments of a step, each operation rounded once."""
    b1, r1, b2, r2 = (np.float32(x) for x in (beta1, 1.0 - beta1, beta2, 1.0 - beta2))
    g = g.astype(np.float32) * np.float32(c)
    return b1 * m.astype(np.float32) + r1 * g, b2 * v.astype(np.float32) + r2 * g * g


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("shift", [0, 3])
@pytest.mark.parametrize("c", [1.0, 0.3])
def test_moments_are_rounded_operation_by_operation(atomo, bits, shift, c):
    """Bit for bit what the same fp32 operations give, whatever form an element goes through: whole chunks, tails, unaligned tensors."""
    lengths, seed, step = [60000, 4097, 33], 77, 6
    state, grads, flats = _case(lengths, torch.float32, torch.float32, bits, False, 23, shift)
    before = _snapshot(flats)
    scale = torch.tensor([5.0, c], device="cuda")
    atomo.atomo_adamw(state, grads, step=step, seed=seed, scale=scale, **HYPER)
    for i, n in enumerate(lengths):
        at, ab = slice(shift, shift + n), slice(shift, shift + -(-n // 32))
        if bits == 32:
            m, v = (before[k][i][at].cpu().numpy() for k in ("m", "v"))
        else:
            m, v = (ref.decode_state(before[k][i][at], before[k + "s"][i][ab]) for k in ("m", "v"))
        m, v = _moments_in_fp32(m, v, grads[i].cpu().numpy(), float(scale[1]), HYPER["beta1"], HYPER["beta2"])
        if bits == 32:
            assert np.array_equal(state.exp_avg[i].cpu().numpy(), m) and np.array_equal(state.exp_avg_sq[i].cpu().numpy(), v)
        else:
            words = ref.philox_words(n, i, step, seed)
            for x, codes, scales, random, keep in ((m, state.exp_avg[i], state.exp_avg_scale[i], words & 0xFFFF, False), (v, state.exp_avg_sq[i], state.exp_avg_sq_scale[i], words >> 16, True)):
                # x / quantum has 24 bits and the random number 16 behind the point: their sum and its floor are exact in 64 bits.  (A value far below its
                # block's largest is first cut to 2^-20 of a quantum, to the nearest.)
                want, quantum, _ = ref.encode_state(x.astype(np.float64), random.astype(np.float64), keep)
                cut = np.round(x.astype(np.float64) / quantum * 2.0 ** 20) / 2.0 ** 20 * quantum
                fine = cut == x
                got = ref.decode_state(codes, scales)
                assert np.array_equal(got[fine], want[fine]) and fine.mean() > 0.9


def test_step_repeats_bit_for_bit_and_follows_its_seed(atomo):
    results = []
    for seed in (7, 7, 8):
        state, grads, flats = _case([10000, 77], torch.bfloat16, torch.float32, 8, True, 21)
        atomo.atomo_adamw(state, grads, step=2, seed=seed, **HYPER)
        results.append([t.view(torch.uint8).clone() for t in state.exp_avg + state.exp_avg_sq])
    assert all(torch.equal(a, b) for a, b in zip(results[0], results[1]))
    assert not all(torch.equal(a, b) for a, b in zip(results[0], results[2]))


def test_step_and_norm_in_a_graph_and_on_another_stream(atomo):
    """Two graphs captured from one context and replayed side by side, against the same calls made directly."""
    from paper_1806_04090_b200 import api
    gen = _gen(22)
    init = [torch.randn(n, generator=gen, device="cuda") for n in (300001, 513)]
    grads = [[torch.randn(p.numel(), generator=gen, device="cuda") for p in init] for _ in range(2)]

    def fresh():
        params = [p.clone() for p in init]
        return params, api.AdamWState.zeros(params, bits=8)

    want = []
    for k in range(2):
        params, state = fresh()
        for _ in range(3):
            scale = atomo.atomo_grad_norm(grads[k], max_norm=1.0)
            atomo.atomo_adamw(state, grads[k], step=1, seed=k, scale=scale, **HYPER)
        want.append(params)
    torch.cuda.synchronize()
    graphs, got = [], []
    for k in range(2):
        params, state = fresh()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            scale = atomo.atomo_grad_norm(grads[k], max_norm=1.0)
            atomo.atomo_adamw(state, grads[k], step=1, seed=k, scale=scale, **HYPER)
        graphs.append((graph, torch.cuda.Stream(), state, scale))
        got.append(params)
    for _ in range(3):
        for graph, stream, _, _ in graphs:
            with torch.cuda.stream(stream):
                graph.replay()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    params, state = fresh()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        scale = atomo.atomo_grad_norm(grads[1], max_norm=1.0, stream=side)
        atomo.atomo_adamw(state, grads[1], step=1, seed=1, scale=scale, stream=side, **HYPER)
    side.synchronize()
    for a, b in zip(want[0] + want[1] + want[1], got[0] + got[1] + params):
        assert torch.equal(a, b)


def test_refused_tensors(atomo):
    from paper_1806_04090_b200 import api
    p, g = torch.zeros(64, device="cuda"), torch.zeros(64, device="cuda")
    state = api.AdamWState.zeros([p])
    for bad in ([], [g, g], [g[:63]], [g.cpu()], [g.double()], [torch.zeros(128, device="cuda")[::2]], [g.int()]):
        with pytest.raises(ValueError):
            atomo.atomo_adamw(state, bad, lr=0.1, step=1)
    with pytest.raises(ValueError):
        atomo.atomo_adamw(state, [g], lr=0.1, step=1, scale=torch.zeros(1, device="cuda"))
    for args in (dict(lr=-1.0, step=1), dict(lr=0.1, step=0), dict(lr=0.1, step=1, beta1=1.0)):
        with pytest.raises(api.AtomoError) as e:
            atomo.atomo_adamw(state, [g], **args)
        assert e.value.code == 1
    for bad in (g.cpu(), g.double(), torch.zeros(128, device="cuda")[::2]):
        for others in (0, 3, 10):
            with pytest.raises(ValueError):
                atomo.atomo_grad_norm([g] * others + [bad] + [g] * others)
    with pytest.raises(api.AtomoError):
        atomo.atomo_grad_norm([])
    with pytest.raises(api.AtomoError):
        atomo.atomo_grad_norm([g], max_norm=0.0)
    # the same memory twice, or a state that lies over another
    with pytest.raises(ValueError, match="overlap"):
        api.AdamWState([p, p], [torch.zeros(64, device="cuda")] * 2, [torch.zeros(64, device="cuda")] * 2)
    with pytest.raises(ValueError, match="overlap"):
        api.AdamWState([p], [p], [torch.zeros(64, device="cuda")])
    flat = torch.zeros(100, device="cuda")
    with pytest.raises(ValueError, match="overlap"):
        api.AdamWState([flat[:64], flat[60:100]], [torch.zeros(64, device="cuda"), torch.zeros(40, device="cuda")], [torch.zeros(64, device="cuda"), torch.zeros(40, device="cuda")])
    with pytest.raises(ValueError):
        api.AdamWState([p], [torch.zeros(64, device="cuda", dtype=torch.bfloat16)], [torch.zeros(64, device="cuda")])
    with pytest.raises(ValueError):
        api.AdamWState([torch.zeros(8, 8, device="cuda").t()[:4]], [torch.zeros(32, device="cuda")], [torch.zeros(32, device="cuda")])


def test_parameters_that_were_given_other_memory(atomo):
    """The call refuses them, and what its description names is still allocated: nothing else gets that memory meanwhile."""
    from paper_1806_04090_b200 import api
    n = 1 << 18
    p, q = torch.nn.Parameter(torch.zeros(n, device="cuda")), torch.nn.Parameter(torch.zeros(77, device="cuda"))
    state = api.AdamWState.zeros([p, q], bits=8, weight_decay=0.0)
    grads = [torch.ones(n, device="cuda"), torch.ones(77, device="cuda")]
    atomo.atomo_adamw(state, grads, lr=0.1, step=1)
    first = p.detach().clone()
    old = p.data_ptr()
    p.data = p.data.clone()
    with pytest.raises(ValueError, match="other memory"):
        atomo.atomo_adamw(state, grads, lr=0.1, step=2)
    assert torch.equal(p.detach(), first)
    assert all(torch.empty(n, device="cuda").data_ptr() != old for _ in range(4))
    moved = api.AdamWState([p, q], state.exp_avg, state.exp_avg_sq, state.exp_avg_scale, state.exp_avg_sq_scale, weight_decay=0.0)
    atomo.atomo_adamw(moved, grads, lr=0.1, step=2)
    assert bool((p < first).all())
    # states: the memory that is described stays allocated
    old = state.exp_avg[0].data_ptr()
    state.exp_avg[0].data = torch.zeros(n, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    assert all(torch.empty(n, dtype=torch.uint8, device="cuda").data_ptr() != old for _ in range(4))
