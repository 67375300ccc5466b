"""64-bit reference of the operators around the exchange, and what the tests of them share."""
import numpy as np
import torch

U32 = 2.0 ** -24                                        # half a unit in the last place, relative
HALF = {t: torch.finfo(t).eps / 2 for t in (torch.float32, torch.bfloat16, torch.float16)}      # the same for a value rounded to a type
# fp16 has no normal numbers below this: rounding is off by half of its smallest number there
TINY = {torch.float32: 2.0 ** -150, torch.bfloat16: 2.0 ** -134, torch.float16: 2.0 ** -25}
TYPES = [torch.float32, torch.bfloat16, torch.float16]
BLOCK = 32


def philox_words(n, tensor, step, seed):
    """The Philox4x32-10 word of each of a parameter's n elements, as include/atomo.h lays out the counter of optimiser states."""
    from oracle import atomo_oracle
    block = np.arange(-(-n // 4), dtype=np.uint64)
    words = atomo_oracle.philox4x32_10(block & np.uint64(0xFFFFFFFF), np.uint64(0x80000000) | (block >> np.uint64(32)), np.full_like(block, tensor),
                                       np.full_like(block, step & 0x7FFFFFFF), seed & 0xFFFFFFFF, seed >> 32)
    return np.stack([np.broadcast_to(w, block.shape) for w in words], axis=1).reshape(-1)[:n]


def adamw(p, g, m, v, lr, step, beta1, beta2, eps, decay, c):
    """(p, m, v) after a step and, for each, how far fp32 arithmetic may be off."""
    m0, g0 = beta1 * m, (1 - beta1) * c * g
    v0, w0 = beta2 * v, (1 - beta2) * (c * g) ** 2
    m1, v1 = m0 + g0, v0 + w0
    root = 1.0 / np.sqrt(1 - beta2 ** step)
    d = np.sqrt(v1) * root + eps
    rate = lr / (1 - beta1 ** step)
    update = rate * m1 / d
    p1 = p - lr * decay * p - update
    # each constant is rounded once, each product and sum once: beta1 m (2 of them) + the sum's; (1 - beta1) c g: 3 + the sum's
    m_off = 4 * U32 * (abs(m0) + abs(g0)) + 2.0 ** -149
    v_off = 6 * U32 * (v0 + w0) + 2.0 ** -148
    # sqrt.approx and the fast division are good to 2 and 4 units, the other factors to one each; v enters by its root
    share = rate * m_off / d + abs(update) * (v_off / np.maximum(2 * v1, 1e-300) * (v1 > 0) + 16 * U32)
    p_off = share + 2 * U32 * (abs(p) + abs(p1) + abs(update)) + 2.0 ** -149
    return (p1, m1, v1), (p_off, m_off, v_off)


def decode_state(codes, scale):
    """fp64 values of an 8-bit state."""
    s = np.ldexp(1.0, scale.view(torch.uint8).cpu().numpy().astype(np.int64) - 127)      # exact, as powers on the GPU are not
    return codes.reshape(-1).double().cpu().numpy() * np.repeat(s, BLOCK)[: codes.numel()]


def encode_state(x, random16, above_zero):
    """What a state x rounds to: (values, quantum of each, how far x / quantum + random lies from a whole number)."""
    n = x.size
    pad = np.zeros(-(-n // BLOCK) * BLOCK)
    pad[:n] = np.abs(x)
    top = pad.reshape(-1, BLOCK).max(1)
    with np.errstate(divide="ignore"):
        e = np.floor(np.log2(top / 1.75)) + 1 - 8           # the largest goes to [224, 448)
    e = np.where(top > 0, e, -127)
    e = np.maximum(np.where(top >= 1.75 * 2.0 ** (e + 8), e + 1, e), -127)
    y = pad / np.repeat(2.0 ** e, BLOCK)
    q = 2.0 ** (np.floor(np.log2(np.maximum(y, 2.0 ** -6))) - 3)
    at = (y / q)[:n] + random16 / 65536.0
    up = np.floor(at) * q[:n]
    if above_zero:
        up = np.where(x > 0, np.maximum(up, 2.0 ** -9), up)
    unit = np.repeat(2.0 ** e, BLOCK)[:n]
    return np.copysign(up, x) * unit, q[:n] * unit, np.abs(at - np.round(at))


def layer_norm(x, weight, bias, eps):
    """(y, mean, rstd) in fp64 and how far y, mean and rstd may be off in fp32 arithmetic."""
    cols = x.shape[1]
    mean = x.mean(1, keepdims=True)
    var = ((x - mean) ** 2).mean(1, keepdims=True)
    rstd = 1 / np.sqrt(var + eps)
    hat = (x - mean) * rstd
    # a thread adds up to 16 values (in the form for long rows cols / 1024), then come five steps in a warp and up to 32 warps
    adds = max(16, -(-cols // 1024)) + 5 + 32 + 3
    mean_off = adds * U32 * np.abs(x).mean(1, keepdims=True)
    # centred values: the mean's error, and a rounding; the variance changes by the square of the former alone
    centred_off = mean_off + U32 * np.abs(x - mean)
    var_off = (adds + 2) * U32 * var + 2 * centred_off ** 2 + 2 * U32 * (var + eps) + 2 * mean_off * np.abs((x - mean).mean(1, keepdims=True))
    rstd_off = rstd * (var_off / (2 * (var + eps)) + 4 * U32)
    hat_off = centred_off * rstd + np.abs(x - mean) * rstd_off + 2 * U32 * np.abs(hat)
    y = hat * weight + bias
    y_off = np.abs(weight) * hat_off + 2 * U32 * (np.abs(hat * weight) + np.abs(bias))
    return (y, mean[:, 0], rstd[:, 0]), (y_off, mean_off[:, 0] + U32 * np.abs(mean[:, 0]), rstd_off[:, 0])


def layer_norm_backward(dy, x, weight, mean, rstd):
    """(dx, dweight, dbias) for given statistics, and how far they may be off."""
    rows, cols = x.shape
    mean, rstd = mean[:, None], rstd[:, None]
    hat, u = (x - mean) * rstd, dy * weight
    a, b = u.mean(1, keepdims=True), (u * hat).mean(1, keepdims=True)
    dx = rstd * (u - a - hat * b)
    adds = max(16, -(-cols // 1024)) + 5 + 32 + 4
    hat_off = 2 * U32 * (np.abs(x - mean) + np.abs(hat / rstd)) * rstd
    a_off = (adds + 1) * U32 * np.abs(u).mean(1, keepdims=True)
    b_off = (adds + 4) * U32 * np.abs(u * hat).mean(1, keepdims=True) + (np.abs(u) * hat_off).mean(1, keepdims=True)
    dx_off = rstd * (U32 * np.abs(u) + a_off + hat_off * np.abs(b) + np.abs(hat) * b_off + 4 * U32 * (np.abs(u) + np.abs(a) + np.abs(hat * b)))
    dw, db = (dy * hat).sum(0), dy.sum(0)
    dw_off = (rows + 4) * U32 * np.abs(dy * hat).sum(0) + (np.abs(dy) * hat_off).sum(0)
    db_off = (rows + 4) * U32 * np.abs(dy).sum(0)
    return (dx, dw, db), (dx_off, dw_off, db_off)


def rounded(off, want, dtype):
    """off, with the rounding of `want` to dtype."""
    return off + HALF[dtype] * (np.abs(want) + off) + TINY[dtype]


def near(got, want, off):
    got = got.detach().double().cpu().numpy().reshape(np.shape(want))
    bad = ~(np.abs(got - want) <= off)
    assert not bad.any(), f"{int(bad.sum())} of {bad.size} off, the worst by {float(np.max((np.abs(got - want) / np.maximum(off, 1e-300)))):.3g} times what may be"
