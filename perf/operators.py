"""The operators on either side of the gradient exchange, as a data-parallel training step of a language model calls them: the two
layers whose weight gradients are sums over the tokens (embedding, layer norm) give gradients that are encoded, and the decoded
mean goes through the global norm into an AdamW step over all parameters.

`listed()` gives fixed cases, `draw(rng)` more of the same ranges, `prepare` what a training or serving program holds before the
call, `run` one pass: the framework's operators where `own` is true, else the same computed by elementary torch operations in 32
bits.  `exact` computes the results in 64 bits from the definitions.

Parameters lie in one buffer, each starting at a multiple of 32 elements, as flat parameter buffers do; the framework gets them as
a list of tensors, the plain form works on the whole buffer at once.  AdamW states in 8 bits are OCP e4m3 numbers with a power of two
(e8m0) for each 32 of them, rounded stochastically with the Philox4x32-10 words of (seed, step, tensor, element); they are returned
in these types, codes and powers of two.
"""
import math

import torch

own = False

BLOCK = 32          # elements that share a power of two
# (rows, cols) of a CIFAR ResNet-18's layers, as the benchmark has them
RESNET18 = ("64x27,4*64x576,128x576,3*128x1152,256x1152,3*256x2304,512x2304,3*512x4608,10x512")


def listed():
    return [
        # a single vector of the smallest configuration: launches and the host's part of the call
        {"name": "norm_4096", "op": "norm", "set": "4096", "grad": "f32"},
        # every parameter of a transformer with an embedding, gradients as the decode leaves them
        {"name": "norm_transformer_133m", "op": "norm", "set": "transformer:1024:8:32000", "grad": "f32"},
        # a handful of small odd tensors with 8-bit states: latency, tails of blocks
        {"name": "adamw8_ragged", "op": "adamw", "set": "1,31,33,1000x3,777x11,4097,513", "param": "bf16", "grad": "f32", "bits": 8, "master": False, "clip": True},
        # the layers of a ResNet-18 in plain fp32 training after clipping
        {"name": "adamw_resnet18", "op": "adamw", "set": RESNET18, "param": "f32", "grad": "f32", "bits": 32, "master": False, "clip": True},
        # a whole model as one vector, states in 8 bits
        {"name": "adamw8_25m", "op": "adamw", "set": "25600000", "param": "f32", "grad": "f32", "bits": 8, "master": False, "clip": False},
        # mixed precision training of a transformer: bf16 weights and gradients, fp32 master copy and states
        {"name": "adamw_transformer_133m", "op": "adamw", "set": "transformer:1024:8:32000", "param": "bf16", "grad": "bf16", "bits": 32, "master": True, "clip": True},
        # serving: the rows of one token for each of sixteen sequences
        {"name": "embedding_serve_16", "op": "embedding", "train": False, "tokens": 16, "vocab": 32000, "width": 4096, "type": "bf16", "zipf": 1.0, "ids": "i64"},
        # training on a small odd vocabulary: lookup, then the gradient of the table
        {"name": "embedding_train_odd", "op": "embedding", "train": True, "tokens": 4001, "vocab": 10007, "width": 515, "type": "f32", "zipf": 1.0, "ids": "i64"},
        # training: 32 sequences of 2048 tokens
        {"name": "embedding_train_64k", "op": "embedding", "train": True, "tokens": 65536, "vocab": 32000, "width": 2048, "type": "bf16", "zipf": 1.1, "ids": "i32"},
        # serving: one token for each of three sequences
        {"name": "layernorm_serve_3", "op": "layernorm", "train": False, "rows": 3, "width": 4096, "type": "bf16", "weight": "bf16"},
        # training, sizes that no tile divides
        {"name": "layernorm_train_odd", "op": "layernorm", "train": True, "rows": 1999, "width": 1023, "type": "f32", "weight": "f32"},
        # training: 16 sequences of 2048 tokens
        {"name": "layernorm_train_32k", "op": "layernorm", "train": True, "rows": 32768, "width": 2048, "type": "bf16", "weight": "f32"},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _some_set(rng):
    if rng.random() < 0.3:
        width = 64 * rng.randint(2, 16)
        return "transformer:%d:%d:%d" % (width, rng.randint(1, 8), _log(rng, 500, 32000))
    total, parts = 0, []
    for _ in range(_log(rng, 1, 150)):
        n = _log(rng, 1, 2.0e7)
        if total + n > 1.2e8:
            n = _log(rng, 1, 2.0e4)
        total += n
        parts.append("%d" % n)
    return ",".join(parts)


def draw(rng):
    op = rng.choice(["norm", "adamw", "adamw", "adamw", "embedding", "embedding", "layernorm", "layernorm"])
    if op == "norm":
        return {"op": op, "set": _some_set(rng), "grad": rng.choice(["f32", "f32", "bf16", "f16"])}
    if op == "adamw":
        param = rng.choice(["f32", "bf16", "f16"])
        grad = rng.choice(["f32", param])
        bits = rng.choice([8, 32])
        return {"op": op, "set": _some_set(rng), "param": param, "grad": grad, "bits": bits, "master": param != "f32" and rng.random() < 0.5, "clip": rng.random() < 0.5}
    if op == "embedding":
        train = rng.random() < 0.7
        vocab, width = _log(rng, 100, 50000), _log(rng, 16, 4096)
        while vocab * width > 6.5e7:
            width = _log(rng, 16, 4096)
        tokens = _log(rng, 1, 65536 if train else 2048)
        while tokens * width > 1.3e8:
            tokens = _log(rng, 1, 65536)
        return {"op": op, "train": train, "tokens": tokens, "vocab": vocab, "width": width, "type": rng.choice(["f32", "bf16", "f16"]),
                "zipf": round(rng.uniform(0.6, 1.3), 2), "ids": rng.choice(["i32", "i64"])}
    train = rng.random() < 0.7
    width = _log(rng, 16, 16384)
    if rng.random() < 0.5:
        width = max(16, width // 16 * 16)
    rows = _log(rng, 1, max(2, min(65536, int(6.0e7 / width)))) if train else _log(rng, 1, 64)
    kind = rng.choice(["f32", "bf16", "f16"])
    return {"op": op, "train": train, "rows": rows, "width": width, "type": kind, "weight": rng.choice(["f32", kind])}


# ---- sizes --------------------------------------------------------------------------------------
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16, "i32": torch.int32, "i64": torch.int64}
BYTES = {"f32": 4, "bf16": 2, "f16": 2, "i32": 4, "i64": 8}


def _lengths(case):
    """(elements, weight decay) of the parameters: matrices are decayed, vectors are not."""
    out = []
    if case["set"].startswith("transformer:"):
        width, blocks, vocab = (int(x) for x in case["set"].split(":")[1:])
        square, wide = (width * width, 0.01), (4 * width * width, 0.01)
        block = [(width, 0.0), (width, 0.0), square, square, square, square, (width, 0.0), (width, 0.0), wide, (4 * width, 0.0), wide, (width, 0.0)]
        return [(vocab * width, 0.01)] + block * blocks + [(width, 0.0), (width, 0.0)]
    for part in case["set"].split(","):
        count, _, shape = part.rpartition("*")
        dims = [int(x) for x in shape.split("x")]
        out += [(math.prod(dims), 0.01 if len(dims) > 1 else 0.0)] * int(count or 1)
    return out


def _starts(lengths):
    starts, at = [], 0
    for n in lengths:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return starts, at


def _zipf(case, dev):
    p = torch.arange(1, case["vocab"] + 1, dtype=torch.float64, device=dev) ** (-case["zipf"])
    return p / p.sum()


# ---- inputs -------------------------------------------------------------------------------------
_contexts = {}


def _context():
    """One library context for the whole program, as a training loop keeps it."""
    from paper_1806_04090_b200 import api
    if 0 not in _contexts:
        _contexts[0] = api.Atomo(0)
    return _contexts[0]


def _randn(gen, n, dev, scale=1.0):
    return torch.randn(n, generator=gen, device=dev, dtype=torch.float32).mul_(scale)


def _pow2(byte):
    """2^(byte - 127) in fp32, byte an integer tensor."""
    return torch.where(byte > 0, byte << 23, 1 << 22).to(torch.int32).view(torch.float32)


def _nearest(x):
    """A state as an earlier step left it: e4m3 codes and the blocks' powers of two."""
    top = x.view(-1, BLOCK).abs().amax(1)
    byte = (((top.view(torch.int32) + 0x200000) >> 23) - 8).clamp_(min=0)
    codes = (x.view(-1, BLOCK) / _pow2(byte)[:, None]).to(torch.float8_e4m3fn).view(-1)
    return codes, byte.to(torch.uint8).view(torch.float8_e8m0fnu)


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed) * 1000003 + 17)
    op = case["op"]
    state = dict(case)
    if op in ("norm", "adamw"):
        sizes = _lengths(case)
        lengths = [n for n, _ in sizes]
        starts, total = _starts(lengths)
        views = lambda flat: [flat[s:s + n] for s, n in zip(starts, lengths)]  # noqa: E731
        inside = torch.zeros(total, dtype=torch.bool, device=dev)
        for v in views(inside):
            v.fill_(True)
        # gradients of a mini-batch: a common scale, some entries far above it
        grad = _randn(gen, total, dev, 1e-3)
        grad[::97] *= 30.0
        grad = (grad * inside).to(TYPES[case["grad"]])
        state.update(total=total, lengths=lengths, starts=starts, grad=grad, grads=views(grad), max_norm=1.0)
        if op == "norm":
            if own:
                state["ctx"] = _context()
            return state
        param = (_randn(gen, total, dev, 0.05) * inside).to(TYPES[case["param"]])
        m = _randn(gen, total, dev, 3e-4) * inside
        v = _randn(gen, total, dev, 1e-3).square_().add_(1e-8) * inside
        state.update(param=param, params=views(param), decay=[d for _, d in sizes], lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, step=100 + int(seed) % 50,
                     seed=int(seed) % (1 << 40), master_flat=None, scale=None)
        if case["master"]:      # the weights are the rounded master copy
            state["master_flat"] = param.float() + _randn(gen, total, dev, 1e-5) * inside
            param.copy_(state["master_flat"])
        if case["clip"]:        # what the global norm of the step left: the norm and the factor of the gradient
            state["scale"] = torch.tensor([2.0 + (int(seed) % 7), 1.0 / (2.0 + (int(seed) % 7))], dtype=torch.float32, device=dev)
        if case["bits"] == 8:
            state["m"], state["m_scale"] = _nearest(m)
            state["v"], state["v_scale"] = _nearest(v)
        else:
            state["m"], state["v"] = m, v
        del m, v, inside
        if own:
            from paper_1806_04090_b200 import api
            state["ctx"] = _context()
            split = lambda flat: [flat[s // BLOCK: (s + n + BLOCK - 1) // BLOCK] for s, n in zip(starts, lengths)]  # noqa: E731
            more = {"exp_avg_scale": split(state["m_scale"]), "exp_avg_sq_scale": split(state["v_scale"])} if case["bits"] == 8 else {}
            state["opt"] = api.AdamWState(state["params"], views(state["m"]), views(state["v"]),
                                          master=views(state["master_flat"]) if case["master"] else None, weight_decay=state["decay"], **more)
        return state
    if op == "embedding":
        kind = TYPES[case["type"]]
        cdf = torch.cumsum(_zipf(case, dev), 0).to(torch.float64)
        rank = torch.searchsorted(cdf, torch.rand(case["tokens"], generator=gen, device=dev, dtype=torch.float64)).clamp_(max=case["vocab"] - 1)
        state["id"] = torch.randperm(case["vocab"], generator=gen, device=dev)[rank].to(TYPES[case["ids"]])
        state["table"] = _randn(gen, case["vocab"] * case["width"], dev, 0.02).to(kind).view(case["vocab"], case["width"])
        state["factor"] = math.sqrt(case["width"])      # embeddings are scaled by the root of their width
        if case["train"]:
            state["dout"] = _randn(gen, case["tokens"] * case["width"], dev, 1e-3).to(kind).view(case["tokens"], case["width"])
    else:
        kind = TYPES[case["type"]]
        rows, width = case["rows"], case["width"]
        # activations of a residual stream: an offset for each row, some channels far above the others
        x = _randn(gen, rows * width, dev).view(rows, width)
        x[:, ::61] *= 8.0
        x += _randn(gen, rows, dev, 0.5)[:, None]
        state.update(x=x.to(kind), weight=(1.0 + _randn(gen, width, dev, 0.1)).to(TYPES[case["weight"]]),
                     bias=_randn(gen, width, dev, 0.1).to(TYPES[case["weight"]]), eps=1e-5)
        if case["train"]:
            state["dy"] = _randn(gen, rows * width, dev, 1e-3).to(kind).view(rows, width)
    if own:
        state["ctx"] = _context()
    return state


# ---- plain forms --------------------------------------------------------------------------------
def _philox(block, tensor, step, seed):
    """The four words of each block of four elements (int64 tensors that hold 32 bits), as a tensor (blocks, 4)."""
    low = 0xFFFFFFFF
    x, y, z, w = block & low, (block >> 32) | 0x80000000, tensor, torch.full_like(block, step & 0x7FFFFFFF)
    k0, k1 = seed & low, (seed >> 32) & low
    for r in range(10):
        a, b = x * 0xD2511F53, z * 0xCD9E8D57       # the low 64 bits of the products, which is all of them
        x, y, z, w = ((b >> 32) & low) ^ y ^ ((k0 + r * 0x9E3779B9) & low), b & low, ((a >> 32) & low) ^ w ^ ((k1 + r * 0xBB67AE85) & low), a & low
    return torch.stack([x, y, z, w], 1)


def _round8(x, random16, codes, scale, keep):
    """Stochastic rounding of a state to e4m3 with a power of two for each block; `keep`: what is above zero stays above zero."""
    mag = x.abs()
    finite = mag < math.inf
    top = torch.where(finite, mag, 0.0).view(-1, BLOCK).amax(1)
    byte = (((top.view(torch.int32) + 0x200000) >> 23) - 8).clamp_(min=0)
    inverse = ((254 - byte) << 23).view(torch.float32)
    # times 2^-120, e4m3's exponent field is that of fp32, subnormal numbers included: its code is the upper 12 bits
    u = (mag.view(-1, BLOCK) * inverse[:, None]).view(-1) * 2.0 ** -120
    code = (u.view(torch.int32) + (random16 << 4)) >> 20
    if keep:
        code = torch.where(mag > 0, code.clamp(min=1), code)
    code = torch.where(finite, code, 0x7F) | torch.where(x < 0, 0x80, 0)
    codes.view(torch.uint8).copy_(code)
    scale.view(torch.uint8).copy_(byte)


def _plain_adamw(s):
    dev = s["grad"].device
    counts = torch.tensor([-(-n // BLOCK) * BLOCK for n in s["lengths"]], device=dev)
    decay = torch.repeat_interleave(torch.tensor(s["decay"], dtype=torch.float32, device=dev), counts)
    g = s["grad"].float()
    if s["scale"] is not None:
        g = g * s["scale"][1]
    if s["bits"] == 8:
        m = s["m"].float() * torch.repeat_interleave(_pow2(s["m_scale"].view(torch.uint8).int()), BLOCK)
        v = s["v"].float() * torch.repeat_interleave(_pow2(s["v_scale"].view(torch.uint8).int()), BLOCK)
    else:
        m, v = s["m"], s["v"]
    m = s["beta1"] * m + (1.0 - s["beta1"]) * g
    v = s["beta2"] * v + (1.0 - s["beta2"]) * g * g
    p = s["param"].float() if s["master_flat"] is None else s["master_flat"]
    t = s["step"]
    p = p - s["lr"] * decay * p - s["lr"] / (1.0 - s["beta1"] ** t) * m / (v.sqrt() / math.sqrt(1.0 - s["beta2"] ** t) + s["eps"])
    if s["bits"] == 8:
        quads = counts // 4
        tensor = torch.repeat_interleave(torch.arange(len(s["lengths"]), device=dev), quads)
        block = torch.arange(s["total"] // 4, device=dev) - torch.repeat_interleave(torch.tensor(s["starts"], device=dev) // 4, quads)
        words = _philox(block, tensor, t, s["seed"]).view(-1)
        _round8(m, (words & 0xFFFF).int(), s["m"], s["m_scale"], False)
        _round8(v, (words >> 16).int(), s["v"], s["v_scale"], True)
    else:
        s["m"].copy_(m)
        s["v"].copy_(v)
    if s["master_flat"] is not None:
        s["master_flat"].copy_(p)
    s["param"].copy_(p)


def _adamw_outputs(s):
    out = {"param": s["param"], "m": s["m"], "v": s["v"]}
    if s["bits"] == 8:
        out.update(m_scale=s["m_scale"], v_scale=s["v_scale"])
    if s["master_flat"] is not None:
        out["master"] = s["master_flat"]
    return out


def _plain_layernorm(s):
    x = s["x"].float()
    mean = x.mean(1)
    centred = x - mean[:, None]
    rstd = 1.0 / (centred.square().mean(1) + s["eps"]).sqrt()
    hat = centred * rstd[:, None]
    w = s["weight"].float()
    out = {"y": (hat * w + s["bias"].float()).to(s["x"].dtype), "mean": mean, "rstd": rstd}
    if s["train"]:
        dy = s["dy"].float()
        u = dy * w
        dx = rstd[:, None] * (u - u.mean(1, keepdim=True) - hat * (u * hat).mean(1, keepdim=True))
        out.update(dx=dx.to(s["x"].dtype), dweight=(dy * hat).sum(0), dbias=dy.sum(0))
    return out


def _plain_embedding(s):
    out = {"out": (s["table"][s["id"]].float() * s["factor"]).to(s["table"].dtype)}
    if s["train"]:
        dtable = torch.zeros(s["vocab"], s["width"], dtype=torch.float32, device=s["id"].device)
        out["dtable"] = dtable.index_add_(0, s["id"], s["dout"].float() * s["factor"])
    return out


def run(state):
    s, op = state, state["op"]
    if op == "norm":
        if own:
            return s["ctx"].atomo_grad_norm(s["grads"], max_norm=s["max_norm"])
        norm = s["grad"].double().square_().sum().sqrt_()       # 64 bits: a sum of a hundred million squares
        return torch.stack([norm, (s["max_norm"] / (norm + 1e-6)).clamp(max=1.0)]).float()
    if op == "adamw":
        if own:
            s["ctx"].atomo_adamw(s["opt"], s["grads"], lr=s["lr"], step=s["step"], beta1=s["beta1"], beta2=s["beta2"], eps=s["eps"], seed=s["seed"], scale=s["scale"])
        else:
            _plain_adamw(s)
        s["step"] += 1
        return _adamw_outputs(s)
    if op == "embedding":
        if not own:
            return _plain_embedding(s)
        out = {"out": s["ctx"].atomo_embedding(s["table"], s["id"], scale=s["factor"])}
        if s["train"]:
            out["dtable"] = s["ctx"].atomo_embedding_backward(s["id"], s["dout"], s["vocab"], scale=s["factor"])
        return out
    if not own:
        return _plain_layernorm(s)
    y, mean, rstd = s["ctx"].atomo_layer_norm(s["x"], s["weight"], s["bias"], eps=s["eps"])
    out = {"y": y, "mean": mean, "rstd": rstd}
    if s["train"]:
        out["dx"], out["dweight"], out["dbias"] = s["ctx"].atomo_layer_norm_backward(s["dy"], s["x"], s["weight"], mean, rstd)
    return out


# ---- 64 bits ------------------------------------------------------------------------------------
def _mul32(a, b):
    """High and low 32 bits of the product of two 32-bit numbers, from 16-bit halves."""
    a0, a1, b0, b1 = a & 0xFFFF, a >> 16, b & 0xFFFF, b >> 16
    mid = a1 * b0 + ((a0 * b0) >> 16)
    mid2 = a0 * b1 + (mid & 0xFFFF)
    return a1 * b1 + (mid >> 16) + (mid2 >> 16), ((mid2 & 0xFFFF) << 16) | ((a0 * b0) & 0xFFFF)


def _exact_words(n, tensor, step, seed, dev):
    """One Philox4x32-10 word for each of a tensor's n elements."""
    block = torch.arange(-(-n // 4), dtype=torch.int64, device=dev)
    c = [block & 0xFFFFFFFF, torch.full_like(block, 1 << 31) | (block >> 32), torch.full_like(block, tensor), torch.full_like(block, step)]
    key = [seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF]
    for _ in range(10):
        h0, l0 = _mul32(c[0], 0xD2511F53)
        h1, l1 = _mul32(c[2], 0xCD9E8D57)
        c = [h1 ^ c[1] ^ key[0], l1, h0 ^ c[3] ^ key[1], l0]
        key = [(key[0] + 0x9E3779B9) & 0xFFFFFFFF, (key[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return torch.stack(c, 1).reshape(-1)[:n]


def _exact_state(x, random16, keep):
    """Codes (the numbers that they stand for) and the exponents of a tensor's blocks: x / 2^e on the grid of e4m3, up with probability of the remainder."""
    n = x.numel()
    pad = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK)).view(-1, BLOCK)
    top = pad.amax(1)
    # the power of two that brings the largest into (224, 448]
    e = torch.where(top > 0, torch.floor(torch.log2(top.clamp(min=1e-300) / 1.75)) + 1 - 8, torch.full_like(top, -127.0))
    e = torch.where(top >= 1.75 * 2.0 ** (e + 8), e + 1, e).clamp(min=-127.0)
    y = (pad / 2.0 ** e[:, None]).view(-1)[:n]
    quantum = 2.0 ** (torch.floor(torch.log2(y.clamp(min=2.0 ** -6))) - 3)
    up = torch.floor(y / quantum + random16.double() / 65536.0) * quantum
    if keep:
        up = torch.where(y > 0, up.clamp(min=2.0 ** -9), up)
    return torch.copysign(up, x), 2.0 ** e


def _exact_adamw(case, s):
    dev = s["grad"].device
    names = ["param", "m", "v"] + (["m_scale", "v_scale"] if s["bits"] == 8 else [])
    out = {k: [] for k in names}
    gs = 1.0 if s["scale"] is None else s["scale"][1].double()
    weight = s["param"] if s["master_flat"] is None else s["master_flat"]
    for i, (start, n) in enumerate(zip(s["starts"], s["lengths"])):
        at = slice(start, start + n)
        blocks = slice(start // BLOCK, (start + n + BLOCK - 1) // BLOCK)
        g = s["grad"][at].double() * gs
        m, v = s["m"][at].double(), s["v"][at].double()
        if s["bits"] == 8:
            m = m * torch.repeat_interleave(2.0 ** (s["m_scale"].view(torch.uint8)[blocks].double() - 127), BLOCK)[:n]
            v = v * torch.repeat_interleave(2.0 ** (s["v_scale"].view(torch.uint8)[blocks].double() - 127), BLOCK)[:n]
        m = torch.lerp(g, m, s["beta1"])
        v = torch.lerp(g * g, v, s["beta2"])
        hat_m, hat_v = m / (1 - s["beta1"] ** s["step"]), v / (1 - s["beta2"] ** s["step"])
        p = weight[at].double() * (1 - s["lr"] * s["decay"][i]) - s["lr"] * hat_m / (torch.sqrt(hat_v) + s["eps"])
        got = {"param": p, "m": m, "v": v}
        if s["bits"] == 8:
            words = _exact_words(n, i, s["step"], s["seed"], dev)
            got["m"], got["m_scale"] = _exact_state(m, words & 0xFFFF, False)
            got["v"], got["v_scale"] = _exact_state(v, words >> 16, True)
        for k in names:
            out[k].append(torch.nn.functional.pad(got[k], (0, 0 if k.endswith("scale") else -n % BLOCK)))
    out = {k: torch.cat(x) for k, x in out.items()}
    if s["master_flat"] is not None:
        out["master"] = out["param"]
    return out


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        norm = torch.linalg.vector_norm(s["grad"].double())
        return torch.stack([norm, torch.minimum(s["max_norm"] / (norm + 1e-6), torch.ones_like(norm))])
    if op == "adamw":
        return _exact_adamw(case, s)
    if op == "embedding":
        out = {"out": torch.index_select(s["table"], 0, s["id"].long()).double() * s["factor"]}
        if s["train"]:
            # rows in the order of their tokens; a token's sum is a difference of running sums
            order = torch.argsort(s["id"].long(), stable=True)
            ends = torch.cumsum(torch.bincount(s["id"].long(), minlength=case["vocab"]), 0)
            parts = []
            for c in range(0, case["width"], 256):
                run_sum = torch.cumsum(torch.cat([torch.zeros_like(s["dout"][:1, c:c + 256]), s["dout"][order, c:c + 256]]).double(), 0)
                total = run_sum[ends]
                parts.append(torch.diff(total, dim=0, prepend=torch.zeros_like(total[:1])))
            out["dtable"] = torch.cat(parts, 1) * s["factor"]
        return out
    x = s["x"].double().requires_grad_(s["train"])
    w, b = s["weight"].double().requires_grad_(s["train"]), s["bias"].double().requires_grad_(s["train"])
    var, mean = torch.var_mean(x, dim=1, correction=0)
    rstd = torch.rsqrt(var + s["eps"])
    y = (x - mean[:, None]) * (rstd[:, None] * w) + b
    out = {"y": y.detach(), "mean": mean.detach(), "rstd": rstd.detach()}
    if s["train"]:
        out["dx"], out["dweight"], out["dbias"] = torch.autograd.grad(y, (x, w, b), s["dy"].double())
    return out


# ---- what a pass cannot do without ----------------------------------------------------------------
def work(case):
    op = case["op"]
    if op == "norm":
        n = float(sum(n for n, _ in _lengths(case)))
        return {"bytes": n * BYTES[case["grad"]] + 8.0, "flops": 2.0 * n}
    if op == "adamw":
        n = float(sum(n for n, _ in _lengths(case)))
        state = 4.0 * (1.0 + 1.0 / BLOCK) if case["bits"] == 8 else 16.0
        weight = 8.0 + BYTES[case["param"]] if case["master"] else 2.0 * BYTES[case["param"]]
        return {"bytes": n * (BYTES[case["grad"]] + state + weight), "flops": 15.0 * n}
    if op == "embedding":
        t, d, size = float(case["tokens"]), float(case["width"]), BYTES[case["type"]]
        seen = float((1.0 - (1.0 - _zipf(case, "cpu")) ** t).sum())       # distinct tokens, on average
        moved = t * BYTES[case["ids"]] + (seen + t) * d * size
        if case["train"]:
            moved += t * BYTES[case["ids"]] + t * d * size + 4.0 * case["vocab"] * d
        return {"bytes": moved, "flops": t * d * (3.0 if case["train"] else 1.0)}
    n, size, wide = float(case["rows"]) * case["width"], BYTES[case["type"]], BYTES[case["weight"]]
    moved = 2.0 * n * size + 2.0 * case["width"] * wide + 8.0 * case["rows"]
    if case["train"]:
        moved += 3.0 * n * size + case["width"] * wide + 8.0 * case["width"] + 8.0 * case["rows"]
    return {"bytes": moved, "flops": (18.0 if case["train"] else 7.0) * n}
