"""Workloads of the operators over tensors held in few bits with a scale per group.

Three operators that follow one another in use: an AdamW step over all tensors of a model (binary32 or 8-bit state,
stochastically rounded low-precision weights), the rounding of weight matrices to 4 bits with group scales, and the
product of activations with such weights.  ``listed`` and ``draw`` give the cases, ``prepare`` a case's inputs, ``run``
one pass: the library's calls where ``own`` is true, elementary torch operations in binary32 where it is false.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
HYPER = dict(lr=1e-4, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=10)
FLOAT = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
SIZE = {"fp32": 4, "bf16": 2, "fp16": 2}
LP = {"bf16": (8, -126, 3.3895313892515355e38), "fp16": (11, -14, 65504.0)}       # precision, emin, largest value
BLOCK = 256                                                                       # elements that share a state scale


# ------------------------------------------------------------------------------------------------ cases
def listed():
    return [
        # one transformer block of the fused-optimizer configuration, binary32 moments and gradients
        dict(name="adamw32_block", op="adamw", sizes="block", bits=32, grad="fp32", lp="bf16", variant="srf", k=4),
        # low-rank adapters and biases: many small tensors of odd sizes, 16-bit gradients
        dict(name="adamw32_adapters", op="adamw", sizes="ragged", count=190, largest=70001, bits=32, grad="bf16", lp="bf16", variant="src", k=3),
        # the same block with 8-bit state, gradients as the backward pass leaves them
        dict(name="adamw8_block", op="adamw", sizes="block", bits=8, grad="bf16", lp="bf16", variant="srf", k=4),
        # a small model's tensors with 8-bit state: launches count
        dict(name="adamw8_small", op="adamw", sizes="ragged", count=48, largest=5000, bits=8, grad="fp16", lp="fp16", variant="srff", k=8),
        # binary32 master weights of a block's wide matrix to 4 bits, power-of-two scales
        dict(name="round4_wide", op="round4", rows=4096, cols=11008, src="fp32", group=32, scale="e8m0", variant="srf", k=4),
        # a fine-tuned bf16 matrix of odd shape, coarse groups with bf16 scales
        dict(name="round4_odd", op="round4", rows=1531, cols=2049, src="bf16", group=128, scale="bf16", variant="src", k=3),
        # one adapter matrix: latency
        dict(name="round4_small", op="round4", rows=64, cols=1024, src="fp16", group=64, scale="bf16", variant="rtne", k=1),
        # one token through a block's square projection
        dict(name="gemv4_square", op="gemv4", m=1, n=4096, k=4096, x="bf16", out="bf16", group=32, scale="e8m0"),
        # one token through the narrowing matrix, coarse groups
        dict(name="gemv4_down", op="gemv4", m=1, n=4096, k=11008, x="fp16", out="fp16", group=128, scale="bf16"),
        # a small batch of tokens through the widening matrix
        dict(name="gemv4_batch8", op="gemv4", m=8, n=11008, k=4096, x="bf16", out="bf16", group=64, scale="bf16"),
        # one token's logits over a large vocabulary, binary32 result
        dict(name="gemv4_vocabulary", op="gemv4", m=1, n=128000, k=4096, x="bf16", out="fp32", group=32, scale="e8m0"),
        # odd everything: a pruned layer
        dict(name="gemv4_odd", op="gemv4", m=3, n=777, k=1001, x="fp16", out="fp16", group=32, scale="bf16"),
    ]


def _log_uniform(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    op = rng.choice(["adamw", "adamw", "round4", "gemv4", "gemv4"])
    variant = rng.choice(["srff", "srf", "src", "rtne"])
    if op == "adamw":
        return dict(op=op, sizes="ragged", count=_log_uniform(rng, 1, 400), largest=_log_uniform(rng, 300, 120000),
                    bits=rng.choice([32, 8]), grad=rng.choice(["fp32", "bf16", "fp16"]), lp=rng.choice(["bf16", "fp16"]),
                    variant=variant, k=rng.choice([1, 2, 3, 4, 8]))
    if op == "round4":
        return dict(op=op, rows=_log_uniform(rng, 1, 5000), cols=_log_uniform(rng, 33, 9000), src=rng.choice(["fp32", "bf16", "fp16"]),
                    group=rng.choice([32, 64, 128]), scale=rng.choice(["e8m0", "bf16"]), variant=variant, k=rng.choice([1, 2, 3, 4, 8]))
    x = rng.choice(["bf16", "fp16"])
    return dict(op=op, m=_log_uniform(rng, 1, 32), n=_log_uniform(rng, 17, 20000), k=_log_uniform(rng, 64, 16000), x=x,
                out=rng.choice([x, "fp32"]), group=rng.choice([32, 64, 128]), scale=rng.choice(["e8m0", "bf16"]))


def _tensor_sizes(case):
    """Element counts of the tensors of an AdamW case."""
    if case["sizes"] == "block":
        return [4096 * 4096, 4096 * 11008, 4096, 4096]
    count, largest = case["count"], case["largest"]
    # a fixed spread from 1 element to `largest`, mostly odd
    return [1 + (largest - 1) * ((7 * i * i + 3 * i) % 97) // 96 for i in range(count)]


def _starts(sizes):
    """Where each tensor begins in the flat buffers: whole blocks apart."""
    at, starts = 0, []
    for n in sizes:
        starts.append(at)
        at += -(-n // BLOCK) * BLOCK
    return starts, at


def work(case):
    if case["op"] == "adamw":
        n = sum(_tensor_sizes(case))
        state = 16 if case["bits"] == 32 else 4 + 16.0 / BLOCK
        return {"bytes": n * (8 + SIZE[case["grad"]] + state + 2), "flops": 14 * n}
    if case["op"] == "round4":
        n = case["rows"] * case["cols"]
        scales = n // case["group"] * (1 if case["scale"] == "e8m0" else 2)
        return {"bytes": n * (2 * SIZE[case["src"]] + 0.5) + scales, "flops": 2 * n}
    m, n, k = case["m"], case["n"], case["k"]
    scales = n * -(-k // case["group"]) * (1 if case["scale"] == "e8m0" else 2)
    return {"bytes": n * k / 2 + scales + 2 * m * k + m * n * SIZE[case["out"]], "flops": 2 * m * n * k}


# ------------------------------------------------------------------------------------------------ inputs
def _generator(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _prepare_adamw(case, seed):
    sizes = _tensor_sizes(case)
    starts, total = _starts(sizes)
    gen = _generator(seed)
    normal = lambda s: torch.randn(total, device=DEV, generator=gen) * s  # noqa: E731
    real = torch.zeros(total, dtype=torch.bool, device=DEV)           # false between one tensor's end and the next one's start
    for a, n in zip(starts, sizes):
        real[a:a + n] = True
    w = normal(0.02) * real
    g = (normal(1e-3) * real).to(FLOAT[case["grad"]])
    m = normal(3e-4) * real
    r = normal(1e-3).abs() * real                                      # root of the second moment
    s = dict(case=case, w=w, g=g, lp=torch.zeros(total, dtype=FLOAT[case["lp"]], device=DEV), seed=seed)
    if case["bits"] == 32:
        s.update(m=m, v=r * r)
    else:
        for name, x in (("m", m), ("v", r)):
            scale = (x.view(-1, BLOCK).abs().amax(1) / 448).clamp_min(2.0 ** -126)
            s[name] = (x.view(-1, BLOCK) / scale[:, None]).clamp(-448, 448).to(torch.float8_e4m3fn).view(-1)
            s[name + "_scale"] = scale
    if own:
        import paper_2504_20634_b200 as fbsr
        part = lambda t: [t[a:a + n] for a, n in zip(starts, sizes)]  # noqa: E731
        more = {}
        if case["bits"] == 8:
            more = {q: [s[q][a // BLOCK:(a + n + BLOCK - 1) // BLOCK] for a, n in zip(starts, sizes)] for q in ("m_scale", "v_scale")}
        s["table"] = fbsr.FbsrAdamwTensors(part(w), part(g), part(s["m"]), part(s["v"]), part(s["lp"]), offsets=starts,
                                           fmt=case["lp"], **more)
    return s


def _prepare_round4(case, seed):
    gen = _generator(seed)
    x = torch.randn(case["rows"], case["cols"], device=DEV, generator=gen) * 0.02
    x = x * torch.exp2(torch.randn(case["rows"], 1, device=DEV, generator=gen))    # rows of different size, as trained weights have
    return dict(case=case, x=x.to(FLOAT[case["src"]]), seed=seed)


def _prepare_gemv4(case, seed):
    """Weights as the rounding leaves them: normally distributed values on the 4-bit grid, scales around 2^-8."""
    gen = _generator(seed)
    m, n, k, group = case["m"], case["n"], case["k"], case["group"]
    blocks = -(-k // 128)
    codes = torch.empty(n, blocks * 64, dtype=torch.uint8, device=DEV)
    lut = _codes_of_normal()
    step = max(1, (1 << 25) // codes.shape[1])
    for a in range(0, n, step):
        part = codes[a:a + step]
        part.copy_(lut[torch.randint(0, lut.numel(), part.shape, device=DEV, generator=gen)])
    canonical = _swap_words(codes)                                     # nothing beyond column k
    canonical[:, (k + 1) // 2:] = 0
    if k % 2:
        canonical[:, k // 2] &= 0x0F
    codes = _swap_words(canonical).contiguous()
    groups = blocks * 128 // group
    if case["scale"] == "e8m0":
        scales = torch.randint(117, 121, (n, groups), device=DEV, generator=gen).to(torch.uint8)
    else:
        scales = (torch.rand(n, groups, device=DEV, generator=gen) + 0.5).mul_(2.0 ** -8).to(torch.bfloat16)
    x = torch.randn(m, k, device=DEV, generator=gen).to(FLOAT[case["x"]])
    return dict(case=case, x=x, codes=codes, scales=scales)


def _codes_of_normal():
    """4096 bytes, each two 4-bit codes, in the proportions that normally distributed values have after rounding."""
    edges = torch.tensor([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0])
    q = (torch.arange(64) + 0.5) / 64
    z = torch.erfinv(2 * q - 1) * math.sqrt(2.0) * 2.2
    code = torch.bucketize(z.abs(), edges) + 8 * (z < 0)
    return (code[:, None] + 16 * code[None, :]).reshape(-1).to(torch.uint8).to(DEV)


def prepare(case, seed):
    return {"adamw": _prepare_adamw, "round4": _prepare_round4, "gemv4": _prepare_gemv4}[case["op"]](case, seed)


# ------------------------------------------------------------------------------------------------ plain forms
def _swap_words(codes):
    """Stored order <-> plain order of 4-bit rows: in each 64 bytes (128 elements) the sixteen 32-bit words lie as the
    transpose of a 4 x 4 square.  Its own inverse."""
    rows, pitch = codes.shape
    return codes.reshape(rows, pitch // 64, 4, 4, 4).transpose(2, 3).reshape(rows, pitch)


def _philox(calls, stream, seed):
    """Philox4x32-10 of the counters (call lo, call hi, stream, 0): [calls, 4] words in int64."""
    low = 0xFFFFFFFF
    c = [calls & low, (calls >> 32) & low, torch.full_like(calls, stream), torch.zeros_like(calls)]
    k0, k1 = seed & low, (seed >> 32) & low
    for _ in range(10):
        p0, p1 = c[0] * 0xD2511F53, c[2] * 0xCD9E8D57                  # the products wrap; their 64 bits are right
        c = [((p1 >> 32) & low) ^ c[1] ^ k0, p1 & low, ((p0 >> 32) & low) ^ c[3] ^ k1, p0 & low]
        k0, k1 = (k0 + 0x9E3779B9) & low, (k1 + 0xBB67AE85) & low
    return torch.stack(c, 1)


def _draws(n, k, seed):
    """k random bits for each of the elements 0 .. n - 1."""
    per_word = 32 // k
    calls = torch.arange(-(-n // (4 * per_word)), device=DEV)
    words = _philox(calls, 0, seed)
    fields = (words[:, :, None] >> (torch.arange(per_word, device=DEV) * k)) & ((1 << k) - 1)
    return fields.reshape(-1)[:n].float()


def _state_draws(n, k, seed):
    """The bits of the two state roundings: 16 bits an element, eight elements a call; low byte, high byte."""
    words = _philox(torch.arange(n // 8, device=DEV), 1, seed)
    halves = torch.stack([words & 0xFFFF, words >> 16], 2).reshape(-1)
    mask = (1 << k) - 1
    return (halves & mask).float(), ((halves >> 8) & mask).float()


def _times_power(a, e):
    half = torch.div(e, 2, rounding_mode="floor")
    return a * torch.exp2(half.float()) * torch.exp2((e - half).float())


def _few_bit_round(y, n, precision, emin, largest, variant, k):
    """The value that y is rounded to: magnitude on the format's grid, round-up decided by the k-bit draw n."""
    a = y.abs()
    e = (torch.frexp(a)[1] - 1).clamp_min(emin)
    sigma = _times_power(a, precision - 1 - e)
    down = torch.floor(sigma)
    delta = sigma - down
    if variant == "srff":
        up = torch.floor(delta * 2.0 ** k) + n >= 2.0 ** k
    elif variant == "srf":
        up = torch.floor(delta * 2.0 ** (k + 1)) + 2 * n + 1 >= 2.0 ** (k + 1)
    elif variant == "src":
        up = torch.round(delta * 2.0 ** k) + n >= 2.0 ** k
    else:
        up = torch.round(sigma) > down
    v = _times_power(down + up, e - (precision - 1)).clamp_max(largest)
    return torch.copysign(v, y)


def _host_scalars():
    b1t, b2t = HYPER["beta1"] ** HYPER["step"], HYPER["beta2"] ** HYPER["step"]
    return HYPER["lr"] / (1 - b1t), 1 / math.sqrt(1 - b2t), 1 - HYPER["beta1"], 1 - HYPER["beta2"]


def _run_adamw(s):
    case = s["case"]
    c1, c2, a1, a2 = _host_scalars()
    g = s["g"].float()
    if case["bits"] == 32:
        m, v = s["m"], s["v"]
    else:
        m = (s["m"].float().view(-1, BLOCK) * s["m_scale"][:, None]).view(-1)
        r = (s["v"].float().view(-1, BLOCK) * s["v_scale"][:, None]).view(-1)
        v = r * r
    m = HYPER["beta1"] * m + a1 * g
    v = HYPER["beta2"] * v + (a2 * g) * g
    r = torch.sqrt(v)
    w = s["w"] * (1 - HYPER["lr"] * HYPER["weight_decay"]) - c1 * (m / (r * c2 + HYPER["eps"]))
    n = w.numel()
    variant, k = case["variant"], case["k"]
    draws = None if variant == "rtne" else _draws(n, k, s["seed"])
    s["w"].copy_(w)
    s["lp"].copy_(_few_bit_round(w, draws, *LP[case["lp"]], variant, k))
    if case["bits"] == 32:
        s["m"].copy_(m)
        s["v"].copy_(v)
        return {q: s[q] for q in ("w", "lp", "m", "v")}
    dm, dr = (None, None) if variant == "rtne" else _state_draws(n, k, s["seed"])
    for name, x, d in (("m", m, dm), ("v", r, dr)):
        scale = (x.view(-1, BLOCK).abs().amax(1) / 448).clamp_min(2.0 ** -126)
        y = (x.view(-1, BLOCK) * (1 / scale)[:, None]).view(-1)
        code = _few_bit_round(y, d, 4, -6, 448.0, variant, k)
        if name == "v":
            code = torch.where((x > 0) & (code == 0), 2.0 ** -9, code)     # a positive root never becomes zero
        s[name].copy_(code)
        s[name + "_scale"].copy_(scale)
    return {q: s[q] for q in ("w", "lp", "m", "v", "m_scale", "v_scale")}


def _largest_scale(src):
    """The largest bf16 whose sixfold is finite in the source's type."""
    return {"fp32": 2.0 ** 125 * 1.328125, "bf16": 2.0 ** 125 * 1.328125, "fp16": 10880.0}[src]


def _run_round4(s):
    case, x = s["case"], s["x"].float()
    rows, cols, group = case["rows"], case["cols"], case["group"]
    padded = -(-cols // 128) * 128
    x = torch.nn.functional.pad(x, (0, padded - cols)).view(rows, padded // group, group)
    amax = x.abs().amax(2)
    if case["scale"] == "e8m0":
        e = (torch.frexp(amax)[1] - 3).clamp(-127, 127)
        scale = torch.exp2(torch.where(amax < 2.0 ** -126, -127, e).float())
    else:
        up = ((amax / 6).view(torch.int32) + 0xFFFF) & ~0xFFFF
        scale = up.view(torch.float32).clamp(2.0 ** -126, _largest_scale(case["src"]))
    y = x * (1 / scale)[:, :, None]
    draws = None if case["variant"] == "rtne" else _draws(rows * padded, case["k"], s["seed"]).view(y.shape)
    v = _few_bit_round(y, draws, 2, 0, 6.0, case["variant"], case["k"]) * scale[:, :, None]
    return {"values": v.view(rows, padded)[:, :cols].to(s["x"].dtype), "scales": scale}


_GRID = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0)


def _weights(s, dtype):
    """The matrix that 4-bit codes and scales stand for, with its padding."""
    case, plain = s["case"], _swap_words(s["codes"])
    grid = torch.tensor(_GRID, dtype=dtype, device=DEV)
    pairs = torch.stack([grid.repeat(16), grid.repeat_interleave(16)], 1)          # both values of a byte
    w = pairs[plain.int()]
    scale = s["scales"].to(dtype)
    if case["scale"] == "e8m0":
        scale = torch.exp2(scale - 127)
    return (w.view(case["n"], -1, case["group"]) * scale[:, :, None]).view(case["n"], -1)


def _run_gemv4(s):
    case = s["case"]
    w = _weights(s, torch.float32)[:, :case["k"]]
    return (s["x"].float() @ w.T).to(FLOAT[case["out"]])


# ------------------------------------------------------------------------------------------------ the library's calls
def _own_adamw(s):
    import paper_2504_20634_b200 as fbsr
    case = s["case"]
    fbsr.fbsr_adamw_multi(s["table"], case["variant"], case["k"], s["seed"], **HYPER)
    return {q: s[q] for q in (("w", "lp", "m", "v") if case["bits"] == 32 else ("w", "lp", "m", "v", "m_scale", "v_scale"))}


def _own_round4(s):
    import paper_2504_20634_b200 as fbsr
    case = s["case"]
    values = torch.empty_like(s["x"])
    codes, scales = fbsr.fbsr_round_w4(s["x"], case["variant"], case["k"], s["seed"], group=case["group"], scale_fmt=case["scale"],
                                       values=values)
    # scales are compared as the values they stand for
    scales = torch.exp2(scales.float() - 127) if case["scale"] == "e8m0" else scales.float()
    return {"values": values, "scales": scales}


def _own_gemv4(s):
    import paper_2504_20634_b200 as fbsr
    case = s["case"]
    return fbsr.fbsr_gemv_w4(s["x"], s["codes"], s["scales"], group=case["group"], out_dtype=FLOAT[case["out"]])


def run(state):
    op = state["case"]["op"]
    if own:
        return {"adamw": _own_adamw, "round4": _own_round4, "gemv4": _own_gemv4}[op](state)
    return {"adamw": _run_adamw, "round4": _run_round4, "gemv4": _run_gemv4}[op](state)


# ------------------------------------------------------------------------------------------------ 64 bits
def _exact_draws(n, k, seed):
    """The draws once more, in numpy's unsigned arithmetic."""
    per_word = 32 // k
    calls = np.arange(-(-n // (4 * per_word)), dtype=np.uint64)
    low, sh = np.uint64(0xFFFFFFFF), np.uint64(32)
    x0, x1 = calls & low, calls >> sh
    x2, x3 = np.zeros_like(calls), np.zeros_like(calls)
    key0, key1 = seed & 0xFFFFFFFF, (seed >> 32) & 0xFFFFFFFF
    for _ in range(10):
        hi_lo_0, hi_lo_2 = x0 * np.uint64(0xD2511F53), x2 * np.uint64(0xCD9E8D57)
        x0, x1, x2, x3 = ((hi_lo_2 >> sh) ^ x1 ^ np.uint64(key0), hi_lo_2 & low,
                          (hi_lo_0 >> sh) ^ x3 ^ np.uint64(key1), hi_lo_0 & low)
        key0, key1 = (key0 + 0x9E3779B9) & 0xFFFFFFFF, (key1 + 0xBB67AE85) & 0xFFFFFFFF
    out = np.empty((calls.size, 4, per_word), dtype=np.float64)
    for w, word in enumerate((x0, x1, x2, x3)):
        for f in range(per_word):
            out[:, w, f] = (word >> np.uint64(f * k)) & np.uint64((1 << k) - 1)
    return torch.from_numpy(out.reshape(-1)[:n]).to(DEV)


def _exact_adamw(case, seed):
    s = _prepare_adamw(case, seed)
    g = s["g"].double()
    if case["bits"] == 32:
        m, v = s["m"].double(), s["v"].double()
    else:
        wide = lambda q: (s[q].double().view(-1, BLOCK) * s[q + "_scale"].double()[:, None]).view(-1)  # noqa: E731
        m, v = wide("m"), wide("v").square()
    # the scalars that the caller gives are binary32 numbers
    lr, b1, b2, eps, wd = (float(np.float32(HYPER[q])) for q in ("lr", "beta1", "beta2", "eps", "weight_decay"))
    t = HYPER["step"]
    m.mul_(b1).add_(g, alpha=1 - b1)
    v.mul_(b2).addcmul_(g, g, value=1 - b2)
    m_hat, v_hat = m / (1 - b1 ** t), v / (1 - b2 ** t)
    w = s["w"].double()
    w = w - lr * wd * w - lr * m_hat / (v_hat.sqrt() + eps)
    # the low-precision weights against the number that they round; 8-bit codes have no value in 64 bits
    if case["bits"] == 32:
        return {"w": w, "lp": w, "m": m, "v": v}
    top = lambda q: (q.view(-1, BLOCK).abs().amax(1) / 448).clamp_min(2.0 ** -126)  # noqa: E731
    return {"w": w, "lp": w, "m": None, "v": None, "m_scale": top(m), "v_scale": top(v.sqrt())}


def _exact_round4(case, seed):
    x = _prepare_round4(case, seed)["x"].double()
    rows, cols, group = case["rows"], case["cols"], case["group"]
    pad = -cols % 128
    x = torch.cat([x, torch.zeros(rows, pad, dtype=torch.float64, device=DEV)], 1).reshape(-1, group)
    amax = x.abs().amax(1, keepdim=True)
    if case["scale"] == "e8m0":
        scale = torch.where(amax > 0, torch.exp2(torch.floor(torch.log2(amax.clamp_min(1e-300))) - 2), 2.0 ** -127).clamp(2.0 ** -127, 2.0 ** 127)
    else:
        ulp = torch.exp2(torch.floor(torch.log2((amax / 6).clamp_min(2.0 ** -126))) - 7)
        scale = (torch.ceil(amax / 6 / ulp) * ulp).clamp(2.0 ** -126, _largest_scale(case["src"]))
    y = (x / scale).abs().clamp_max(6.0)
    grid = torch.tensor(_GRID[:8], dtype=torch.float64, device=DEV)
    at = (torch.searchsorted(grid, y, right=True) - 1).clamp(0, 6)                # neighbours on the grid
    lo, hi = grid[at], grid[at + 1]
    delta = (y - lo) / (hi - lo)
    k = case["k"]
    if case["variant"] == "rtne":
        up = (delta > 0.5) | ((delta == 0.5) & (at % 2 == 1))
    else:
        n = _exact_draws(x.numel(), k, seed).view_as(y)
        d = torch.round(delta * 2.0 ** k) * 2.0 ** -k if case["variant"] == "src" else delta
        up = d + (n + (0.5 if case["variant"] == "srf" else 0.0)) * 2.0 ** -k >= 1
    v = torch.where(up, hi, lo) * scale * torch.where(x < 0, -1.0, 1.0)
    return {"values": v.view(rows, -1)[:, :cols], "scales": scale.view(rows, -1)}


def _exact_gemv4(case, seed):
    s = _prepare_gemv4(case, seed)
    n, k, group = case["n"], case["k"], case["group"]
    words = s["codes"].view(torch.int32).view(n, -1, 4, 4).transpose(2, 3).reshape(n, -1)      # plain order, eight codes a word
    code = (words[:, :, None] >> (4 * torch.arange(8, device=DEV, dtype=torch.int32))) & 15
    code = code.view(n, -1)
    w = torch.tensor(_GRID, dtype=torch.float64, device=DEV)[code]
    scale = s["scales"].double()
    if case["scale"] == "e8m0":
        scale = 2.0 ** (scale - 127)
    w *= scale.repeat_interleave(group, 1)
    return torch.mm(s["x"].double(), w[:, :k].T)


def exact(case, seed):
    return {"adamw": _exact_adamw, "round4": _exact_round4, "gemv4": _exact_gemv4}[case["op"]](case, seed)
