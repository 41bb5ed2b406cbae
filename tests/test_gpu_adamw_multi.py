"""fbsr_adamw_multi: one AdamW step over many tensors, binary32 and 8-bit state.

Values are compared with the formulas in binary64; what is rounded to few bits is compared code by code with the oracle
applied to the values that were rounded.
"""
import ctypes

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

HYPER = dict(lr=1e-3, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.1, step=3)
EPS32 = 2.0 ** -24
SIZES = (1, 255, 256, 257, 1023, 1024, 1025, 5000, 8192, 70001)
GRAD = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    from oracle import capi
    import gpu_util
    module.fbsr, module.capi, module.gu = fbsr, capi, gpu_util


def make(sizes, seed, bits=32, grad="fp32", lp="bf16", misalign=0, fresh=False):
    """Tensors of the given sizes, `misalign` elements off their storage's start, and the table over them."""
    gen = torch.Generator(device="cuda").manual_seed(seed)

    def place(x):
        raw = torch.empty(x.numel() + misalign, dtype=x.dtype, device="cuda")
        raw[misalign:] = x
        return raw[misalign:]

    t = {k: [] for k in ("w", "g", "m", "v", "lp", "ms", "vs")}
    for n in sizes:
        z = torch.randn(4, max(n, 1), device="cuda", generator=gen)[:, :n]
        blocks = -(-n // 256)
        t["w"].append(place(z[0] * 0.02))
        t["g"].append(place((z[1] * 1e-2).to(GRAD[grad])))
        if bits == 32:
            t["m"].append(place(z[2] * (0 if fresh else 1e-3)))
            t["v"].append(place((z[3] * (0 if fresh else 1e-2)) ** 2))
        else:
            code = lambda x: x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8) * (0 if fresh else 1)  # noqa: E731
            t["m"].append(place(code(z[2] * 100)))
            t["v"].append(place(code(z[3].abs() * 100)))
            scale = torch.rand(2, max(blocks, 1), device="cuda", generator=gen)[:, :blocks] * (0 if fresh else 1)
            t["ms"].append((scale[0] * 1e-5).contiguous())
            t["vs"].append((scale[1] * 1e-4).contiguous())
        t["lp"].append(place(torch.zeros(n, dtype=fbsr.CODE_DTYPE[lp], device="cuda")))
    more = dict(m_scale=t["ms"], v_scale=t["vs"]) if bits == 8 else {}
    t["table"] = fbsr.FbsrAdamwTensors(t["w"], t["g"], t["m"], t["v"], t["lp"], fmt=lp, **more)
    return t


def offsets_of(sizes):
    out, at = [], 0
    for n in sizes:
        out.append(at)
        at += -(-n // 256) * 256
    return out


def host(x):
    if x.dtype in (torch.bfloat16, torch.float16):
        return x.float().cpu().numpy()
    return gu.to_np(x)


def scalars(h):
    b1, b2, lr = h["beta1"], h["beta2"], h["lr"]
    return lr / (1 - b1 ** h["step"]), 1 / np.sqrt(1 - b2 ** h["step"]), b1, b2, 1 - b1, 1 - b2, h["eps"], 1 - lr * h["weight_decay"]


def step64(w, g, m, v, h):
    """The step in binary64 from binary32 inputs, and a bound on what binary32 operations may be off: every product,
    sum, quotient and root has one rounding of 2^-24, every host scalar one more."""
    c1, c2, b1, b2, a1, a2, eps, decay = scalars(h)
    w, g, m, v = (np.asarray(x, dtype=np.float64) for x in (w, g, m, v))
    m1, v1 = b1 * m + a1 * g, b2 * v + a2 * g * g
    r = np.sqrt(v1)
    d = r * c2 + eps
    w1 = w * decay - c1 * m1 / d
    tiny = 2.0 ** -126
    em = EPS32 * (3 * np.abs(b1 * m) + 3 * np.abs(a1 * g)) + tiny      # the scalar, the product (unless fused), the sum
    ev = EPS32 * (3 * b2 * v + 4 * a2 * g * g) + tiny
    # root: half of v's relative error and its own; d: the product, c2 and the sum; then the quotient, c1 and the fma
    er = 0.5 * ev / np.maximum(r, 1e-150) + EPS32 * r
    ed = er * c2 + EPS32 * (3 * r * c2 + 2 * d)
    ew = c1 * (em / d + np.abs(m1) / d * (ed / d + 3 * EPS32)) + EPS32 * (3 * np.abs(w * decay) + np.abs(w1)) + tiny
    return (w1, m1, v1, r), (ew, em, ev, er)


def within(got, want, bound, what):
    off = np.abs(np.asarray(got, dtype=np.float64) - want)
    bad = ~(off <= 1.05 * bound)                 # 5 % for the second-order terms
    assert not bad.any(), "%s: %d of %d off, worst %g of the bound" % (what, bad.sum(), bad.size, np.nanmax(off / bound))


@pytest.mark.parametrize("variant,k", [("srff", 1), ("srf", 2), ("src", 3), ("srf", 4), ("srff", 5), ("src", 6), ("srf", 8),
                                       ("src", 9), ("srff", 10), ("srf", 13), ("src", 16), ("rtne", 4), ("rta", 1), ("rto", 1)])
@pytest.mark.parametrize("lp", ["bf16", "fp16", "e4m3", "e5m2", "b8p4"])
def test_binary32_state_is_the_single_tensor_step_bit_for_bit(variant, k, lp):
    """Without decay each tensor's step is the oracle's Adam step at the tensor's offset."""
    h = dict(HYPER, weight_decay=0.0)
    for q in ("lr", "beta1", "beta2", "eps"):                # that entry point takes binary32 scalars
        h[q] = float(np.float32(h[q]))
    t = make(SIZES, seed=5, lp=lp)
    before = [[host(x[i]).copy() for x in (t["w"], t["g"], t["m"], t["v"])] for i in range(len(SIZES))]
    fbsr.fbsr_adamw_multi(t["table"], variant, k, 77, **h)
    torch.cuda.synchronize()
    for i, off in enumerate(offsets_of(SIZES)):
        w, g, m, v = before[i]
        codes = capi.adam_update(w, g, m, v, lp, variant, k, 77, off, h["lr"], h["beta1"], h["beta2"], h["eps"], h["step"])
        for name, want in (("w", w), ("m", m), ("v", v)):
            assert np.array_equal(host(t[name][i]).view(np.uint32), want.view(np.uint32)), (name, i)
        gu.assert_codes_equal(t["lp"][i], codes, "lp of tensor %d" % i)


@pytest.mark.parametrize("grad", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("misalign", [0, 1])
@pytest.mark.parametrize("scaled", [False, True])
def test_binary32_state_against_binary64(grad, misalign, scaled):
    t = make(SIZES, seed=6, grad=grad, misalign=misalign)
    gs = torch.tensor([0.37], device="cuda") if scaled else None
    before = [[host(x[i]).copy() for x in (t["w"], t["g"], t["m"], t["v"])] for i in range(len(SIZES))]
    fbsr.fbsr_adamw_multi(t["table"], "srf", 4, 3, grad_scale=gs, **HYPER)
    torch.cuda.synchronize()
    for i, off in enumerate(offsets_of(SIZES)):
        w, g, m, v = before[i]
        if scaled:
            g = (g * np.float32(0.37)).astype(np.float32)
        want, bound = step64(w, g, m, v, HYPER)
        for q, name in enumerate(("w", "m", "v")):
            within(host(t[name][i]), want[q], bound[q], "%s of tensor %d" % (name, i))
        gu.assert_codes_equal(t["lp"][i], capi.fbsr_round(host(t["w"][i]), "bf16", "srf", 4, 3, offset=off), "lp %d" % i)


def state_words(seed, offset, n):
    out = np.empty(-(-n // 2) + 1, dtype=np.uint32)
    capi.lib().fbsr_oracle_random_words(seed, offset // 2, out.size, 1, ctypes.c_void_p(out.ctypes.data))
    return out.view(np.uint16)[:n]


def packed_fields(n, k):
    """Draws n packed as the supplied-bits entry point of the oracle wants them."""
    dpw = 32 // k
    words = np.zeros(-(-n.size // dpw), dtype=np.uint32)
    for f in range(dpw):
        part = n[f::dpw].astype(np.uint32) << np.uint32(f * k)
        words[:part.size] |= part
    return words


@pytest.mark.parametrize("variant,k", [("srff", 1), ("srf", 4), ("src", 3), ("srf", 8), ("src", 7), ("rtne", 4), ("rta", 16), ("rto", 2)])
@pytest.mark.parametrize("grad,misalign", [("fp32", 0), ("bf16", 0), ("fp16", 3)])
def test_8bit_state_codes_and_scales(variant, k, grad, misalign):
    t = make(SIZES, seed=8, bits=8, grad=grad, misalign=misalign)
    before = [[host(x[i]).copy() for x in (t["w"], t["g"], t["m"], t["v"], t["ms"], t["vs"])] for i in range(len(SIZES))]
    fbsr.fbsr_adamw_multi(t["table"], variant, k, 21, **HYPER)
    torch.cuda.synchronize()
    f = np.float32
    b1, b2, a1, a2 = f(HYPER["beta1"]), f(HYPER["beta2"]), f(1 - HYPER["beta1"]), f(1 - HYPER["beta2"])
    for i, (n, off) in enumerate(zip(SIZES, offsets_of(SIZES))):
        w, g, cm, cv, ms, vs = before[i]
        rep = lambda s: np.repeat(s, 256)[:n]  # noqa: E731
        m = capi.decode_array("e4m3", cm) * rep(ms)
        root = capi.decode_array("e4m3", cv) * rep(vs)
        v = root * root
        want, bound = step64(w, g, m, v, HYPER)
        within(host(t["w"][i]), want[0], bound[0], "w of tensor %d" % i)
        gu.assert_codes_equal(t["lp"][i], capi.fbsr_round(host(t["w"][i]), "bf16", variant, k, 21, offset=off), "lp %d" % i)
        # the binary32 values that are rounded, operation by operation
        m1 = b1 * m + a1 * g
        v1 = b2 * v + (a2 * g) * g
        draws = state_words(21, off, n)
        for x, got, scale, shift, positive in ((m1, t["m"][i], t["ms"][i], 0, False), (np.sqrt(v1), t["v"][i], t["vs"][i], 8, True)):
            assert x.dtype == np.float32
            pad = np.zeros(-(-n // 256) * 256, dtype=np.float32)
            pad[:n] = np.abs(x)
            s = np.maximum(pad.reshape(-1, 256).max(1) * (f(1) / f(448)), f(2.0 ** -126))
            assert np.array_equal(host(scale), s), "scale of tensor %d" % i
            y = x * rep(f(1) / s)
            bits = (draws >> np.uint16(shift)) & np.uint16((1 << k) - 1 if k < 16 else 0xFFFF)
            code = capi.fbsr_round_bits(y, "e4m3", variant, k, packed_fields(bits, k))
            if positive:
                code = np.where((x > 0) & (code == 0), 1, code).astype(np.uint8)
            gu.assert_codes_equal(got, code, "%s of tensor %d" % ("v" if positive else "m", i))


@pytest.mark.parametrize("misalign", [4, 8, 16])
@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("grad", ["fp32", "bf16"])
def test_alignments_between_element_and_vector(misalign, bits, grad):
    """Pointers that allow 16-byte copies, vector stores, or one of the two, give what aligned tensors give."""
    t, u = (make(SIZES, seed=40, bits=bits, grad=grad, misalign=x) for x in (misalign, 0))
    for x in (t, u):
        fbsr.fbsr_adamw_multi(x["table"], "src", 4, 9, **HYPER)
    for q in ("w", "m", "v", "lp", "ms", "vs"):
        for a, b in zip(t[q], u[q]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), q


def test_roots_and_quotients_of_the_8bit_step_are_rounded_correctly():
    """One element a block is not zero: its scale is the root of the new second moment over 448; with c1 a power of two and
    no weight before, the new weight is the quotient."""
    blocks = 1 << 16
    gen = torch.Generator(device="cuda").manual_seed(5)
    g = torch.zeros(blocks, 256, device="cuda")
    g[:, 3] = torch.randn(blocks, device="cuda", generator=gen) * torch.exp2(torch.rand(blocks, device="cuda", generator=gen) * 60 - 40)
    n = g.numel()
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    w, ms, vs = z(torch.float32), z(torch.float32, blocks), z(torch.float32, blocks)
    t = fbsr.FbsrAdamwTensors([w], [g.view(-1)], [z(torch.uint8)], [z(torch.uint8)], None, m_scale=[ms], v_scale=[vs])
    fbsr.fbsr_adamw_multi(t, "rtne", 1, 0, lr=2.0 ** -10, beta1=0.9, beta2=0.999, eps=1e-8, weight_decay=0.0, step=10 ** 6)
    f = np.float32
    x = host(g[:, 3])
    v = (f(1 - 0.999) * x) * x
    root = np.sqrt(v)
    assert np.array_equal(host(vs), np.maximum(root * (f(1) / f(448)), f(2.0 ** -126)))
    q = (f(1 - 0.9) * x) / (root + f(1e-8))                  # c2 is one by then
    assert np.array_equal(host(w.view(blocks, 256)[:, 3]), -q * f(2.0 ** -10))


def test_second_moments_outside_the_fast_root():
    """Very small and very large gradients: the moments' scales and signs hold, an overflowing second moment moves nothing."""
    n = 1024
    g = torch.zeros(n, device="cuda")
    g[0], g[1], g[256], g[512], g[513] = 1e-18, -1e-22, 3e38, -2e19, 1e-3
    z = lambda dt, k=n: torch.zeros(k, dtype=dt, device="cuda")  # noqa: E731
    w, m, v, ms, vs = z(torch.float32) + 0.5, z(torch.uint8), z(torch.uint8), z(torch.float32, 4), z(torch.float32, 4)
    t = fbsr.FbsrAdamwTensors([w], [g], [m], [v], None, m_scale=[ms], v_scale=[vs])
    fbsr.fbsr_adamw_multi(t, "rtne", 1, 0, **dict(HYPER, weight_decay=0.0, step=1))
    assert torch.isfinite(w).all() and torch.isfinite(ms).all() and torch.isfinite(vs).all()
    # -1e-22 beside 1e-18 is -0.0448 = -1.43 2^-5 in units of the scale: exponent field 2, 3.5 eighths (to the nearest, 3), signed
    assert int(m[1]) == 0x93 and int(m[256]) == 0x7E and int(m[512]) == 0xFE
    # (1e-3 3e38) 3e38 overflows, (1e-3 2e19) 2e19 = 4e35 does not: its weight takes the first step's lr
    assert int(v[256]) == 0x7E and float(w[256]) == 0.5 and abs(float(w[512]) - 0.501) < 1e-6
    f = np.float32
    assert float(vs[0]) == np.sqrt((f(1 - 0.999) * f(1e-18)) * f(1e-18)) * (f(1) / f(448))


def test_fresh_8bit_state_steps_as_binary32_does():
    """From zero state the first step's moments are one product each, the same whatever the state's width."""
    a, b = make((4096, 33), 9, bits=8, fresh=True), make((4096, 33), 9, bits=32, fresh=True)
    for q in ("w", "g"):                             # the two have drawn different numbers so far
        for x, y in zip(a[q], b[q]):
            y.copy_(x)
    h = dict(HYPER, step=1)
    for t in (a, b):
        fbsr.fbsr_adamw_multi(t["table"], "srf", 4, 1, **h)
    for x, y in zip(a["w"], b["w"]):
        assert torch.equal(x, y)


def test_a_positive_second_moment_never_vanishes():
    """One large and many tiny gradients in a block: the tiny roots are below half of the smallest code."""
    n = 256
    w, g = torch.zeros(n, device="cuda"), torch.full((n,), 1e-9, device="cuda")
    g[7] = 1e3
    m, v = torch.zeros(n, dtype=torch.uint8, device="cuda"), torch.zeros(n, dtype=torch.uint8, device="cuda")
    ms, vs = torch.zeros(1, device="cuda"), torch.zeros(1, device="cuda")
    for variant in ("rtne", "srff", "srf"):
        v.zero_()
        t = fbsr.FbsrAdamwTensors([w], [g], [m], [v], None, m_scale=[ms], v_scale=[vs])
        fbsr.fbsr_adamw_multi(t, variant, 2, 5, **dict(HYPER, step=1))
        assert (v != 0).all()
    g.zero_()
    v.zero_()
    vs.zero_()
    fbsr.fbsr_adamw_multi(t, "srf", 2, 5, **HYPER)
    assert (v == 0).all() and float(vs) == 2.0 ** -126          # a zero root stays zero


@pytest.mark.parametrize("bits", [32, 8])
def test_special_gradients_stay_in_their_elements(bits):
    sizes = (600,)
    t, u = make(sizes, 12, bits=bits), make(sizes, 12, bits=bits)
    for i, value in ((3, float("nan")), (300, float("inf")), (301, float("-inf"))):
        t["g"][0][i] = value
        u["g"][0][i] = 0.0
    for x in (t, u):
        fbsr.fbsr_adamw_multi(x["table"], "src", 3, 4, **HYPER)
    keep = torch.ones(600, dtype=torch.bool, device="cuda")
    keep[[3, 300, 301]] = False
    assert torch.isnan(t["w"][0][3]) and torch.isnan(t["w"][0][300]) and int(t["lp"][0][3]) == 0x7FC0
    assert torch.equal(t["w"][0][keep], u["w"][0][keep])
    if bits == 32:
        assert torch.equal(t["m"][0][keep], u["m"][0][keep])
    else:
        code = t["m"][0].view(torch.uint8)
        assert int(code[3]) & 0x7F == 0x7F and int(code[300]) == 0x7E and int(code[301]) == 0xFE
        assert torch.equal(code[keep][:200], u["m"][0][keep][:200])          # the block's scale ignores them
        assert torch.isfinite(t["ms"][0]).all() and torch.isfinite(t["vs"][0]).all()


@pytest.mark.parametrize("count", [0, 1, 48, 49, 400, 401, 900])
def test_many_tensors(count):
    """More tensors than a launch takes, empty ones among them; nothing outside the tensors is written."""
    sizes = [(37 * i) % 700 for i in range(count)]
    gen = torch.Generator(device="cuda").manual_seed(1)
    total = sum(sizes) + 16 * count
    base = torch.randn(total + 1, device="cuda", generator=gen)
    w, m, v = base.clone(), base * 1e-3, base ** 2
    lp = torch.full((total + 1,), 0xA5A5 - 65536, dtype=torch.int16, device="cuda").view(torch.uint16)
    inside = torch.zeros(total + 1, dtype=torch.bool, device="cuda")
    cut, at = [], 0
    for n in sizes:
        cut.append(slice(at, at + n))
        inside[at:at + n] = True
        at += n + 16
    part = lambda x: [x[s] for s in cut]  # noqa: E731
    t = fbsr.FbsrAdamwTensors(part(w), part(base), part(m), part(v), part(lp), offsets=[0] * count)
    before = fbsr.fbsr_launch_count()
    fbsr.fbsr_adamw_multi(t, "rtne", 1, 0, **HYPER)
    torch.cuda.synchronize()
    launches = -(-count // 400) if any(sizes) else 0
    assert fbsr.fbsr_launch_count() - before == launches
    want, bound = step64(host(base), host(base), host(base * 1e-3), host(base ** 2), HYPER)
    sel = inside.cpu().numpy()
    within(host(w)[sel], want[0][sel], bound[0][sel], "w")
    assert torch.equal(w[~inside], base[~inside]) and (lp.view(torch.int16)[~inside] == 0xA5A5 - 65536).all()
    assert np.array_equal(host(lp)[sel], capi.fbsr_round(host(w)[sel], "bf16", "rtne", 1, 0))


@pytest.mark.parametrize("bits,grad,misalign", [(32, "fp32", 0), (32, "bf16", 1), (8, "bf16", 0), (8, "fp16", 8), (8, "fp32", 3)])
@pytest.mark.parametrize("variant,k,lp", [("srf", 4, "bf16"), ("src", 3, "e4m3"), ("srff", 8, "fp16"), ("srf", 5, "bf16"), ("rto", 1, "fp16")])
def test_one_large_call_is_many_small_ones(bits, grad, misalign, variant, k, lp):
    """A call over about a million elements gives a warp four rows, a call over half of that one: the same bits."""
    sizes, names = (1_000_001, 300, 70001, 1025), ("w", "g", "m", "v", "lp", "ms", "vs")
    t, u = make(sizes, 9, bits, grad, lp, misalign), make(sizes, 9, bits, grad, lp, misalign)
    fbsr.fbsr_adamw_multi(t["table"], variant, k, 77, **HYPER)
    half = 500_224                               # a multiple of 256
    for i, start in enumerate(offsets_of(sizes)):
        for lo, hi in ((0, half), (half, sizes[i])) if i == 0 else ((0, sizes[i]),):
            part = {q: [u[q][i][lo // 256:-(-hi // 256)] if q in ("ms", "vs") else u[q][i][lo:hi]] for q in names if u[q]}
            more = dict(m_scale=part["ms"], v_scale=part["vs"]) if bits == 8 else {}
            one = fbsr.FbsrAdamwTensors(part["w"], part["g"], part["m"], part["v"], part["lp"], fmt=lp, offsets=[start + lo], **more)
            fbsr.fbsr_adamw_multi(one, variant, k, 77, **HYPER)
    for q in names:
        for a, b in zip(t[q], u[q]):
            assert torch.equal(a.view(torch.uint8), b.view(torch.uint8)), q


def test_without_low_precision_copies_and_with_other_gradients():
    t = make((1000, 10), 3)
    x = fbsr.FbsrAdamwTensors(t["w"], t["g"], t["m"], t["v"], [t["lp"][0], None])
    other = [torch.zeros_like(g) for g in t["g"]]
    x.set_grads(other)
    m = [y.clone() for y in t["m"]]
    fbsr.fbsr_adamw_multi(x, "srf", 4, 0, **HYPER)
    for y, z in zip(t["m"], m):
        assert torch.allclose(y, z * 0.9, rtol=1e-6)
    assert (t["lp"][1].view(torch.int16) == 0).all() and (t["lp"][0].view(torch.int16) != 0).any()


def test_on_another_stream():
    t, u = make(SIZES, 30), make(SIZES, 30)
    fbsr.fbsr_adamw_multi(u["table"], "srf", 4, 3, **HYPER)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        fbsr.fbsr_adamw_multi(t["table"], "srf", 4, 3, **HYPER)
    torch.cuda.current_stream().wait_stream(s)
    for q in ("w", "m", "v"):
        assert all(torch.equal(a, b) for a, b in zip(t[q], u[q]))


def test_refusals():
    t = make((300,), 2)
    args = dict(HYPER)
    run = lambda table=t["table"], variant="srf", k=4, **kw: fbsr.fbsr_adamw_multi(table, variant, k, 0, **dict(args, **kw))  # noqa: E731
    before = t["w"][0].clone()
    for kw, status in ((dict(k=0), 1), (dict(k=17), 1), (dict(variant=6), 1), (dict(step=0), 1)):
        with pytest.raises(fbsr.FbsrError) as e:
            run(**kw)
        assert e.value.status == status
    x = fbsr.FbsrAdamwTensors(t["w"], t["g"], t["m"], t["v"], t["lp"], offsets=[8])
    with pytest.raises(fbsr.FbsrError) as e:
        run(x)
    assert e.value.status == 1
    u = make((300,), 2, bits=8)
    with pytest.raises(fbsr.FbsrError) as e:
        run(u["table"], k=9)                                  # nine bits do not fit the state's draws
    assert e.value.status == 2
    run(u["table"], variant="rtne", k=9)
    assert torch.equal(t["w"][0], before)
    for bad in (dict(g=[t["g"][0][:-1]]), dict(m=[t["m"][0].double()]), dict(lp=[t["w"][0]]), dict(v=[t["v"][0].cpu()]),
                dict(w=[t["w"][0].view(150, 2).t()]), dict(g=[])):
        full = dict(w=t["w"], g=t["g"], m=t["m"], v=t["v"], lp=t["lp"])
        full.update(bad)
        with pytest.raises((TypeError, ValueError)):
            fbsr.FbsrAdamwTensors(**full)
    with pytest.raises(ValueError):
        fbsr.FbsrAdamwTensors(u["w"], u["g"], u["m"], u["v"], u["lp"], m_scale=u["ms"])
    with pytest.raises((TypeError, ValueError)):
        run(grad_scale=torch.ones(2, device="cuda"))
