"""The operators over many tensors and 4-bit matrices at the ends of what they accept."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    from oracle import capi
    import gpu_util
    module.fbsr, module.capi, module.gu = fbsr, capi, gpu_util


def test_repeated_and_overlapping_rows_are_refused_before_a_launch():
    """One token broadcast over a batch, windows of a sequence, and results that would lie on one another."""
    w = torch.randn(48, 256, device="cuda")
    codes, scales = fbsr.fbsr_round_w4(w, "srf", 4, 1)
    token = torch.randn(256, device="cuda").to(torch.bfloat16)
    windows = torch.randn(512, device="cuda").to(torch.bfloat16).unfold(0, 256, 8)
    one = torch.empty(48, device="cuda", dtype=torch.bfloat16)
    before = fbsr.fbsr_launch_count()
    for x in (token.expand(8, -1), windows):
        with pytest.raises(TypeError):
            fbsr.fbsr_gemv_w4(x, codes, scales)
        with pytest.raises(TypeError):
            fbsr.fbsr_round_w4(x, "srf", 4, 1)
    with pytest.raises(TypeError):
        fbsr.fbsr_gemv_w4(token.repeat(8, 1), codes, scales, out=one.expand(8, -1))
    with pytest.raises(TypeError):
        fbsr.fbsr_round_w4(w, "srf", 4, 1, values=w[0].clone().expand(48, -1))
    assert fbsr.fbsr_launch_count() == before
    # what a caller does instead, and single rows, which have no stride to speak of
    y = fbsr.fbsr_gemv_w4(token.expand(8, -1).contiguous(), codes, scales)
    assert torch.equal(y, y[:1].expand(8, -1))
    assert torch.equal(fbsr.fbsr_gemv_w4(token.expand(1, -1), codes, scales), fbsr.fbsr_gemv_w4(token, codes, scales)[None])


def states(w, g, code_m, scale_m, code_v, scale_v):
    """The table of one tensor with 8-bit state out of numpy arrays, and its tensors."""
    t = [torch.from_numpy(np.ascontiguousarray(x)).cuda() for x in (w, g, code_m, code_v, scale_m, scale_v)]
    lp = torch.empty(w.size, dtype=torch.bfloat16, device="cuda")
    table = fbsr.FbsrAdamwTensors([t[0]], [t[1]], [t[2]], [t[3]], [lp], m_scale=[t[4]], v_scale=[t[5]])
    return table, t, lp


@pytest.mark.parametrize("eps", [0.0, 1e-45, 1e-40, 1.17e-38, 2.0 ** -126, 1e-8, -1e-3])
def test_quotients_of_the_8bit_step_at_the_ends_of_the_range(eps):
    """Denominators that are zero, subnormal and negative, moments that are infinite and quotients that overflow: the step is
    the header's, operation by operation, whatever the neighbours are."""
    f = np.float32
    n = 256 * 6 + 9
    rng = np.random.default_rng(1)
    w = np.full(n, 0.5, f)
    g = np.zeros(n, f)
    code_m, code_v = np.zeros(n, np.uint8), np.zeros(n, np.uint8)
    scale_m, scale_v = np.zeros(7, f), np.zeros(7, f)
    g[3:700:5] = f(1e-30)                                    # its square underflows, the first moment does not
    g[256:512:7] = rng.normal(size=37).astype(f) * f(1e-3)
    code_m[512:768], scale_m[2] = 0x38, f(1e35)              # 1e35 over a zero root
    code_m[768:1024:3], scale_m[3] = 0x7E, f(1e36)           # 448e36 is beyond binary32: an infinite first moment
    code_v[768:1024], scale_v[3] = 0x38, f(1.0)
    code_m[1024:1280:9], scale_m[4] = 0xB8, f(1e-3)
    code_v[1024:1280], scale_v[4] = 0x38, f(1e-2)
    g[1300:1310] = 1e-18                                     # roots above zero, below the fast root's range
    w[1400::2] = -0.0
    table, t, lp = states(w, g, code_m, scale_m, code_v, scale_v)
    # c1 is a power of two, c2 and the decay are one: every operation below is rounded as the step's is
    fbsr.fbsr_adamw_multi(table, "rtne", 1, 0, lr=2.0 ** -10, beta1=0.9, beta2=0.999, eps=eps, weight_decay=0.0, step=10 ** 6)
    torch.cuda.synchronize()
    with np.errstate(all="ignore"):
        m = f(0.9) * (capi.decode_array("e4m3", code_m) * np.repeat(scale_m, 256)[:n]) + f(1 - 0.9) * g
        root = capi.decode_array("e4m3", code_v) * np.repeat(scale_v, 256)[:n]
        v = f(0.999) * (root * root) + (f(1 - 0.999) * g) * g
        d = np.sqrt(v) + f(eps)
        want = w - f(2.0 ** -10) * (m / d)
    assert all(x.dtype == f for x in (m, v, d, want))
    got = gu.to_np(t[0])
    assert np.array_equal(np.isnan(got), np.isnan(want))
    ok = ~np.isnan(want)
    assert np.array_equal(got[ok], want[ok]), np.nonzero(got[ok] != want[ok])[0][:5]
    if eps > 0:
        assert ok.all() and np.isinf(want[512:768]).any() and np.isinf(want[768:1024]).any()
    with np.errstate(invalid="ignore"):
        gu.assert_codes_equal(lp.view(torch.uint16), capi.fbsr_round(got, "bf16", "rtne", 1, 0))


def test_a_row_of_2_to_31_columns():
    """The largest row: its first and last thousand elements round as they do by themselves, codes, scales and values."""
    n, part = 1 << 31, 1024
    x = torch.zeros(1, n, dtype=torch.bfloat16, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    x[0, :part] = torch.randn(part, device="cuda", generator=gen)
    x[0, -part:] = torch.randn(part, device="cuda", generator=gen)
    values = torch.full_like(x, 9.0)
    codes, scales = fbsr.fbsr_round_w4(x, "srf", 4, 5, values=values)
    for at in (0, n - part):
        own = torch.empty(1, part, dtype=torch.bfloat16, device="cuda")
        c, s = fbsr.fbsr_round_w4(x[:, at:at + part].contiguous(), "srf", 4, 5, offset=at, values=own)
        assert torch.equal(codes[:, at // 2:(at + part) // 2], c) and torch.equal(scales[:, at // 32:(at + part) // 32], s)
        assert torch.equal(values[:, at:at + part], own)
    assert not codes[0, part // 2:-part // 2].any() and not values[0, part:-part].any()


@pytest.mark.parametrize("bits", [32, 8])
@pytest.mark.parametrize("step,beta2", [(1, 0.999), (10 ** 4, 0.9999), (10 ** 5, 0.9999), (10 ** 6, 0.999999), (2 ** 31 - 1, 0.9999999)])
def test_late_steps(bits, step, beta2):
    """The bias corrections of early and late steps, against binary64."""
    from test_gpu_adamw_multi import HYPER, make, setup_module as prepare_module, step64, within
    import test_gpu_adamw_multi
    prepare_module(test_gpu_adamw_multi)
    h = dict(HYPER, step=step, beta2=beta2)
    t = make((70001,), 3, bits=bits)
    w, g, m, v = (gu.to_np(t[q][0]).copy() for q in ("w", "g", "m", "v"))
    if bits == 8:
        rep = lambda s: np.repeat(gu.to_np(s), 256)[:70001]  # noqa: E731
        m = capi.decode_array("e4m3", m) * rep(t["ms"][0])
        root = capi.decode_array("e4m3", v) * rep(t["vs"][0])
        v = root * root
    fbsr.fbsr_adamw_multi(t["table"], "srf", 4, 1, **h)
    torch.cuda.synchronize()
    want, bound = step64(w, g, m, v, h)
    within(gu.to_np(t["w"][0]), want[0], bound[0], "w")


def test_every_root_of_two_binades_as_the_8bit_step_uses_it():
    """Second moments over all 2^24 numbers of [1, 4), and times 4^-48 and 4^62.  With eps = -2^n the denominator is the root's
    distance from the lower end of its range, exactly, so that one unit of the root shows in the quotient and in the weight."""
    f = np.float32
    target = np.arange(0x3F800000, 0x40800000, dtype=np.uint32).view(f)
    # v' = fl(fl(V / 2) + fl(fl(g / 2) g)): V the square of a code, the largest with V / 2 below 0.97 of the target, g the rest
    code = np.arange(0x30, 0x48, dtype=np.uint8)
    halves = (f(0.5) * capi.decode_array("e4m3", code) ** 2).astype(f)
    at = np.searchsorted(halves, target.astype(np.float64) * 0.97, side="right") - 1
    assert at.min() >= 0 and halves[-1] > 4
    half = halves[at]
    second = lambda g: half + (f(0.5) * g) * g  # noqa: E731
    middle = np.sqrt(2.0 * (target.astype(np.float64) - half)).astype(f)
    g = middle.copy()
    for step in (-3, -2, -1, 1, 2, 3):
        other = (middle.view(np.uint32) + np.uint32(step & 0xFFFFFFFF)).view(f)
        g = np.where((second(g) != target) & (second(other) == target), other, g)
    reached = second(g) == target
    assert reached.all()
    root = np.sqrt(second(g))
    with np.errstate(divide="ignore"):
        want = -f(2.0 ** -10) * (g / (root - f(1)))
    assert want.dtype == f
    blocks = target.size // 256
    for n in (0, -48, 62):
        s = f(2.0 ** n)
        table, t, _ = states(np.zeros_like(g), g * s, np.zeros(target.size, np.uint8), np.zeros(blocks, f), code[at], np.full(blocks, s))
        fbsr.fbsr_adamw_multi(table, "rtne", 1, 0, lr=2.0 ** -10, beta1=0.0, beta2=0.5, eps=-2.0 ** n, weight_decay=0.0, step=2000)
        got = gu.to_np(t[0])
        assert np.array_equal(got, want), "2^%d: %d of %d differ" % (n, (got != want).sum(), want.size)
