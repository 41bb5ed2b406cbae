"""fbsr_round_w4: codes, scales and values of 4-bit matrices against the oracle, bit for bit."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    import gpu_util
    import w4_util
    module.fbsr, module.gu, module.w4 = fbsr, gpu_util, w4_util


def matrix(rows, cols, seed, src, spread=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(rows, cols, device="cuda", generator=gen) * torch.exp2(torch.randn(rows, cols, device="cuda", generator=gen) * spread)
    return x.to(TORCH[src])


def stored(t):
    return (t.view(torch.int16).cpu().numpy().view(np.uint16) if t.dtype == torch.bfloat16 else t.cpu().numpy())


def check(x, group, scale_fmt, variant, k, seed=7, offset=0, what=""):
    src = {v: n for n, v in TORCH.items()}[x.dtype]
    rows, cols = x.shape
    pad = fbsr.fbsr_w4_padded(cols)
    raw, out = gu.guarded(rows * pad // 2, torch.uint8)
    out = out.view(rows, pad // 2)
    val = torch.full_like(x, 9.0)
    codes, scales = fbsr.fbsr_round_w4(x, variant, k, seed, offset=offset, group=group, scale_fmt=scale_fmt, values=val, out=out)
    torch.cuda.synchronize()
    code, ecale, s = w4.expect(x.float().cpu().numpy(), group, scale_fmt, variant, k, seed, offset, src)
    assert np.array_equal(stored(scales), ecale), what + " scales"
    got = w4.unpack(codes.cpu().numpy())
    assert np.array_equal(got, code), "%s: %d codes differ" % (what, (got != code).sum())
    assert gu.canaries_intact(raw, rows * pad // 2, torch.uint8)
    want = (torch.from_numpy(w4.GRID[code].astype(np.float32) * np.repeat(s, group, axis=1)))[:, :cols].to(TORCH[src])
    assert torch.equal(torch.isnan(val.cpu()), torch.isnan(want))
    ok = ~torch.isnan(want)
    assert torch.equal(val.cpu()[ok], want[ok]), what + " values"
    # without values the same codes
    again, scales2 = fbsr.fbsr_round_w4(x, variant, k, seed, offset=offset, group=group, scale_fmt=scale_fmt)
    assert torch.equal(again, codes) and torch.equal(scales2.view(torch.uint8), scales.view(torch.uint8))


@pytest.mark.parametrize("variant", ["srff", "srf", "src"])
@pytest.mark.parametrize("k", range(1, 17))
def test_every_variant_and_draw_width(variant, k):
    check(matrix(37, 300, k, "fp32"), 32, "e8m0", variant, k, offset=128 * k, what="%s k=%d" % (variant, k))
    check(matrix(5, 129, k, "bf16"), 64, "bf16", variant, k, what="%s k=%d" % (variant, k))


@pytest.mark.parametrize("variant", ["rtne", "rta", "rto"])
def test_deterministic_modes(variant):
    x = matrix(20, 520, 3, "fp32", spread=0.5)
    x[:, ::5] = torch.tensor([0.25, 0.75, 2.5, 5.0], device="cuda").repeat(20, 26) * 2.0 ** -3       # ties
    x[:, 0] = 4.0 * 2.0 ** -3
    check(x, 128, "e8m0", variant, 1)
    check(x, 32, "bf16", variant, 9)


@pytest.mark.parametrize("src", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("scale_fmt", ["e8m0", "bf16"])
def test_types_groups_and_shapes(src, group, scale_fmt):
    for rows, cols in ((1, 1), (1, 127), (3, 128), (2, 129), (70, 31), (513, 384), (9, 2049)):
        check(matrix(rows, cols, rows + cols, src), group, scale_fmt, "srf", 4, seed=1 << 40, offset=1280, what="%d x %d" % (rows, cols))


@pytest.mark.parametrize("src", ["fp32", "bf16"])
def test_strided_and_misaligned_rows(src):
    base = matrix(40, 700, 1, src)
    for x in (base[:, 1:430], base[::3, 8:520], base[5:6, 3:300], base[:, 64:192]):
        check(x, 32, "bf16", "src", 3)


@pytest.mark.parametrize("src", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("scale_fmt", ["e8m0", "bf16"])
@pytest.mark.parametrize("group", [32, 128])
def test_special_values(src, scale_fmt, group):
    x = matrix(12, 256, 2, src)
    big = {"fp32": 3.4e38, "bf16": 3.38e38, "fp16": 65504.0}[src]
    small = {"fp32": 1e-45, "bf16": 9.2e-41, "fp16": 6e-8}[src]
    x[0, 5] = float("nan")
    x[1, 40] = float("inf")
    x[2] = float("-inf")                                        # a row without finite values
    x[3] = 0.0
    x[4, :128] = small
    x[5, ::2] = big
    x[6, 130] = -big
    x[7, 3], x[7, 4] = float("nan"), float("inf")
    x[8] = -0.0
    x[9] *= 2.0 ** -100 if src != "fp16" else 2.0 ** -12
    check(x, group, scale_fmt, "srf", 4)
    check(x, group, scale_fmt, "rtne", 4)


def test_large_matrix_by_rows():
    """Rows rounded in one call and in two calls with their offsets give the same bytes."""
    x = matrix(2000, 1111, 4, "fp32")
    codes, scales = fbsr.fbsr_round_w4(x, "srf", 3, 11, offset=256)
    a = 777
    c2, s2 = fbsr.fbsr_round_w4(x[a:], "srf", 3, 11, offset=256 + a * fbsr.fbsr_w4_padded(1111))
    assert torch.equal(codes[a:], c2) and torch.equal(scales[a:], s2)


def test_empty_and_refused_calls():
    x = matrix(4, 128, 1, "fp32")
    for shape in ((0, 128), (4, 0)):
        c, s = fbsr.fbsr_round_w4(x[:shape[0], :shape[1]], "srf", 4, 0)
        assert c.numel() == 0 and s.numel() == 0
    for kw, status in ((dict(variant=6), 1), (dict(k_bits=0), 1), (dict(k_bits=17), 1), (dict(group=48), 2), (dict(offset=64), 1),
                       (dict(offset=1 << 63), 1)):
        with pytest.raises(fbsr.FbsrError) as e:
            fbsr.fbsr_round_w4(x, **dict(dict(variant="srf", k_bits=4, seed=0), **kw))
        assert e.value.status == status, kw
    odd = torch.empty(4 * 64 + 8, dtype=torch.uint8, device="cuda")[8:].view(4, 64)
    with pytest.raises(fbsr.FbsrError) as e:
        fbsr.fbsr_round_w4(x, "srf", 4, 0, out=odd)
    assert e.value.status == 3
    for bad in (dict(scale_fmt="fp32"), dict(values=x[:, :5]), dict(values=x.bfloat16()), dict(out=torch.empty(4, 32, dtype=torch.uint8, device="cuda")),
                dict(scales=torch.empty(4, 4, device="cuda"))):
        with pytest.raises((TypeError, ValueError)):
            fbsr.fbsr_round_w4(x, "srf", 4, 0, **bad)
    for src in (x.double(), x.cpu(), x.t(), x[0]):
        with pytest.raises((TypeError, ValueError)):
            fbsr.fbsr_round_w4(src, "srf", 4, 0)
