"""fbsr_gemv_w4: products with 4-bit matrices against binary64."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

TORCH = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}
UNIT = {"fp32": 2.0 ** -24, "bf16": 2.0 ** -8, "fp16": 2.0 ** -11}     # half an ulp: 2^-P
TINY = {"fp32": 2.0 ** -149, "bf16": 2.0 ** -133, "fp16": 2.0 ** -25}


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    import gpu_util
    import w4_util
    module.fbsr, module.gu, module.w4 = fbsr, gpu_util, w4_util


def weights(n, k, seed, group=32, scale_fmt="e8m0", lo=-9, hi=-3):
    """Random codes (zero beyond column k) and scales: (codes, scales, binary64 values)."""
    rng = np.random.default_rng(seed)
    pad = w4.padded(k)
    plain = rng.integers(0, 16, size=(n, pad)).astype(np.uint8)
    plain[:, k:] = 0
    codes = w4.pack(plain) if n else np.zeros((0, pad // 2), np.uint8)
    if scale_fmt == "e8m0":
        s = rng.integers(127 + lo, 127 + hi, size=(n, pad // group)).astype(np.uint8)
        st = torch.from_numpy(s).cuda()
    else:
        s = ((2.0 ** rng.uniform(lo, hi, size=(n, pad // group))).astype(np.float32).view(np.uint32) >> 16).astype(np.uint16)
        st = torch.from_numpy(s.view(np.int16).copy()).cuda().view(torch.bfloat16)
    return torch.from_numpy(codes).cuda(), st, (w4.GRID[plain] * np.repeat(w4.scale_values(s, scale_fmt), group, axis=1))[:, :k]


def activations(m, k, seed, x_type, spread=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(m, k, device="cuda", generator=gen) * torch.exp2(torch.randn(m, k, device="cuda", generator=gen) * spread)
    return x.to(TORCH[x_type])


def bound(x, w, want, out_type):
    """Exact products; up to 32 of them summed in the matrix unit (2^-23 a step, it may truncate), then one multiply-add a
    group in each of eight warps and eight additions; small bfloat16 elements to 2^-40 of their row's largest; the result
    rounded once."""
    k = x.shape[1]
    mass = np.abs(x) @ np.abs(w).T
    top = np.abs(x).max(1, keepdims=True) if k else np.zeros((x.shape[0], 1))
    steps = 2 * 32 + -(-k // 32) / 8 + 2 + 8
    inner = steps * 2.0 ** -24 * mass + 2.0 ** -40 * top * np.abs(w).sum(1)[None, :]
    return inner + UNIT[out_type] * (np.abs(want) + inner) + TINY[out_type]


def check(x, codes, scales, w, group, out_type, what="", misalign=0, pad_y=0):
    m, n = x.shape[0], w.shape[0]
    dt = TORCH[out_type]
    raw, flat = gu.guarded(m * (n + pad_y), dt, misalign=misalign)
    flat.view(torch.uint8).fill_(gu.CANARY)
    out = flat.view(m, n + pad_y)[:, :n]
    y = fbsr.fbsr_gemv_w4(x, codes, scales, group=group, out=out)
    torch.cuda.synchronize()
    assert y is out
    xd = x.double().cpu().numpy()
    want = xd @ w.T
    off = np.abs(out.double().cpu().numpy() - want)
    lim = bound(xd, w, want, out_type)
    assert (off <= lim).all(), "%s: %d off, worst %.2f of the bound" % (what, (off > lim).sum(), (off / lim).max())
    assert gu.canaries_intact(raw, m * (n + pad_y), dt, misalign=misalign)
    if pad_y and m:
        assert (flat.view(torch.uint8).view(m, -1)[:, n * dt.itemsize:] == gu.CANARY).all()      # nothing between the rows
    again = fbsr.fbsr_gemv_w4(x, codes, scales, group=group, out_dtype=dt)
    assert torch.equal(again, out), what + ": not reproducible"


@pytest.mark.parametrize("x_type", ["bf16", "fp16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("scale_fmt", ["e8m0", "bf16"])
@pytest.mark.parametrize("out_type", ["fp32", "same"])
def test_types_groups_and_shapes(x_type, group, scale_fmt, out_type):
    out_type = x_type if out_type == "same" else out_type
    for m, n, k in ((1, 1, 1), (1, 16, 128), (1, 17, 129), (2, 300, 1001), (3, 64, 31), (7, 33, 4096), (8, 100, 1024), (1, 5, 9000)):
        codes, scales, w = weights(n, k, n + k, group, scale_fmt)
        check(activations(m, k, m, x_type), codes, scales, w, group, out_type, "%d %d %d" % (m, n, k))


@pytest.mark.parametrize("x_type", ["bf16", "fp16"])
@pytest.mark.parametrize("m", [9, 15, 16, 17, 31, 32, 33, 64, 70])
def test_more_rows(x_type, m):
    for n, k in ((50, 520), (200, 2300)):
        codes, scales, w = weights(n, k, m)
        check(activations(m, k, m, x_type), codes, scales, w, 32, "fp32", "%d %d %d" % (m, n, k))


@pytest.mark.parametrize("m,n,k", [(1, 4096, 4096), (1, 1024, 4096), (1, 256, 14336), (4, 20000, 512), (16, 5000, 1500), (1, 40000, 640),
                                   (2, 128, 40000), (32, 64, 70001), (1, 9, 200000)])
def test_wide_and_long(m, n, k):
    codes, scales, w = weights(n, k, 4, 64, "bf16")
    check(activations(m, k, 2, "bf16"), codes, scales, w, 64, "fp32", "%d %d %d" % (m, n, k))


# Shapes of the kernel for many rows of W: tiles of 16 rows spread over 148 CTAs, of which each CTA's runs of 512 columns are cut
# into sixteen shares; tiles that one warp has, that two have and that all have, a last tile of 4, 11 and 3 rows, a last run of
# less than 512 columns, and tiles of a single run.
@pytest.mark.parametrize("m,n,k,x_type,group,scale_fmt", [
    (1, 9460, 4001, "bf16", 32, "e8m0"), (1, 4731, 8190, "fp16", 128, "bf16"), (1, 9460, 4096, "bf16", 32, "bf16"),
    (3, 9460, 4001, "fp16", 64, "bf16"), (8, 9460, 4096, "bf16", 64, "bf16"), (5, 75000, 300, "bf16", 32, "e8m0"),
    (1, 100003, 130, "fp16", 64, "e8m0"), (2, 2368, 16384, "bf16", 128, "e8m0")])
def test_many_rows_of_w(m, n, k, x_type, group, scale_fmt):
    codes, scales, w = weights(n, k, 11, group, scale_fmt)
    x = activations(m, k, 5, x_type)
    raw, flat = gu.guarded(m * n, torch.float32)
    flat.view(torch.uint8).fill_(gu.CANARY)
    out = fbsr.fbsr_gemv_w4(x, codes, scales, group=group, out=flat.view(m, n))
    torch.cuda.synchronize()
    xd = x.double().cpu().numpy()
    want, mass = xd @ w.T, np.abs(xd) @ np.abs(w).T
    # as in bound(), but all of a row's groups may be one warp's, and up to sixteen sums are joined
    steps = 2 * 32 + -(-k // 32) + -(-k // 128) + 16
    inner = steps * 2.0 ** -24 * mass + 2.0 ** -40 * np.abs(xd).max(1, keepdims=True) * np.abs(w).sum(1)[None, :]
    lim = inner + UNIT["fp32"] * (np.abs(want) + inner) + TINY["fp32"]
    off = np.abs(out.double().cpu().numpy() - want)
    assert (off <= lim).all(), "%d off, worst %.2f of the bound" % ((off > lim).sum(), (off / lim).max())
    assert gu.canaries_intact(raw, m * n, torch.float32)
    assert torch.equal(fbsr.fbsr_gemv_w4(x, codes, scales, group=group, out_dtype=torch.float32), out)


def test_strides_and_alignment():
    codes, scales, w = weights(130, 777, 1)
    for x_type in ("bf16", "fp16"):
        base = activations(12, 1000, 3, x_type)
        for x in (base[:5, 1:778], base[::3, 8:785], base[2:3, 5:782]):
            check(x, codes, scales, w, 32, "fp32", "strided x")
            check(x, codes, scales, w, 32, x_type, "strided y", misalign=1, pad_y=3)


def test_wide_range_of_bfloat16():
    """Rows of very large and very small numbers, and within a row elements 2^30 apart."""
    codes, scales, w = weights(64, 512, 5)
    x = activations(6, 512, 1, "bf16")
    x[0] *= 2.0 ** 100
    x[1] *= 2.0 ** -120
    x[2, 1:] *= 2.0 ** -30
    x[3] = 0.0
    x[4] = (torch.arange(512, device="cuda") % 2).to(torch.bfloat16) * 2.0 ** -130      # subnormal
    x[5, 7] = 3e38
    wide = w.copy()
    wide[:, 7] = 0.0                                             # the large element meets zero weights
    plain = w4.unpack(codes.cpu().numpy())
    plain[:, 7] = 0
    check(x, torch.from_numpy(w4.pack(plain)).cuda(), scales, wide, 32, "fp32", "range")


def test_extreme_scales():
    codes, scales, w = weights(40, 256, 6, lo=-127, hi=-120)
    check(activations(2, 256, 1, "fp16"), codes, scales, w, 32, "fp32", "small scales")
    codes, scales, w = weights(40, 256, 6, lo=90, hi=110)
    check(activations(2, 256, 1, "bf16"), codes, scales, w, 32, "fp32", "large scales")
    scales.zero_()                                               # byte 0: 2^-127
    w0 = w4.GRID[w4.unpack(codes.cpu().numpy())] * 2.0 ** -127
    check(activations(2, 256, 1, "fp16"), codes, scales, w0, 32, "fp32", "byte 0")


@pytest.mark.parametrize("x_type", ["bf16", "fp16"])
@pytest.mark.parametrize("scale_fmt", ["e8m0", "bf16"])
def test_special_values_go_where_the_formula_takes_them(x_type, scale_fmt):
    codes, scales, w = weights(40, 300, 7, 32, scale_fmt)
    x = activations(4, 300, 1, x_type)
    clean = fbsr.fbsr_gemv_w4(x, codes, scales)
    bad = scales.clone()
    if scale_fmt == "e8m0":
        bad[13, 2] = 255
    else:
        bad[13, 2] = float("nan")
    y = fbsr.fbsr_gemv_w4(x, codes, bad)
    assert torch.isnan(y[:, 13]).all()
    keep = torch.arange(40, device="cuda") != 13
    assert torch.equal(y[:, keep], clean[:, keep])
    x[1, 3], x[2, 299] = float("nan"), float("inf")
    y = fbsr.fbsr_gemv_w4(x, codes, scales, out_dtype=torch.float32).cpu().double().numpy()
    assert np.isnan(y[1]).all() and np.isfinite(y[[0, 3]]).all()
    with np.errstate(invalid="ignore"):
        want = np.inf * w[:, 299]
    assert np.array_equal(np.isnan(y[2]), np.isnan(want)) and np.array_equal(y[2][~np.isnan(want)], want[~np.isnan(want)])


def test_of_a_rounded_matrix_and_one_dimension():
    """Round, multiply: the product is that of the values that the rounding reports."""
    gen = torch.Generator(device="cuda").manual_seed(3)
    src = torch.randn(77, 391, device="cuda", generator=gen)
    val = torch.empty_like(src)
    for group, scale_fmt in ((32, "e8m0"), (128, "bf16")):
        codes, scales = fbsr.fbsr_round_w4(src, "srf", 4, 3, group=group, scale_fmt=scale_fmt, values=val)
        x = activations(1, 391, 2, "bf16")
        check(x, codes, scales, val.double().cpu().numpy(), group, "fp32")
        one = fbsr.fbsr_gemv_w4(x[0], codes, scales, group=group)
        assert one.shape == (77,) and torch.equal(one, fbsr.fbsr_gemv_w4(x, codes, scales, group=group)[0])


def test_on_another_stream():
    codes, scales, w = weights(500, 2000, 1)
    x = activations(2, 2000, 1, "fp16")
    want = fbsr.fbsr_gemv_w4(x, codes, scales)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        y = fbsr.fbsr_gemv_w4(x, codes, scales)
    torch.cuda.current_stream().wait_stream(s)
    assert torch.equal(y, want)


def test_empty_and_refused_calls():
    codes, scales, w = weights(40, 256, 1)
    x = activations(2, 256, 1, "bf16")
    assert fbsr.fbsr_gemv_w4(x[:0], codes, scales).shape == (0, 40)
    assert fbsr.fbsr_gemv_w4(x, codes[:0], scales[:0]).shape == (2, 0)
    none = torch.empty(40, 0, dtype=torch.uint8, device="cuda")
    y = torch.ones(2, 41, device="cuda")
    assert (fbsr.fbsr_gemv_w4(x[:, :0], none, none, out=y[:, :40]) == 0).all() and (y[:, 40] == 1).all()
    with pytest.raises(fbsr.FbsrError) as e:
        fbsr.fbsr_gemv_w4(x, codes, torch.zeros(40, 256 // 16, dtype=torch.uint8, device="cuda"), group=16)
    assert e.value.status == 2
    shifted = torch.empty(40 * 128 + 8, dtype=torch.uint8, device="cuda")[8:].view(40, 128)
    with pytest.raises(fbsr.FbsrError) as e:
        fbsr.fbsr_gemv_w4(x, shifted, scales)
    assert e.value.status == 3
    odd = torch.empty(40 * 8 + 1, dtype=torch.uint8, device="cuda")[1:].view(40, 8)
    with pytest.raises(fbsr.FbsrError) as e:
        fbsr.fbsr_gemv_w4(x, codes, odd)
    assert e.value.status == 3
    for args, kw in (((x.float(), codes, scales), {}), ((x[:, :100], codes, scales), {}), ((x, codes, scales[:, :4]), {}),
                     ((x, codes, scales.int()), {}), ((x, codes.cpu(), scales), {}), ((x.t(), codes, scales), {}),
                     ((x, codes, scales), dict(out=torch.empty(2, 39, device="cuda"))),
                     ((x, codes, scales), dict(out_dtype=torch.float64)), ((x, codes[:, ::2], scales), {})):
        with pytest.raises((TypeError, ValueError)):
            fbsr.fbsr_gemv_w4(*args, **kw)
