"""The operators' C entry points refuse bad arguments by a status, before anything touches a device (runs without a GPU),
and the plain-numpy 4-bit helpers of the GPU tests are what the header says."""
import ctypes

import numpy as np
import pytest

FP32, BF16, FP16 = 0x20, 0, 1
OK, INVALID, UNSUPPORTED, ALIGNMENT, TOO_LARGE = 0, 1, 2, 3, 6
A = 4096                       # an address that is aligned and never read


@pytest.fixture(scope="module")
def b():
    from paper_2504_20634_b200 import binding, build
    build.build()
    return binding


def adamw(b, count=1, state_bits=32, g_fmt=FP32, fmt=BF16, variant=1, k=4, step=1, grad_scale=None, null=False, **fields):
    t = (b.FbsrAdamwTensor * max(count, 1))()
    for d in t:
        d.w = d.g = d.m = d.v = d.m_scale = d.v_scale = d.w_lp = A
        d.n, d.offset = 8, 0
        for name, value in fields.items():
            setattr(d, name, value)
    return b._L.fbsr_adamw_multi(None if null else t, count, state_bits, g_fmt, fmt, variant, k, 0, 1e-3, 0.9, 0.999, 1e-8, 0.0,
                                 step, grad_scale, None)


def test_adamw_multi(b):
    for kw in (dict(fmt=5), dict(fmt=-1), dict(variant=6), dict(k=0), dict(k=17), dict(step=0), dict(null=True), dict(offset=128),
               dict(w=None), dict(g=None), dict(m=None), dict(v=None), dict(state_bits=8, m_scale=None),
               dict(state_bits=8, v_scale=None)):
        assert adamw(b, **kw) == INVALID, kw
    for kw in (dict(g_fmt=2), dict(state_bits=16), dict(state_bits=8, k=9)):
        assert adamw(b, **kw) == UNSUPPORTED, kw
    for kw in (dict(w=A + 2), dict(m=A + 1), dict(v=A + 2), dict(g=A + 2), dict(g_fmt=BF16, g=A + 1), dict(w_lp=A + 1), dict(grad_scale=A + 2),
               dict(state_bits=8, m_scale=A + 2)):
        assert adamw(b, **kw) == ALIGNMENT, kw
    assert adamw(b, n=1 << 41) == TOO_LARGE
    assert adamw(b, count=40, n=1 << 40) == TOO_LARGE
    # nothing to do: no tensors, or tensors without elements, whatever their pointers
    assert adamw(b, count=0, null=True) == OK
    assert adamw(b, n=0, w=None, g=None) == OK
    assert adamw(b, n=0, count=500) == OK


def test_adamw_multi_checks_every_tensor_before_it_launches(b):
    t = (b.FbsrAdamwTensor * 2)()
    for d in t:
        d.w = d.g = d.m = d.v = A
        d.n = 8
    t[1].offset = 8
    before = b.fbsr_launch_count()
    assert b._L.fbsr_adamw_multi(t, 2, 32, FP32, BF16, 1, 4, 0, 1e-3, 0.9, 0.999, 1e-8, 0.0, 1, None, None) == INVALID
    assert b.fbsr_launch_count() == before


def round_w4(b, src=A, fmt=FP32, ld=128, rows=4, cols=128, codes=A, scales=A, scale_fmt=0, group=32, values=None, vld=0, variant=1, k=4, offset=0):
    return b._L.fbsr_round_w4(src, fmt, ld, rows, cols, codes, scales, scale_fmt, group, values, vld, variant, k, 0, offset, None)


def test_round_w4(b):
    for kw in (dict(variant=-1), dict(variant=6), dict(k=0), dict(k=17), dict(src=None), dict(codes=None), dict(scales=None), dict(ld=127),
               dict(offset=64), dict(offset=1 << 63), dict(values=A, vld=100)):
        assert round_w4(b, **kw) == INVALID, kw
    for kw in (dict(fmt=2), dict(group=16), dict(group=256), dict(scale_fmt=2)):
        assert round_w4(b, **kw) == UNSUPPORTED, kw
    for kw in (dict(src=A + 2), dict(fmt=BF16, src=A + 1), dict(codes=A + 8), dict(scale_fmt=1, scales=A + 1), dict(values=A + 2, vld=128)):
        assert round_w4(b, **kw) == ALIGNMENT, kw
    assert round_w4(b, rows=1 << 39) == TOO_LARGE and round_w4(b, cols=1 << 33, ld=1 << 33) == TOO_LARGE
    assert round_w4(b, rows=(1 << 30) + 1) == TOO_LARGE
    assert round_w4(b, rows=0, src=None) == OK and round_w4(b, cols=0, src=None) == OK
    assert [b.fbsr_w4_padded(c) for c in (0, 1, 127, 128, 129, 4096)] == [0, 128, 128, 128, 256, 4096]


def gemv_w4(b, x=A, fmt=BF16, ldx=256, m=1, codes=A, scales=A, scale_fmt=0, group=32, n=16, k=256, y=A, out=FP32, ldy=16):
    return b._L.fbsr_gemv_w4(x, fmt, ldx, m, codes, scales, scale_fmt, group, n, k, y, out, ldy, None)


def test_gemv_w4(b):
    for kw in (dict(x=None), dict(codes=None), dict(scales=None), dict(y=None), dict(ldx=255, m=2), dict(ldy=15)):
        assert gemv_w4(b, **kw) == INVALID, kw
    for kw in (dict(fmt=FP32), dict(fmt=2), dict(out=2), dict(group=8), dict(scale_fmt=-1)):
        assert gemv_w4(b, **kw) == UNSUPPORTED, kw
    for kw in (dict(x=A + 1), dict(codes=A + 4), dict(scales=A + 2), dict(y=A + 2), dict(scale_fmt=1, scales=A + 4)):
        assert gemv_w4(b, **kw) == ALIGNMENT, kw
    assert gemv_w4(b, n=1 << 31, ldy=1 << 31) == TOO_LARGE and gemv_w4(b, k=1 << 29, ldx=1 << 29) == TOO_LARGE
    assert gemv_w4(b, m=0, x=None, y=None) == OK and gemv_w4(b, n=0, ldy=0, y=None) == OK


def test_the_table_refuses_what_is_not_on_a_device(b):
    import torch
    x = torch.zeros(4)
    with pytest.raises(TypeError):
        b.FbsrAdamwTensors([x], [x], [x], [x])
    with pytest.raises((TypeError, ValueError)):
        b.fbsr_round_w4(torch.zeros(4, 4), "srf", 4, 0)
    with pytest.raises((TypeError, ValueError)):
        b.fbsr_gemv_w4(torch.zeros(1, 4, dtype=torch.bfloat16), torch.zeros(4, 64, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8))


def test_order_of_codes_and_values_of_the_helpers():
    import w4_util as w4
    rng = np.random.default_rng(0)
    plain = rng.integers(0, 16, size=(3, 256)).astype(np.uint8)
    codes = w4.pack(plain)
    assert codes.shape == (3, 128) and np.array_equal(w4.unpack(codes), plain)
    # element 32 j + 8 t + i of a block of 128: bits [4 i, 4 i + 4) of the 32-bit word at place 4 t + j
    words = codes.view(np.uint32)
    for block, j, t, i in ((0, 0, 0, 0), (0, 3, 1, 5), (1, 2, 3, 7)):
        assert (int(words[1, 16 * block + 4 * t + j]) >> (4 * i)) & 15 == plain[1, 128 * block + 32 * j + 8 * t + i]
    assert [float(w4.GRID[c]) for c in range(8)] == [0, 0.5, 1, 1.5, 2, 3, 4, 6]


def test_rounding_of_the_helpers_against_the_grid():
    """The oracle's run-time format stands for E2M1: nearest-even codes are the nearest grid points, ties to the even code."""
    import w4_util as w4
    x = np.arange(-8, 8.001, 1 / 64, dtype=np.float32)
    x = np.concatenate([x, np.zeros(-x.size % 32, np.float32)])
    x[-1] = 6.0                                              # the scale is one: 2^(floor(log2 8) - 2) = 2 in the groups beyond 4
    groups = np.stack([np.concatenate([x[i:i + 31], [np.float32(4.0)]]) for i in range(0, x.size - 31, 31)])
    groups = groups[np.abs(groups).max(1) < 8]
    code, stored, s = w4.expect(groups, 32, "e8m0", "rtne", 1, 0, 0, "fp32")
    assert (stored[:, 0] == 127).all()
    got = w4.GRID[code[:, :32]]
    mags = w4.GRID[:8]
    a = np.minimum(np.abs(groups), 6.0).astype(np.float64)
    d = np.abs(a[:, :, None] - mags)
    best = d.min(2)
    assert np.array_equal(np.abs(np.abs(got) - a), best)
    tie = (d == best[:, :, None]).sum(2) == 2
    assert tie.any() and ((code[:, :32] & 1)[tie] == 0).all()
    assert np.array_equal(np.signbit(got), np.signbit(groups))
