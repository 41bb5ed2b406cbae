"""fbsr_attend_kv where weights or sizes of values lie far apart, held to a bound that counts by weighted values: a value that is large but
weighs nothing allows nothing, so a row of zeros, or sums that were not scaled when the maximum moved, cannot pass.

The bound, before the last rounding.  With p_t the weights (their sum is 1), s_t the scale of row t of v (4 bits: 2 to the largest exponent
of its groups' scales) and c_td = v_td / s_t:

    (2^-11 + 2 E + S) sum_t p_t |v_td|  +  2^-33 M sum_t |c_td|,        M = max_t p_t max(s_t, 2^-60)

2^-11: half a step of binary16 for p_t s_t.  The second term: the kernel's maximum is taken over x + log2(max(s, 2^-60)) and moves so that the
largest p_t s_t of a part is 2^8 or more, and a weight below binary16's normal range is off by 2^-25 at most, 2^-33 of that.  E: the
error of a score, dim products summed a step of eight at a time and a handful of roundings of it, and that of the exponential.  S: sums
in binary32 over steps of 16 tokens, in each of which a sum may be cut off (2^-23) and scaled (2^-24), for numerator and denominator, and
joined from up to 16 parts."""
import pytest
import torch

import test_gpu_attend_kv as few

pytestmark = pytest.mark.gpu


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    import kv_util
    module.fbsr, module.kv = fbsr, kv_util
    few.fbsr, few.kv = fbsr, kv_util


def row_scales(cache, table_row, length):
    at = torch.arange(length, device="cuda")
    s = cache.v_scales[table_row.long()[at // cache.page], :, at % cache.page].double()         # [length, kv heads, groups]
    return s[..., 0] if cache.bits == 8 else torch.exp2(torch.floor(torch.log2(s.amax(-1))))


def attend(q, k, v, s, scale):
    """One sequence, every query sees every token: (result in binary64, bound before the last rounding)."""
    share = q.shape[1] // k.shape[1]
    k, v, s, q = k.repeat_interleave(share, 1), v.repeat_interleave(share, 1), s.repeat_interleave(share, 1), q.double()
    x = torch.einsum("ihd,thd->iht", q, k) * scale
    p = torch.softmax(x, -1)
    size = (torch.einsum("ihd,thd->iht", q.abs(), k.abs()) * abs(scale)).amax(-1, keepdim=True)
    out, w = torch.einsum("iht,thd->ihd", p, v), torch.einsum("iht,thd->ihd", p, v.abs())
    n, dim = v.shape[0], v.shape[2]
    errors = 2.0 ** -11 + 2 * ((dim / 8 + 8) * 2.0 ** -23 * size + 2.0 ** -20) + (3 * n / 16 + 32) * 2.0 ** -23
    most = (p * s.t().clamp_min(2.0 ** -60)).amax(-1, keepdim=True)
    codes = (v.abs() / s[..., None]).sum(0)
    return out, errors * w + 2.0 ** -33 * most * codes


def check(got, q, cache, table_row, length, scale, told=0.85):
    """Within the bound and half a step of q's type; and the bound tells a zero result, or one of twice the size, from the right one for `told` of
    all elements at least."""
    k, v = few.sequence(cache, table_row, length)
    want, bound = attend(q, k, v, row_scales(cache, table_row, length), scale)
    info = torch.finfo(q.dtype)
    bound = torch.maximum(want.abs() * info.eps, torch.full_like(want, info.smallest_normal * info.eps)) / 2 + bound
    assert bool(torch.isfinite(got).all())
    share = float(((got.double() - want).abs() / bound).max())
    assert share <= 1, share
    assert float((bound < want.abs() / 4).double().mean()) >= told


# Queries of one sequence that make each kernel: up to 8 and 16 rows, 32, 64 and 128 of them along the lanes, several tiles of rows.
ROWS = [3, 11, 24, 50, 100, 150]


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("share", ROWS)
def test_sizes_of_values_far_apart(bits, share):
    """Rows of v from 2^-40 to 2^30; rows of zeros, one of which takes nearly all of the weight; sizes of queries from 2^-60 to 2^30."""
    n, dim, page = 400, 128, 8
    gen = few.generator(share)
    k = torch.randn(n, 1, dim, device="cuda", generator=gen)
    v = torch.randn(n, 1, dim, device="cuda", generator=gen) * torch.exp2(torch.randint(-40, 30, (n, 1, 1), device="cuda", generator=gen).float())
    v[::7] = 0
    k[14] = 3.0
    cache = fbsr.FbsrKvCache.empty(n // page, 1, dim, page, bits)
    fbsr.fbsr_round_kv(cache, k, v, torch.arange(n, device="cuda"), "rtne", 1, 0)
    table = torch.arange(n // page, device="cuda").int()[None]
    length = torch.tensor([n], dtype=torch.int32, device="cuda")
    for q_scale in (1.0, 2.0 ** -60, 2.0 ** 30):
        q = (torch.randn(1, share, dim, device="cuda", generator=gen).abs() * q_scale).bfloat16()
        got = fbsr.fbsr_attend_kv(q, cache, table, length, scale=0.125 / q_scale)
        check(got, q, cache, table[0], n, 0.125 / q_scale)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("share", ROWS)
@pytest.mark.parametrize("order", ["rising", "falling", "one"])
def test_maxima_that_move(bits, share, order):
    """Scores that rise along the sequence by 80 times the query's first element, values that shrink as they do: every tile moves the
    maximum and scales the sums.  One sequence in chunks, and 160 of them, a chunk each."""
    page, n, dim = 32, 1280, 64
    ramp = torch.linspace(0, 80, n, device="cuda")
    ramp = {"rising": ramp, "falling": ramp.flip(0), "one": torch.where(torch.arange(n, device="cuda") == 777, 60.0, 0.0)}[order]
    k = torch.zeros(n, 1, dim, device="cuda")
    k[:, 0, 0] = ramp
    k[:, 0, 1:] = 0.05 * torch.randn(n, dim - 1, device="cuda", generator=few.generator(4))
    v = torch.randn(n, 1, dim, device="cuda", generator=few.generator(5)) * torch.exp2(-ramp / 4)[:, None, None]
    cache = fbsr.FbsrKvCache.empty(n // page, 1, dim, page, bits)
    fbsr.fbsr_round_kv(cache, k, v, torch.arange(n, device="cuda"), "rtne", 1, 0)
    for batch in (1, 160):
        q = torch.randn(batch, share, dim, device="cuda", generator=few.generator(6)).bfloat16()        # binary16 results would be subnormal
        q[:, :, 0] = torch.tensor([1.0, -1.0, 4.0, 0.1], device="cuda").repeat(38)[:share]
        table = torch.arange(n // page, device="cuda").int()[None].expand(batch, -1).contiguous()
        got = fbsr.fbsr_attend_kv(q, cache, table, torch.full((batch,), n, dtype=torch.int32, device="cuda"), scale=1.0)
        for b in {0, batch // 3, batch - 1}:
            check(got[b:b + 1], q[b:b + 1], cache, table[b], n, 1.0)
