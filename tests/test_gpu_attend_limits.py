"""fbsr_attend_kv at the ends of what it accepts: the longest sequences, and sizes of queries and keys at the ends of their types."""
import pytest
import torch

import test_gpu_attend_kv as few

pytestmark = pytest.mark.gpu


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    import kv_util
    module.fbsr, module.kv = fbsr, kv_util
    few.fbsr, few.kv = fbsr, kv_util


@pytest.mark.parametrize("queries,share", [(1, 1), (5, 4)])
def test_the_longest_sequence(queries, share):
    """2^31 - 65536 tokens, out of a table that repeats one page and ends with another, whose keys score 48 more: the tokens before it
    weigh 2^31 e^-40 at most, so the result is that of the last page alone, which only the last of the joined chunks holds."""
    page, dim, width = 65536, 64, 32767
    gen = few.generator(1)
    k, v = (0.25 * torch.randn(2 * page, 1, dim, device="cuda", generator=gen) for _ in range(2))
    k[page:, :, 0] += 12.0
    v[:page] += 5.0
    cache = fbsr.FbsrKvCache.empty(2, 1, dim, page, 4)
    fbsr.fbsr_round_kv(cache, k, v, torch.arange(2 * page, device="cuda"), "rtne", 1, 0)
    q = (0.25 * torch.randn(queries, share, dim, device="cuda", generator=gen)).half()
    q[:, :, 0] = 4.0
    table = torch.zeros(1, width, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    got = fbsr.fbsr_attend_kv(q, cache, table, torch.tensor([width * page], dtype=torch.int32, device="cuda"), scale=1.0)
    few.compare(got, q, cache, table[:, -1:], [page], [queries], scale=1.0)


@pytest.mark.parametrize("bits", [8, 4])
@pytest.mark.parametrize("share", [3, 11, 24, 100])
def test_large_queries_and_small_keys(bits, share):
    """Queries near the largest bfloat16 number over keys near the smallest scale, with scores of some tens: what turns a sum of products into
    a score passes 2^100, and is not to be multiplied by the sum before the key's scale."""
    n, dim, page = 300, 64, 16
    gen = few.generator(2)
    k = torch.randn(n, 1, dim, device="cuda", generator=gen) * 2.0 ** -122
    v = torch.randn(n, 1, dim, device="cuda", generator=gen)
    width = -(-n // page)
    cache = fbsr.FbsrKvCache.empty(width, 1, dim, page, bits)
    fbsr.fbsr_round_kv(cache, k, v, torch.arange(n, device="cuda"), "rtne", 1, 0)
    table = torch.arange(width, device="cuda").int()[None]
    q = (torch.randn(1, share, dim, device="cuda", generator=gen) * 2.0 ** 124).bfloat16()
    got = fbsr.fbsr_attend_kv(q, cache, table, torch.tensor([n], dtype=torch.int32, device="cuda"), scale=1.0)
    few.compare(got, q, cache, table, [n], [1], scale=1.0)
