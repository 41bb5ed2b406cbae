"""Results beside their sources in one buffer give what results of their own give; those that lie on them are refused and nothing is launched."""
import pytest
import torch

import test_gpu_attend_kv as few

pytestmark = pytest.mark.gpu


def setup_module(module):
    import paper_2504_20634_b200 as fbsr
    import kv_util
    module.fbsr, module.kv = fbsr, kv_util
    few.fbsr, few.kv = fbsr, kv_util


def refused(call):
    before = fbsr.fbsr_launch_count()
    with pytest.raises(fbsr.FbsrError):
        call()
    assert fbsr.fbsr_launch_count() == before


def test_attention():
    cache = few.random_cache(12, 2, 64, 16, 8, 5)
    table = torch.randperm(12, device="cuda").int().view(2, 6)
    lengths = torch.tensor([90, 33], dtype=torch.int32, device="cuda")
    room = torch.randn(8, 2, 4, 64, device="cuda").half()
    q = room[:, 0].clone()
    want = fbsr.fbsr_attend_kv(q, cache, table, lengths)
    for view in (room[:, 1], room[:, 1].flip(0)[:, :2].repeat(1, 2, 1), torch.empty(4, 8, 64, dtype=torch.float16, device="cuda").transpose(0, 1)):
        fbsr.fbsr_attend_kv(room[:, 0], cache, table, lengths, out=view)
        assert torch.equal(view, want) and torch.equal(room[:, 0], q)
    flat = room.view(-1)
    for out in (room[:, 0], flat[1:1 + 8 * 512 - 512 + 256].as_strided((8, 4, 64), (512, 64, 1), 1), flat[64:64 + 2048].view(8, 4, 64)):
        refused(lambda: fbsr.fbsr_attend_kv(room[:, 0], cache, table, lengths, out=out))


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_rows_read_back(dtype):
    cache = few.random_cache(6, 3, 64, 16, 4, 5)
    slots = torch.randperm(96, device="cuda")[:40]
    want = fbsr.fbsr_read_kv(cache, slots, dtype)
    for room in (torch.zeros(40, 2, 3, 64, dtype=dtype, device="cuda"), torch.zeros(40, 3, 2, 64, dtype=dtype, device="cuda").transpose(1, 2)):
        k, v = fbsr.fbsr_read_kv(cache, slots, k=room[:, 0], v=room[:, 1])
        assert torch.equal(k, want[0]) and torch.equal(v, want[1])
    room = torch.zeros(41, 3, 64, dtype=dtype, device="cuda")
    refused(lambda: fbsr.fbsr_read_kv(cache, slots, k=room[:40], v=room[1:]))
    refused(lambda: fbsr.fbsr_read_kv(cache, slots, k=room[:40], v=room[:40]))


@pytest.mark.parametrize("dtype", [torch.float32, torch.float16])
def test_values_beside_their_sources(dtype):
    room = torch.randn(6, 700, device="cuda").to(dtype)
    x = room[:, :300].clone()
    want = torch.empty_like(x)
    codes, scales = fbsr.fbsr_round_i8(x, "srf", 4, 1, values=want)
    got = fbsr.fbsr_round_i8(room[:, :300], "srf", 4, 1, values=room[:, 300:600])
    assert torch.equal(got[0], codes) and torch.equal(got[1], scales) and torch.equal(room[:, 300:600], want) and torch.equal(room[:, :300], x)
    refused(lambda: fbsr.fbsr_round_i8(room[:, :300], "srf", 4, 1, values=room[:, 299:599]))
    refused(lambda: fbsr.fbsr_round_i8(room[:5, :300], "srf", 4, 1, values=room[1:, :300]))


@pytest.mark.parametrize("m", [2, 40])
def test_products_beside_their_sources(m):
    room = torch.randint(-127, 128, (m, 512), dtype=torch.int8, device="cuda")
    w = torch.randint(-127, 128, (64, 256), dtype=torch.int8, device="cuda")
    one = torch.ones(64, device="cuda")
    a = room[:, :256].clone()
    want = fbsr.fbsr_gemm_i8(a, one[:m], w, one)
    y = room.view(torch.bfloat16)[:, 128:192]
    assert torch.equal(fbsr.fbsr_gemm_i8(room[:, :256], one[:m], w, one, out=y), want) and torch.equal(room[:, :256], a)
    refused(lambda: fbsr.fbsr_gemm_i8(room[:, :256], one[:m], w, one, out=room.view(torch.bfloat16)[:, 127:191]))
    refused(lambda: fbsr.fbsr_gemm_i8(a, one[:m], w, one, out=w.view(torch.bfloat16).view(-1)[:64 * m].view(m, 64)))
