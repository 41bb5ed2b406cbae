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
