"""What the binding hands to the C entry points of the operators over many tensors and 4-bit matrices, and what it refuses
before it gets there (runs without a GPU: host tensors stand in for those of a device)."""
import random

import pytest
import torch


class OnDevice:
    """A host tensor that says it lies on a device."""
    is_cuda = True

    def __init__(self, t):
        self.t = t

    def __getattr__(self, name):
        return getattr(self.t, name)


@pytest.fixture(scope="module")
def b():
    from paper_2504_20634_b200 import binding, build
    build.build()
    return binding


def matrix(b, t):
    return b._matrix(OnDevice(t), (t.dtype,), "x")


def test_rows_that_overlap_or_repeat_are_refused(b):
    x = torch.zeros(64, dtype=torch.bfloat16)
    for t in (x.expand(8, -1), x.unfold(0, 16, 8), x.unfold(0, 63, 1), x[:1].expand(4, 1), x.as_strided((3, 16), (15, 1))):
        with pytest.raises(TypeError):
            matrix(b, t)


def test_leading_dimensions(b):
    x = torch.zeros(12, 100)
    for t, ld in ((x, 100), (x[::3], 300), (x[:, 7:50], 100), (x[2:3, 5:9], 4), (x[0].expand(1, -1), 100), (x[:0], 100), (x[:, :1], 100),
                  (x.as_strided((4, 16), (16, 1)), 16), (x[:1, :1].expand(1, 1), 1)):
        assert matrix(b, t) == (t.data_ptr(), ld), (t.shape, t.stride())
    for t in (x[:, :0], x[:0, :0], x.as_strided((5, 0), (0, 1))):      # nothing to read, whatever the stride
        assert matrix(b, t)[1] >= 0
    with pytest.raises(TypeError):
        matrix(b, x.t())


def test_rows_as_handed_over_end_inside_the_storage(b):
    rng = random.Random(3)
    flat = torch.zeros(400)
    taken = 0
    for _ in range(3000):
        rows, cols, ld = rng.randint(1, 9), rng.randint(1, 40), rng.randint(0, 45)
        if (rows - 1) * ld + cols > flat.numel():
            continue
        t = flat.as_strided((rows, cols), (ld, 1))
        try:
            address, given = matrix(b, t)
        except TypeError:
            assert rows > 1 and ld < cols
            continue
        taken += 1
        assert (address - flat.data_ptr()) // 4 + (rows - 1) * given + cols <= flat.numel()
        assert rows == 1 or given == ld
    assert taken > 500


def test_the_host_part_of_a_late_step_costs_what_an_early_one_does(b):
    """beta^step is not formed step by step: 2^31 - 1 products take seconds, and a call launches after them."""
    import time
    t = (b.FbsrAdamwTensor * 1)()                            # a tensor without elements: nothing is launched
    for beta1, beta2 in ((0.9, 1.0 - 2.0 ** -40), (1.0 - 2.0 ** -50, 0.999)):
        start = time.perf_counter()
        assert b._L.fbsr_adamw_multi(t, 1, 32, 0x20, 0, 1, 4, 0, 1e-3, beta1, beta2, 1e-8, 0.0, 2 ** 31 - 1, None, None) == 0
        assert time.perf_counter() - start < 0.2


def test_powers_of_beta_give_the_scalars_of_the_single_tensor_step(b):
    """pow in binary64 and repeated products round to the same binary32 scalars."""
    import numpy as np
    f = np.float32
    steps = list(range(1, 1500)) + [10 ** 4, 12345, 10 ** 5, 10 ** 6]
    for beta1, beta2 in ((0.9, 0.999), (0.5, 0.95), (0.8, 0.9999), (0.98, 0.99999)):
        b1, b2, lr = float(f(beta1)), float(f(beta2)), float(f(1e-3))
        for step in steps:
            got = b.fbsr_adam_scalars(lr, b1, b2, step)
            assert got[0] == f(lr / (1 - b1 ** step)) and got[1] == f(1 / np.sqrt(1 - b2 ** step)), (beta1, beta2, step)


def test_results_written_over_their_source_are_refused(b):
    a, other, invalid = 4096, 8192, 1
    before = b.fbsr_launch_count()
    assert b._L.fbsr_round_w4(a, 0x20, 128, 4, 128, other, other, 0, 32, a, 128, 1, 4, 0, 0, None) == invalid       # values on src
    assert b._L.fbsr_gemv_w4(a, 0, 256, 1, other, other, 0, 32, 16, 256, a, 0x20, 16, None) == invalid               # y on x
    assert b.fbsr_launch_count() == before


def table(b, w, m=None, v=None, lp=None, **more):
    like = lambda given: [torch.zeros_like(t) for t in w] if given is None else given  # noqa: E731
    lists = [[OnDevice(t) for t in x] for x in (w, like(None), like(m), like(v))]
    return b.FbsrAdamwTensors(*lists, None if lp is None else [t if t is None else OnDevice(t) for t in lp], **more)


def test_a_tensor_listed_twice_or_lying_on_another_is_refused(b):
    flat, other = torch.zeros(1000), torch.zeros(600)
    apart = [flat[:300], flat[300:600], other, flat[600:600], flat[600:]]
    table(b, apart)                                          # neighbours and empty tensors are no overlap
    for w in ([flat, other, flat], [flat, flat], [flat[:301], flat[300:600]], [other, flat[:600], flat[599:]]):
        with pytest.raises(ValueError):
            table(b, w)
    for more in (dict(m=apart), dict(v=apart), dict(lp=[None, flat.view(torch.bfloat16)[:300], None, None, None])):
        with pytest.raises(ValueError):
            table(b, apart, **more)
    # 8-bit state: codes in one buffer behind one another, then scales that two tensors share
    w, codes, scales = [torch.zeros(300), torch.zeros(500)], torch.zeros(1600, dtype=torch.uint8), torch.zeros(8)
    part = lambda x, cut: [OnDevice(x[a:e]) for a, e in cut]  # noqa: E731
    state = [part(codes, ((0, 300), (300, 800))), part(codes, ((800, 1100), (1100, 1600)))]
    lists = [[OnDevice(t) for t in w], [OnDevice(torch.zeros_like(t)) for t in w], *state]
    b.FbsrAdamwTensors(*lists, m_scale=part(scales, ((0, 2), (2, 4))), v_scale=part(scales, ((4, 6), (6, 8))))
    with pytest.raises(ValueError):
        b.FbsrAdamwTensors(*lists, m_scale=part(scales, ((0, 2), (1, 3))), v_scale=part(scales, ((4, 6), (6, 8))))


def test_offsets_outside_the_stream_are_refused(b):
    w = [torch.zeros(300), torch.zeros(10)]
    t = table(b, w, offsets=[0, 2 ** 64 - 256])
    assert t.array[1].offset == 2 ** 64 - 256
    for offsets in ([-256, 0], [0, 2 ** 64], [0, -2 ** 64]):
        with pytest.raises(ValueError):
            table(b, w, offsets=offsets)
