"""Results that lie on what a call reads, or on one another, are refused by the C entry points whatever their strides, and results that
lie beside it in one buffer are not (runs without a GPU: a refused call touches no device)."""
import random

import pytest

from test_answer_refusals import A, BF16, FP32, INVALID, WORKSPACE, b, desc, refused    # noqa: F401 (b: a fixture)

HEADS, DIM = 2, 128                              # of the cache that desc describes


def attend(b, q, q_strides, out, out_strides, total, heads=HEADS):
    """A call that asks for a workspace and gives none: what passes the look for overlaps ends there."""
    return b._L.fbsr_attend_kv(q, *q_strides, BF16, total, heads, desc(b), A, 200, 200, A, 1, None, 256, None, 0, 0.1, out, *out_strides, A, 0, None)


def rows_of(base, strides, tokens, heads):
    return [base + 2 * (t * strides[0] + h * strides[1]) for t in range(tokens) for h in range(heads)]


def overlap(q, out):
    return any(x < y + 2 * DIM and y < x + 2 * DIM for x in q for y in out)


def test_attend_agrees_with_every_pair_of_rows(b):
    rng = random.Random(1)
    seen = {True: 0, False: 0}
    for i in range(4000):
        tokens, heads = rng.randint(1, 5), rng.choice([2, 4])
        inner = rng.choice([DIM, DIM, DIM + 8, 2 * DIM, 3 * DIM + 5])
        outer = heads * inner * rng.choice([1, 2, 3]) + rng.choice([0, 0, 64, 7])
        out_strides = rng.choice([(outer, inner), (inner, tokens * inner + rng.choice([0, 64, 300]))])
        # queries of the same strides, of others, repeated, or in the other direction
        q_strides = rng.choice([out_strides, out_strides, (outer + 128, inner), (0, inner), (-outer, inner), (outer, -inner), (DIM, 5 * DIM), (96, 40)])
        out = 1 << 20
        q = out + 2 * rng.choice([DIM, -DIM, inner, -inner, heads * inner, 2 * heads * inner, rng.randint(-4 * outer, 4 * outer)])
        mine, theirs = rows_of(q, q_strides, tokens, heads), rows_of(out, out_strides, tokens, heads)
        bad = overlap(mine, theirs)
        seen[bad] += 1
        assert attend(b, q, q_strides, out, out_strides, tokens, heads) == (INVALID if bad else WORKSPACE), (q - out, q_strides, out_strides, tokens, heads)
    assert min(seen.values()) > 500


def test_attend_looks_at_large_tensors_at_once(b):
    """2^24 rows beside one another in one buffer, and one element on."""
    tokens, heads, row = 1 << 19, 32, 32 * DIM
    strides = (2 * row, DIM)
    assert attend(b, 1 << 20, strides, (1 << 20) + 2 * row, strides, tokens, heads) == WORKSPACE
    assert attend(b, 1 << 20, strides, (1 << 20) + 2 * row - 2, strides, tokens, heads) == INVALID
    assert attend(b, 1 << 20, strides, (1 << 20) + 2 * row + 2, strides, tokens, heads) == INVALID
    # 2^63 bytes apart: no product wraps, neither to what lies there nor past it
    far = (1 << 62, DIM)
    assert attend(b, 1 << 20, far, (1 << 20) + 2 * row, strides, 3, heads) == WORKSPACE
    assert attend(b, 1 << 20, far, (1 << 20) + 2 * row - 2, strides, 3, heads) == INVALID


def test_what_is_read_back_lies_apart(b):
    def read(v, strides, k_strides=(256, 128), fmt=BF16, tokens=4):
        return b._L.fbsr_read_kv(desc(b), A, tokens, 16 * A, *k_strides, v, *strides, fmt, None)
    for v, strides in ((16 * A, (256, 128)), (16 * A + 2, (256, 128)), (16 * A - 2, (256, 128)), (16 * A + 3 * 512, (256, 128)), (16 * A + 256, (512, 128)),
                       (16 * A - 3 * 512, (256, 128)), (16 * A + 4 * 512 - 2, (1024, 512)), (16 * A, (0, 128)), (16 * A + 7 * 256, (-256, 128))):
        assert read(v, strides) == INVALID, (v - 16 * A, strides)
    assert read(16 * A + 2 * 4 * 256, (256, 128), fmt=FP32) == INVALID                   # rows of twice the bytes


def test_values_and_products_lie_apart_from_their_sources(b):
    def round_i8(values, vld, ld=100, fmt=FP32):
        return b._L.fbsr_round_i8(16 * A, fmt, ld, 4, 100, A, A, values, vld, 1, 4, 1, 0, None)
    for values, vld, ld in ((16 * A, 100, 100), (16 * A + 4, 100, 100), (16 * A - 4, 100, 100), (16 * A + 3 * 400, 100, 100), (16 * A + 396, 200, 200),
                            (16 * A + 404, 200, 200), (16 * A + 400, 150, 200), (16 * A - 3 * 1200, 300, 200)):
        assert round_i8(values, vld, ld) == INVALID, (values - 16 * A, vld, ld)

    def gemm_i8(y, ldy=5, m=4, lda=128, ldw=128, fmt=BF16):
        return b._L.fbsr_gemm_i8(16 * A, lda, m, A, 32 * A, ldw, 5, A, 128, y, fmt, ldy, None)
    for y, kw in ((16 * A, {}), (32 * A, {}), (16 * A + 510, {}), (16 * A - 2, {}), (32 * A + 4 * 128 + 126, {}), (16 * A + 126, dict(lda=256, ldy=128)),
                  (16 * A + 128 - 10 + 2, dict(lda=256, ldy=128, m=100)), (32 * A - 8, dict(fmt=FP32))):
        assert gemm_i8(y, **kw) == INVALID, (y, kw)
