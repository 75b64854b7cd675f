"""GPU: attention of few rows in bf16 against 64 bits, with the weights' rounding not allowed for as one of bf16.

Tolerance: that of test_gpu_kv, but for the weights.  A weight p is the sum of two numbers of bf16: its upper half, from which it is less
than 2^-7 p away, and that rest, rounded, which is off by 2^-8 of itself at most: 2^-15 p.  (A rest below 2^-24 p is taken as that: 2^-24 p more.)"""
import numpy as np
import pytest

from tests import kv_ref as K
from tests.ops_ref import U32, UBF
from tests.test_gpu_kv import Case, ctx, f64, vf  # noqa: F401
from tests.test_gpu_kv_shared import shared_case

pytestmark = pytest.mark.gpu


def check(c, q, got, causal=True, window=0):
    k, v = c.values()
    scale = float(np.float32(c.dim ** -0.5))
    want, mag, size = K.attend(f64(q), k, v, c.table, c.keys, c.page, c.heads, causal, window, scale, c.offsets)
    live = np.zeros(c.tokens, bool)
    for first, rows in K.spans(c.offsets, len(c.new), c.tokens):
        live[first:first + rows] = True
    weight = 2 * (c.dim + 8) * U32 * size + (8 + max(int(c.keys.max()), 1)) * U32 + 2.0 ** -15 + 2.0 ** -24
    tol = weight * mag + UBF * np.abs(want)
    err = np.abs(f64(got) - want)[live]
    assert (err <= tol[live] + 1e-30).all(), float((err / (tol[live] + 1e-30)).max())


CASES = [
    # cache, heads, kv_heads, dim, new, keys, page, causal, window
    ("bf16", 8, 2, 64, [1], [60], 16, True, 0),
    ("bf16", 8, 2, 128, [1, 4, 2], [7, 40, 700], 16, True, 0),
    ("e4m3", 8, 2, 128, [1, 1, 0, 3], [33, 64, 5, 1000], 64, True, 0),
    ("bf16", 4, 2, 45, [3, 8], [9, 30], 16, True, 5),
    ("e4m3", 2, 2, 200, [9, 16], [40, 20], 16, True, 0),
    ("bf16", 3, 3, 256, [2, 5], [50, 12], 16, False, 0),
    ("bf16", 16, 1, 32, [1, 1], [9000, 20], 64, True, 0),     # shared along the keys
    ("bf16", 4, 2, 64, [1] * 1100, [12] * 1100, 16, True, 0),   # a wave a sequence
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c)[:60])
def test_weights_of_few_rows(vf, ctx, case):  # noqa: F811
    cache, heads, kv_heads, dim, new, keys, page, causal, window = case
    c = Case(vf, "bf16", cache, heads, kv_heads, dim, new, keys, page)
    q = c.matrix(heads * dim, scale=1.5)
    table, lengths = c.where()
    got = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, causal=causal, window=window, offsets=c.dev(c.offsets), longest=max(new))
    check(c, q, got, causal, window)


@pytest.mark.parametrize("cache,dim", [("bf16", 64), ("e4m3", 128)])
def test_weights_of_sequences_that_share_pages(vf, ctx, cache, dim):  # noqa: F811
    c = shared_case(vf, "bf16", cache, 8, 2, dim, 70, 5, 60, 16, 1, 900)
    q = c.matrix(8 * dim, scale=1.5)
    check(c, q, vf.vf_kv_attend(ctx, c.cache, q, *c.where()))


def test_visible_infinities_stay(vf, ctx):  # noqa: F811
    """A value that is infinite, behind keys that all rows see: the formula's infinity, also where its weight is a number of bf16."""
    for sign in (1.0, -1.0):
        c = Case(vf, "bf16", "bf16", 4, 2, 64, [1], [64], 16, ragged=False)
        c.k[:] = 0.0                    # (all weights are the same, 1 before they are divided by their sum)
        c.v[c.table[0, 0], 1, 3, 5] = sign * np.inf
        c.pool()
        q = c.matrix(256)
        got = f64(vf.vf_kv_attend(ctx, c.cache, q, *c.where())).reshape(4, 64)
        assert (got[2:, 5] == sign * np.inf).all() and np.isfinite(np.delete(got, 5, 1)).all() and np.isfinite(got[:2]).all()
