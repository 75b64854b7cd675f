"""GPU: calls of the attention operators that mean the same as another, and places and types that a call leaves to them (tolerances: test_gpu_kv)."""
import pytest

from tests.test_gpu_kv import Case, ctx, vf  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32")])
@pytest.mark.parametrize("new,keys", [([1, 3], [40, 9]), ([40, 70], [50, 129])])
def test_a_window_without_causality_is_none(vf, ctx, kind, cache, new, keys):  # noqa: F811
    c = Case(vf, kind, cache, 4, 2, 64, new, keys, 16)
    q = c.matrix(256, scale=1.5)
    table, lengths = c.where()
    got = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, causal=False, window=5, offsets=c.dev(c.offsets))
    c.check_attend(ctx, q, got, False, 0)


@pytest.mark.parametrize("dim", [65, 72, 73, 75, 78, 79, 80, 82, 85, 87, 88, 90])
def test_heads_whose_rows_are_no_multiple_of_three(vf, ctx, dim):  # noqa: F811
    """fp32 with many rows and places, where a lane takes three numbers of a value: rows of 72, 80, 88 and 96."""
    for causal, window in ((True, 0), (True, 33), (False, 0)):
        c = Case(vf, "fp32", "fp32", 4, 2, dim, [40, 1, 33, 0, 150], [60, 20, 33, 7, 600], 16, extra=40)
        q = c.matrix(4 * dim, scale=1.5)
        table, lengths = c.where()
        got = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, causal=causal, window=window, offsets=c.dev(c.offsets))
        c.check_attend(ctx, q, got, causal, window)
