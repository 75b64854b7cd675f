"""GPU: single tokens of sequences that share pages, as a search's rows do, against 64 bits (tolerances: test_gpu_kv).

Sequences that begin with the same page go together where their keys and values are many by the sizes that the host knows, which are the
table's; most of these tables is empty."""
import numpy as np
import pytest

from tests import kv_ref as K
from tests.test_gpu_kv import Case, ctx, vf  # noqa: F401

pytestmark = pytest.mark.gpu


def shared_case(vf, kind, cache, heads, kv_heads, dim, rows, parents, longest, page, seed, entries):  # noqa: F811
    """`rows` sequences behind `parents` prefixes of several lengths: whole pages of the prefix, then pages of their own."""
    rng = np.random.default_rng([rows, parents, longest, seed])
    prefix = rng.integers(0, longest + 1, parents)
    prefix[0] = longest
    who = rng.integers(0, parents, rows)
    keys = prefix[who] + rng.integers(0 if parents > 1 else 1, 2 * page, rows)   # some have a page more, some end in the prefix's last one
    keys[rng.integers(rows)] = 0
    c = Case(vf, kind, cache, heads, kv_heads, dim, [1] * rows, keys, page, seed=seed, ragged=False)
    table = np.full((rows, entries), K.NONE, np.int32)
    table[:, :c.table.shape[1]] = c.table
    for r in range(rows):
        same = np.flatnonzero(who == who[r])[0]
        whole = min(prefix[who[r]], keys[r], keys[same]) // page
        table[r, :whole] = table[same, :whole]
    c.table = table
    c.pool()
    return c


CASES = [
    # kind, cache, heads, kv_heads, dim, rows, parents, longest, page, window, entries
    ("bf16", "bf16", 8, 2, 64, 70, 5, 300, 16, 0, 900),
    ("bf16", "bf16", 16, 2, 64, 40, 1, 700, 16, 0, 1800),
    ("bf16", "e4m3", 4, 4, 128, 100, 7, 200, 32, 0, 600),
    ("bf16", "bf16", 6, 2, 80, 33, 3, 150, 16, 0, 2700),
    ("bf16", "bf16", 4, 2, 64, 64, 4, 300, 16, 100, 900),
    ("fp32", "fp32", 8, 2, 64, 70, 6, 200, 16, 0, 600),
    ("fp32", "e4m3", 4, 2, 40, 50, 4, 100, 16, 37, 2700),
    ("bf16", "bf16", 8, 2, 256, 40, 3, 200, 64, 0, 120),
    ("bf16", "bf16", 2, 1, 32, 1500, 20, 100, 16, 0, 360),
    ("bf16", "bf16", 3, 1, 16, 4096, 300, 40, 16, 0, 390),
]


@pytest.mark.parametrize("case", CASES, ids=lambda c: "-".join(str(x) for x in c))
def test_sequences_that_share_pages(vf, ctx, case):  # noqa: F811
    kind, cache, heads, kv_heads, dim, rows, parents, longest, page, window, entries = case
    c = shared_case(vf, kind, cache, heads, kv_heads, dim, rows, parents, longest, page, 1, entries)
    each = kv_heads * K.width_of(c.fmt, dim) * 2 * {"fp32": 4, "bf16": 2, "e4m3": 1}[cache]
    assert rows * entries * page * each >= 384 << 20
    q = c.matrix(heads * dim, scale=1.5)
    table, lengths = c.where()
    got = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, window=window)
    c.check_attend(ctx, q, got, True, window)
    again = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, window=window)
    assert c.torch.equal(got, again)
    # one at a time, as few keys: the other way
    apart = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, window=window, longest_kv=1)
    c.check_attend(ctx, q, apart, True, window)


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_missing_pages_and_what_is_not_finite(vf, ctx, kind):  # noqa: F811
    """In the middle of what is shared: entries that are no page, keys and values that are not finite, in one sequence or in all."""
    import torch
    for what in ("gone", "wrong", "first gone", "value", "key", "own value"):
        c = shared_case(vf, kind, kind, 8, 2, 64, 48, 3, 200, 16, 2, 1100)
        r = int(np.argmax(c.keys))
        if what == "gone":
            c.table[r, 3] = -1
        elif what == "wrong":
            c.table[r, 3] = 10 ** 7
        elif what == "first gone":
            c.table[r, 0] = -1
        elif what == "value":
            c.v[c.table[r, 4], 1, 5, 3] = float("inf")
        elif what == "key":
            c.k[c.table[r, 4], 1, 5, 3] = float("nan")
        else:
            c.v[c.table[r, (c.keys[r] - 1) // 16], 1, (c.keys[r] - 1) % 16, 3] = float("nan")
        c.pool()
        q = c.matrix(8 * 64)
        table, lengths = c.where()
        got = vf.vf_kv_attend(ctx, c.cache, q, table, lengths)
        torch.cuda.synchronize()
        c.check_attend(ctx, q, got)


def test_two_streams_and_a_graph(vf):  # noqa: F811
    """The same call on another stream than the tensors', and captured: replays between eager calls of other sizes on the same context."""
    import torch
    side = torch.cuda.Stream()
    ctx = vf.vf_create(0, stream=side)   # noqa: F811
    c = shared_case(vf, "bf16", "bf16", 8, 2, 64, 70, 5, 300, 16, 3, 900)
    other = shared_case(vf, "bf16", "bf16", 8, 2, 64, 40, 3, 900, 16, 4, 1500)
    q, p = c.matrix(512), other.matrix(512)
    where, there = c.where(), other.where()
    eager = vf.vf_kv_attend(ctx, c.cache, q, *where)      # (the context gets its scratch)
    want = eager.clone()
    c.check_attend(ctx, q, eager)
    torch.cuda.synchronize()
    buf = q.clone()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = vf.vf_kv_attend(ctx, c.cache, buf, *where)
    for k in (1.0, 0.0, -1.0, 1.0):
        buf.copy_(q * k)
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            g.replay()
        other.check_attend(ctx, p, vf.vf_kv_attend(ctx, other.cache, p, *there))
        torch.cuda.synchronize()
        if k == 1.0:
            assert torch.equal(got, want)
        else:
            c.check_attend(ctx, buf, got)
    vf.vf_destroy(ctx)
