"""The attention value network's keeping of lengths, pages and rows on the CPU, with the operators' rules for pages and positions in place of the
operators: a stage's prediction is the sum of all stages' first features that it sees, whole numbers, so that every value is exact."""
import numpy as np
import pytest
import torch

from paper_2011_14486_amd import attention


NAN = float("nan")


class Pool:
    """A cache of one number a token."""

    def __init__(self, pages, page):
        self.k, self.page = torch.full((pages, 1, page, 8), float("nan")), page
        self.tensors = (self.k, None)


class Thing:
    pass


def network(monkeypatch, capturing=False):
    net = object.__new__(attention.AttentionValue)
    net.ctx, net.torch, net.blocks, net.kv_heads, net.head_dim = Thing(), torch, [None], 1, 8
    net.ctx.device, net.ctx.torch = torch.device("cpu"), torch
    net.not_there = torch.zeros(3, dtype=torch.int32), torch.tensor([NAN, NAN, 0.0])
    net.ctx.empty = lambda shape, dtype: torch.full(shape, float("nan"))
    net.capturing, net.pages = capturing, []
    monkeypatch.setattr(attention.AttentionValue, "_capturing", lambda self: self.capturing, raising=False)

    def cache(fmt, head_dim, k, v):
        c = Pool(0, k.shape[2])
        c.k, c.tensors = k, (k, v)
        return c

    monkeypatch.setattr(attention.vf, "KvCache", cache)

    def tokens(x, caches, table, lengths, offsets, longest, longest_kv):
        pool, wide = caches[0].k, table.shape[1]
        page, n, each = pool.shape[2], len(lengths), len(x) // len(lengths)
        net.pages.append(pool.shape[0])
        out = torch.full((len(x),), float("nan"))
        for write in (True, False):
            for s in range(n):
                first, end = (s * each, (s + 1) * each) if offsets is None else (int(offsets[s]), int(offsets[s + 1]))
                if not 0 <= first <= end <= len(x):
                    continue
                length = min(max(int(lengths[s]), 0), wide * page)
                place = lambda t: (int(table[s, t // page]), t % page)   # noqa: E731
                for i in range(end - first):
                    t = length - (end - first) + i
                    if write and t >= 0 and 0 <= place(t)[0] < len(pool):
                        pool[place(t)[0], 0, place(t)[1], 0] = x[first + i, 0]
                    if not write:
                        keys = [pool[place(u)[0], 0, place(u)[1], 0] if 0 <= place(u)[0] < len(pool) else float("nan") for u in range(t + 1)]
                        out[first + i] = float(sum(keys))
        return out

    net._tokens = tokens
    return net


def state_of(rows, stages, page=16):
    wide = -(-stages // page)
    return attention.AttentionState(torch, [Pool(rows * wide, page)], rows, wide, torch.device("cpu"))


def value_of(xs):
    return float(sum(sum(xs[:t + 1]) for t in range(len(xs))))


def stages(rng, n):
    return torch.from_numpy(rng.integers(-9, 10, (n, 3)).astype(np.float32))


def test_a_state_is_used_again(monkeypatch):
    """Rows that fork to a short one have the place of a short one, however long the longest has been, and ragged calls add what rows have got."""
    net, rng = network(monkeypatch), np.random.default_rng(1)
    state = state_of(4, 32)
    net.fork(state, torch.zeros(2, dtype=torch.int32))
    first = stages(rng, 33)
    net.score(first, 2, 30, torch.tensor([0, 30, 33], dtype=torch.int32), state)
    net.fork(state, torch.tensor([1], dtype=torch.int32))
    keep = first[30:33, 0].tolist()
    for _ in range(29):
        y = stages(rng, 1)
        keep.append(float(y[0, 0]))
        assert net.extend(y, state).tolist() == [value_of(keep)]
    with pytest.raises(ValueError):
        net.extend(stages(rng, 1), state)      # 33 stages
    assert state.lengths.tolist() == [32]
    # a further search from nothing
    state.lengths.zero_()
    state.total.zero_()
    x = stages(rng, 32)
    assert net.score(x, 1, state=state).tolist() == [value_of(x[:, 0].tolist())]
    with pytest.raises(ValueError):
        net.extend(stages(rng, 1), state)


def test_turns_of_the_longest_row(monkeypatch):
    """Ragged calls in which another row is the longest each time."""
    net, rng = network(monkeypatch), np.random.default_rng(2)
    state = state_of(2, 32)
    kept = [[], []]
    for counts in ([20, 1], [1, 20], [5, 5]):
        x = stages(rng, sum(counts))
        off = np.concatenate([[0], np.cumsum(counts)])
        got = net.score(x, 2, max(counts), torch.from_numpy(off.astype(np.int32)), state)
        for r in range(2):
            kept[r] += x[off[r]:off[r + 1], 0].tolist()
        assert got.tolist() == [value_of(k) for k in kept]
    with pytest.raises(ValueError):
        net.score(stages(rng, 8), 2, 7, torch.tensor([0, 7, 8], dtype=torch.int32), state)
    assert state.lengths.tolist() == [26, 26]


def test_ragged_sequences_without_a_longest(monkeypatch):
    """Without `longest` it is looked up: pages for the tokens there are, and a state's place is each row's own."""
    net, rng = network(monkeypatch), np.random.default_rng(3)
    counts = rng.integers(0, 40, 200)
    counts[7] = 300
    x = stages(rng, int(counts.sum()))
    off = np.concatenate([[0], np.cumsum(counts)])
    got = net.score(x, 200, offsets=torch.from_numpy(off.astype(np.int32)))
    assert got.tolist() == [value_of(x[a:b, 0].tolist()) for a, b in zip(off[:-1], off[1:])]
    assert net.pages[-1] <= len(x) // 16 + 200
    state = state_of(6, 32)
    net.fork(state, torch.zeros(6, dtype=torch.int32))
    for counts in ([20, 30, 5, 0, 1, 16], [12, 2, 3, 32, 1, 16]):
        x = stages(rng, sum(counts))
        off = np.concatenate([[0], np.cumsum(counts)])
        net.score(x, 6, offsets=torch.from_numpy(off.astype(np.int32)), state=state)
    assert state.lengths.tolist() == [32, 32, 8, 32, 2, 32] and state.longest == 32
    with pytest.raises(ValueError):
        net.score(x[:3], 6, offsets=torch.tensor([0, 0, 0, 0, 0, 0, 3], dtype=torch.int32), state=state)


def test_ranges_in_any_order(monkeypatch):
    """Ranges that lie in no order, that leave rows out, and ones that do not lie in the tokens."""
    net, rng = network(monkeypatch), np.random.default_rng(4)
    x = stages(rng, 100)
    off = torch.tensor([3, 40, 90, 90, 200], dtype=torch.int32)
    for more in (dict(), dict(longest=50), dict(longest=100)):
        got = net.score(x, 4, offsets=off, **more)
        assert got.tolist() == [value_of(x[a:b, 0].tolist()) for a, b in ((3, 40), (40, 90), (90, 90), (0, 0))]


def test_captured_calls_look_nothing_up(monkeypatch):
    """While a stream is captured all tokens are taken as the longest, and nothing is read back."""
    net, rng = network(monkeypatch, capturing=True), np.random.default_rng(5)
    x = stages(rng, 60)
    off = torch.tensor([0, 25, 60], dtype=torch.int32)
    want = [value_of(x[:25, 0].tolist()), value_of(x[25:, 0].tolist())]
    monkeypatch.setattr(torch.Tensor, "__int__", lambda self: pytest.fail("looked up"))
    taken = []
    net._tokens = lambda x, caches, table, lengths, offsets, longest, longest_kv: (taken.append((longest, tuple(table.shape))), x[:, 0])[1]
    net.score(x, 2, offsets=off)
    assert taken == [(60, (2, 4))]


def same(got, want):
    return np.array_equal(np.array(got.tolist()), np.array(want), equal_nan=True)


def test_a_longest_below_the_truth(monkeypatch):
    """Sequences with more tokens have NaN as their value, never another number, and a state's row is not lengthened by them; without offsets the
    host knows better."""
    net, rng = network(monkeypatch), np.random.default_rng(6)
    counts = [20, 50, 33, 32, 0]
    x = stages(rng, sum(counts))
    off = np.concatenate([[0], np.cumsum(counts)])
    each, offsets = [value_of(x[a:b, 0].tolist()) for a, b in zip(off[:-1], off[1:])], torch.from_numpy(off.astype(np.int32))
    assert same(net.score(x, 5, 32, offsets), [each[0], NAN, NAN, each[3], 0.0])
    assert same(net.score(x, 5, 1, offsets), [NAN, NAN, NAN, NAN, 0.0])
    got = net.score(x[:120], 3, 10)
    assert same(got, [value_of(x[a:a + 40, 0].tolist()) for a in (0, 40, 80)])
    state = state_of(5, 48)
    net.fork(state, torch.zeros(5, dtype=torch.int32))
    got = net.score(x, 5, 40, offsets, state)
    assert same(got, [each[0], NAN, each[2], each[3], 0.0]) and same(state.total, got.tolist())
    assert state.lengths.tolist() == [20, 0, 33, 32, 0] and state.longest == 40
    more = stages(rng, 5)
    keep = [x[a:b, 0].tolist() + [float(v)] for a, b, v in zip(off[:-1], off[1:], more[:, 0])]
    assert same(net.extend(more, state), [value_of(k) if r != 1 else NAN for r, k in enumerate(keep)])


def test_replays_past_the_place(monkeypatch):
    """A captured extension that is replayed more often than there is place for: NaN from there on, and pages that rows share stay as they were."""
    net, rng = network(monkeypatch), np.random.default_rng(7)
    state = state_of(4, 16)
    net.fork(state, torch.zeros(1, dtype=torch.int32))
    x = stages(rng, 16)
    net.score(x, 1, state=state)
    net.fork(state, torch.zeros(4, dtype=torch.int32))      # (four rows of 16 stages that share one full page)
    before = state.caches[0].k.clone()
    net.capturing = True
    for _ in range(3):
        assert same(net.extend(stages(rng, 4), state), [NAN] * 4)
    assert torch.equal(before.nan_to_num(-1e9), state.caches[0].k.nan_to_num(-1e9))
    # and rows with some place left, replayed on the same tensors
    state = state_of(2, 16)
    net.fork(state, torch.zeros(2, dtype=torch.int32))
    x = stages(rng, 2 * 14)
    net.capturing = False
    net.score(x, 2, state=state)
    net.capturing = True
    keep = [x[:14, 0].tolist(), x[14:, 0].tolist()]
    lengths, total = state.lengths, state.total
    for turn in range(4):
        y = stages(rng, 2)
        got = net.extend(y, state)
        keep = [k + [float(v)] for k, v in zip(keep, y[:, 0])]
        assert same(got, [value_of(k) if turn < 2 else NAN for k in keep])
        assert state.lengths is lengths and state.total is total
    # what replays have added the host does not know: calls after them go by the rows' own lengths too
    net.capturing = False
    state.longest = 1
    assert same(net.extend(stages(rng, 2), state), [NAN, NAN])


@pytest.mark.parametrize("kind", [torch.int32, torch.int64])
def test_parents_that_are_not_there(monkeypatch, kind):
    """-1 begins from nothing; any other parent that is no row makes a row whose value is NaN; the same parent may come many times."""
    net, rng = network(monkeypatch), np.random.default_rng(8)
    state = state_of(7, 48)
    net.fork(state, torch.zeros(3, dtype=kind))
    counts = [20, 32, 0]
    x = stages(rng, sum(counts))
    off = np.concatenate([[0], np.cumsum(counts)])
    net.score(x, 3, 32, torch.from_numpy(off.astype(np.int32)), state)
    prefix = [x[a:b, 0].tolist() for a, b in zip(off[:-1], off[1:])]
    parents = [1, -1, 3, 1, -2, 0, 2 ** 31 - 1]
    net.fork(state, torch.tensor(parents, dtype=kind))
    y = stages(rng, 7)
    want = [value_of(([] if p == -1 else prefix[p]) + [float(v)]) if -1 <= p < 3 else NAN for p, v in zip(parents, y[:, 0])]
    assert same(net.extend(y, state), want)
    assert state.lengths.tolist() == [33, 1, 1, 33, 1, 21, 1]
    # a state without rows, and rows from nothing again
    net.fork(state, torch.zeros(0, dtype=kind))
    assert net.extend(y[:0], state).shape == (0,)
    net.fork(state, torch.tensor([-1, 0], dtype=kind))
    assert same(net.extend(y[:2], state), [float(y[0, 0]), NAN])
