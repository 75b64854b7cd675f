"""GPU: the attention value network's places - ragged sequences without a longest, one that is too small, states that are used again, captured calls
that are replayed past the place - against the same sequences scored another way (tolerances: test_gpu_attention_value)."""
import numpy as np
import pytest

from tests.test_gpu_attention_value import dev, predictions
from tests.test_gpu_ssm_value import bf16, close, ctx, vf  # noqa: F401

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def weights():
    from paper_2011_14486_amd import inputs
    return inputs.attention_weights(32, 96, 2, 4, 2, 64, 64, seed=4)


def ragged(counts, seed=1):
    import torch
    x = bf16(np.random.default_rng(seed).standard_normal((int(sum(counts)), 32)))
    off = np.concatenate([[0], np.cumsum(counts)])
    return x, dev(off, torch.int32), off


def test_ragged_sequences_without_a_longest(vf, ctx, weights):  # noqa: F811
    import torch
    from paper_2011_14486_amd import attention
    net = attention.AttentionValue(ctx, weights)
    counts = np.random.default_rng(2).integers(0, 51, 2000)
    counts[[0, 999]] = 0, 50
    x, off, _ = ragged(counts)
    x = dev(x)
    net.score(x, 2000, 50, off)
    torch.cuda.synchronize()
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    got = net.score(x, 2000, offsets=off)
    torch.cuda.synchronize()
    # (keys and values: 2 x 2000 x 4 pages x 16 x 2 x 64 x 2 bytes = 66 MB; what 50,000 tokens have at a time in a block, 512 + 256 + 4 x 96 numbers of
    # bf16 and as many of 8 bits, 180; with all tokens taken as the longest keys and values would be 51 GB)
    assert torch.cuda.max_memory_allocated() - held < 400 << 20
    assert torch.equal(got, net.score(x, 2000, 50, off)) and got[0] == 0
    # one sequence much longer than the others
    counts[5] = 1000
    x, off, _ = ragged(counts)
    x = dev(x)
    torch.cuda.reset_peak_memory_stats()
    held = torch.cuda.memory_allocated()
    got = net.score(x, 2000, offsets=off)
    torch.cuda.synchronize()
    assert torch.cuda.max_memory_allocated() - held < 400 << 20
    assert torch.equal(got, net.score(x, 2000, 1000, off, net.state(2000, 1000))) and torch.isfinite(got).all()
    small, off3, _ = ragged([20, 1, 0, 37], 3)
    each = predictions(weights, small, [20, 1, 0, 37], False)
    want = np.array([each[:20].sum(), each[20], 0.0, each[21:].sum()])
    close(net.score(dev(small), 4, offsets=off3).cpu().numpy(), want, np.sqrt((each ** 2).mean()), np.array([20, 1, 1, 37]))
    state = net.state(4, 40)
    got = net.score(dev(small), 4, offsets=off3, state=state)
    close(got.cpu().numpy(), want, np.sqrt((each ** 2).mean()), np.array([20, 1, 1, 37]))
    assert state.longest == 37 and state.lengths.tolist() == [20, 1, 0, 37]


def test_a_longest_below_the_truth(vf, ctx, weights):  # noqa: F811
    import torch
    from paper_2011_14486_amd import attention
    net = attention.AttentionValue(ctx, weights)
    counts = [20, 50, 33, 32, 0]
    x, off, _ = ragged(counts)
    right = net.score(dev(x), 5, offsets=off)
    got = net.score(dev(x), 5, 32, off)
    assert torch.isnan(got[[1, 2]]).all() and torch.equal(got[[0, 3, 4]], right[[0, 3, 4]])
    state = net.state(5, 64)
    got = net.score(dev(x), 5, 40, off, state)
    assert torch.isnan(got[1]) and torch.equal(got[[0, 2, 3, 4]], right[[0, 2, 3, 4]]) and state.lengths.tolist() == [20, 0, 33, 32, 0]
    assert torch.equal(net.score(dev(x[:120]), 3, 5), net.score(dev(x[:120]), 3))


def test_a_state_is_used_again(vf, ctx, weights):  # noqa: F811
    import torch
    from paper_2011_14486_amd import attention
    net = attention.AttentionValue(ctx, weights)
    state = net.state(4, 32)
    net.fork(state, torch.zeros(2, dtype=torch.int32, device="cuda"))
    x, off, _ = ragged([30, 3])
    net.score(dev(x), 2, 30, off, state)
    net.fork(state, torch.ones(1, dtype=torch.int32, device="cuda"))
    y = bf16(np.random.default_rng(5).standard_normal((29, 32)))
    for i in range(29):
        got = net.extend(dev(y[i:i + 1]), state)
    whole = np.concatenate([x[30:], y])
    each = predictions(weights, whole, [32], False)
    close(got.cpu().numpy(), np.array([each.sum()]), np.sqrt((each ** 2).mean()), 32)
    with pytest.raises(ValueError):
        net.extend(dev(y[:1]), state)


def test_captured_calls(vf, weights):  # noqa: F811
    """Ragged scores and extensions in graphs: every replay against the eager call, past the state's place NaN, shared pages as they were."""
    import torch
    from paper_2011_14486_amd import attention
    side = torch.cuda.Stream()
    ctx = vf.vf_create(0, stream=side)   # noqa: F811
    net = attention.AttentionValue(ctx, weights)
    x, off, _ = ragged([20, 0, 45, 3, 33])
    x = dev(x)
    other = off.clone()
    other[1:4] = torch.tensor([15, 15, 60], dtype=torch.int32)   # the same tokens dealt otherwise
    offs = [off, other]
    for longest in (None, 60):
        net.score(x, 5, longest, off)
        buf, at = x.clone(), off.clone()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = net.score(buf, 5, longest, at)
        for turn, k in enumerate((1.0, -0.5, 2.0, 1.0, 0.0)):
            buf.copy_(x * k)
            at.copy_(offs[turn & 1])
            torch.cuda.synchronize()
            g.replay()
            torch.cuda.synchronize()
            replayed = got.clone()
            assert torch.equal(replayed, net.score(x * k, 5, 60, offs[turn & 1])) and torch.isfinite(replayed).all()
            x.float().sum().item()
    # four rows that share a full page, and two with place for two stages more
    y = dev(bf16(np.random.default_rng(6).standard_normal((4, 32))))
    for rows, begin, left in ((4, 16, 0), (2, 14, 2)):
        state = net.state(4, 16)
        if rows == 4:
            net.fork(state, torch.zeros(1, dtype=torch.int32, device="cuda"))
            net.score(x[:16], 1, state=state)
            net.fork(state, torch.zeros(4, dtype=torch.int32, device="cuda"))
        else:
            net.fork(state, torch.zeros(2, dtype=torch.int32, device="cuda"))
            net.score(x[:28], 2, state=state)
        first, before = state.total.clone(), [c.k.clone() for c in state.caches]
        eager = [first]
        z = y[:rows].clone()
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            got = net.extend(z, state)
        assert state.captured
        torch.cuda.synchronize()
        for turn in range(4):
            g.replay()
            torch.cuda.synchronize()
            if turn < left:
                eager.append(got.clone())
                assert torch.isfinite(got).all()
            else:
                assert torch.isnan(got).all() and torch.isnan(state.total).all()
        assert state.lengths.tolist() == [16] * rows
        if left == 0:
            assert all(torch.equal(a, c.k) for a, c in zip(before, state.caches))
        else:
            again = net.state(4, 32)
            net.fork(again, torch.zeros(2, dtype=torch.int32, device="cuda"))
            assert torch.equal(net.score(x[:28], 2, state=again), eager[0])
            for want in eager[1:]:
                assert torch.equal(net.extend(z, again), want)
        torch.cuda.synchronize()
        assert torch.isnan(net.extend(z, state)).all()      # an eager call behind the replays
    vf.vf_destroy(ctx)


@pytest.mark.parametrize("fmt", [1, 2])
def test_parents_that_are_not_there(vf, ctx, weights, fmt):  # noqa: F811
    """-1 begins from nothing; any other parent that is no row makes a row whose value is NaN; the others are as without these."""
    import torch
    from paper_2011_14486_amd import attention
    net = attention.AttentionValue(ctx, weights)
    x, off, _ = ragged([20, 32, 0])
    y = dev(bf16(np.random.default_rng(7).standard_normal((7, 32))))
    got = []
    for parents in ([1, -1, 3, 1, -2, 0, 2 ** 31 - 1], [1, 2, 2, 1, 2, 0, 2]):     # (row 2 has nothing either)
        state = net.state(7, 48, fmt=fmt)
        net.fork(state, torch.zeros(3, dtype=torch.int32, device="cuda"))
        net.score(dev(x), 3, 32, off, state)
        net.fork(state, dev(np.array(parents), torch.int32))
        got.append(net.extend(y, state))
        assert state.lengths.tolist() == [33, 1, 1, 33, 1, 21, 1]
    there = [0, 1, 3, 5]
    assert torch.equal(got[0][there], got[1][there]) and torch.isfinite(got[1]).all() and torch.isnan(got[0][[2, 4, 6]]).all()
    net.fork(state, torch.zeros(0, dtype=torch.int32, device="cuda"))
    net.fork(state, dev(np.array([-1]), torch.int32))
    assert torch.equal(net.extend(y[1:2], state), net.extend(y[1:2], net.state(1, 48, fmt=fmt)))
