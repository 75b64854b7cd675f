"""GPU: the attention value network, whole sequences, single stages and forks, against the formulas in 64 bits.

The oracle rounds where the network does (bf16, 8 bits).  Where the two differ by a rounding of bf16 (2^-8) a number may fall on the
other side of a border of the 8-bit grid: one in 2^-8 / 2^-3 = 32 of them, by 2^-3 of itself, 0.022 of the whole in root mean square.
Two blocks' worth of such roundings (five each: queries, keys, values, outputs, units) and those of input and head: under sqrt(12) of it, 0.076; 0.12 is
allowed, and a single prediction three times that.  Values that the network gives for the same sequences in two ways differ by no more."""
import numpy as np
import pytest

from tests import kv_ref as K
from tests.test_gpu_ssm_value import bf16, close, ctx, norm, rounded, vf  # noqa: F401

pytestmark = pytest.mark.gpu


def predictions(w, x, lens, eight):
    """Per token of sequences one behind the other, from nothing; x float64 [tokens][F]."""
    H, G, D = (w[k] for k in ("heads", "kv_heads", "head_dim"))
    h, out = bf16(rounded(x, 2) @ rounded(w["w_in"], 3).T), None
    pos = np.concatenate([np.arange(n) for n in lens])
    held = (lambda v: rounded(v.reshape(-1, D), 2).reshape(v.shape)) if eight else bf16

    def normed(gain):
        nonlocal h
        s = h if out is None else h + out
        h = bf16(s)
        return rounded(norm(s, gain), 2)

    for b in w["blocks"]:
        qkv = bf16(normed(b["gain"]) @ rounded(b["w_qkv"], 3).T)
        q, k = (K.turned(p.reshape(len(x), -1, D), pos, w["freq"], False, 1.0)[0] for p in (qkv[:, :H * D], qkv[:, H * D:(H + G) * D]))
        q, k, v = bf16(q), held(k), held(qkv[:, (H + G) * D:].reshape(len(x), G, D))
        y, first = np.zeros((len(x), H, D)), 0
        for n in lens:
            for i in range(first, first + n):
                for hd in range(H):
                    z = k[first:i + 1, hd * G // H] @ q[i, hd] * D ** -0.5
                    p = np.exp(z - z.max())
                    y[i, hd] = p / p.sum() @ v[first:i + 1, hd * G // H]
            first += n
        out = bf16(rounded(bf16(y.reshape(len(x), -1)), 2) @ rounded(b["w_out"], 3).T)
        if w["hidden"]:
            u = np.maximum(bf16(normed(b["gain_up"]) @ rounded(b["w_up"], 3).T), 0.0)
            out = bf16(rounded(u, 2) @ rounded(b["w_down"], 3).T)
    return (normed(w["gain"]) @ rounded(w["w_head"], 3).T)[:, 0] + w["b_head"][0]


def dev(v, t=None):
    import torch
    return torch.from_numpy(np.ascontiguousarray(v)).to(t or torch.bfloat16).cuda()


SIZES = [(64, 256, 2, 4, 2, 64, 384, 2), (32, 96, 2, 3, 3, 40, 0, 1), (16, 64, 1, 8, 1, 128, 100, 1)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_prefixes_forks_extensions(vf, ctx, size):  # noqa: F811
    """Ragged prefixes, then rounds of a beam: fork, extend, fork to fewer; every value against the whole sequence's."""
    import torch
    from paper_2011_14486_amd import attention, inputs
    F, width, blocks, heads, kv_heads, D, hidden, fmt = size
    w = inputs.attention_weights(F, width, blocks, heads, kv_heads, D, hidden, seed=3)
    net = attention.AttentionValue(ctx, w)
    rng = np.random.default_rng(5)
    lens = [20, 1, 0, 37, 12, 32]
    x = bf16(rng.standard_normal((sum(lens), F)))
    state = net.state(17, 50, fmt=fmt)
    net.fork(state, dev(np.zeros(6), torch.int32))
    off = np.concatenate([[0], np.cumsum(lens)])
    got = net.score(dev(x), 6, max(lens), dev(off, torch.int32), state)
    each = predictions(w, x, lens, fmt == 2)
    size_of = np.sqrt((each ** 2).mean())
    sums = lambda e, ls: np.array([e[a:a + k].sum() for a, k in zip(np.concatenate([[0], np.cumsum(ls)]).astype(int), ls)])   # noqa: E731
    close(got.cpu().numpy(), sums(each, lens), size_of, np.maximum(lens, 1))
    assert float(got[2]) == 0.0
    kept = [x[a:a + k] for a, k in zip(off, lens)]
    for rows in (17, 5, 5, 17, 9):
        parents = rng.integers(0, len(kept), rows)
        net.fork(state, dev(parents, torch.int32))
        new = bf16(rng.standard_normal((rows, F)))
        got = net.extend(dev(new), state)
        kept = [np.concatenate([kept[p], new[r:r + 1]]) for r, p in enumerate(parents)]
        counts = [len(v) for v in kept]
        all_x = np.concatenate(kept)
        want = sums(predictions(w, all_x, counts, fmt == 2), counts)
        close(got.cpu().numpy(), want, size_of, np.array(counts))
        assert state.lengths.tolist() == counts
        # a page that a row goes on in is no other row's
        table, mine = state.table.cpu().numpy(), []
        for r, n in enumerate(counts):
            mine += table[r, (n - 1) // 16:].tolist()
        assert len(set(mine)) == len(mine)
        # and the whole sequences at once
        whole = net.score(dev(all_x), rows, max(counts), dev(np.concatenate([[0], np.cumsum(counts)]), torch.int32))
        if fmt == 1:
            close(whole.cpu().numpy(), want, size_of, np.array(counts))


def test_uniform_sequences_and_refusals(vf, ctx):  # noqa: F811
    import torch
    from paper_2011_14486_amd import attention, inputs
    w = inputs.attention_weights(64, 128, 2, 2, hidden=64, seed=1)
    net = attention.AttentionValue(ctx, w)
    x = bf16(np.random.default_rng(2).standard_normal((8 * 50, 64)))
    got = net.score(dev(x), 8)
    each = predictions(w, x, [50] * 8, False)
    close(got.cpu().numpy(), each.reshape(8, 50).sum(1), np.sqrt((each ** 2).mean()), 50)
    state = net.state(8, 64)
    again = net.score(dev(x), 8, state=state)
    assert torch.equal(got, again) and state.longest == 50
    with pytest.raises(ValueError):
        net.score(dev(x[:8 * 15]), 8, state=state)          # 65 stages
    with pytest.raises(ValueError):
        net.score(dev(x[:7]), 7, state=state)               # another number of rows
    with pytest.raises(ValueError):
        net.score(dev(x[:9]), 8)
    with pytest.raises(ValueError):
        net.fork(state, dev(np.zeros(9), torch.int32))
    assert torch.equal(net.score(dev(x[:0]), 8, state=state), state.total)
    assert net.score(dev(x[:0]), 0).shape == (0,)


def test_replays_equal_eager_calls(vf):  # noqa: F811
    """Extensions in a graph, replayed with other inputs between eager calls."""
    import torch
    from paper_2011_14486_amd import attention, inputs
    side = torch.cuda.Stream()
    ctx = vf.vf_create(0, stream=side)   # noqa: F811
    net = attention.AttentionValue(ctx, inputs.attention_weights(32, 96, 2, 4, 2, 64, 128, seed=2))
    rng = np.random.default_rng(1)
    x0, y0 = dev(rng.standard_normal((10 * 37, 32))), dev(rng.standard_normal((40, 32)))
    parents = dev(rng.integers(0, 10, 40), torch.int32)

    def start():
        s = net.state(40, 50)
        net.fork(s, torch.zeros(10, dtype=torch.int32, device="cuda"))
        net.score(x0, 10, state=s)
        net.fork(s, parents)
        return s

    kept = start()
    lengths, total = kept.lengths.clone(), kept.total.clone()
    y = y0.clone()
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = net.extend(y, kept)
    for k in (1.0, 0.5, 1.0, -2.0, 0.25):
        y.copy_(y0 * k)
        kept.lengths.copy_(lengths)
        kept.total.copy_(total)
        g.replay()
        replayed = got.clone()
        torch.cuda.synchronize()
        other = start()
        eager = net.extend(y0 * k, other)
        torch.cuda.synchronize()
        assert torch.equal(replayed, eager) and torch.equal(kept.total, other.total) and torch.equal(kept.lengths, other.lengths)
        x0.float().sum().item()
    vf.vf_destroy(ctx)
