"""GPU: the state-space value network, whole sequences and single stages, against the formulas in 64 bits.

The oracle rounds where the network does (bf16, 8 bits).  Where the two differ by a rounding of bf16 (2^-8) a number may fall on the
other side of a border of the 8-bit grid: one in 2^-8 / 2^-3 = 32 of them, by 2^-3 of itself, 0.022 of the whole in root mean square.
Three blocks' worth of such roundings (two each) and those of input and head: under sqrt(8) of it, 0.063; 0.12 is allowed, and a
single prediction three times that."""
import numpy as np
import pytest

from tests import ops_ref as R

pytestmark = pytest.mark.gpu
RMS, ONE = 0.12, 0.36


@pytest.fixture(scope="module")
def vf():
    import paper_2011_14486_amd as pkg
    return pkg.load()


@pytest.fixture(scope="module")
def ctx(vf):
    c = vf.vf_create(0)
    yield c
    vf.vf_destroy(c)


def bf16(v):
    import torch
    return torch.from_numpy(np.ascontiguousarray(v)).to(torch.bfloat16).double().numpy()


def rounded(v, fmt):
    codes, scales = R.quantize(np.asarray(v, np.float64), fmt)
    return (codes * np.ldexp(1.0, scales.astype(int) - 127)[..., None]).reshape(v.shape[0], -1)[:, :v.shape[1]]


def norm(x, gain):
    return x / np.sqrt((x * x).mean(1, keepdims=True) + 1e-5) * gain


def predictions(w, x, spans):
    """Per token, sequences from nothing; x float64 [tokens][F]."""
    H, P, G, N = (w[k] for k in ("heads", "head_dim", "groups", "n_state"))
    inner, C = H * P, H * P + 2 * G * N
    h = bf16(rounded(x, 2) @ rounded(w["w_in"], 3).T)
    out = None
    for b in w["blocks"]:
        s = h if out is None else h + out
        proj = bf16(rounded(norm(s, b["gain"]), 2) @ rounded(b["w_proj"], 3).T)
        h = bf16(s)
        y, *_ = R.ssm((H, P, G, N, b["conv_w"].shape[1]), {k: np.asarray(v, np.float64) for k, v in b.items()}, proj[:, inner:inner + C],
                      proj[:, inner + C:], proj[:, :inner], spans, None, [-1] * len(spans))
        out = bf16(rounded(norm(bf16(y), b["gain_out"]), 2) @ rounded(b["w_out"], 3).T)
    return (rounded(norm(h + out, w["gain"]), 2) @ rounded(w["w_head"], 3).T)[:, 0] + w["b_head"][0]


def close(got, want, each, count):
    """Sums over `count` predictions whose root mean square is `each`."""
    err = np.abs(np.asarray(got, np.float64) - want) / (each * np.sqrt(count))
    assert np.sqrt((err ** 2).mean()) <= RMS and err.max() <= ONE, (np.sqrt((err ** 2).mean()), err.max())


SIZES = [(64, 256, 2, 4, 64, 1, 64, 4), (32, 96, 3, 2, 48, 2, 16, 4), (16, 64, 1, 3, 20, 1, 12, 3)]


@pytest.mark.parametrize("size", SIZES, ids=str)
def test_prefixes_then_extensions(vf, ctx, size):
    """Ragged prefixes, then three rounds of a beam of extensions with shared parents; every value against the whole sequence's."""
    import torch
    from paper_2011_14486_amd import inputs, ssm
    F, width, blocks, heads, P, G, N, W = size
    w = inputs.ssm_weights(F, width, blocks, heads, P, G, N, W, seed=3)
    net = ssm.SsmValue(ctx, w)
    rng = np.random.default_rng(5)
    lens = [20, 1, 0, 37, 12]
    n, rows, rounds = len(lens), 9, 3
    first = np.concatenate([[0], np.cumsum(lens)])
    x = bf16(rng.standard_normal((first[-1], F)))
    dev = lambda v, t=torch.bfloat16: torch.from_numpy(np.ascontiguousarray(v)).to(t).cuda()   # noqa: E731
    prefixes = net.state(n)
    got = net.score(dev(x), n_seq=n, longest=max(lens), offsets=dev(first, torch.int32), state_out=prefixes)
    each = predictions(w, x, list(zip(first[:-1], lens)))
    size_of = np.sqrt((each ** 2).mean())
    want = np.array([each[a:a + k].sum() for a, k in zip(first, lens)])
    close(got.cpu().numpy(), want, size_of, np.maximum(lens, 1))
    assert float(got[2]) == 0.0
    # extensions: row r of a round continues row parents[r] of the one before
    kept, state = [x[a:a + k] for a, k in zip(first, lens)], prefixes
    for k in range(rounds):
        parents = rng.integers(0, len(kept), rows)
        new = bf16(rng.standard_normal((rows, F)))
        nxt = net.state(rows + 2)
        to = rng.permutation(rows + 2)[:rows]
        got = net.extend(dev(new), state, dev(parents, torch.int32), nxt, dev(to, torch.int32))
        kept = [np.concatenate([kept[p], new[r:r + 1]]) for r, p in enumerate(parents)]
        all_x, counts = np.concatenate(kept), [len(v) for v in kept]
        at = np.concatenate([[0], np.cumsum(counts)[:-1]])
        each = predictions(w, all_x, list(zip(at, counts)))
        want = np.array([each[a:a + c].sum() for a, c in zip(at, counts)])
        close(got.cpu().numpy(), want, size_of, np.array(counts))
        # and the whole sequences by the scan
        whole = net.score(dev(all_x), n_seq=rows, longest=max(counts), offsets=dev(np.append(at, len(all_x)), torch.int32))
        close(whole.cpu().numpy(), want, size_of, np.array(counts))
        # the next round's parents in the order of rows
        state = ssm.SsmState([tuple(t[dev(to, torch.int64)].contiguous() for t in b) for b in nxt.blocks], nxt.total[dev(to, torch.int64)])


def test_uniform_sequences(vf, ctx):
    """The layout of the recurrent scorer's inputs, [M][T][F]."""
    import torch
    from paper_2011_14486_amd import inputs, ssm
    w = inputs.ssm_weights(64, 128, 2, 2, seed=1)
    net = ssm.SsmValue(ctx, w)
    M, T = 8, 50
    x = bf16(np.random.default_rng(2).standard_normal((M * T, 64)))
    got = net.score(torch.from_numpy(x).to(torch.bfloat16).cuda().reshape(M, T, 64).reshape(M * T, 64), n_seq=M).cpu().numpy()
    each = predictions(w, x, [(T * m, T) for m in range(M)])
    close(got, each.reshape(M, T).sum(1), np.sqrt((each ** 2).mean()), T)
