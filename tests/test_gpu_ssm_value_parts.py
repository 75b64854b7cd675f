"""GPU: the state-space value network call by call.  Every operator that score and extend call is written down with what it took and
gave; each result is compared with the formula in 64 bits on the very inputs that it took, within that operator's own roundings (as
derived in test_gpu_norm_mx and test_gpu_ssm), and what each took has to be what the network's formula says."""
import numpy as np
import pytest

from tests import ops_ref as R
from tests.test_gpu_norm_mx import NORM, check_mx
from tests.test_gpu_ssm_value_slots import ctx, i32, vf  # noqa: F401

pytestmark = pytest.mark.gpu


def f64(t):
    return t.double().cpu().numpy()


def values(m):
    return R.mx_values(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.fmt, m.cols)


class Recorded:
    """The operators' calls while it is entered: (name, arguments, result)."""
    NAMES = {"vf_mx_quantize": ("x", "fmt"), "vf_mx_matmul": ("a", "w", "bias", "out_type"),
             "vf_rms_norm": ("x", "gain", "eps", "residual", "sum_out", "out_type"),
             "vf_ssm_scan": ("layer", "xbc", "dt", "z", "n_seq", "longest", "offsets", "state", "slots", "state_out", "slots_out"),
             "vf_ssm_step": ("layer", "xbc", "dt", "z", "state", "slots", "state_out", "slots_out")}

    def __init__(self, monkeypatch, binding):
        self.calls = []
        for name, order in self.NAMES.items():
            monkeypatch.setattr(binding, name, self.wrap(name, order, getattr(binding, name)))

    def wrap(self, name, order, fn):
        def call(ctx, *args, **kw):  # noqa: F811
            given = dict(zip(order, args), **kw)
            if given.get("state") is not None:      # (it may be left in its own place)
                given["before"] = tuple(t.clone() for t in given["state"])
            out = fn(ctx, *args, **kw)
            self.calls.append((name, given, out))
            return out
        return call


def check_quantize(given, q):
    codes, scales = R.quantize(f64(given["x"]), q.fmt)
    assert q.fmt == given["fmt"] and np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(R.code_values(q.codes.cpu().numpy(), q.fmt), codes)


def check_matmul(given, y):
    a, w = values(given["a"]), values(given["w"])
    b = 0.0 if given.get("bias") is None else f64(given["bias"])
    want, mag, K = a @ w.T + b, np.abs(a) @ np.abs(w).T + np.abs(b), a.shape[1]
    wide = given.get("out_type", 1) == 0
    tol = (K + 2) * 2.0 ** -23 * mag + (0 if wide else 7 * 2.0 ** -13 * mag + R.UBF * (1 + 1e-3) * np.abs(want))
    assert (np.abs(f64(y) - want) <= tol).all()


def check_norm(given, result):
    q, total = result
    s = f64(given["x"]) + (0.0 if given.get("residual") is None else f64(given["residual"]))
    check_mx(None, q, s / np.sqrt((s * s).mean(1, keepdims=True) + given.get("eps", 1e-5)) * f64(given["gain"]), NORM)
    assert (total is None) == (given.get("residual") is None)
    if total is not None:
        assert (np.abs(f64(total) - s) <= (R.UBF + R.U32) * np.abs(s)).all()


def check_scan(given, out, spans, chunks):
    la = given["layer"]
    lay = dict(zip(("conv_w", "conv_b", "a", "d", "dt_bias"), (f64(t) for t in la.tensors)))
    n = len(spans)
    slots = list(range(n)) if given.get("slots") is None else given["slots"].tolist()
    before = given.get("before")
    want, conv, st, omag, smag = R.ssm((la.heads, la.head_dim, la.groups, la.n_state, la.taps), lay, f64(given["xbc"]), f64(given["dt"]),
                                       f64(given["z"]), spans, None if before is None else tuple(f64(t) for t in before), slots)
    base = (128 + max([c for _, c in spans] + [1]) + la.n_state) * R.U32
    live = ~np.isnan(want)
    assert (np.abs(f64(out) - want)[live] <= (((4 * R.UBF if chunks else 0) + base) * omag + R.UBF * np.abs(want))[live]).all()
    if given.get("state_out") is not None:
        to = np.arange(n) if given.get("slots_out") is None else np.asarray(given["slots_out"].tolist())
        kept = to >= 0
        got = tuple(f64(t)[to[kept]] for t in given["state_out"])
        assert np.array_equal(got[0], conv[kept])
        assert (np.abs(got[1] - st[kept]) <= (((3 * 2.0 ** -16 if chunks else 0) + base) * smag)[kept]).all()


def same(a, b):
    """One and the same piece of memory."""
    return a.data_ptr() == b.data_ptr() and a.shape == b.shape and a.stride() == b.stride()


def check_network(net, x, calls, spans, chunks):
    """All calls of one pass; returns the tokens' predictions."""
    todo = list(calls)

    def take(name):
        got, given, out = todo.pop(0)
        assert got == name
        {"vf_mx_quantize": check_quantize, "vf_mx_matmul": check_matmul, "vf_rms_norm": check_norm}.get(name, lambda *_: None)(given, out)
        return given, out

    q, rows = take("vf_mx_quantize")
    assert same(q["x"], x) and rows.fmt == 2
    m, h = take("vf_mx_matmul")
    assert m["a"] is rows and m["w"] is net.w_in and m.get("bias") is None
    out = None
    for k, (gain, w_proj, layer, gain_out, w_out) in enumerate(net.blocks):
        n, (rows, total) = take("vf_rms_norm")
        assert n["gain"] is gain and n["out_type"] == 2 and (n["x"] is h and n.get("residual") is None if k == 0 else n["x"] is out and n["residual"] is h)
        h = h if total is None else total
        m, proj = take("vf_mx_matmul")
        assert m["a"] is rows and m["w"] is w_proj and m.get("bias") is None
        name, given, y = todo.pop(0)
        inner, C = layer.heads * layer.head_dim, layer.channels
        assert name in ("vf_ssm_scan", "vf_ssm_step") and given["layer"] is layer and same(given["z"], proj[:, :inner])
        assert same(given["xbc"], proj[:, inner:inner + C]) and same(given["dt"], proj[:, inner + C:])
        check_scan(given, y, spans, chunks)
        n, (rows, total) = take("vf_rms_norm")
        assert n["x"] is y and n["gain"] is gain_out and n.get("residual") is None and n["out_type"] == 2
        m, out = take("vf_mx_matmul")
        assert m["a"] is rows and m["w"] is w_out and m.get("bias") is None
    n, (rows, _) = take("vf_rms_norm")
    assert n["x"] is out and n["residual"] is h and n["gain"] is net.gain
    m, y = take("vf_mx_matmul")
    assert m["a"] is rows and m["w"] is net.w_head and m["bias"] is net.b_head and m["out_type"] == 0 and not todo
    return f64(y)[:, 0]


def check_weights(net, w):
    def four(m, v):
        codes, scales = R.quantize(v.astype(np.float64), 3)
        assert m.fmt == 3 and m.cols == v.shape[1] and np.array_equal(m.scales.cpu().numpy(), scales)
        assert np.array_equal(R.code_values(m.codes.cpu().numpy(), 3), codes)

    four(net.w_in, w["w_in"])
    four(net.w_head, w["w_head"])
    assert np.array_equal(f64(net.gain), w["gain"]) and np.array_equal(f64(net.b_head), w["b_head"]) and len(net.blocks) == len(w["blocks"])
    for (gain, w_proj, layer, gain_out, w_out), b in zip(net.blocks, w["blocks"]):
        four(w_proj, b["w_proj"])
        four(w_out, b["w_out"])
        assert np.array_equal(f64(gain), b["gain"]) and np.array_equal(f64(gain_out), b["gain_out"])
        for t, name in zip(layer.tensors, ("conv_w", "conv_b", "a", "d", "dt_bias")):
            assert np.array_equal(f64(t), b[name])
        assert (layer.heads, layer.head_dim, layer.groups, layer.n_state) == tuple(w[k] for k in ("heads", "head_dim", "groups", "n_state"))


def close(value, each, before=0.0):
    """A value against the sum of its predictions: an fp32 addition for each."""
    tol = (len(each) + 2) * 2.0 ** -24 * (np.abs(each).sum() + abs(before))
    assert abs(float(value) - (each.sum() + before)) <= tol


@pytest.mark.parametrize("size", [(64, 256, 2, 4, 64, 1, 64, 4), (32, 96, 3, 2, 48, 2, 16, 4), (16, 64, 1, 3, 20, 1, 12, 3)], ids=str)
def test_every_call_of_the_network(vf, ctx, monkeypatch, size):  # noqa: F811
    """Ragged prefixes, their continuation in place, extensions from some slots into others, and uniform sequences."""
    import torch
    from paper_2011_14486_amd import binding, inputs, ssm
    F, width, blocks, heads, P, G, N, W = size
    w = inputs.ssm_weights(F, width, blocks, heads, P, G, N, W, seed=4)
    net = ssm.SsmValue(ctx, w)
    check_weights(net, w)
    in_chunks = P % 16 == 0 and N % 16 == 0 and W <= 4
    rec = Recorded(monkeypatch, binding)
    stages = lambda n, s: torch.from_numpy(np.random.default_rng(s).standard_normal((n, F))).to(torch.bfloat16).cuda()   # noqa: E731

    def run(call, x, spans, chunks):
        rec.calls.clear()
        got = call(x)
        return got, check_network(net, x, rec.calls, spans, chunks)

    lens = [20, 1, 0, 37, 12]
    first = np.concatenate([[0], np.cumsum(lens)])
    spans = list(zip(first[:-1], lens))
    state = net.state(5)
    offsets = i32(*first)
    got, each = run(lambda x: net.score(x, 5, 37, offsets, state_out=state), stages(70, 1), spans, in_chunks)
    for s, (a, n) in enumerate(spans):
        close(got[s], each[a:a + n])
    assert torch.equal(state.total, got)
    # on from the states, which are left in their own places
    before = f64(state.total)
    got, each = run(lambda x: net.score(x, 5, 37, offsets, state=state, state_out=state), stages(70, 2), spans, in_chunks)
    for s, (a, n) in enumerate(spans):
        close(got[s], each[a:a + n], before[s])
    assert torch.equal(state.total, got)
    # one more stage of some rows
    before, left = f64(state.total), net.state(9)
    slots, to = [4, 0, -1, 4, 2, 1, 3], [8, -1, 0, 3, 2, 5, 1]
    got, each = run(lambda x: net.extend(x, state, i32(*slots), left, i32(*to)), stages(7, 3), [(r, 1) for r in range(7)], False)
    for r in range(7):
        close(got[r], each[r:r + 1], before[slots[r]] if slots[r] >= 0 else 0.0)
        assert to[r] < 0 or float(left.total[to[r]]) == float(got[r])
    # and of all rows, in place
    before = f64(left.total)
    got, each = run(lambda x: net.extend(x, left, None, left), stages(9, 4), [(r, 1) for r in range(9)], False)
    for r in range(9):
        close(got[r], each[r:r + 1], before[r])
    assert torch.equal(left.total, got)
    got, each = run(lambda x: net.score(x, 6), stages(60, 5), [(10 * m, 10) for m in range(6)], in_chunks)
    for m in range(6):
        close(got[m], each[10 * m:10 * m + 10])
