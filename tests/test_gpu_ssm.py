"""GPU: convolution with selective scan, whole sequences and single tokens, against the recurrence in 64 bits.

Tolerances go by the same sums over magnitudes (ops_ref.ssm).  Token by token in fp32: each of x, B, C is a sum of W + 1 terms
through silu (slope at most 1.1, exponential and reciprocal about 16 roundings): under 30 of 2^-24 of its magnitude each; the step
under 10, decays under 30 over the memory's length, one more per token and per n of the sums: (128 + T + N) 2^-24.
In chunks (bf16): x, B, C, their products within a chunk and the state before a chunk are rounded to bf16 (2^-8 each, at most
four of them meet in a product); what the state takes up is in two parts of 8 bits each, so three errors of 2^-16.  An
output in bf16 is rounded once more."""
import numpy as np
import pytest

from tests import ops_ref as R

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def vf():
    import paper_2011_14486_amd as pkg
    return pkg.load()


@pytest.fixture(scope="module")
def ctx(vf):
    c = vf.vf_create(0)
    yield c
    vf.vf_destroy(c)


class Case:
    """Inputs of one call: sizes (H, P, G, N, W), lengths of the sequences, type."""

    def __init__(self, vf, sizes, lens, kind, gate=True, plain=False, gap=0, slots=0, seed=0, scale=1.0):
        import torch
        H, P, G, N, W = sizes
        C = H * P + 2 * G * N
        rng = np.random.default_rng([H, P, G, N, W, len(lens), seed])
        self.vf, self.sizes, self.lens, self.kind = vf, sizes, list(lens), kind
        self.dtype = torch.bfloat16 if kind == "bf16" else torch.float32
        lay = dict(conv_w=rng.uniform(-1, 1, (C, W)) / np.sqrt(W), a=-rng.uniform(1, 16, H))
        if not plain:
            dt0 = np.exp(rng.uniform(np.log(0.001), np.log(0.1), H))
            lay.update(conv_b=rng.uniform(-0.5, 0.5, C), d=rng.standard_normal(H), dt_bias=np.log(np.expm1(dt0)))
        dev = {k: torch.from_numpy(v).float().cuda() for k, v in lay.items()}
        self.layer = vf.SsmLayer(H, P, G, N, **dev)
        self.lay = {k: v.double().cpu().numpy() for k, v in dev.items()}
        self.first = np.concatenate([[0], np.cumsum(lens)[:-1]]).astype(int) + gap
        self.tokens = int(np.sum(lens)) + 2 * gap
        # views of a wider matrix, as a projection leaves them, with NaN in the rows and columns of nobody
        wide = torch.full((self.tokens, 3 + H * P + C + H + 2), float("nan"), dtype=self.dtype, device="cuda")
        body = torch.from_numpy(rng.standard_normal((self.tokens - 2 * gap, H * P + C + H)) * scale).to(self.dtype).cuda()
        wide[gap:self.tokens - gap, 3:-2] = body
        self.z = wide[:, 3:3 + H * P] if gate else None
        self.xbc, self.dt = wide[:, 3 + H * P:3 + H * P + C], wide[:, 3 + H * P + C:-2]
        self.state = None
        if slots:
            self.state = (torch.from_numpy(rng.standard_normal((slots, C, W - 1))).to(self.dtype).cuda(),
                          torch.from_numpy(rng.standard_normal((slots, H, P, N))).float().cuda())
        self.offsets = torch.from_numpy(np.concatenate([self.first, [self.tokens - gap]]).astype(np.int32)).cuda()

    def ref(self, slots=None, state="own"):
        f = lambda t: None if t is None else t.double().cpu().numpy()   # noqa: E731
        st = self.state if isinstance(state, str) else state
        return R.ssm(self.sizes, self.lay, f(self.xbc), f(self.dt), f(self.z), list(zip(self.first, self.lens)),
                     None if st is None else (f(st[0]), f(st[1])),
                     list(range(len(self.lens))) if slots is None else list(slots))

    def check(self, out, ref, chunks, state=None, rows=None):
        """out, and state = (conv, ssm) of the sequences in order, against the reference."""
        want, conv, st, omag, smag = ref
        T, N = max(self.lens + [1]), self.sizes[3]
        base = (128 + T + N) * R.U32
        u = R.UBF if self.kind == "bf16" else R.U32
        live = ~np.isnan(want)
        got = out.double().cpu().numpy()
        err, tol = np.abs(got - want)[live], ((4 * R.UBF if chunks else 0) + base) * omag[live] + u * np.abs(want)[live]
        assert (err <= tol).all(), (float(np.nanmax(err / tol)), err.max())
        if state is not None:
            c, s = (t.double().cpu().numpy() for t in state)
            assert np.array_equal(c, conv)
            tol = ((3 * 2.0 ** -16 if chunks else 0) + base) * smag
            assert (np.abs(s - st) <= tol).all(), float((np.abs(s - st) / np.maximum(tol, 1e-300)).max())


def in_chunks(kind, sizes):
    """The documented rule for sequences on the matrix cores."""
    return kind == "bf16" and sizes[1] % 16 == 0 and sizes[3] % 16 == 0 and sizes[4] <= 4


# (H, P, G, N, W): odd sizes token by token, sizes that run in chunks, shared groups, all numbers of taps
SIZES = [(1, 1, 1, 1, 1), (2, 3, 1, 5, 2), (3, 17, 1, 30, 4), (4, 40, 2, 24, 3), (2, 100, 2, 129, 4), (1, 256, 1, 256, 8),
         (1, 16, 1, 32, 4), (4, 64, 1, 64, 4), (6, 64, 2, 128, 4), (3, 48, 1, 96, 2), (5, 32, 5, 32, 1), (8, 64, 1, 32, 8),
         (2, 64, 1, 256, 4), (7, 16, 1, 160, 3), (2, 128, 1, 64, 4), (1, 256, 1, 256, 4), (3, 80, 1, 16, 4),
         (2, 112, 2, 48, 4)]
LENS = [[1], [2], [50, 50], [64], [65, 0, 1, 63, 2], [7, 130, 3], [33, 31, 32, 96, 97]]


@pytest.mark.parametrize("sizes", SIZES, ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_scan(vf, ctx, sizes, kind):
    import torch
    H, P, G, N, W = sizes
    for k, lens in enumerate(LENS):
        c = Case(vf, sizes, lens, kind, gate=k % 2 == 0, plain=k % 3 == 2, gap=k % 2, slots=len(lens) if k != 3 else 0, seed=k)
        new = c.layer.state(len(lens), c.dtype)
        for t in new:
            t.fill_(float("nan"))
        big = torch.full((c.tokens, H * P + 3), 5.0, dtype=c.dtype, device="cuda")
        out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), longest=max(lens), offsets=c.offsets, state=c.state,
                             state_out=new, out=big[:, 1:1 + H * P])
        c.check(out, c.ref(), in_chunks(kind, sizes), new)
        assert bool((big[:, 0] == 5).all()) and bool((big[:, 1 + H * P:] == 5).all())
        if k % 2:  # rows that belong to no sequence are not written
            assert bool((big[0] == 5).all()) and bool((big[-1] == 5).all())


@pytest.mark.parametrize("sizes", [(4, 64, 1, 64, 4), (3, 17, 1, 30, 4), (8, 64, 1, 128, 4)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_uniform_sequences_without_offsets_and_state(vf, ctx, sizes, kind):
    c = Case(vf, sizes, [50] * 9, kind)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=9)
    c.check(out, c.ref(), in_chunks(kind, sizes))


@pytest.mark.parametrize("sizes,kind", [((2, 64, 1, 128, 4), "bf16"), ((4, 32, 2, 64, 4), "bf16"), ((1, 48, 1, 32, 2), "bf16"),
                                        ((2, 20, 1, 12, 4), "fp32")], ids=str)
@pytest.mark.parametrize("lens", [[3000], [2500, 10, 0, 1700]], ids=str)
def test_long_sequences(vf, ctx, sizes, kind, lens):
    """A few sequences that are long (split along their length on the matrix cores)."""
    c = Case(vf, sizes, lens, kind, slots=len(lens))
    new = c.layer.state(len(lens), c.dtype)
    args = dict(n_seq=len(lens), longest=max(lens), offsets=c.offsets, state=c.state, state_out=new)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
    ref = c.ref()
    c.check(out, ref, in_chunks(kind, sizes), new)
    # told that the sequences are shorter than they are, and longer: the same results in other ways
    for longest in (100, 100000):
        again = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **dict(args, longest=longest))
        c.check(again, ref, in_chunks(kind, sizes), new)


@pytest.mark.parametrize("sizes", [(1, 1, 1, 1, 1), (3, 17, 1, 30, 4), (4, 64, 2, 64, 4), (32, 64, 1, 128, 4), (2, 100, 1, 129, 2),
                                   (1, 256, 1, 256, 8)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("rows", [1, 5, 300])
def test_step_from_shared_parents(vf, ctx, sizes, kind, rows):
    import torch
    if rows == 300 and sizes[0] == 32:
        rows = 40
    rng = np.random.default_rng(rows)
    c = Case(vf, sizes, [1] * rows, kind, slots=3)
    slots = rng.integers(-1, 3, rows)
    to = rng.permutation(rows + 4)[:rows]
    to[::3] = -1
    new = c.layer.state(rows + 4, c.dtype)
    for t in new:
        t.fill_(3.0)
    i32 = lambda v: torch.from_numpy(np.asarray(v, np.int32)).cuda()   # noqa: E731
    out = vf.vf_ssm_step(ctx, c.layer, c.xbc, c.dt, c.z, state=c.state, slots=i32(slots), state_out=new, slots_out=i32(to))
    ref = c.ref(slots)
    c.check(out, ref, False)
    want, conv, st, omag, smag = ref
    kept = np.flatnonzero(to >= 0)
    got = tuple(t.double().cpu().numpy() for t in new)
    assert np.array_equal(got[0][to[kept]], conv[kept])
    assert (np.abs(got[1][to[kept]] - st[kept]) <= (129 + sizes[3]) * R.U32 * smag[kept]).all()
    rest = np.setdiff1d(np.arange(rows + 4), to[kept])
    assert (got[0][rest] == 3).all() and (got[1][rest] == 3).all()


@pytest.mark.parametrize("sizes", [(4, 64, 2, 64, 4), (3, 17, 1, 30, 4), (2, 32, 1, 32, 8)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_state_in_place_token_by_token_equals_the_sequence(vf, ctx, sizes, kind):
    """A prompt, then single tokens, then a prompt of two tokens (shorter than the convolution), all in one state buffer."""
    import torch
    n, T = 6, 40
    H, P = sizes[0], sizes[1]
    c = Case(vf, sizes, [T] * n, kind)
    state = c.layer.state(n + 2, c.dtype)
    slots = torch.tensor([3, 0, 7, 1, 2, 5], dtype=torch.int32, device="cuda")
    out = torch.empty((n, T, H * P), dtype=c.dtype, device="cuda")
    part = lambda t, i, j: t.reshape(n, T, -1)[:, i:j].reshape(n * (j - i), -1)   # noqa: E731
    first = vf.vf_ssm_scan(ctx, c.layer, part(c.xbc, 0, 30), part(c.dt, 0, 30), part(c.z, 0, 30), n_seq=n, state_out=state, slots_out=slots)
    out[:, :30] = first.reshape(n, 30, -1)
    for t in range(30, 38):
        y = vf.vf_ssm_step(ctx, c.layer, part(c.xbc, t, t + 1), part(c.dt, t, t + 1), part(c.z, t, t + 1), state=state, slots=slots,
                           state_out=state, slots_out=slots)
        out[:, t] = y
    y = vf.vf_ssm_scan(ctx, c.layer, part(c.xbc, 38, 40), part(c.dt, 38, 40), part(c.z, 38, 40), n_seq=n, state=state, slots=slots,
                       state_out=state, slots_out=slots)
    out[:, 38:] = y.reshape(n, 2, -1)
    at = slots.long()
    c.check(out.reshape(n * T, -1), c.ref(), in_chunks(kind, sizes), (state[0][at], state[1][at]))
    assert not state[0][[4, 6]].any() and not state[1][[4, 6]].any()


@pytest.mark.parametrize("sizes,rows", [((4, 16, 1, 16, 4), 2600), ((4, 24, 2, 40, 3), 2100), ((8, 20, 1, 10, 8), 1300)], ids=str)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_steps_of_many_rows(vf, ctx, sizes, rows, kind):
    """More rows than workgroups: a workgroup takes several, from shared parents into slots of their own, then in place."""
    import torch
    rng = np.random.default_rng(rows)
    c = Case(vf, sizes, [1] * rows, kind, slots=7)
    slots = rng.integers(-1, 7, rows)
    new = c.layer.state(rows, c.dtype)
    out = vf.vf_ssm_step(ctx, c.layer, c.xbc, c.dt, c.z, state=c.state, slots=torch.from_numpy(slots.astype(np.int32)).cuda(), state_out=new)
    c.check(out, c.ref(slots), False, new)
    before = tuple(t.clone() for t in new)
    out = vf.vf_ssm_step(ctx, c.layer, c.xbc, c.dt, c.z, state=new, state_out=new)
    c.check(out, c.ref(range(rows), before), False, new)


@pytest.mark.parametrize("sizes,kind,lens", [((4, 17, 1, 30, 4), "fp32", [2, 3, 0, 1] * 800), ((2, 64, 1, 64, 4), "bf16", [9, 0, 40, 33] * 300),
                                             ((5, 64, 1, 128, 2), "bf16", [50] * 150), ((3, 30, 1, 20, 2), "bf16", [1] * 3000)],
                         ids=["few tokens", "chunks, some empty", "chunks, uniform", "one token"])
def test_many_short_sequences(vf, ctx, sizes, kind, lens):
    """More sequences than workgroups."""
    c = Case(vf, sizes, lens, kind)
    new = c.layer.state(len(lens), c.dtype)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), longest=max(lens), offsets=c.offsets, state_out=new)
    ref = c.ref()
    c.check(out, ref, in_chunks(kind, sizes) and max(lens) > 8, new)
    if len(set(lens)) == 1:
        out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n_seq=len(lens), state_out=new)
        c.check(out, ref, in_chunks(kind, sizes) and max(lens) > 8, new)


@pytest.mark.parametrize("kind,sizes", [("bf16", (4, 64, 1, 64, 4)), ("fp32", (3, 17, 1, 30, 4))], ids=str)
def test_bad_slots_and_offsets(vf, ctx, kind, sizes):
    """Slots that are not there read as NaN and are not written; ranges that are not there are empty."""
    import torch
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")   # noqa: E731
    lens = [20, 20, 20, 20]
    c = Case(vf, sizes, lens, kind, slots=4)
    new = c.layer.state(4, c.dtype)
    args = dict(n_seq=4, longest=20, state=c.state, state_out=new)
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, offsets=c.offsets, slots=i32([0, 4, -2, 2 ** 31 - 1]),
                         slots_out=i32([4, 1, 2, -5]), **args)
    want = c.ref([0, -1, -1, -1])
    c.check(out[:20], tuple(v[:20] if v.shape[0] == 80 else v[:1] for v in want), in_chunks(kind, sizes))
    assert bool(out[20:].isnan().all())
    assert bool(new[1][1:3].isnan().all()) and not new[1][[0, 3]].any() and not new[0][[0, 3]].any()
    out = torch.full_like(out, 2.0)
    for t in new:
        t.zero_()
    for off in ([0, 20, 15, 30, 90], [-3, 20, 40, 60, 2 ** 31 - 1], [0, -20, 40, -1, -1]):
        o = np.array(off, dtype=np.int64)
        empty = [s for s in range(4) if o[s] < 0 or o[s + 1] < o[s] or o[s + 1] > 80]
        out.fill_(2.0)
        vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, offsets=i32(off), out=out, **args)
        written = np.zeros(80, bool)
        for s in range(4):
            if s not in empty:
                written[o[s]:o[s + 1]] = True
        got = out.float().cpu().numpy()
        assert (got[~written] == 2).all() and np.isfinite(got).all()
        for s in empty:
            assert torch.equal(new[0][s], c.state[0][s]) and torch.equal(new[1][s], c.state[1][s])


@pytest.mark.parametrize("kind,sizes", [("bf16", (4, 64, 1, 64, 4)), ("fp32", (3, 17, 1, 30, 4))], ids=str)
def test_nan_and_large_steps_stay_where_they_are(vf, ctx, kind, sizes):
    """A NaN in one sequence reaches that sequence only; steps so large that the state is forgotten at once, and so
    small that nothing is, give what the formulas say."""
    import torch
    lens = [40, 70, 40]
    c = Case(vf, sizes, lens, kind, seed=4)
    args = dict(n_seq=3, longest=70, offsets=c.offsets)
    c.dt[40:110] = 60.0      # e^(60 a) = 0: only the token itself counts
    c.dt[110:150] = -60.0    # a step of e^-60: nothing is taken up
    clean = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
    c.check(clean, c.ref(), in_chunks(kind, sizes))
    c.xbc[60, 0] = float("nan")
    hurt = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
    assert torch.equal(hurt[:40], clean[:40]) and torch.equal(hurt[110:], clean[110:])
    assert torch.equal(hurt[40:60, 1:], clean[40:60, 1:]) or in_chunks(kind, sizes)
    assert bool(hurt[60, :1].isnan().all())


@pytest.mark.parametrize("sizes", [(4, 64, 1, 64, 4), (2, 64, 1, 128, 4), (3, 48, 1, 32, 2), (1, 16, 1, 256, 4)], ids=str)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")], ids=str)
@pytest.mark.parametrize("lens", [[100], [70, 40]], ids=str)
def test_what_is_not_finite_reaches_no_token_before_its_own(vf, ctx, sizes, value, lens):
    """In chunks: x, B, C, step or gate of one token; outputs before it are as without, and from it on NaN or infinite where the
    formulas have it."""
    import torch
    H, P, G, N, W = sizes
    c = Case(vf, sizes, lens, "bf16", seed=5)
    args = dict(n_seq=len(lens), longest=max(lens), offsets=c.offsets)
    clean = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
    for part, col, at in ((c.xbc, 5, 45), (c.xbc, H * P - 1, 33), (c.xbc, H * P + 3, 50), (c.xbc, H * P + G * N + 2, 20), (c.dt, 0, 41),
                          (c.z, 7, 35)):
        if part is c.dt and value < 0:
            continue    # a step of zero
        kept = part[at, col].clone()
        part[at, col] = value
        hurt = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, **args)
        part[at, col] = kept
        assert torch.equal(hurt[:at], clean[:at])
        assert torch.equal(hurt[lens[0]:], clean[lens[0]:])
        if part is c.z:
            got = torch.ones_like(hurt[at], dtype=torch.bool)
            got[col] = False
            assert torch.equal(hurt[at][got], clean[at][got]) and torch.equal(hurt[at + 1:], clean[at + 1:])
            if value > 0 or value != value:
                assert not bool(hurt[at, col].isfinite())
        elif part is c.xbc and col < H * P:
            others = torch.ones(H * P, dtype=torch.bool, device="cuda")
            others[col] = False
            assert torch.equal(hurt[:, others], clean[:, others])
            if value > 0 or value != value:
                lasting = hurt[at:lens[0], col]
                assert not bool(lasting.isfinite().any())


def test_no_sequences_and_empty_ones(vf, ctx):
    import torch
    c = Case(vf, (2, 16, 1, 32, 4), [5], "bf16", slots=3)
    y = vf.vf_ssm_scan(ctx, c.layer, c.xbc[:0], c.dt[:0], c.z[:0], n_seq=0)
    assert y.shape == (0, 32)
    new = c.layer.state(3, c.dtype)
    y = vf.vf_ssm_scan(ctx, c.layer, c.xbc[:0], c.dt[:0], None, n_seq=3, state=c.state, state_out=new)
    torch.cuda.synchronize()
    assert y.shape == (0, 32) and torch.equal(new[0], c.state[0]) and torch.equal(new[1], c.state[1])
    y = vf.vf_ssm_scan(ctx, c.layer, c.xbc[:0], c.dt[:0], None, n_seq=3, state_out=new)
    torch.cuda.synchronize()
    assert not new[0].any() and not new[1].any()


@pytest.mark.parametrize("lens", [[40] * 5, [2000]], ids=str)
def test_scan_in_a_graph(vf, lens):
    """Captured on a stream of its own, replayed with other inputs between eager calls."""
    import torch
    side = torch.cuda.Stream()
    x = vf.vf_create(0, stream=side)
    c = Case(vf, (2, 64, 1, 64, 4), lens, "bf16", slots=len(lens))
    new = c.layer.state(len(lens), c.dtype)
    dt = c.dt.clone()
    call = lambda d: vf.vf_ssm_scan(x, c.layer, c.xbc, d, c.z, n_seq=len(lens), state=c.state, state_out=new)   # noqa: E731
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        out = call(dt)
    for k in (0.0, 1.0, 0.0, -2.0):
        dt.copy_(c.dt + k)
        for t in new:
            t.zero_()
        g.replay()
        torch.cuda.synchronize()
        got, kept = out.clone(), [t.clone() for t in new]
        c2 = c.dt + k
        keep, c.dt = c.dt, c2
        ref = c.ref()
        c.dt = keep
        c.check(got, ref, True, kept)
        eager = call(c2)
        torch.cuda.synchronize()
        c.check(eager, ref, True, new)
    vf.vf_destroy(x)
