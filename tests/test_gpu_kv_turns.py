"""GPU: the attention operators where workgroups go on to further sequences, caches whose places pass 32 bits, other streams, graphs, and the
network's run of them at sizes where every way is taken."""
import numpy as np
import pytest

from tests.test_gpu_kv import Case, ctx, f64, rope_of, vf  # noqa: F401

pytestmark = pytest.mark.gpu


def test_more_sequences_than_workgroups(vf, ctx):  # noqa: F811
    """A row that sees one key gives its value, as it is: single tokens of a million sequences appended, read, and attended to."""
    import torch
    n = (1 << 20) + 77
    cache = vf.KvCache.zeros(vf.VF_BF16, n, 16, 1, 8)
    g = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn((n, 24), generator=g, device="cuda").bfloat16()
    table, lengths = torch.randperm(n, generator=g, device="cuda").to(torch.int32)[:, None], torch.ones(n, dtype=torch.int32, device="cuda")
    assert vf.vf_kv_append(ctx, cache, x[:, 8:16], x[:, 16:], table, lengths) is None
    k, v = vf.vf_kv_read(ctx, cache, table, lengths, n)
    assert torch.equal(k, x[:, 8:16]) and torch.equal(v, x[:, 16:])
    assert torch.equal(vf.vf_kv_attend(ctx, cache, x[:, :8], table, lengths), v)
    m = n // 20 * 20   # 20 rows a sequence: the way through the LDS
    out = vf.vf_kv_attend(ctx, cache, x[:m, :8], table[:m // 20], lengths[:m // 20], causal=False)
    assert torch.equal(out.reshape(-1, 20, 8), v[:m // 20, None].expand(-1, 20, 8))


@pytest.mark.parametrize("fmt", [1, 2])
def test_places_behind_32_bits(vf, ctx, fmt):  # noqa: F811
    """A cache of more than 2^31 numbers (2^32 bytes of codes): the same sequences in its last pages and in a small cache."""
    import torch
    pages = 133000 if fmt == 1 else 263000
    large = vf.KvCache(fmt, 128, *(torch.empty((pages, 8, 16, 128), dtype=torch.bfloat16 if fmt == 1 else torch.uint8, device="cuda") for _ in range(2)),
                       *(() if fmt == 1 else (torch.empty((pages, 8, 16, 4), dtype=torch.uint8, device="cuda") for _ in range(2))))
    small = vf.KvCache.zeros(fmt, 50, 16, 8, 128)
    rng = np.random.default_rng(2)
    new = torch.from_numpy(rng.standard_normal((400, 48 * 128))).bfloat16().cuda()
    q, k, v = new[:, :32 * 128], new[:, 32 * 128:40 * 128], new[:, 40 * 128:]
    order = torch.from_numpy(rng.permutation(50)[:26].astype(np.int32)).cuda().reshape(2, 13)
    lengths = torch.full((2,), 200, dtype=torch.int32, device="cuda")
    rope, _ = rope_of(vf, 128)
    got = []
    for cache, table in ((large, order + (pages - 50)), (small, order)):
        turned = vf.vf_kv_append(ctx, cache, k, v, table, lengths, q=q, rope=rope)
        got.append([turned, *vf.vf_kv_read(ctx, cache, table, lengths, 400), vf.vf_kv_attend(ctx, cache, turned, table, lengths),
                    vf.vf_kv_attend(ctx, cache, turned[198:200], table, lengths),
                    vf.vf_kv_attend(ctx, cache, turned[:2], table, lengths, longest_kv=10 ** 6)])
    for a, b in zip(*got):
        assert torch.equal(a, b) and torch.isfinite(a.float()).all()


def test_rows_of_a_long_cache(vf, ctx):  # noqa: F811
    """Shared along the keys by many workgroups: 1, 5 and 40 rows behind 70,000 keys, in all types."""
    for kind, cache in (("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32")):
        for rows in (1, 5, 40):
            c = Case(vf, kind, cache, 4, 2, 64, [rows, 1], [70000, 3], 64, ragged=True)
            q = c.matrix(256, scale=1.5)
            table, lengths = c.where()
            c.check_attend(ctx, q, vf.vf_kv_attend(ctx, c.cache, q, table, lengths, offsets=c.dev(c.offsets)))


@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("group", [3, 16, 17, 64])
def test_many_heads_of_one(vf, ctx, kind, group):  # noqa: F811
    """Row blocks that end inside a token's heads."""
    c = Case(vf, kind, kind, 2 * group, 2, 32, [1, 13, 4], [40, 90, 4], 16)
    q = c.matrix(2 * group * 32, scale=1.5)
    table, lengths = c.where()
    for window in (0, 7):
        c.check_attend(ctx, q, vf.vf_kv_attend(ctx, c.cache, q, table, lengths, window=window, offsets=c.dev(c.offsets)), True, window)
    c.check_attend(ctx, q, vf.vf_kv_attend(ctx, c.cache, q, table, lengths, causal=False, offsets=c.dev(c.offsets)), False)


def test_ragged_sequences_in_any_order(vf, ctx):  # noqa: F811
    """Enough row blocks for several rounds of workgroups, where sequences with most keys come first: 64 and 65 sequences."""
    rng = np.random.default_rng(4)
    for n in (64, 65):
        new, keys = rng.integers(0, 60, n), rng.integers(0, 150, n)
        c = Case(vf, "bf16", "bf16", 16, 4, 64, new, new + keys, 16)
        q = c.matrix(1024, scale=1.5)
        table, lengths = c.where()
        c.check_attend(ctx, q, vf.vf_kv_attend(ctx, c.cache, q, table, lengths, offsets=c.dev(c.offsets), longest=59, longest_kv=209))


@pytest.mark.parametrize("kind,cache", [("bf16", "bf16"), ("bf16", "e4m3"), ("fp32", "fp32")])
def test_other_streams_and_graphs(vf, kind, cache):  # noqa: F811
    """A context on a stream of its own, tensors of the current one; the run append, attend, read captured and replayed with other inputs between
    eager calls, two graphs on one context in turn."""
    import torch
    side = torch.cuda.Stream()
    ctx = vf.vf_create(0, stream=side)   # noqa: F811
    cases = [Case(vf, kind, cache, 8, 2, 64, [3, 1, 40], [3, 9000, 100], 16, seed=s, ragged=True) for s in (1, 2)]
    rope, _ = rope_of(vf, 64)
    graphs = []
    for c in cases:
        proj, (table, lengths), off = c.matrix(12 * 64), c.where(), c.dev(c.offsets)
        buf = proj.clone()

        def run(x, c=c, table=table, lengths=lengths, off=off):
            q = vf.vf_kv_append(ctx, c.cache, x[:, 512:640], x[:, 640:], table, lengths, q=x[:, :512], rope=rope, offsets=off)
            return q, vf.vf_kv_attend(ctx, c.cache, q, table, lengths, offsets=off), *vf.vf_kv_read(ctx, c.cache, table, lengths, c.tokens, offsets=off, out_type=c.fmt & 1)

        rows = [r for a, n in zip(c.offsets[:-1], c.new) for r in range(a, a + n)]
        run(buf)                      # (the context gets its scratch)
        torch.cuda.synchronize()
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=side):
            out = run(buf)
        graphs.append((g, run, buf, proj, out, rows))
    for k in (1.0, -0.5, 2.0):
        for g, run, buf, proj, out, rows in graphs:
            buf.copy_(proj * k)
            torch.cuda.synchronize()
            with torch.cuda.stream(side):
                g.replay()
            torch.cuda.synchronize()
            replayed = [t[rows].clone() for t in out]
            for a, b in zip(replayed, run(proj * k)):
                torch.cuda.synchronize()
                assert torch.equal(a, b[rows])
    vf.vf_destroy(ctx)


def test_two_contexts_at_once(vf):  # noqa: F811
    """Two contexts on streams of their own, calls in turn without waiting: each has scratch of its own."""
    import torch
    made = []
    for s in range(2):
        st = torch.cuda.Stream()
        c = Case(vf, "bf16", "bf16", 8, 2, 128, [1], [20000], 64, seed=s, ragged=False)
        made.append((vf.vf_create(0, stream=st), st, c, c.matrix(1024), c.where(), []))
    torch.cuda.synchronize()
    for _ in range(20):
        for ctx, st, c, q, where, outs in made:   # noqa: F811
            with torch.cuda.stream(st):
                outs.append(vf.vf_kv_attend(ctx, c.cache, q, *where))
    torch.cuda.synchronize()
    for ctx, st, c, q, where, outs in made:
        c.check_attend(ctx, q, outs[0])
        assert all(torch.equal(o, outs[0]) for o in outs)
        vf.vf_destroy(ctx)


def test_in_place_and_far_positions(vf, ctx):  # noqa: F811
    """Queries turned in place in their wide matrix, and positions up to 2^30, whose angles are as right as the first ones'."""
    import torch
    c = Case(vf, "fp32", "fp32", 6, 2, 96, [20, 30], [20, 130], 16)
    proj = c.matrix(10 * 96)
    rope, f = rope_of(vf, 64, True)
    table, lengths = c.where()
    q, k, v = proj[:, :576], proj[:, 576:768], proj[:, 768:]
    apart = vf.vf_kv_append(ctx, c.cache, k, v, table, lengths, q=q, rope=rope, offsets=c.dev(c.offsets))
    same = vf.vf_kv_append(ctx, c.cache, k, v, table, lengths, q=q, rope=rope, offsets=c.dev(c.offsets), q_out=q)
    assert same is q and torch.equal(q[2:-2], apart[2:-2])
    pages = (1 << 30) // 1024
    cache = vf.KvCache.zeros(vf.VF_FP32, 2, 1024, 1, 8)
    table = torch.full((1, pages), -1, dtype=torch.int32, device="cuda")
    table[0, -1] = 1
    x = torch.randn((5, 24), device="cuda")
    freq = torch.tensor([1.0, 0.3, 0.01, 1e-4], dtype=torch.float64, device="cuda")
    at = torch.tensor([1 << 30], dtype=torch.int32, device="cuda")
    got = vf.vf_kv_append(ctx, cache, x[:, 8:16], x[:, 16:], table, at, q=x[:, :8], rope=vf.Rope(freq))
    pos = np.arange((1 << 30) - 5, 1 << 30)[:, None]
    # (numpy takes the angle's product in 64 bits too, so both have its rounding: 2^-53 of 2^30, and 2^-23 is allowed for it)
    c64, s64 = np.cos(pos * f64(freq)), np.sin(pos * f64(freq))
    a, b = f64(x[:, :4]), f64(x[:, 4:8])
    want = np.concatenate((a * c64 - b * s64, b * c64 + a * s64), 1)
    size = np.tile(np.abs(a) + np.abs(b), 2)
    assert (np.abs(f64(got) - want) <= (4 * 2.0 ** -24 + 2.0 ** -23) * size).all()
    rk, rv = vf.vf_kv_read(ctx, cache, table, at, 5, out_type=0)
    assert torch.equal(rv, x[:, 16:])
    out = vf.vf_kv_attend(ctx, cache, got, table, at, window=1, longest_kv=1 << 30)
    # (one key: its weight p times the value, times 1 / p: three roundings)
    assert (np.abs(f64(out) - f64(rv)) <= 4 * 2.0 ** -24 * np.abs(f64(rv))).all()


@pytest.mark.parametrize("cache", ["fp32", "e4m3"])
@pytest.mark.parametrize("dim", [9, 32, 40, 64, 80, 96, 128])
def test_rows_of_32_a_wave(vf, ctx, cache, dim):  # noqa: F811
    """fp32 with tables of more than 512 places: ragged rows, windows, all keys, pages that are missing or none, numbers that are not finite."""
    heads = 6
    new, keys = [40, 1, 33, 0, 150], [60, 20, 33, 7, 600]
    for window, causal in ((0, True), (21, True), (0, False)):
        c = Case(vf, "fp32", cache, heads, 2, dim, new, keys, 16, extra=40)
        q = c.matrix(heads * dim, scale=1.5)
        table, lengths = c.where()
        got = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, causal=causal, window=window, offsets=c.dev(c.offsets))
        c.check_attend(ctx, q, got, causal, window)
    for where, entry in (((0, 1), -1), ((4, 20), 10 ** 7), ((4, 37), -1)):
        c = Case(vf, "fp32", cache, heads, 2, dim, new, keys, 16, extra=40)
        c.table[where] = entry
        c.pool()
        q = c.matrix(heads * dim)
        table, lengths = c.where()
        c.check_attend(ctx, q, vf.vf_kv_attend(ctx, c.cache, q, table, lengths, offsets=c.dev(c.offsets)))
    for what in (float("inf"), float("nan")):
        c = Case(vf, "fp32", cache, heads, 2, dim, new, keys, 16, extra=40)
        clean = f64(vf.vf_kv_attend(ctx, c.cache, q, *c.where(), offsets=c.dev(c.offsets)))
        for t in (5, 33, 59):
            c.v[c.table[0, t // 16], 0, t % 16, dim // 2] = what
        c.pool()
        got = f64(vf.vf_kv_attend(ctx, c.cache, q, *c.where(), offsets=c.dev(c.offsets)))
        first = int(c.offsets[0])
        for r in range(c.tokens - 4):
            row = first + r
            hit = r < 40 and any(t <= 20 + r for t in (5, 33, 59))
            for h in range(heads):
                a, b = got[row, h * dim:(h + 1) * dim], clean[row, h * dim:(h + 1) * dim]
                if hit and h < heads // 2:
                    assert not np.isfinite(a[dim // 2])
                else:
                    assert np.array_equal(a, b)


def test_outputs_in_place(vf, ctx):  # noqa: F811
    """Outputs in the queries' place, in every way that attention takes."""
    for kind, new, keys, extra in (("bf16", [1], [40], 1), ("bf16", [1], [9000], 1), ("bf16", [3, 40, 200], [9, 40, 700], 1), ("fp32", [3, 40], [9, 40], 1),
                                   ("fp32", [40, 200], [40, 700], 40), ("bf16", [1] * 2100, [20] * 2100, 1)):
        c = Case(vf, kind, kind, 8, 2, 64, new, keys, 16, extra=extra, ragged=len(new) < 9)
        q = c.matrix(512)
        kept = q.clone()
        table, lengths = c.where()
        off = c.dev(c.offsets)
        apart = vf.vf_kv_attend(ctx, c.cache, q, table, lengths, offsets=off)
        assert vf.vf_kv_attend(ctx, c.cache, q, table, lengths, offsets=off, out=q) is q
        live = slice(2, -2) if c.offsets is not None else slice(None)
        assert c.torch.equal(q[live], apart[live]) and not c.torch.equal(q[live], kept[live])
