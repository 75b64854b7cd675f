"""GPU: sequence operators at sizes where a workgroup takes more than one tile, row or part (test_host_ops_ways pins that they do), against
64 bits.  Tolerances are those of test_gpu_norm_mx and test_gpu_ssm."""
import numpy as np
import pytest

from tests import ops_ref as R
from tests.test_gpu_norm_mx import NORM, check_mx, ctx, vf  # noqa: F401
from tests.test_gpu_ssm import Case

pytestmark = pytest.mark.gpu

# products in large tiles, more of them than workgroups, (M, N, K): K ends inside a stage, a block and a group of four stages; 17,
# 8, 5 and 4 stages
LARGE = [(7950, 4103, 2080), (7950, 4103, 930), (8100, 4097, 545), (7937, 4200, 400)]
SMALL = [(3000, 700, 545), (4200, 4103, 2080)]    # in small ones: few, and more than workgroups
# norms of more rows than workgroups hold at a time, (rows, width): one, two, four, eight, 16 waves a row, four chunks a thread
NORMS = [(2 * 8192 + 3, 512), (2 * 4096 + 5, 1000), (2 * 2048 + 3, 2048), (2 * 1024 + 3, 5000), (2 * 512 + 3, 8200), (512 + 3, 16389)]
# sequences in chunks, more than workgroups: (H, P, G, N, W), number
CHUNKS = [((4, 64, 1, 64, 4), 4500), ((4, 64, 2, 128, 4), 2301), ((3, 32, 1, 32, 2), 4500)]


def operands(vf, ctx, M, N, K, a_fmt):  # noqa: F811
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(M + N + K + a_fmt)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=g)   # noqa: E731
    return (vf.vf_mx_quantize(ctx, draw(M, K) * draw(K).exp(), a_fmt), vf.vf_mx_quantize(ctx, draw(N, K) / K ** 0.5, 3), draw(N))


def reference(vf, ctx, a, w, bias=0.0):  # noqa: F811
    """The product in 64 bits, and of the magnitudes, for some scattered rows (all columns), and these rows."""
    import torch
    from tests.ops_ref import mx_values
    M = a.codes.shape[0]
    at = np.unique(np.concatenate([np.arange(0, M, 61), np.arange(max(0, M - 300), M)]))
    rows = torch.from_numpy(at).cuda()
    av = mx_values(a.codes[rows].cpu().numpy(), a.scales[rows].cpu().numpy(), a.fmt, a.cols)
    wv = mx_values(w.codes.cpu().numpy(), w.scales.cpu().numpy(), w.fmt, w.cols)
    av, wv = torch.from_numpy(av).cuda(), torch.from_numpy(wv).cuda()
    b = torch.as_tensor(bias, device="cuda").double()
    return av @ wv.t().contiguous() + b, av.abs() @ wv.abs().t().contiguous() + b.abs(), rows


def close(got, want, mag, K, a_fmt, out_type):
    tol = (K + 2) * 2.0 ** -23 * mag
    if out_type == 1:
        tol = tol + (7 * 2.0 ** -13 * mag if a_fmt == 2 else 0) + R.UBF * (1 + 1e-3) * want.abs()
    err = (got.double() - want).abs()
    assert bool((err <= tol).all()), float((err / tol).max())


@pytest.mark.parametrize("M,N,K", LARGE + SMALL)
@pytest.mark.parametrize("a_fmt,out_type", [(2, 1), (3, 1), (3, 0), (2, 0)])
def test_products(vf, ctx, M, N, K, a_fmt, out_type):  # noqa: F811
    import torch
    a, w, bias = operands(vf, ctx, M, N, K, a_fmt)
    big = torch.full((M + 1, N + 3), 7.0, dtype=torch.float32 if out_type == 0 else torch.bfloat16, device="cuda")
    got = vf.vf_mx_matmul(ctx, a, w, bias, out_type, out=big[:M, 1:1 + N])
    want, mag, rows = reference(vf, ctx, a, w, bias)
    close(got[rows], want, mag, K, a_fmt, out_type)
    assert bool((big[M] == 7).all()) and bool((big[:, 0] == 7).all()) and bool((big[:, 1 + N:] == 7).all())
    # every row: the rows of a in another order give the same numbers in that order
    order = torch.randperm(M, generator=torch.Generator().manual_seed(1)).cuda()
    other = vf.vf_mx_matmul(ctx, a._replace(codes=a.codes[order], scales=a.scales[order]), w, bias, out_type)
    assert torch.equal(other, got[order])


@pytest.mark.parametrize("M,N,K", [LARGE[0], LARGE[2], SMALL[0], (64, 90, 288)], ids=str)
@pytest.mark.parametrize("a_fmt,out_type", [(2, 1), (3, 1), (2, 0)])
def test_scales_from_end_to_end(vf, ctx, M, N, K, a_fmt, out_type):  # noqa: F811
    """Scale bytes from 0 to 254, those of a row and a column together near 2^0; a NaN scale reaches its row or column only."""
    import torch
    a, w, _ = operands(vf, ctx, M, N, K, a_fmt)
    rng = np.random.default_rng(K)
    kb = a.scales.shape[1]
    base = np.concatenate([[0, 254, 127], rng.integers(0, 255, kb - 3)])
    near = lambda c, n: np.clip(c + rng.integers(-5, 6, (n, kb)), 0, 254).astype(np.uint8)   # noqa: E731
    a = a._replace(scales=torch.from_numpy(near(base, M)).cuda())
    w = w._replace(scales=torch.from_numpy(near(254 - base, N)).cuda())
    assert {0, 254} <= set(a.scales[:, :2].unique().tolist())
    got = vf.vf_mx_matmul(ctx, a, w, None, out_type)
    want, mag, rows = reference(vf, ctx, a, w)
    close(got[rows], want, mag, K, a_fmt, out_type)
    a.scales[M - 2, kb - 1] = a.scales[5, 0] = w.scales[N - 3, kb // 2] = 255
    hurt = vf.vf_mx_matmul(ctx, a, w, None, out_type)
    hit = torch.zeros((M, N), dtype=torch.bool, device="cuda")
    hit[[5, M - 2]] = True
    hit[:, N - 3] = True
    assert bool(hurt[hit].isnan().all()) and torch.equal(hurt[~hit], got[~hit])


@pytest.mark.parametrize("rows,width", NORMS)
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_norms(vf, ctx, rows, width, kind):  # noqa: F811
    """All types of output, the sum over x or the residual; a third of the rows, and all of them against other launches."""
    import torch
    dtype, ut = (torch.bfloat16, R.UBF) if kind == "bf16" else (torch.float32, R.U32)
    g = torch.Generator(device="cuda")
    g.manual_seed(width)
    x0, r0 = (torch.randn(rows, width, device="cuda", generator=g).to(dtype) for _ in range(2))
    gain = 1 + 0.2 * torch.randn(width, device="cuda", generator=g)
    s = x0.double() + r0.double()
    want = s / (s * s).mean(1, keepdim=True).add(1e-5).sqrt() * gain.double()
    for out_type, u in ((0, R.U32), (1, R.UBF), (2, None), (3, None)):
        x, r = x0.clone(), r0.clone()
        y, total = vf.vf_rms_norm(ctx, x, gain, residual=r, sum_out=x if out_type % 2 else r, out_type=out_type)
        assert bool(((total.double() - s).abs() <= (ut + R.U32) * s.abs()).all())
        assert torch.equal(r if out_type % 2 else x, r0 if out_type % 2 else x0)
        if u is not None:
            assert bool(((y.double() - want).abs() <= (u + NORM) * want.abs()).all())
            continue
        some = slice(rows - 40, rows)
        check_mx(vf, y._replace(codes=y.codes[some], scales=y.scales[some]), want[some].cpu().numpy(), NORM)
        for i in range(0, rows, 401):     # few rows in a launch of their own
            part, _ = vf.vf_rms_norm(ctx, x0[i:i + 401], gain, residual=r0[i:i + 401], out_type=out_type)
            assert torch.equal(part.codes, y.codes[i:i + 401]) and torch.equal(part.scales, y.scales[i:i + 401])


@pytest.mark.parametrize("sizes,n", CHUNKS, ids=str)
@pytest.mark.parametrize("ragged", [True, False])
def test_sequences_in_chunks(vf, ctx, sizes, n, ragged):  # noqa: F811
    """From states in other slots into slots in another order; some sequences against the recurrence, all of them against calls
    with fewer."""
    import torch
    rng = np.random.default_rng(n)
    lens = [int(v) for v in rng.integers(0, 45, n)] if ragged else [33] * n
    if ragged:
        lens[::7], lens[-1], lens[0] = [0] * len(lens[::7]), 70, 40
    c = Case(vf, sizes, lens, "bf16", slots=1, seed=3)
    H, P, G, N, W = sizes
    g = torch.Generator(device="cuda")
    g.manual_seed(n)
    c.state = (torch.randn(n, H * P + 2 * G * N, W - 1, device="cuda", generator=g).bfloat16(), torch.randn(n, H, P, N, device="cuda", generator=g))
    slots, to = rng.integers(-1, n, n), rng.permutation(n)
    to[::5] = -1
    i32 = lambda v: torch.from_numpy(np.asarray(v, np.int32)).cuda()   # noqa: E731
    new = c.layer.state(n, c.dtype)
    off = c.offsets if ragged else None
    out = vf.vf_ssm_scan(ctx, c.layer, c.xbc, c.dt, c.z, n, 70 if ragged else None, off, c.state, i32(slots), new, i32(to))
    assert bool(out.isfinite().all())
    # the same in four calls
    again, out2 = c.layer.state(n, c.dtype), torch.empty_like(out)
    for part in np.array_split(np.arange(n), 4):
        a, b = part[0], part[-1] + 1
        rows = slice(int(c.first[a]), int(c.first[b - 1] + lens[b - 1]))
        out2[rows] = vf.vf_ssm_scan(ctx, c.layer, c.xbc[rows], c.dt[rows], c.z[rows], len(part), 70 if ragged else None,
                                    i32(np.append(c.first[part], rows.stop) - rows.start) if ragged else None,
                                    c.state, i32(slots[part]), again, i32(to[part]))
    assert torch.equal(out, out2) and torch.equal(new[0], again[0]) and torch.equal(new[1], again[1])
    # some by the recurrence: first, last, and in between
    some = np.unique(np.concatenate([[0, 1, n - 2, n - 1], rng.integers(0, n, 12)]))
    f = lambda t: t.double().cpu().numpy()   # noqa: E731
    rows = np.concatenate([np.arange(c.first[s], c.first[s] + lens[s]) for s in some])
    at = torch.from_numpy(rows).cuda()
    taken = torch.from_numpy(np.maximum(slots[some], 0)).cuda()
    spans = list(zip(np.concatenate([[0], np.cumsum([lens[s] for s in some])[:-1]]), [lens[s] for s in some]))
    ref = R.ssm(sizes, c.lay, f(c.xbc[at]), f(c.dt[at]), f(c.z[at]), spans, (f(c.state[0][taken]), f(c.state[1][taken])),
                [i if slots[s] >= 0 else -1 for i, s in enumerate(some)])
    c.check(out[at], ref, True)
    want, conv, st, omag, smag = ref
    kept = [i for i, s in enumerate(some) if to[s] >= 0]
    dst = torch.from_numpy(to[some[kept]]).cuda()
    assert np.array_equal(f(new[0][dst]), conv[kept])
    assert (np.abs(f(new[1][dst]) - st[kept]) <= (3 * 2.0 ** -16 + (128 + 70 + N) * R.U32) * smag[kept]).all()
    idle = np.setdiff1d(np.arange(n), to[to >= 0])
    assert not new[1][torch.from_numpy(idle).cuda()].any()
