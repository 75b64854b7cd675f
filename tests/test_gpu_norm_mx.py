"""GPU: norm with residual, microscaled quantization and product against 64 bits.

Tolerances.  norm: with s = fl(x + r) one rounding; the sum of squares adds at most 32 numbers a thread, 6 levels
over the lanes and 16 waves, all positive: 54 roundings at most, halved by the root; root, division and the two products 4
more, the mean and eps 2: under 40 roundings of 2^-24 relative to the value, and one of the output's type.
product: the terms are exact (4 + 2 significant bits and powers of two); K additions in some order, each at
most 2^-23 (truncated) of a partial sum of at most sum |a w|, the bias one more, and one rounding of the output.  8-bit
rows with outputs in bf16: of eight neighbouring terms seven may lose what is below 2^-13 of the largest."""
import numpy as np
import pytest

from tests import ops_ref as R

pytestmark = pytest.mark.gpu
BF = 2.0 ** -8
NORM = 40 * R.U32


@pytest.fixture(scope="module")
def vf():
    import paper_2011_14486_amd as pkg
    return pkg.load()


@pytest.fixture(scope="module")
def ctx(vf):
    c = vf.vf_create(0)
    yield c
    vf.vf_destroy(c)


def make(rng, rows, cols, dtype, size=None):
    import torch
    x = rng.standard_normal((rows, cols)) * (np.exp(rng.standard_normal(cols)) if size is None else size)
    return torch.from_numpy(x).to(dtype).cuda()


def f64(t):
    return t.double().cpu().numpy()


def norm_ref(x, r, gain, eps):
    s = x if r is None else x + r
    return s / np.sqrt((s * s).mean(-1, keepdims=True) + eps) * (1.0 if gain is None else gain), s


def check_mx(vf, q, y, rel):
    """q holds y quantized: scales those of the blocks' largest magnitudes (either neighbour where `rel` reaches over a
    power of two), values within half a step of the grid."""
    rows, cols = y.shape
    codes, scales = q.codes.cpu().numpy(), q.scales.cpu().numpy()
    emax, most, _, _ = R.FORMATS[q.fmt]
    v = np.zeros((rows, scales.shape[1] * 32))
    v[:, :cols] = y
    v = v.reshape(rows, -1, 32)
    top = np.abs(v).max(-1)
    low, high = (np.maximum(np.floor(np.log2(np.maximum(top * f, 1e-300))) - emax, -127) for f in (1 - rel, 1 + rel))
    e = scales.astype(np.float64) - 127
    assert ((e >= low) & (e <= high)).all()
    m = v / 2.0 ** e[..., None]
    got = R.code_values(codes, q.fmt)
    want = np.clip(m, -most, most)
    assert (np.abs(got - want) <= 0.5 * R.grid_step(want, q.fmt) * (1 + 1e-12) + rel * np.abs(m)).all()
    assert not got.reshape(rows, -1)[:, cols:].any()


@pytest.mark.parametrize("rows,width", [(1, 1), (1, 1024), (3, 31), (5, 33), (2, 257), (7, 1111), (65, 64), (130, 512), (9, 2048),
                                        (3, 8192), (2, 8200), (2, 16389), (1, 32768)])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
def test_norm(vf, ctx, rows, width, kind):
    import torch
    dtype, ut = (torch.bfloat16, BF) if kind == "bf16" else (torch.float32, R.U32)
    rng = np.random.default_rng([rows, width])
    x, r = make(rng, rows, width, dtype), make(rng, rows, width, dtype)
    gain = torch.from_numpy(1 + 0.2 * rng.standard_normal(width)).float().cuda()
    want, s = norm_ref(f64(x), f64(r), f64(gain), 1e-5)
    for out_type, u in ((vf.VF_BF16, BF), (vf.VF_FP32, R.U32)):
        y, total = vf.vf_rms_norm(ctx, x, gain, 1e-5, residual=r, out_type=out_type)
        assert (np.abs(f64(y) - want) <= (u + NORM) * np.abs(want)).all()
        assert (np.abs(f64(total) - s) <= (ut + R.U32) * np.abs(s)).all()
    for fmt in (vf.VF_E4M3, vf.VF_E2M1):
        q, total2 = vf.vf_rms_norm(ctx, x, gain, 1e-5, residual=r, out_type=fmt)
        check_mx(vf, q, want, NORM)
        assert torch.equal(total, total2)
    # without residual and gain, nothing but the output is written
    y, none = vf.vf_rms_norm(ctx, x, out_type=vf.VF_FP32)
    want, _ = norm_ref(f64(x), None, None, 1e-5)
    assert none is None and (np.abs(f64(y) - want) <= (R.U32 + NORM) * np.abs(want)).all()


def test_norm_views_and_in_place(vf, ctx):
    """Rows at odd distances and odd addresses; the sum over the residual itself; nothing outside the views changes."""
    import torch
    rng = np.random.default_rng(3)
    for dtype, u in ((torch.bfloat16, BF), (torch.float32, R.U32)):
        big, res = make(rng, 21, 1201, dtype, 1.0), make(rng, 21, 1203, dtype, 1.0)
        x, r = big[:, 3:1103], res[:, 5:1105]
        b0, r0 = big.clone(), res.clone()
        outbig = torch.full((21, 1301), 7.0, dtype=dtype, device="cuda")
        want, s = norm_ref(f64(x), f64(r), None, 1e-6)
        y, total = vf.vf_rms_norm(ctx, x, None, 1e-6, residual=r, sum_out=r, out=outbig[:, 1:1101])
        assert total is r and torch.equal(big, b0)
        assert (np.abs(f64(y) - want) <= (u + NORM) * np.abs(want)).all() and (np.abs(f64(r) - s) <= (u + R.U32) * np.abs(s)).all()
        assert torch.equal(res[:, :5], r0[:, :5]) and torch.equal(res[:, 1105:], r0[:, 1105:])
        assert bool((outbig[:, :1] == 7).all()) and bool((outbig[:, 1101:] == 7).all())
        # the sum over x, the output over x's neighbour type
        x2 = b0.clone()[:, 3:1103]
        vf.vf_rms_norm(ctx, x2, None, 1e-6, residual=r0[:, 5:1105], sum_out=x2)
        assert torch.equal(x2, total)


def test_norm_zero_rows_infinities_and_nan(vf, ctx):
    import torch
    x = torch.zeros((6, 100), device="cuda")
    x[1, 3], x[2, 3], x[3, 3], x[4] = float("inf"), float("nan"), 1e30, 1e-25
    y, _ = vf.vf_rms_norm(ctx, x, None, 1e-5)
    y = f64(y)
    assert (y[0] == 0).all() and (y[5] == 0).all()
    assert np.isnan(y[1, 3]) and (np.delete(y[1], 3) == 0).all()       # inf * 0 in its place, zero elsewhere
    assert np.isnan(y[2]).all()
    assert y[3, 3] == 0                                               # the square of 1e30 is infinite in 32 bits
    assert np.allclose(y[4], 1e-25 / np.sqrt(1e-5), rtol=1e-5)
    q, _ = vf.vf_rms_norm(ctx, x, None, 1e-5, out_type=vf.VF_E4M3)
    s = q.scales.cpu().numpy()
    assert (s[0] == 0).all() and s[1, 0] == 255 and (s[1, 1:] == 0).all() and (s[2] == 255).all()
    assert not q.codes[0].any() and not q.codes[2].any()
    # eps = 0 with a zero row: 0 * infinity
    y, _ = vf.vf_rms_norm(ctx, torch.zeros((1, 8), device="cuda"), None, 0.0)
    assert np.isnan(f64(y)).all()
    for shape in ((0, 100), (0, 5000)):
        y, _ = vf.vf_rms_norm(ctx, torch.empty(shape, device="cuda"))
        assert y.shape == shape


def block_edges(fmt):
    """Blocks of 32 with ties, values next to ties, subnormal codes, saturated tops, tiny and huge scales."""
    emax, most, emin, frac = R.FORMATS[fmt]
    rows = []
    grid = [0.0] + [np.ldexp(1 + f / 2 ** frac, e) for e in range(emin, emax + 1) for f in range(2 ** frac)]
    grid = np.array([g for g in grid if g <= most] + [np.ldexp(f / 2 ** frac, emin) for f in range(1, 2 ** frac)])
    grid.sort()
    ties = (grid[1:] + grid[:-1]) / 2
    for values in (grid, ties, ties * (1 + 2.0 ** -20), ties * (1 - 2.0 ** -20), -ties):
        for i in range(0, len(values), 30):
            rows.append(np.concatenate((values[i:i + 30], np.zeros(max(0, 30 - len(values[i:i + 30]))), [most, -most])))
    rows.append(np.concatenate((np.linspace(most, np.ldexp(1.0, emax + 1) * (1 - 2.0 ** -20), 31), [0.0])))   # cut to the largest
    rows.append(np.full(32, 0.0))
    rows.append(np.where(np.arange(32) % 2, 0.0, -0.0))
    base = np.array(rows)
    parts = [base]
    for p in (-60, -100, -126, -133, -140, 60, 110):
        parts.append(base * 2.0 ** p)
    x = np.concatenate(parts).astype(np.float32)
    bad = np.tile(base[:1], (3, 1)).astype(np.float32)
    bad[0, 4], bad[1, 5], bad[2, 31] = np.inf, np.nan, -np.inf
    return np.concatenate((x, bad))


@pytest.mark.parametrize("fmt", [2, 3])
def test_quantize_edges(vf, ctx, fmt):
    import torch
    x = block_edges(fmt)
    q = vf.vf_mx_quantize(ctx, torch.from_numpy(x).cuda(), fmt)
    codes, scales = R.quantize(x.astype(np.float64), fmt)
    assert np.array_equal(q.scales.cpu().numpy(), scales)
    assert np.array_equal(R.code_values(q.codes.cpu().numpy(), fmt), codes)
    # and the values that the codes stand for, in both types
    want = R.mx_values(q.codes.cpu().numpy(), scales, fmt, 32)
    y = vf.vf_mx_dequantize(ctx, q, vf.VF_FP32).cpu().numpy().astype(np.float64)
    fine = np.isfinite(want)
    tiny = np.abs(want) < 2.0 ** -126        # (a subnormal result is the nearest one)
    assert np.array_equal(fine, np.isfinite(y)) and np.array_equal(y[fine & ~tiny], want[fine & ~tiny])
    assert (np.abs(y - want)[fine & tiny] <= 2.0 ** -150).all()


@pytest.mark.parametrize("rows,cols", [(1, 1), (3, 8), (5, 31), (4, 32), (7, 33), (2, 100), (64, 1000), (3, 4099)])
@pytest.mark.parametrize("kind", ["bf16", "fp32"])
@pytest.mark.parametrize("fmt", [2, 3])
def test_quantize_shapes(vf, ctx, rows, cols, kind, fmt):
    import torch
    dtype = torch.bfloat16 if kind == "bf16" else torch.float32
    rng = np.random.default_rng([rows, cols, fmt])
    whole = make(rng, rows, cols + 5, dtype)
    x = whole[:, 3:3 + cols]
    q = vf.vf_mx_quantize(ctx, x, fmt)
    codes, scales = R.quantize(f64(x), fmt)
    assert np.array_equal(q.scales.cpu().numpy(), scales) and np.array_equal(R.code_values(q.codes.cpu().numpy(), fmt), codes)
    out = torch.full((rows, cols + 3), 9.0, dtype=dtype, device="cuda")
    vf.vf_mx_dequantize(ctx, q, vf.VF_BF16 if kind == "bf16" else vf.VF_FP32, out=out[:, 1:1 + cols])
    assert np.array_equal(f64(out[:, 1:1 + cols]), R.mx_values(q.codes.cpu().numpy(), scales, fmt, cols))
    assert bool((out[:, :1] == 9).all()) and bool((out[:, 1 + cols:] == 9).all())


def test_all_codes_have_their_values(vf, ctx):
    import torch
    for fmt, nb in ((vf.VF_E4M3, 32), (vf.VF_E2M1, 16)):
        codes = torch.arange(256, dtype=torch.uint8, device="cuda").reshape(-1, nb)
        for s in (0, 1, 100, 127, 200, 254, 255):
            scales = torch.full((codes.shape[0], 1), s, dtype=torch.uint8, device="cuda")
            y = vf.vf_mx_dequantize(ctx, vf.MX(codes, scales, fmt, 32), vf.VF_FP32).cpu().numpy().astype(np.float64)
            want = R.mx_values(codes.cpu().numpy(), scales.cpu().numpy(), fmt, 32)
            with np.errstate(over="ignore"):
                want = want.astype(np.float32).astype(np.float64)
            assert np.array_equal(y, want, equal_nan=True)


def product(vf, ctx, M, N, K, a_fmt, seed=0, bias=True):
    import torch
    rng = np.random.default_rng([M, N, K, a_fmt, seed])
    a = vf.vf_mx_quantize(ctx, make(rng, M, K, torch.float32), a_fmt)
    w = vf.vf_mx_quantize(ctx, make(rng, N, K, torch.float32, 1 / np.sqrt(K)), vf.VF_E2M1)
    b = torch.from_numpy(rng.standard_normal(N)).float().cuda() if bias else None
    av, wv = (R.mx_values(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.fmt, K) for m in (a, w))
    want = av @ wv.T + (0 if b is None else f64(b))
    mag = np.abs(av) @ np.abs(wv).T + (0 if b is None else np.abs(f64(b)))
    return a, w, b, want, mag


@pytest.mark.parametrize("M,N,K", [(1, 1, 1), (1, 64, 128), (3, 17, 33), (4, 100, 1024), (16, 16, 31), (17, 130, 129), (33, 48, 160),
                                   (64, 256, 512), (100, 1000, 520), (129, 129, 993), (257, 300, 256), (300, 520, 1000),
                                   (512, 512, 640), (1000, 260, 96)])
@pytest.mark.parametrize("a_fmt", [2, 3])
def test_product(vf, ctx, M, N, K, a_fmt):
    import torch
    a, w, b, want, mag = product(vf, ctx, M, N, K, a_fmt)
    tol = (K + 2) * 2.0 ** -23 * mag
    y = vf.vf_mx_matmul(ctx, a, w, bias=b, out_type=vf.VF_FP32)
    assert (np.abs(f64(y) - want) <= tol).all()
    if a_fmt == 2:
        tol = tol + 7 * 2.0 ** -13 * mag
    big = torch.full((M, N + 7), 5.0, dtype=torch.bfloat16, device="cuda")
    vf.vf_mx_matmul(ctx, a, w, bias=b, out=big[:, 3:3 + N])
    assert (np.abs(f64(big[:, 3:3 + N]) - want) <= tol + BF * np.abs(want) * (1 + 1e-3)).all()
    assert bool((big[:, :3] == 5).all()) and bool((big[:, 3 + N:] == 5).all())


@pytest.mark.parametrize("M,N,K", [(2100, 2100, 160), (2048, 2048, 256), (2000, 2049, 993), (16500, 255, 96), (1800, 2310, 33)])
@pytest.mark.parametrize("a_fmt", [2, 3])
def test_product_in_tiles(vf, ctx, M, N, K, a_fmt):
    """Sizes that are cut into large tiles: edges in every direction, ends of k inside a stage."""
    test_product(vf, ctx, M, N, K, a_fmt)


@pytest.mark.parametrize("M,N,K", [(4, 64, 384), (300, 512, 1056), (1500, 700, 260), (2300, 2000, 416)])
@pytest.mark.parametrize("a_fmt", [2, 3])
def test_product_of_whole_numbers_is_exact(vf, ctx, M, N, K, a_fmt):
    """Codes of small whole numbers and scales of one: every partial sum is exact, so any order gives the same."""
    import torch
    rng = np.random.default_rng([M, N, K])
    kb = (K + 31) // 32
    pick = np.array([0, 2, 4, 5, 6, 7, 10, 12, 14])            # 0, 1, 2, 3, 4, 6, -1, -2, -4 as 4-bit codes
    values = np.array([0, 1, 2, 3, 4, 6, -1, -2, -4.0])

    def draw(rows):
        i = rng.integers(0, 9, (rows, kb * 32))
        i[:, K:] = 0
        n = pick[i]
        return values[i], torch.from_numpy((n[:, 0::2] | n[:, 1::2] << 4).astype(np.uint8)).cuda()

    one = lambda rows: torch.full((rows, kb), 127, dtype=torch.uint8, device="cuda")   # noqa: E731
    av, ac = draw(M)
    wv, wc = draw(N)
    if a_fmt == 2:
        a = vf.vf_mx_quantize(ctx, torch.from_numpy(av[:, :K]).float().cuda(), a_fmt)
        av = R.mx_values(a.codes.cpu().numpy(), a.scales.cpu().numpy(), 2, kb * 32)
    else:
        a = vf.MX(ac, one(M), a_fmt, K)
    y = vf.vf_mx_matmul(ctx, a, vf.MX(wc, one(N), 3, K), out_type=vf.VF_FP32)
    assert np.array_equal(f64(y), av @ wv.T)


def test_product_scales(vf, ctx):
    """Scales far apart from block to block and row to row, up to both ends; a NaN scale reaches its row and column only."""
    import torch
    rng = np.random.default_rng(5)
    M, N, K = 70, 90, 288
    a, w, _, _, _ = product(vf, ctx, M, N, K, 2, bias=False)
    sa = torch.from_numpy(rng.integers(97, 158, tuple(a.scales.shape)).astype(np.uint8)).cuda()
    sw = torch.from_numpy(rng.integers(97, 158, tuple(w.scales.shape)).astype(np.uint8)).cuda()
    a, w = a._replace(scales=sa), w._replace(scales=sw)
    av, wv = (R.mx_values(m.codes.cpu().numpy(), m.scales.cpu().numpy(), m.fmt, K) for m in (a, w))
    y = f64(vf.vf_mx_matmul(ctx, a, w, out_type=vf.VF_FP32))
    assert (np.abs(y - av @ wv.T) <= (K + 2) * 2.0 ** -23 * (np.abs(av) @ np.abs(wv).T)).all()
    sa[5, 3] = 255
    sw[7, 8] = 255
    y2 = f64(vf.vf_mx_matmul(ctx, a, w, out_type=vf.VF_FP32))
    hit = np.zeros((M, N), bool)
    hit[5], hit[:, 7] = True, True
    assert np.isnan(y2[hit]).all() and np.array_equal(y2[~hit], y[~hit])


def test_other_streams_and_a_graph(vf):
    """Inputs made on one stream, a context on another, results used on the first; a captured chain replayed."""
    import torch
    side = torch.cuda.Stream()
    c = vf.vf_create(0, stream=side)
    rng = np.random.default_rng(8)
    x0, r0 = make(rng, 500, 1000, torch.bfloat16), make(rng, 500, 1000, torch.bfloat16)
    w = vf.vf_mx_quantize(c, make(rng, 300, 1000, torch.bfloat16, 0.03), vf.VF_E2M1)

    def chain(ctx, x, r):
        q, s = vf.vf_rms_norm(ctx, x, residual=r, out_type=vf.VF_E4M3)
        return vf.vf_mx_matmul(ctx, q, w), s

    want = None
    for k in range(5):
        x = x0 * (1.0 + k)      # made on the current stream right before
        y, s = chain(c, x, r0)
        got = (y + 0, s + 0)    # read on the current stream right behind
        del x, y, s
        torch.cuda.synchronize()
        if k == 0:
            want = got
    c2 = vf.vf_create(0)
    y, s = chain(c2, x0, r0)
    assert torch.equal(y, want[0]) and torch.equal(s, want[1])
    vf.vf_destroy(c2)
    g = torch.cuda.CUDAGraph()
    xin = x0.clone()
    with torch.cuda.graph(g, stream=side):
        gy, gs = chain(c, xin, r0)
    for k in (1, 0, 2, 0):
        xin.copy_(x0 * (1.0 + k))
        g.replay()
        ey, es = chain(c, x0 * (1.0 + k), r0)
        assert torch.equal(gy, ey) and torch.equal(gs, es)
        torch.cuda.synchronize()
    vf.vf_destroy(c)


@pytest.mark.parametrize("M,N,K", [(33, 4112, 96), (129, 2100, 512), (257, 1300, 333), (640, 520, 2049), (1025, 4100, 64), (2100, 4097, 160)])
@pytest.mark.parametrize("a_fmt", [2, 3])
@pytest.mark.parametrize("out_type", [0, 1])
def test_product_in_small_and_large_tiles(vf, ctx, M, N, K, a_fmt, out_type):
    """Sizes on both sides of the lines between the ways; sums of K exact products in fp32 (2^-24 each of the magnitudes' sum, four
    waves' parts), the cut of the 8-bit terms (2^-13 of each) where the output is bf16, and the output's rounding."""
    import torch
    rng = np.random.default_rng([M, N, K])
    a, w = (vf.vf_mx_quantize(ctx, torch.from_numpy(rng.standard_normal(s)).float().cuda(), f) for s, f in (((M, K), a_fmt), ((N, K), 3)))
    bias = torch.from_numpy(rng.standard_normal(N)).float().cuda()
    big = torch.full((M + 1, N + 3), 7.0, dtype=torch.float32 if out_type == 0 else torch.bfloat16, device="cuda")
    got = vf.vf_mx_matmul(ctx, a, w, bias, out_type, out=big[:M, 1:1 + N]).double()
    av, wv = (vf.vf_mx_dequantize(ctx, m, vf.VF_FP32).double() for m in (a, w))
    want = av @ wv.t().contiguous() + bias.double()
    mag = av.abs() @ wv.abs().t().contiguous() + bias.double().abs()
    cut = 2.0 ** -13 if a_fmt == 2 and out_type == 1 else 0.0
    tol = ((K + 8) * R.U32 + cut) * mag + (R.U32 if out_type == 0 else R.UBF) * want.abs()
    assert bool(((got - want).abs() <= tol).all()), float(((got - want).abs() / tol).max())
    assert bool((big[M] == 7).all()) and bool((big[:, 0] == 7).all()) and bool((big[:, 1 + N:] == 7).all())
