"""Performance cases of the sequence operators: the parts of a state-space value network.

A case is a dict of plain values.  `op` names the operator:

  norm      vf_rms_norm: residual's addition, root-mean-square norm, output in the type or in 8 or 4 bits with scales
  quantize  vf_mx_quantize (and vf_mx_dequantize, which gives the values that the codes stand for)
  product   vf_mx_matmul: rows in 8 or 4 bits times weights in 4 bits
  scan      vf_ssm_scan: short causal convolution and selective state space scan over whole sequences
  step      vf_ssm_step: the same for one more token of every row, from parents' states into the rows' own

With `own` false run() computes the operators in elementary torch operations; with `own` true it
makes the library's calls.  exact() follows the definitions in 64 bits, the recurrence token by token.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda" if torch.cuda.is_available() else "cpu"
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
BYTES = {"bf16": 2.0, "fp32": 4.0, "e4m3": 1.0 + 1.0 / 32, "e2m1": 0.5 + 1.0 / 32}
# microscaled formats: exponent and value of the largest number, smallest normal exponent, fraction bits
FORMATS = {"e4m3": (8, 448.0, -6, 3), "e2m1": (2, 6.0, 0, 1)}
E2M1 = [0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0]
EPS = 1e-5
CHUNK = 64


def listed():
    return [
        # one token of a decision that is taken alone: two small launches
        dict(name="norm_token", op="norm", rows=1, width=1024, type="bf16", residual=True, out="e4m3"),
        # all tokens of a batch of prompts, the plain residual norm
        dict(name="norm_prompt", op="norm", rows=32768, width=2048, type="bf16", residual=True, out="bf16"),
        # activations of an odd number of rows and columns in 8 bits
        dict(name="quantize_rows", op="quantize", rows=333, cols=1000, type="bf16", format="e4m3"),
        # a large weight matrix into 4 bits, as when a model is loaded
        dict(name="quantize_weights", op="quantize", rows=8192, cols=4096, type="bf16", format="e2m1"),
        # the in-projection of a few single tokens (gate, x, B, C and steps of 32 heads of 64)
        dict(name="product_tokens", op="product", M=4, N=4384, K=1024, a="e4m3", out="bf16", bias=False),
        # the same projection for an odd batch of tokens, both sides in 4 bits
        dict(name="product_4bit", op="product", M=5000, N=4384, K=4096, a="e2m1", out="bf16", bias=True),
        # the largest product: prompts against a wide layer
        dict(name="product_prompt", op="product", M=16384, N=8192, K=4096, a="e4m3", out="bf16", bias=False),
        # 16,384 sequences of 50 layers scored from their first layer, as the recurrent network's are
        dict(name="scan_stages", op="scan", seqs=16384, longest=50, ragged=False, heads=4, head_dim=64, groups=1, n_state=64,
             taps=4, type="bf16", gate=True, initial=False, final=False),
        # one long prompt: few rows, a long axis
        dict(name="scan_prompt", op="scan", seqs=1, longest=16384, ragged=False, heads=32, head_dim=64, groups=1, n_state=128,
             taps=4, type="bf16", gate=True, initial=False, final=True),
        # ragged pipelines continued from their prefixes, odd sizes, 32 bits
        dict(name="scan_ragged", op="scan", seqs=37, longest=300, ragged=True, heads=5, head_dim=40, groups=1, n_state=24,
             taps=3, type="fp32", gate=False, initial=True, final=True),
        # one candidate behind one prefix
        dict(name="step_token", op="step", rows=1, slots=4, heads=32, head_dim=64, groups=1, n_state=128, taps=4, type="bf16"),
        # a beam's extensions: 1024 rows continue 64 parents' states into slots of their own
        dict(name="step_beam", op="step", rows=1024, slots=64, heads=32, head_dim=64, groups=1, n_state=128, taps=4, type="bf16"),
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "quantize", "product", "product", "scan", "scan", "step"])
    if op == "norm":
        rows, width = _log(rng, 1, 32768), _log(rng, 16, 8192)
        rows = max(1, min(rows, 64 * 1024 * 1024 // width))
        return dict(op=op, rows=rows, width=width, type=rng.choice(["bf16", "bf16", "fp32"]), residual=rng.random() < 0.7,
                    out=rng.choice(["bf16", "fp32", "e4m3", "e2m1"]))
    if op == "quantize":
        rows, cols = _log(rng, 1, 8192), _log(rng, 8, 8192)
        rows = max(1, min(rows, 32 * 1024 * 1024 // cols))
        return dict(op=op, rows=rows, cols=cols, type=rng.choice(["bf16", "bf16", "fp32"]), format=rng.choice(["e4m3", "e2m1"]))
    if op == "product":
        N, K = _log(rng, 64, 8192), _log(rng, 64, 4096)
        if rng.random() < 0.5:  # widths are mostly multiples of a power of two, sometimes odd
            N, K = (N + 63) // 64 * 64, (K + 127) // 128 * 128
        return dict(op=op, M=_log(rng, 1, 16384), N=N, K=K, a=rng.choice(["e4m3", "e2m1"]),
                    out=rng.choice(["bf16", "bf16", "fp32"]), bias=rng.random() < 0.5)
    groups = rng.choice([1, 1, 1, 2])
    heads = groups * rng.choice([1, 2, 3, 4, 5, 8, 16])
    if rng.random() < 0.6:
        head_dim, n_state, kind = rng.choice([32, 64, 64, 128]), rng.choice([16, 32, 64, 128]), "bf16"
    else:
        head_dim, n_state, kind = rng.randint(3, 100), rng.randint(1, 128), rng.choice(["bf16", "fp32"])
    taps = rng.choice([4, 4, 4, 2, 3, 1])
    if op == "step":
        rows = max(1, min(_log(rng, 1, 1024), (1 << 27) // (heads * head_dim * n_state)))
        return dict(op=op, rows=rows, slots=_log(rng, 1, 64), heads=heads, head_dim=head_dim, groups=groups, n_state=n_state,
                    taps=taps, type=kind)
    longest = _log(rng, 1, 16384)
    seqs = max(1, min(_log(rng, 1, 4096), (1 << 18) // longest, (1 << 27) // (heads * head_dim * n_state)))
    return dict(op=op, seqs=seqs, longest=longest, ragged=rng.random() < 0.5, heads=heads, head_dim=head_dim, groups=groups,
                n_state=n_state, taps=taps, type=kind, gate=rng.random() < 0.6, initial=rng.random() < 0.5,
                final=rng.random() < 0.5)


# ------------------------------------------------------------------ inputs

def _gen(seed):
    return torch.Generator(device=DEV).manual_seed(seed)


def _normal(g, *shape, std=1.0, dtype=torch.float32):
    return (torch.randn(shape, generator=g, device=DEV) * std).to(dtype)


def _lengths(case):
    """Lengths of the sequences, by the case alone: one has the longest, some are short or empty."""
    n, top = case["seqs"], case["longest"]
    if not case["ragged"]:
        return np.full(n, top, np.int64)
    rng = np.random.default_rng([n, top, case["heads"]])
    lens = rng.integers(0, top + 1, n)
    lens[rng.integers(n)] = top
    if n > 2:
        lens[int(np.argmin(lens))] = 0
    return lens


def _layer(case, g):
    """Weights of the convolution and the scan: decays of 1 to 16 per unit of time, steps of 0.001 to 0.1 and more."""
    H, P, G, N, W = (case[k] for k in ("heads", "head_dim", "groups", "n_state", "taps"))
    C = H * P + 2 * G * N
    step = torch.exp(torch.rand(H, generator=g, device=DEV) * math.log(100.0) + math.log(0.001))
    return dict(conv_w=(torch.rand((C, W), generator=g, device=DEV) * 2 - 1) / math.sqrt(W),
                conv_b=(torch.rand(C, generator=g, device=DEV) * 2 - 1) / math.sqrt(W),
                a=-(1.0 + 15.0 * torch.rand(H, generator=g, device=DEV)), d=1.0 + _normal(g, H, std=0.2),
                dt_bias=step + torch.log(-torch.expm1(-step)))


def prepare(case, seed):
    g, op = _gen(seed), case["op"]
    s = dict(case=case)
    if op in ("norm", "quantize"):
        rows, cols, t = case["rows"], case["width"] if op == "norm" else case["cols"], TYPES[case["type"]]
        # a few columns are much larger than the others, as in a network's residual stream
        size = torch.exp(_normal(g, cols, std=0.7))
        s["x"] = (_normal(g, rows, cols) * size).to(t)
        if op == "norm":
            s["gain"] = 1.0 + _normal(g, cols, std=0.2)
            s["residual"] = (_normal(g, rows, cols) * size).to(t) if case["residual"] else None
        return s
    if op == "product":
        M, N, K = case["M"], case["N"], case["K"]
        s["a"] = _pack(_normal(g, M, K) * torch.exp(_normal(g, K, std=0.5)), case["a"])
        s["w"] = _pack(_normal(g, N, K, std=1.0 / math.sqrt(K)), "e2m1")
        s["bias"] = _normal(g, N) if case["bias"] else None
        return s
    H, P, G, N, W = (case[k] for k in ("heads", "head_dim", "groups", "n_state", "taps"))
    C, t = H * P + 2 * G * N, TYPES[case["type"]]
    s["layer"] = _layer(case, g)
    if op == "step":
        tokens, gate, n, slots, n_out = case["rows"], True, case["rows"], case["slots"], case["rows"]
        s["slots"] = torch.randint(slots, (n,), generator=g, device=DEV, dtype=torch.int32)
    else:
        lens = _lengths(case)
        tokens, gate, n, slots = int(lens.sum()), case["gate"], case["seqs"], case["seqs"] if case["initial"] else 0
        n_out = n if case["final"] else 0
        s["offsets"] = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)).to(DEV) if case["ragged"] else None
        s["slots"] = torch.randperm(n, generator=g, device=DEV).to(torch.int32) if slots else None
    # the in-projection's output [gate | x B C | steps]; its parts are views
    proj = _normal(g, tokens, (H * P if gate else 0) + C + H, dtype=t)
    s["z"] = proj[:, :H * P] if gate else None
    s["xbc"], s["dt"] = proj[:, -C - H:-H], proj[:, -H:]
    s["state"] = (_normal(g, slots, C, W - 1, dtype=t), _normal(g, slots, H, P, N)) if slots else None
    s["state_out"] = (torch.empty((n_out, C, W - 1), dtype=t, device=DEV),
                      torch.empty((n_out, H, P, N), device=DEV)) if n_out else None
    return s


# ------------------------------------------------------------------ plain forms

def _scale_exponents(v, fmt):
    """Exponent of the scale of every block of 32 columns, and whether the block holds only finite values."""
    top = v.abs().amax(-1)
    fine = torch.isfinite(top)
    e = torch.frexp(torch.where(fine & (top > 0), top, 2.0 ** -140))[1] - 1 - FORMATS[fmt][0]
    return e.clamp(-127, 127), fine


def _quantized(x, fmt):
    """x [rows][cols] as the values of the format: (codes' values [rows][blocks][32], exponents [rows][blocks], finite)."""
    _, most, emin, frac = FORMATS[fmt]
    cols = x.shape[1]
    v = torch.nn.functional.pad(x, (0, -cols % 32)).reshape(x.shape[0], -1, 32)
    e, fine = _scale_exponents(v, fmt)
    v = torch.where(fine[..., None], torch.ldexp(v, -e[..., None]), 0.0)
    grid = torch.ldexp(torch.ones_like(v), (torch.frexp(v)[1] - 1).clamp(min=emin) - frac)
    return (torch.round(v / grid) * grid).clamp(-most, most), e, fine


def _values(x, fmt):
    """The values that x has in a microscaled format."""
    q, e, fine = _quantized(x, fmt)
    v = torch.where(fine[..., None], torch.ldexp(q, e[..., None]), math.nan)
    return v.reshape(x.shape[0], -1)[:, :x.shape[1]]


def _pack(x, fmt):
    """(codes, scales, format, columns): e4m3 a byte a value, e2m1 two values a byte with the even column in the low half."""
    q, e, fine = _quantized(x, fmt)
    scales = torch.where(fine, e + 127, 255).to(torch.uint8)
    if fmt == "e4m3":
        codes = q.to(torch.float8_e4m3fn).view(torch.uint8).reshape(x.shape[0], -1)
    else:
        half = torch.tensor(E2M1[:8], device=q.device)
        c = torch.searchsorted(half, q.abs().contiguous()) + 8 * torch.signbit(q)
        c = c.reshape(x.shape[0], -1, 2)
        codes = (c[..., 0] | c[..., 1] << 4).to(torch.uint8)
    return codes, scales, fmt, x.shape[1]


def _unpack(packed, dtype=torch.float32):
    codes, scales, fmt, cols = packed
    if fmt == "e4m3":
        v = codes.view(torch.float8_e4m3fn).to(dtype)
    else:
        c = codes.to(torch.int64)
        v = torch.tensor(E2M1, device=codes.device, dtype=dtype)[torch.stack((c & 15, c >> 4), -1)]
    v = v.reshape(codes.shape[0], -1, 32)
    return torch.ldexp(v, scales.to(torch.int32)[..., None] - 127).reshape(codes.shape[0], -1)[:, :cols]


def _plain_norm(s):
    case, x = s["case"], s["x"].float()
    if s["residual"] is not None:
        x = x + s["residual"].float()
    y = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS) * s["gain"]
    out = y.to(TYPES[case["out"]]) if case["out"] in TYPES else _values(y, case["out"]).to(torch.bfloat16)
    return (out, x.to(s["x"].dtype)) if s["residual"] is not None else out


def _plain_product(s):
    y = _unpack(s["a"]) @ _unpack(s["w"]).t()
    if s["bias"] is not None:
        y = y + s["bias"]
    return y.to(TYPES[s["case"]["out"]])


def _silu(x):
    return x / (1.0 + torch.exp(-x))


def _softplus(x):
    return torch.clamp(x, min=0.0) + torch.log1p(torch.exp(-x.abs()))


def _convolved(padded, layer):
    """silu of the causal convolution of [..][W - 1 + T][C]."""
    w = layer["conv_w"]
    return _silu((padded.unfold(1, w.shape[1], 1) * w).sum(-1) + layer["conv_b"])


def _plain_scan(s):
    """In chunks: products within a chunk, the states at the chunks' starts by one product with the decays between them."""
    case, layer = s["case"], s["layer"]
    H, P, G, N, W = (case[k] for k in ("heads", "head_dim", "groups", "n_state", "taps"))
    n, T, C, t = case["seqs"], case["longest"], s["xbc"].shape[1], s["xbc"].dtype
    tokens = s["xbc"].shape[0]
    if s["offsets"] is None:
        start = torch.arange(n, device=DEV) * T
        length = torch.full((n,), T, device=DEV)
    else:
        off = s["offsets"].long()
        start, length = off[:-1], off[1:] - off[:-1]
    Q = min(CHUNK, T)
    nc = -(-T // Q)
    at = torch.arange(nc * Q, device=DEV)
    live = at < length[:, None]                                              # [n][nc Q]
    rows = (start[:, None] + at).clamp(max=max(tokens - 1, 0))
    old_conv = torch.zeros((n, W - 1, C), device=DEV)
    old = torch.zeros((n, H, P, N), device=DEV)
    if s["state"] is not None:
        old_conv = s["state"][0][s["slots"].long()].float().transpose(1, 2)
        old = s["state"][1][s["slots"].long()]
    padded = torch.cat((old_conv, s["xbc"][rows].float() * live[..., None]), 1)  # [n][W - 1 + nc Q][C]
    u = _convolved(padded, layer) * live[..., None]
    x = u[..., :H * P].reshape(n, nc, Q, H, P).transpose(2, 3)               # [n][nc][H][Q][P]
    B = u[..., H * P:H * P + G * N].reshape(n, nc, Q, G, N).transpose(2, 3)  # [n][nc][G][Q][N]
    Cm = u[..., H * P + G * N:].reshape(n, nc, Q, G, N).transpose(2, 3)
    dt = (_softplus(s["dt"][rows].float() + layer["dt_bias"]) * live[..., None]).reshape(n, nc, Q, H).transpose(2, 3)
    cum = (dt.double() * layer["a"].double()[:, None]).cumsum(-1)            # [n][nc][H][Q]
    total = torch.nn.functional.pad(cum[..., -1].transpose(1, 2).cumsum(-1), (1, 0))  # [n][H][nc + 1]
    per = H // G
    grow = lambda v: v.repeat_interleave(per, 2) if per > 1 else v           # noqa: E731  groups to heads
    causal = torch.ones((Q, Q), dtype=torch.bool, device=DEV).tril()
    decay = torch.exp((cum[..., :, None] - cum[..., None, :]).masked_fill(~causal, -math.inf)).float()
    mix = grow(Cm @ B.transpose(-1, -2).contiguous()) * decay * dt[..., None, :]
    y = mix @ x
    weight = (torch.exp(cum[..., -1:] - cum) * dt).float()
    local = (x * weight[..., None]).transpose(-1, -2).contiguous() @ grow(B)  # [n][nc][H][P][N]
    states = torch.cat((old[:, :, None], local.transpose(1, 2)), 2).reshape(n, H, nc + 1, P * N)
    later = torch.ones((nc + 1, nc + 1), dtype=torch.bool, device=DEV).tril()
    passed = torch.exp((total[..., :, None] - total[..., None, :]).masked_fill(~later, -math.inf)).float()
    states = (passed @ states).reshape(n, H, nc + 1, P, N)                   # before chunk i; the last: behind all
    before = states[:, :, :-1].transpose(1, 2)                               # [n][nc][H][P][N]
    y = y + torch.exp(cum).float()[..., None] * (grow(Cm) @ before.transpose(-1, -2).contiguous())
    y = (y + x * layer["d"][:, None, None]).transpose(2, 3).reshape(n, nc * Q, H * P)
    y = y[live] if s["offsets"] is not None else y[:, :T].reshape(n * T, H * P)
    if s["z"] is not None:
        y = y * _silu(s["z"].float())
    if not case["final"]:
        return y.to(t)
    last = padded.gather(1, (length[:, None] + torch.arange(W - 1, device=DEV))[..., None].expand(n, W - 1, C))
    return y.to(t), last.transpose(1, 2).to(t).contiguous(), states[:, :, -1].contiguous()


def _plain_step(s):
    case, layer = s["case"], s["layer"]
    H, P, G, N = (case[k] for k in ("heads", "head_dim", "groups", "n_state"))
    n, t, slots = case["rows"], s["xbc"].dtype, s["slots"].long()
    window = torch.cat((s["state"][0][slots].float(), s["xbc"].float()[..., None]), -1)   # [n][C][W]
    u = _silu((window * layer["conv_w"]).sum(-1) + layer["conv_b"])
    x = u[:, :H * P].reshape(n, H, P, 1)
    B = u[:, H * P:H * P + G * N].reshape(n, G, 1, N).repeat_interleave(H // G, 1)
    Cm = u[:, H * P + G * N:].reshape(n, G, 1, N).repeat_interleave(H // G, 1)
    dt = _softplus(s["dt"].float() + layer["dt_bias"])
    S = s["state"][1][slots] * torch.exp(dt * layer["a"])[..., None, None] + dt[..., None, None] * x * B
    y = ((S * Cm).sum(-1) + x[..., 0] * layer["d"][:, None]).reshape(n, H * P) * _silu(s["z"].float())
    return y.to(t), window[..., 1:].to(t), S


def run(state):
    s, case = state, state["case"]
    op = case["op"]
    if not own:
        if op == "quantize":
            return _values(s["x"].float(), case["format"]).to(torch.bfloat16)
        return {"norm": _plain_norm, "product": _plain_product, "scan": _plain_scan, "step": _plain_step}[op](s)
    vf, ctx = _library()
    if op == "norm":
        fmt = _type_ids(vf)[case["out"]]
        y, total = vf.vf_rms_norm(ctx, s["x"], s["gain"], EPS, residual=s["residual"], out_type=fmt)
        if case["out"] in FORMATS:
            y = vf.vf_mx_dequantize(ctx, y)
        return (y, total) if total is not None else y
    if op == "quantize":
        return vf.vf_mx_dequantize(ctx, vf.vf_mx_quantize(ctx, s["x"], _type_ids(vf)[case["format"]]))
    if op == "product":
        ids = _type_ids(vf)
        a, w = (vf.MX(codes, scales, ids[fmt], cols) for codes, scales, fmt, cols in (s["a"], s["w"]))
        return vf.vf_mx_matmul(ctx, a, w, bias=s["bias"], out_type=ids[case["out"]])
    if "made" not in s:  # the layer's description, which a program keeps with the weights
        s["made"] = vf.SsmLayer(*(case[k] for k in ("heads", "head_dim", "groups", "n_state")), **s["layer"])
    layer = s["made"]
    if op == "step":
        y = vf.vf_ssm_step(ctx, layer, s["xbc"], s["dt"], z=s["z"], state=s["state"], slots=s["slots"], state_out=s["state_out"])
    else:
        y = vf.vf_ssm_scan(ctx, layer, s["xbc"], s["dt"], z=s["z"], n_seq=case["seqs"], longest=case["longest"],
                           offsets=s["offsets"], state=s["state"], slots=s["slots"], state_out=s["state_out"])
    return (y, *s["state_out"]) if s["state_out"] is not None else y


def _type_ids(vf):
    return {"fp32": vf.VF_FP32, "bf16": vf.VF_BF16, "e4m3": vf.VF_E4M3, "e2m1": vf.VF_E2M1}


_held = []


def _library():
    """The library and the context that a program keeps."""
    if not _held:
        import paper_2011_14486_amd as pkg
        vf = pkg.load()
        _held.extend((vf, vf.vf_create(0)))
    return _held


# ------------------------------------------------------------------ work

def work(case):
    op = case["op"]
    if op == "norm":
        each = BYTES[case["type"]] * (3 if case["residual"] else 1) + BYTES[case["out"]]
        return dict(bytes=case["rows"] * case["width"] * each + 4.0 * case["width"], flops=5.0 * case["rows"] * case["width"])
    if op == "quantize":  # the values in, codes out; codes in, the values out as bf16
        n = float(case["rows"] * case["cols"])
        return dict(bytes=n * (BYTES[case["type"]] + 2 * BYTES[case["format"]] + 2.0), flops=3.0 * n)
    if op == "product":
        M, N, K = float(case["M"]), case["N"], case["K"]
        return dict(bytes=M * K * BYTES[case["a"]] + N * K * BYTES["e2m1"] + M * N * BYTES[case["out"]], flops=2.0 * M * N * K)
    H, P, G, N, W = (case[k] for k in ("heads", "head_dim", "groups", "n_state", "taps"))
    C, size = H * P + 2 * G * N, BYTES[case["type"]]
    state = 4.0 * H * P * N + size * C * (W - 1)
    if op == "step":
        tokens, gate = case["rows"], True
        states = case["rows"] + min(case["rows"], case["slots"])
    else:
        tokens, gate = float(_lengths(case).sum()), case["gate"]
        states = case["seqs"] * (int(case["initial"]) + int(case["final"]))
    return dict(bytes=tokens * size * (C + H + H * P * (2 if gate else 1)) + states * state,
                flops=tokens * (5.0 * H * P * N + 2.0 * W * C))


# ------------------------------------------------------------------ the definitions in 64 bits

def _exact_values(y, fmt):
    """Nearest values of the format by comparing with all of them; ties to the even code."""
    emax, _, _, _ = FORMATS[fmt]
    if fmt == "e2m1":
        table = torch.tensor(E2M1[:8], dtype=torch.float64, device=y.device)
    else:
        table = torch.arange(127, dtype=torch.uint8, device=y.device).view(torch.float8_e4m3fn).double()
    mid = (table[1:] + table[:-1]) / 2
    cols = y.shape[1]
    v = torch.nn.functional.pad(y, (0, -cols % 32)).reshape(y.shape[0], -1, 32)
    top = v.abs().amax(-1, keepdim=True)
    e = (torch.floor(torch.log2(top)) - emax).clamp(-127, 127)
    m = v.abs() / torch.exp2(e)
    above, upto = torch.searchsorted(mid, m, right=True), torch.searchsorted(mid, m)
    code = torch.where(upto % 2 == 0, upto, above)
    return (torch.copysign(table[code], v) * torch.exp2(e)).reshape(y.shape[0], -1)[:, :cols]


def _exact_scan(s, n, T, lengths, starts, slots, gate):
    """Token by token.  A sequence that has ended keeps its state."""
    case, layer = s["case"], {k: v.double() for k, v in s["layer"].items()}
    H, P, G, N, W = (case[k] for k in ("heads", "head_dim", "groups", "n_state", "taps"))
    C = H * P + 2 * G * N
    tokens = s["xbc"].shape[0]
    past = torch.zeros((n, C, W - 1), dtype=torch.float64, device=DEV)
    S = torch.zeros((n, H, P, N), dtype=torch.float64, device=DEV)
    if s["state"] is not None:
        past, S = s["state"][0].double()[slots], s["state"][1].double()[slots]
    out = torch.zeros((tokens, H * P), dtype=torch.float64, device=DEV)
    for k in range(T):
        who = torch.arange(n, device=DEV) if int(lengths.min()) > k else torch.nonzero(lengths > k)[:, 0]
        row = starts[who] + k
        window = torch.cat((past[who], s["xbc"][row].double()[..., None]), -1)
        past[who] = window[..., 1:]
        v = torch.einsum("ncw,cw->nc", window, layer["conv_w"]) + layer["conv_b"]
        v = v * torch.sigmoid(v)
        x = v[:, :H * P].reshape(-1, H, P)
        B = v[:, H * P:H * P + G * N].reshape(-1, G, N)
        Cm = v[:, H * P + G * N:].reshape(-1, G, N)
        dt = torch.logaddexp(s["dt"][row].double() + layer["dt_bias"], torch.zeros((), dtype=torch.float64, device=DEV))
        add = (dt[..., None] * x).reshape(-1, G, H // G * P)[..., None] * B[:, :, None]
        now = S[who] * torch.exp(dt * layer["a"])[..., None, None] + add.reshape(-1, H, P, N)
        S[who] = now
        y = (now.reshape(-1, G, H // G * P, N) * Cm[:, :, None]).sum(-1).reshape(-1, H, P)
        out[row] = (y + layer["d"][:, None] * x).reshape(-1, H * P)
    if gate:
        z = s["z"].double()
        out = out * z * torch.sigmoid(z)
    return out, past, S


def exact(case, seed):
    s = prepare(case, seed)
    op = case["op"]
    if op == "norm":
        x = s["x"].double()
        if s["residual"] is not None:
            x = x + s["residual"].double()
        y = x / torch.sqrt(x.square().sum(-1, keepdim=True) / x.shape[1] + EPS) * s["gain"].double()
        y = _exact_values(y, case["out"]) if case["out"] in FORMATS else y
        return (y, x) if s["residual"] is not None else y
    if op == "quantize":
        return _exact_values(s["x"].double(), case["format"])
    if op == "product":
        y = torch.nn.functional.linear(_unpack(s["a"], torch.float64), _unpack(s["w"], torch.float64))
        return y if s["bias"] is None else y + s["bias"].double()
    if op == "step":
        n = case["rows"]
        return _exact_scan(s, n, 1, torch.ones(n, device=DEV), torch.arange(n, device=DEV), s["slots"].long(), True)
    lens = _lengths(case)
    starts = torch.from_numpy(np.concatenate([[0], np.cumsum(lens)[:-1]])).to(DEV)
    got = _exact_scan(s, case["seqs"], case["longest"], torch.from_numpy(lens).to(DEV), starts,
                      None if s["slots"] is None else s["slots"].long(), case["gate"])
    return got if case["final"] else got[0]
