"""The sequence operators written out in 64 bits with numpy, and the magnitudes that rounding errors go by."""
import numpy as np

U32, UBF = 2.0 ** -24, 2.0 ** -8   # largest relative error of one rounding
FORMATS = {2: (8, 448.0, -6, 3), 3: (2, 6.0, 0, 1)}   # VF_E4M3, VF_E2M1: emax, largest, least exponent, fraction bits


def grid_step(v, fmt):
    """Distance of the format's numbers around |v| (an array)."""
    _, _, emin, frac = FORMATS[fmt]
    _, e = np.frexp(v)
    return np.ldexp(1.0, np.maximum(np.where(v == 0, emin, e - 1), emin) - frac)


def quantize(x, fmt):
    """x float64 [rows][cols] -> (values of the codes [rows][kb][32], scale bytes [rows][kb])."""
    emax, most, _, _ = FORMATS[fmt]
    rows, cols = x.shape
    kb = (cols + 31) // 32
    v = np.zeros((rows, kb * 32))
    v[:, :cols] = x
    v = v.reshape(rows, kb, 32)
    codes, scales = np.zeros_like(v), np.zeros((rows, kb), np.uint8)
    for r in range(rows):
        for b in range(kb):
            block = v[r, b]
            if not np.isfinite(block).all():
                scales[r, b] = 255
                continue
            top = np.abs(block).max()
            e = -127 if top == 0 else max(int(np.floor(np.log2(top))) - emax, -127)
            scales[r, b] = e + 127
            m = block / 2.0 ** e
            step = grid_step(m, fmt)
            codes[r, b] = np.clip(np.rint(m / step) * step, -most, most)   # rint: ties to even
    return codes, scales


def code_values(codes, fmt):
    """uint8 codes [rows][...] -> float64 values [rows][kb][32]."""
    if fmt == 3:
        table = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
        n = np.stack((codes & 15, codes >> 4), -1).reshape(codes.shape[0], -1)
        v = np.where(n & 8, -1.0, 1.0) * table[n & 7]
    else:
        e, f = (codes >> 3) & 15, codes & 7
        v = np.where(e > 0, np.ldexp(1.0 + f / 8.0, e.astype(int) - 7), np.ldexp(f / 8.0, -6))
        v = np.where((e == 15) & (f == 7), np.nan, v) * np.where(codes & 128, -1.0, 1.0)
    return v.reshape(codes.shape[0], -1, 32)


def mx_values(codes, scales, fmt, cols):
    v = code_values(codes, fmt) * np.where(scales == 255, np.nan, np.ldexp(1.0, scales.astype(int) - 127))[..., None]
    return v.reshape(codes.shape[0], -1)[:, :cols]


def silu(x):
    with np.errstate(over="ignore"):
        return x / (1.0 + np.exp(-x))


def ssm(sizes, layer, xbc, dt, z, spans, state, slots):
    """sizes = (H, P, G, N, W); layer, inputs float64; spans = [(first, count)]; state = (conv, ssm) or None;
    slots = slot of every sequence or -1.  Returns out, the sequences' (conv, ssm), and for each of out and ssm
    the same sums of magnitudes."""
    H, P, G, N, W = sizes
    C = H * P + 2 * G * N
    n = len(spans)
    out, omag = np.full((xbc.shape[0], H * P), np.nan), np.zeros((xbc.shape[0], H * P))
    conv, st, smag = np.zeros((n, C, W - 1)), np.zeros((n, H, P, N)), np.zeros((n, H, P, N))
    bias = layer["conv_b"] if layer.get("conv_b") is not None else np.zeros(C)
    dtb = layer["dt_bias"] if layer.get("dt_bias") is not None else np.zeros(H)
    dd = layer["d"] if layer.get("d") is not None else np.zeros(H)
    group = np.arange(H) // (H // G)
    for s, (first, count) in enumerate(spans):
        past = np.zeros((C, W - 1))
        if state is not None and slots[s] >= 0:
            past, st[s] = state[0][slots[s]], state[1][slots[s]]
            smag[s] = np.abs(st[s])
        for t in range(first, first + count):
            window = np.concatenate((past, xbc[t][:, None]), 1)
            past = window[:, 1:]
            u = silu((window * layer["conv_w"]).sum(1) + bias)
            um = (np.abs(window) * np.abs(layer["conv_w"])).sum(1) + np.abs(bias)
            parts = []
            for q in (u, um):
                parts += [q[:H * P].reshape(H, P), q[H * P:H * P + G * N].reshape(G, N)[group], q[H * P + G * N:].reshape(G, N)[group]]
            x, B, Cm, xm, Bm, Cmm = parts
            step = np.logaddexp(dt[t] + dtb, 0.0)
            a = np.exp(step * layer["a"])[:, None, None]
            st[s] = a * st[s] + step[:, None, None] * x[:, :, None] * B[:, None, :]
            smag[s] = a * smag[s] + step[:, None, None] * xm[:, :, None] * Bm[:, None, :]
            y = (st[s] * Cm[:, None, :]).sum(-1) + dd[:, None] * x
            ym = (smag[s] * Cmm[:, None, :]).sum(-1) + np.abs(dd)[:, None] * xm
            gate = silu(z[t]) if z is not None else 1.0
            out[t], omag[t] = y.reshape(-1) * gate, ym.reshape(-1) * np.abs(gate)
        conv[s] = past
    return out, conv, st, omag, smag
