"""The attention operators written out in 64 bits with numpy, and the magnitudes that rounding errors go by."""
import numpy as np

from tests.ops_ref import mx_values, quantize

NONE = -1   # an entry of a table that is no page


def width_of(fmt, dim):
    """Elements of a row of the cache."""
    return (dim + 31) // 32 * 32 if fmt == 2 else (dim + 7) // 8 * 8


def turned(x, pos, freq, interleaved, magnitude):
    """x [rows][heads][dim] at positions pos [rows]; returns the turned numbers and the same sums of magnitudes."""
    r = 2 * len(freq)
    angle = pos[:, None] * freq
    c, s = magnitude * np.cos(angle)[:, None], magnitude * np.sin(angle)[:, None]
    out, mag = x.copy(), np.abs(x)
    first, second = (slice(0, r, 2), slice(1, r, 2)) if interleaved else (slice(0, r // 2), slice(r // 2, r))
    a, b = x[..., first], x[..., second]
    out[..., first], out[..., second] = a * c - b * s, b * c + a * s
    both = (np.abs(a) + np.abs(b)) * abs(magnitude)
    mag[..., first], mag[..., second] = both, both
    return out, mag


def spans(offsets, n_seq, tokens):
    """(first, rows) of every sequence; ranges that do not lie in the tokens are empty."""
    if offsets is None:
        each = tokens // n_seq if n_seq else 0
        return [(s * each, each) for s in range(n_seq)]
    made = []
    for b, e in zip(offsets[:-1], offsets[1:]):
        fine = 0 <= b <= e <= tokens
        made.append((int(b), int(e - b)) if fine else (0, 0))
    return made


def length_of(lengths, s, table, page):
    return int(min(max(int(lengths[s]), 0), table.shape[1] * page))


def places(offsets, lengths, table, page, tokens):
    """Per row of the call: (sequence, position) or None for rows of no sequence."""
    at = [None] * tokens
    for s, (first, rows) in enumerate(spans(offsets, len(lengths), tokens)):
        for i in range(rows):
            at[first + i] = (s, length_of(lengths, s, table, page) - rows + i)
    return at


def keys_of(pool, table, page, s, length, pages):
    """Keys or values of a sequence [length][heads][dim] from pool [pages][heads][page][dim] in float64; of a page that is not there
    zeros, of an entry that is no page NaN."""
    out = np.zeros((length, pool.shape[1], pool.shape[3]))
    there = np.ones(length, bool)
    for t0 in range(0, length, page):
        e, n = int(table[s, t0 // page]), min(page, length - t0)
        if e == NONE:
            there[t0:t0 + n] = False
        elif 0 <= e < pages:
            out[t0:t0 + n] = pool[e][:, :n].transpose(1, 0, 2)
        else:
            out[t0:t0 + n] = np.nan
    return out, there


def attend(q, k_pool, v_pool, table, lengths, page, heads, causal, window, scale, offsets):
    """q [tokens][heads dim]; pools [pages][kv_heads][page][dim].  Returns out, sum of weights times |values|, and the largest sum of
    magnitudes of a row's scores, each [tokens][heads ..]; rows of no sequence are NaN."""
    tokens, kv, dim, pages = q.shape[0], k_pool.shape[1], k_pool.shape[3], k_pool.shape[0]
    group = heads // kv
    out, mag = np.full((tokens, heads, dim), np.nan), np.zeros((tokens, heads, dim))
    size = np.zeros((tokens, heads))
    for s, (first, rows) in enumerate(spans(offsets, len(lengths), tokens)):
        length = length_of(lengths, s, table, page)
        k, there = keys_of(k_pool, table, page, s, length, pages)
        v, _ = keys_of(v_pool, table, page, s, length, pages)
        t = np.arange(length)
        for i in range(rows):
            pos = length - rows + i
            seen = there.copy()
            if causal:
                seen &= t <= pos
                if window:
                    seen &= t > pos - window
            for h in range(heads):
                qr = q[first + i].reshape(heads, dim)[h]
                kk, vv = k[seen, h // group], v[seen, h // group]
                z = scale * (kk @ qr)
                if len(z) == 0 or (z == -np.inf).all():
                    out[first + i, h] = 0.0
                    continue
                with np.errstate(invalid="ignore", over="ignore"):
                    p = np.exp(z - np.nanmax(z)) if not np.isnan(z).any() else np.full(len(z), np.nan)
                    p = p / p.sum()
                    out[first + i, h] = p @ vv
                    mag[first + i, h] = p @ np.abs(vv)
                    size[first + i, h] = np.max(scale * (np.abs(kk) @ np.abs(qr)))
    return out.reshape(tokens, -1), mag.reshape(tokens, -1), np.repeat(size, dim, 1).reshape(tokens, -1)


def cache_values(fmt, dim, rows, scales):
    """Rows of a cache [..][w] as float64 [..][dim]: numbers, or codes with scales."""
    if fmt != 2:
        return rows[..., :dim].astype(np.float64)
    shape = rows.shape[:-1]
    return mx_values(rows.reshape(-1, rows.shape[-1]), scales.reshape(-1, scales.shape[-1]), 2, dim).reshape(*shape, dim)


def eight_bits(x):
    """x [rows][dim] as 8-bit floats with scales: (values, steps between the format's numbers there, scale bytes)."""
    from tests.ops_ref import grid_step
    codes, scales = quantize(x, 2)
    e = np.ldexp(1.0, scales.astype(int) - 127)[..., None]
    step = grid_step(codes, 2) * e
    return (codes * e).reshape(len(x), -1)[:, :x.shape[1]], step.reshape(len(x), -1)[:, :x.shape[1]], scales
