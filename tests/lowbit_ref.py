"""Plain implementations, in 64 bits, of the operators on few bits: quantisation in blocks, products of
quantised matrices, AdamW with 8-bit moments, embedding lookup and gradient.  Values in 8 bits are held
as the float64 values they stand for."""
import numpy as np
import torch

BLOCK = 128
E4M3, E5M2 = 0, 1
TORCH8 = (torch.float8_e4m3fn, torch.float8_e5m2)
TOP = (448.0, 57344.0)
LOW = (-6, -14)            # exponent of the smallest normal value
DIGITS = (3, 2)            # mantissa digits


def scale_for(amax, fmt):
    """The smallest power of two, at least 2^-126, that brings amax to TOP at most; 1 where amax is 0."""
    f, e = np.frexp(amax / TOP[fmt])
    e = np.maximum(np.where(f == 0.5, e - 1, e), -126)
    return np.where(amax == 0, 1.0, np.ldexp(1.0, e))


def step_at(y, fmt):
    _, e = np.frexp(np.abs(y))
    return np.ldexp(1.0, np.maximum(e - 1, LOW[fmt]) - DIGITS[fmt])


def quantize(x, fmt, tile):
    """x [rows, cols] float64 -> (values / scale rounded to nearest even, scales [col blocks, rows or row blocks])."""
    r, c = x.shape
    rp, cp = -(-r // tile) * tile, -(-c // BLOCK) * BLOCK
    p = np.zeros((rp, cp))
    p[:r, :c] = x
    p = p.reshape(rp // tile, tile, cp // BLOCK, BLOCK)
    fin = np.isfinite(p)
    s = scale_for(np.where(fin, np.abs(p), 0).max(axis=(1, 3), keepdims=True), fmt)
    with np.errstate(invalid="ignore"):
        y = np.where(fin, p, 0) / s
        step = step_at(y, fmt)
        q = np.where(fin, np.round(y / step) * step, np.nan)
    return q.reshape(rp, cp)[:r, :c], s[:, 0, :, 0].T.copy()


def widen(q, s, tile):
    """Values times their scales."""
    r, c = q.shape
    full = np.repeat(np.repeat(s.T, tile, axis=0)[:r], BLOCK, axis=1)[:, :c]
    return q * full


def bytes_of(q, fmt, pitch, fill=0):
    """q (exact values of the format) as bytes with a row pitch."""
    b = torch.full((q.shape[0], pitch), fill, dtype=torch.uint8)
    b[:, :q.shape[1]] = torch.as_tensor(q).float().to(TORCH8[fmt]).view(torch.uint8)
    return b


def mix32(x):
    x = np.asarray(x, dtype=np.uint64) & np.uint64(0xFFFFFFFF)
    low = np.uint64(0xFFFFFFFF)
    x = ((x ^ (x >> np.uint64(16))) * np.uint64(0x7FEB352D)) & low
    x = ((x ^ (x >> np.uint64(15))) * np.uint64(0x846CA68B)) & low
    return x ^ (x >> np.uint64(16))


def random_halves(n, seed, step):
    i = np.arange(n, dtype=np.uint64)
    low = np.uint64(0xFFFFFFFF)
    key = mix32((seed + step * 0x9E3779B9) & 0xFFFFFFFF)
    h = mix32((i & low) ^ ((key + (i >> np.uint64(32)) * np.uint64(0x85EBCA77)) & low))
    return (h >> np.uint64(16)).astype(np.float64), (h & np.uint64(0xFFFF)).astype(np.float64)


def round_moment(x, fmt, u):
    """Stochastic rounding of blocks of 128: (values, scales).  u: 16 random bits an element."""
    n = x.size
    nb = -(-n // BLOCK)
    fin = np.isfinite(x)
    p = np.zeros(nb * BLOCK)
    p[:n] = np.where(fin, np.abs(x), 0)
    s = scale_for(p.reshape(nb, BLOCK).max(axis=1), fmt)
    y = np.where(fin, np.abs(x), 0) / np.repeat(s, BLOCK)[:n]
    fine = 2.0 ** (-149 - (-120, -112)[fmt])                  # float32's last digit below the smallest normal value
    y = np.where(y < 2.0 ** LOW[fmt], np.round(y / fine) * fine, y)
    step = step_at(y, fmt)
    q = np.minimum(np.floor(y / step + (u + 0.5) / 65536) * step, TOP[fmt])
    if fmt == E5M2:
        q = np.where((x > 0) & (q == 0), 2.0 ** (LOW[fmt] - DIGITS[fmt]), q)
    return np.where(fin, np.where(x < 0, -q, q), np.nan), s


def adamw8(w, m, ms, v, vs, g, wd, seed, lr, beta1, beta2, eps, step):
    """One step; every operation is done in 64 bits and rounded to float32, as the definition asks.
    m, v: values; ms, vs: scales of blocks of 128.  Returns (w, m, ms, v, vs)."""
    def R(x):
        with np.errstate(over="ignore"):
            return np.asarray(x, dtype=np.float64).astype(np.float32).astype(np.float64)
    lr, b1, b2, eps, wd = (float(np.float32(x)) for x in (lr, beta1, beta2, eps, wd))
    c1, c2 = float(np.float32(1 / (1 - b1 ** step))), float(np.float32(1 / (1 - b2 ** step)))
    o1, o2 = float(np.float32(1 - b1)), float(np.float32(1 - b2))
    n = w.size
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        m = R(m * np.repeat(ms, BLOCK)[:n])
        v = R(v * np.repeat(vs, BLOCK)[:n])
        m = R(R(b1 * m) + R(o1 * g))
        v = R(R(b2 * v) + R(R(o2 * g) * g))
        upd = R(R(lr * R(m * c1)) / R(R(np.sqrt(R(v * c2))) + eps))
        w = R(R(w - R(R(lr * wd) * w)) - upd)
    um, uv = random_halves(n, seed, step)
    qm, sm = round_moment(m, E4M3, um)
    qv, sv = round_moment(v, E5M2, uv)
    return w, qm, sm, qv, sv


def embedding(ids, table, scale):
    out = np.zeros((len(ids), table.shape[1]))
    ok = (ids >= 0) & (ids < len(table))
    out[ok] = float(np.float32(scale)) * table[ids[ok]]
    return out


def embedding_grad(ids, dout, vocab, scale):
    out = np.zeros((vocab, dout.shape[1]))
    ok = (ids >= 0) & (ids < vocab)
    np.add.at(out, ids[ok], dout[ok])
    return float(np.float32(scale)) * out
