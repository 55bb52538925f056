"""Plain implementations, in 64 bits, of the rotary positions, the dropout, the gated recurrence and the routing to experts,
with the bounds on float32 kernels' errors that their tests use.  A rounding to T is off by UNIT[T] of the value at most."""
import math

import numpy as np
import torch

HALVES, PAIRS = 0, 1
PLAIN, COMPLEMENT = 0, 1
F32 = 2.0 ** -24
UNIT = {0: 2.0 ** -8, 1: F32}                       # by precision: bf16, float
DTYPE = {0: torch.bfloat16, 1: torch.float32}


def rounded(a, prec):
    """a as T holds it, in float64."""
    return torch.as_tensor(np.asarray(a, dtype=np.float64)).to(DTYPE[prec]).double().numpy()


# ---- rotary ----

def frequencies(rot, base=10000.0, factor=1.0, original=0, low=1.0, high=32.0):
    """Radians a position."""
    out = []
    for i in range(rot // 2):
        f = base ** (-2.0 * i / rot)
        if factor > 1:
            keep = min(1.0, max(0.0, (original * f / (2 * math.pi) - low) / (high - low))) if original else 0.0
            f *= keep + (1 - keep) / factor
        out.append(f)
    return np.array(out)


def rotary(x, positions, freq, rot, layout, amplitude=1.0, back=False):
    """x [rows, heads, head_dim], positions [rows] -> y, and a bound on a kernel's error before y's own rounding.

    A kernel's cosine and sine are within 2^-22: two units of the last place of 1, and the angle's rounding (an eighth of a
    turn to 24 bits).  Amplitude, products and the sum add three roundings of at most A (|x_a| + |x_b|) each; the frequencies, held here
    in 53 bits, leave the angle uncertain by 2^-52 of itself."""
    angle = positions[:, None].astype(np.float64) * freq[None, :]
    c, s = amplitude * np.cos(angle)[:, None], (-1 if back else 1) * amplitude * np.sin(angle)[:, None]
    h = rot // 2
    a, b = (slice(0, h), slice(h, rot)) if layout == HALVES else (slice(0, rot, 2), slice(1, rot, 2))
    y, bound = x.copy(), np.zeros_like(x)
    y[..., a] = x[..., a] * c - x[..., b] * s
    y[..., b] = x[..., b] * c + x[..., a] * s
    bound[..., a] = bound[..., b] = abs(amplitude) * (np.abs(x[..., a]) + np.abs(x[..., b])) * (2.0 ** -22 + 3 * F32 + np.abs(angle)[:, None] * 2.0 ** -52)
    return y, bound


# ---- dropout ----

def philox(counter, key):
    """Philox4x32-10 on whole numbers of Python or arrays of uint64: four words."""
    c = [np.asarray(x, dtype=np.uint64) for x in counter]
    k = list(key)
    low, up = np.uint64(0xFFFFFFFF), np.uint64(32)
    for _ in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        c = [(p1 >> up) ^ c[1] ^ np.uint64(k[0]), p1 & low, (p0 >> up) ^ c[3] ^ np.uint64(k[1]), p0 & low]
        k = [(k[0] + 0x9E3779B9) & 0xFFFFFFFF, (k[1] + 0xBB67AE85) & 0xFFFFFFFF]
    return c


def kept(rows, cols, p, seed, offset):
    """Which elements are kept, and 1 / (1 - p) as it is taken."""
    groups = -(-cols // 8)
    offset %= 2 ** 64
    row, group = np.meshgrid(np.arange(rows), np.arange(groups), indexing="ij")
    words = philox((group, row, np.full_like(row, offset & 0xFFFFFFFF), np.full_like(row, offset >> 32)), (seed & 0xFFFFFFFF, seed >> 32))
    bits = np.zeros((rows, groups, 8), dtype=np.uint64)
    for j in range(8):
        bits[:, :, j] = (words[j // 2] >> np.uint64(16 * (j % 2))) & np.uint64(0xFFFF)
    limit = int(np.rint(np.float64(np.float32(p)) * 65536))
    return bits.reshape(rows, groups * 8)[:, :cols] >= limit, (65536.0 / (65536 - limit) if limit < 65536 else 0.0)


# ---- recurrence ----

def sigmoid(x):
    with np.errstate(over="ignore"):
        return 1 / (1 + np.exp(-x))


def recurrence(f, x, g, h0, offsets, mode):
    """f, x, g [rows, d] (g None: no gate), h0 [n_seq, d], offsets [n_seq + 1] -> dict of y, h, before (h of the token
    before), h_last, and bounds on a float32 kernel's errors: of h (`e_h`), and of y before its rounding (`e_y`).

    A kernel's gates have a relative error of gate_error(f); a step's product and sum and, where stretches are joined,
    the products of a stretch's decays round a few times, each by F32 of at most `habs`, the recurrence of the absolute values.  Those errors
    decay like h itself, so they obey the recurrence too."""
    a, rest = sigmoid(f), sigmoid(-f)
    b = rest * x if mode == COMPLEMENT else x
    h, before, e_h, h_last, habs_all = np.zeros_like(f), np.zeros_like(f), np.zeros_like(f), h0.copy(), np.zeros_like(f)
    for s in range(len(offsets) - 1):
        state, habs, err = h0[s].copy(), np.abs(h0[s]), np.zeros(f.shape[1])
        for t in range(offsets[s], offsets[s + 1]):
            before[t] = state
            size = a[t] * habs + np.abs(b[t])
            err = a[t] * err + gate_error(f[t]) * (a[t] * rest[t] * habs + np.abs(b[t])) + 8 * F32 * size
            state, habs = a[t] * state + b[t], size
            h[t], e_h[t], habs_all[t] = state, err, habs
        h_last[s] = state
    y, e_y = h, e_h
    if g is not None:
        gate = g * sigmoid(g)
        y, e_y = h * gate, e_h * np.abs(gate) + np.abs(h * gate) * (gate_error(g) + 3 * F32)
    return dict(a=a, rest=rest, h=h, before=before, y=y, h_last=h_last, e_h=e_h, e_y=e_y, habs=habs_all)


def gate_error(f):
    """Relative error of a kernel's sigmoid: the exponential (2^-22 and the rounding of its argument, |f| 2^-23), sum, reciprocal
    (2^-23) and product."""
    return 2.0 ** -21 + np.abs(f) * 2.0 ** -23


def recurrence_backward(f, x, g, h0, offsets, mode, dy, dh_last, fwd):
    """Gradients and bounds on a float32 kernel's errors before their rounding: {name: (value, bound)}."""
    a, rest, before, h = fwd["a"], fwd["rest"], fwd["before"], fwd["h"]
    gate = g * sigmoid(g) if g is not None else np.ones_like(f)
    u = dy * gate
    e_u = np.abs(u) * (gate_error(g) + 3 * F32) if g is not None else np.zeros_like(u)
    dh, e_dh, dh0, e_dh0 = np.zeros_like(f), np.zeros_like(f), dh_last.copy(), np.zeros_like(dh_last)
    for s in range(len(offsets) - 1):
        carry, size, err = dh_last[s].copy(), np.abs(dh_last[s]), np.zeros(f.shape[1])
        for t in range(offsets[s + 1] - 1, offsets[s] - 1, -1):
            now, much = u[t] + carry, np.abs(u[t]) + size
            here = err + e_u[t] + F32 * much
            dh[t], e_dh[t] = now, here
            carry, size = a[t] * now, a[t] * much
            err = a[t] * here + (gate_error(f[t]) * rest[t] + 8 * F32) * size
        dh0[s], e_dh0[s] = carry, err
    e_before = np.zeros_like(f)
    for s in range(len(offsets) - 1):
        lo, hi = offsets[s], offsets[s + 1]
        e_before[lo + 1:hi] = fwd["e_h"][lo:hi - 1] if hi > lo else 0
    diff = before - x if mode == COMPLEMENT else before
    size = np.abs(before) + np.abs(x) if mode == COMPLEMENT else np.abs(before)
    ar = a * rest
    out = {"df": (dh * diff * ar, ar * (e_dh * np.abs(diff) + np.abs(dh) * e_before) + ar * np.abs(dh) * size * (2 * gate_error(f) + 6 * F32)),
           "dx": (dh * rest, e_dh * rest + np.abs(dh) * rest * (gate_error(f) + 2 * F32)) if mode == COMPLEMENT else (dh, e_dh),
           "dh0": (dh0, e_dh0)}
    if g is not None:
        sg = sigmoid(g)
        slope = sg * (1 + g * (1 - sg))
        out["dg"] = (dy * h * slope, np.abs(dy * slope) * fwd["e_h"] + np.abs(dy * h) * (np.abs(sg) + np.abs(g) * sg * (1 - sg)) * (3 * gate_error(g) + 6 * F32)
                     + np.abs(dy * slope) * fwd["habs"] * 4 * F32)
    return out


# ---- experts ----

def expert_plan(ids, n_experts, capacity, align, slots):
    """ids [n, k] -> slot_of, source, offsets, counts, choice by choice."""
    flat = ids.reshape(-1)
    lists = [[] for _ in range(n_experts)]
    for i, e in enumerate(flat):
        if 0 <= e < n_experts:
            lists[e].append(i)
    counts = np.array([len(x) for x in lists])
    room = np.full(n_experts, capacity) if capacity else -(-counts // align) * align
    offsets = np.concatenate([[0], np.cumsum(room)])
    slot_of, source = np.full(len(flat), -1), np.full(slots, -1)
    for e, x in enumerate(lists):
        for r, i in enumerate(x[:capacity] if capacity else x):
            slot_of[i], source[offsets[e] + r] = offsets[e] + r, i
    return slot_of.reshape(ids.shape), source, offsets, counts


def combine(slot_of, weights, z, resid):
    """y and a bound on a float32 kernel's error before y's rounding: a rounding for each addition of what it adds up to."""
    n, k = slot_of.shape
    y = np.zeros((n, z.shape[1])) if resid is None else resid.copy()
    size = np.abs(y)
    for t in range(n):
        for j in range(k):
            if slot_of[t, j] >= 0:
                w = 1.0 if weights is None else weights[t, j]
                y[t] += w * z[slot_of[t, j]]
                size[t] += np.abs(w * z[slot_of[t, j]])
    return y, (k + 1) * F32 * size
