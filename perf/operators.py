"""The operators of a training step kept in few bits, and the two ends of the token table, as they are measured.

  emb_fwd   rows of the token table, scaled
  emb_bwd   the table's gradient, summed over the tokens that are alike
  adamw8    AdamW over many tensors at once, moments in 8 bits with a scale for each 128 elements
  quant     matrices in 8-bit floating point with a scale for each 1 x 128 or 128 x 128 elements, as stored and transposed
  gemm8     C = A B^T of such matrices

`run` computes them in plain torch operations; where `own` is set, through paper_2204_06514_b200's entry points.
"""
import math

import numpy as np
import torch

own = False

BLOCK = 128
E4M3, E5M2 = 0, 1
TORCH8 = (torch.float8_e4m3fn, torch.float8_e5m2)
TOP = (448.0, 57344.0)          # largest finite value of the two formats


def listed():
    return [
        # a few sequences' next tokens looked up at once: latency is all there is
        {"name": "emb_fwd_128x256_f32", "op": "emb_fwd", "n": 128, "vocab": 1000, "d": 256, "f32": True, "pad": 0.1},
        # the 124M model's batch: 16 x 1024 tokens of hidden size 768
        {"name": "emb_fwd_16384x768", "op": "emb_fwd", "n": 16384, "vocab": 50304, "d": 768, "f32": False, "pad": 0.0},
        # the same batch's gradient, the table's untouched rows zeroed
        {"name": "emb_bwd_16384x768", "op": "emb_bwd", "n": 16384, "vocab": 50304, "d": 768, "f32": False, "pad": 0.0, "acc": False},
        # a long ragged batch added to the output head's gradient of a tied table, a tenth of it padding
        {"name": "emb_bwd_61237x2048_acc", "op": "emb_bwd", "n": 61237, "vocab": 50304, "d": 2048, "f32": False, "pad": 0.1, "acc": True},
        # every tensor of a two-layer model of hidden size 250 (odd sizes, short biases): 28 tensors in one call
        {"name": "adamw8_28_tensors_d250", "op": "adamw8", "d": 250, "ff": 1000, "layers": 2, "vocab": 0, "bf16_grad": False, "step": 7},
        # the weights of one block of hidden size 4096: 201 million elements
        {"name": "adamw8_block_d4096", "op": "adamw8", "d": 4096, "ff": 16384, "layers": 1, "vocab": 0, "bf16_grad": False, "step": 100},
        # sixteen rows of activations before one decode-like product
        {"name": "quant_rows_16x768", "op": "quant", "rows": 16, "cols": 768, "f32": False, "tile": 1, "fmt": E4M3, "straight": True, "transposed": False},
        # an activation matrix for the forward product (rows) and the weight gradient (columns) from one reading
        {"name": "quant_both_8192x4096", "op": "quant", "rows": 8192, "cols": 4096, "f32": False, "tile": 1, "fmt": E4M3, "straight": True, "transposed": True},
        # a float32 master weight, 128 x 128 blocks, as stored (input gradient) and transposed (forward)
        {"name": "quant_weight_f32_4100x4096", "op": "quant", "rows": 4100, "cols": 4096, "f32": True, "tile": 128, "fmt": E4M3, "straight": True, "transposed": True},
        # sixteen tokens through a 4096 x 4096 projection
        {"name": "gemm8_16x4096x4096", "op": "gemm8", "m": 16, "n": 4096, "k": 4096, "fa": E4M3, "fb": E4M3, "b_block": 128, "f32": False, "acc": False, "bias": True},
        # the first MLP product of a block of hidden size 4096 on 8192 tokens, with its bias
        {"name": "gemm8_8192x16384x4096", "op": "gemm8", "m": 8192, "n": 16384, "k": 4096, "fa": E4M3, "fb": E4M3, "b_block": 128, "f32": False, "acc": False, "bias": True},
        # a weight gradient on a ragged batch of 5000 tokens: activations times e5m2 gradients, added to a float32 gradient
        {"name": "gemm8_wgrad_4096x1000x5000", "op": "gemm8", "m": 4096, "n": 1000, "k": 5000, "fa": E4M3, "fb": E5M2, "b_block": 1, "f32": True, "acc": True, "bias": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["emb_fwd", "emb_bwd", "adamw8", "quant", "gemm8"])
    if op in ("emb_fwd", "emb_bwd"):
        c = {"op": op, "n": _log(rng, 1, 60000), "vocab": _log(rng, 2, 50000), "d": _log(rng, 1, 2040), "f32": rng.random() < 0.3,
             "pad": rng.choice([0.0, 0.1, 0.5])}
        if rng.random() < 0.5:
            c["d"] = (c["d"] + 63) // 64 * 64
        if op == "emb_bwd":
            c["acc"] = rng.random() < 0.5
        return c
    if op == "adamw8":
        d = _log(rng, 4, 2000)
        return {"op": op, "d": d, "ff": _log(rng, d, 4 * d), "layers": rng.randint(1, 3), "vocab": 0 if rng.random() < 0.5 else _log(rng, 16, 20000),
                "bf16_grad": rng.random() < 0.4, "step": _log(rng, 1, 20000)}
    if op == "quant":
        straight = rng.random() < 0.7
        return {"op": op, "rows": _log(rng, 1, 9000), "cols": _log(rng, 1, 4500), "f32": rng.random() < 0.3, "tile": rng.choice([1, 1, 128]),
                "fmt": rng.choice([E4M3, E4M3, E5M2]), "straight": straight, "transposed": not straight or rng.random() < 0.6}
    f32 = rng.random() < 0.4
    return {"op": op, "m": _log(rng, 1, 8000), "n": _log(rng, 8, 8000), "k": _log(rng, 16, 6000), "fa": rng.choice([E4M3, E4M3, E5M2]), "fb": rng.choice([E4M3, E4M3, E5M2]),
            "b_block": rng.choice([1, 128]), "f32": f32, "acc": f32 and rng.random() < 0.5, "bias": not f32 and rng.random() < 0.5}


def _up(x, a):
    return (x + a - 1) // a * a


def _sizes(c):
    """Element counts and weight decays of a model's tensors, in the framework's order."""
    d, f, one = c["d"], c["ff"], []
    if c["vocab"]:
        one += [(c["vocab"] * d, 0.1)]
    for _ in range(c["layers"]):
        one += [(d, 0.0), (d, 0.0), (3 * d * d, 0.1), (3 * d, 0.0), (d * d, 0.1), (d, 0.0), (d, 0.0), (d, 0.0), (d * f, 0.1), (f, 0.0), (f * d, 0.1), (d, 0.0)]
    if c["layers"] > 1:
        one += [(d, 0.0), (d, 0.0)]
        one += [(d * d, 0.1), (d, 0.0)]
    return one


def _distinct(n, vocab):
    """How many ids of Zipf's distribution n draws are expected to touch."""
    k = np.arange(1, vocab + 1, dtype=np.float64)
    p = np.log1p(1.0 / k) / math.log(vocab + 1)
    return float(np.sum(-np.expm1(n * np.log1p(-np.minimum(p, 1 - 1e-12)))))


def work(c):
    if c["op"] in ("emb_fwd", "emb_bwd"):
        es = 4 if c["f32"] else 2
        live = max(1.0, c["n"] * (1 - c["pad"]))
        rows = min(_distinct(live, c["vocab"]), live)
        if c["op"] == "emb_fwd":
            return {"bytes": 4.0 * c["n"] + (rows + c["n"]) * c["d"] * es, "flops": live * c["d"]}
        table = 2 * rows * c["d"] * 4 if c["acc"] else c["vocab"] * c["d"] * 4
        return {"bytes": 4.0 * c["n"] + live * c["d"] * es + table, "flops": live * c["d"]}
    if c["op"] == "adamw8":
        n = sum(n for n, _ in _sizes(c))
        return {"bytes": n * (16.0 if c["bf16_grad"] else 18.0) + 16.0 * sum(-(-n // BLOCK) for n, _ in _sizes(c)), "flops": 16.0 * n}
    if c["op"] == "quant":
        r, k, t = c["rows"], c["cols"], c["tile"]
        scales = (-(-k // BLOCK) * -(-r // t)) * c["straight"] + (-(-r // BLOCK) * -(-k // t)) * c["transposed"]
        return {"bytes": r * k * ((4.0 if c["f32"] else 2.0) + c["straight"] + c["transposed"]) + 4.0 * scales, "flops": 2.0 * r * k}
    m, n, k = c["m"], c["n"], c["k"]
    kb = -(-k // BLOCK)
    es = 4 if c["f32"] else 2
    return {"bytes": float(m * k + n * k + 4 * kb * (m + -(-n // c["b_block"])) + m * n * es * (2 if c["acc"] else 1) + 2 * n * c["bias"]), "flops": 2.0 * m * n * k}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _ids(c, g, dev):
    """Token ids of Zipf's distribution, frequent ones anywhere in the table; a share of them is padding (-1)."""
    u = torch.rand(c["n"], generator=g, device=dev, dtype=torch.float64)
    rank = torch.exp(u * math.log(c["vocab"] + 1)).long().clamp_(1, c["vocab"]) - 1
    place = torch.randperm(c["vocab"], generator=g, device=dev)
    ids = place[rank].to(torch.int32)
    if c["pad"]:
        ids = torch.where(torch.rand(c["n"], generator=g, device=dev) < c["pad"], torch.full_like(ids, -1), ids)
    return ids


def _pow2(field):
    """2^(field - 127) for exponent fields 1 .. 254."""
    return (field << 23).to(torch.int32).view(torch.float32)


def _scale_field(amax, fmt):
    """Exponent field of the smallest power of two s with amax / s <= TOP (at least 2^-126; 1 for a block of zeros)."""
    bits = amax.view(torch.int32).to(torch.int64)
    field = ((bits + 0x1FFFFF) >> 23) - (8, 15)[fmt]
    return torch.where(bits == 0, torch.full_like(field, 127), field.clamp(min=1))


def _quantized(x, fmt):
    """x [rows, k] float32 -> values in 8 bits [rows, k], scales [k blocks, rows]: one for each 128 elements of a row."""
    r, k = x.shape
    kb = -(-k // BLOCK)
    xp = torch.nn.functional.pad(x, (0, kb * BLOCK - k)).view(r, kb, BLOCK)
    fin = torch.isfinite(xp)
    field = _scale_field(torch.where(fin, xp.abs(), torch.zeros_like(xp)).amax(dim=2), fmt)
    y = xp * _pow2(254 - field).unsqueeze(2)
    y = torch.where(fin, y, torch.full_like(y, math.nan))
    return y.view(r, kb * BLOCK)[:, :k].to(TORCH8[fmt]), _pow2(field).t().contiguous()


def _quantized_square(x, fmt):
    """x [rows, k] float32 -> values in 8 bits, scales [k blocks, row blocks]: one for each 128 x 128 elements."""
    r, k = x.shape
    rb, kb = -(-r // BLOCK), -(-k // BLOCK)
    xp = torch.nn.functional.pad(x, (0, kb * BLOCK - k, 0, rb * BLOCK - r)).view(rb, BLOCK, kb, BLOCK)
    fin = torch.isfinite(xp)
    field = _scale_field(torch.where(fin, xp.abs(), torch.zeros_like(xp)).amax(dim=(1, 3)), fmt)
    y = xp * _pow2(254 - field).view(rb, 1, kb, 1)
    y = torch.where(fin, y, torch.full_like(y, math.nan))
    return y.reshape(rb * BLOCK, kb * BLOCK)[:r, :k].to(TORCH8[fmt]), _pow2(field).t().contiguous()


def _matrix(rows, cols, g, dev):
    """Activations or gradients: normal, a few columns and rows much larger than the rest, some exact zeros."""
    x = torch.randn((rows, cols), generator=g, device=dev)
    x *= torch.exp(1.5 * torch.randn((1, cols), generator=g, device=dev))
    x *= torch.exp(0.7 * torch.randn((rows, 1), generator=g, device=dev))
    x[:, ::61] = 0
    return x


def _pitched(q, pitch):
    """q [rows, k] in memory of `pitch` elements a row."""
    buf = torch.zeros((q.shape[0], pitch), dtype=torch.uint8, device=q.device)
    buf[:, :q.shape[1]] = q.view(torch.uint8)
    return buf


def prepare(c, seed):
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 1009 + 17)
    s = {"c": c, "op": c["op"], "dev": dev}
    if c["op"] in ("emb_fwd", "emb_bwd"):
        t = torch.float32 if c["f32"] else torch.bfloat16
        s["ids"] = _ids(c, g, dev)
        s["scale"] = math.sqrt(c["d"])
        if c["op"] == "emb_fwd":
            s["table"] = (0.02 * torch.randn((c["vocab"], c["d"]), generator=g, device=dev)).to(t)
            s["out"] = torch.empty((c["n"], c["d"]), dtype=t, device=dev)
        else:
            s["dout"] = torch.randn((c["n"], c["d"]), generator=g, device=dev).to(t)
            s["dtable"] = torch.randn((c["vocab"], c["d"]), generator=g, device=dev) if c["acc"] else torch.empty((c["vocab"], c["d"]), device=dev)
    elif c["op"] == "adamw8":
        sizes = _sizes(c)
        at = np.concatenate([[0], np.cumsum([_up(n, BLOCK) for n, _ in sizes])]).tolist()   # every tensor starts a block of its own
        n = at[-1]
        s["w"] = 0.02 * torch.randn(n, generator=g, device=dev)
        # gradients of very different sizes within a block, some of them exactly zero
        grad = 1e-3 * torch.randn(n, generator=g, device=dev) * torch.exp(2.0 * torch.randn(n, generator=g, device=dev))
        grad[::37] = 0
        s["g"] = grad.to(torch.bfloat16) if c["bf16_grad"] else grad
        # moments as an earlier step left them
        m0 = 1e-3 * torch.randn(n, generator=g, device=dev)
        v0 = (2e-3 * torch.randn(n, generator=g, device=dev)).square() + 1e-9
        if c["step"] == 1:
            m0.zero_(); v0.zero_()
        qm, sm = _quantized(m0.view(1, n), E4M3)
        qv, sv = _quantized(v0.view(1, n), E5M2)
        s["m"], s["m_scale"], s["v"], s["v_scale"] = qm.view(n), sm.view(-1), qv.view(n), sv.view(-1)
        s["wc"] = torch.zeros(n, dtype=torch.bfloat16, device=dev)
        s["tensors"] = [(a, k, wd, 1 + i) for i, ((k, wd), a) in enumerate(zip(sizes, at))]
        # what is behind a tensor's last element is nobody's: zeros that stay
        for a, k, _, _ in s["tensors"]:
            e = a + _up(k, BLOCK)
            s["w"][a + k:e] = 0; s["m"][a + k:e].view(torch.uint8).zero_(); s["v"][a + k:e].view(torch.uint8).zero_()
        s["hp"] = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=c["step"])
    elif c["op"] == "quant":
        r, k, t = c["rows"], c["cols"], c["tile"]
        x = _matrix(r, k, g, dev)
        s["x"] = x if c["f32"] else x.to(torch.bfloat16)
        if c["straight"]:
            s["q"] = torch.empty((r, _up(k, 16)), dtype=torch.uint8, device=dev)
            s["s"] = torch.empty((-(-k // BLOCK), -(-r // t)), device=dev)
        if c["transposed"]:
            s["qt"] = torch.empty((k, _up(r, 16)), dtype=torch.uint8, device=dev)
            s["st"] = torch.empty((-(-r // BLOCK), -(-k // t)), device=dev)
    else:
        m, n, k = c["m"], c["n"], c["k"]
        a, sa = _quantized(_matrix(m, k, g, dev), c["fa"])
        w = 0.02 * torch.randn((n, k), generator=g, device=dev) if c["b_block"] == BLOCK else _matrix(n, k, g, dev)
        b, sb = (_quantized_square if c["b_block"] == BLOCK else _quantized)(w, c["fb"])
        s["a"], s["sa"], s["b"], s["sb"] = _pitched(a, _up(k, 16)), sa, _pitched(b, _up(k, 16)), sb
        s["bias"] = torch.randn(n, generator=g, device=dev).to(torch.bfloat16) if c["bias"] else None
        t = torch.float32 if c["f32"] else torch.bfloat16
        s["out"] = torch.randn((m, n), generator=g, device=dev).to(t) if c["acc"] else torch.empty((m, n), dtype=t, device=dev)
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _plain_emb_fwd(s):
    ids, vocab = s["ids"].long(), s["c"]["vocab"]
    ok = (ids >= 0) & (ids < vocab)
    rows = s["table"][ids.clamp(0, vocab - 1)].float() * s["scale"]
    return torch.where(ok.unsqueeze(1), rows, torch.zeros_like(rows)).to(s["table"].dtype)


def _plain_emb_bwd(s):
    ids, c = s["ids"].long(), s["c"]
    ok = (ids >= 0) & (ids < c["vocab"])
    dout = s["dout"].float()
    dout = torch.where(ok.unsqueeze(1), dout, torch.zeros_like(dout))
    total = torch.zeros((c["vocab"], c["d"]), device=s["dev"]).index_add_(0, ids.clamp(0, c["vocab"] - 1), dout) * s["scale"]
    s["dtable"] = s["dtable"] + total if c["acc"] else total
    return s["dtable"]


_LOW = 0xFFFFFFFF


def _mix(x):
    """32-bit multiply-xorshift mix of whole numbers held in 64 bits."""
    x = ((x ^ (x >> 16)) * 0x7FEB352D) & _LOW
    x = ((x ^ (x >> 15)) * 0x846CA68B) & _LOW
    return x ^ (x >> 16)


def _mix_one(x):
    return int(_mix(x & _LOW))


def _rounded(x, scale_field, bits, fmt):
    """Stochastic rounding of x / 2^(field - 127) to 8 bits; `bits`: 16 random ones. Elements that are not finite become NaN."""
    shift = (20, 21)[fmt]
    y = x.abs() * _pow2(254 - scale_field) * (2.0 ** -120, 2.0 ** -112)[fmt]
    code = (y.view(torch.int32).to(torch.int64) + (bits << (shift - 16)) + (1 << (shift - 17))) >> shift
    code = code.clamp(max=(0x7E, 0x7B)[fmt])
    if fmt == E5M2:
        code = torch.where((x > 0) & (code == 0), torch.ones_like(code), code)
    code = torch.where(torch.isfinite(x), code, torch.full_like(code, 0x7F))
    code = torch.where(x < 0, code | 0x80, code)
    return code.to(torch.uint8).view(TORCH8[fmt])


def _scale_of(x, fmt):
    fin = torch.isfinite(x)
    return _scale_field(torch.where(fin, x.abs(), torch.zeros_like(x)).amax(dim=1, keepdim=True), fmt)


def _plain_adamw8(s):
    hp = s["hp"]
    f32 = lambda x: torch.tensor(x, dtype=torch.float32, device=s["dev"])  # noqa: E731  (float32 constants, as the definition has them)
    lr, b1, b2, eps = (f32(hp[k]) for k in ("lr", "beta1", "beta2", "eps"))
    b1d, b2d = float(np.float32(hp["beta1"])), float(np.float32(hp["beta2"]))
    ib1, ib2 = f32(1.0 / (1.0 - b1d ** hp["step"])), f32(1.0 / (1.0 - b2d ** hp["step"]))
    one = f32(1.0)
    for a, n, wd, seed in s["tensors"]:
        nb, e = -(-n // BLOCK), a + _up(n, BLOCK)
        blk = slice(a // BLOCK, e // BLOCK)
        idx = torch.arange(nb * BLOCK, device=s["dev"])
        key = _mix_one(seed + hp["step"] * 0x9E3779B9)
        h = _mix((idx & _LOW) ^ ((key + (idx >> 32) * 0x85EBCA77) & _LOW)).view(nb, BLOCK)
        g = s["g"][a:e].float().view(nb, BLOCK)
        live = (idx < n).view(nb, BLOCK)
        g = torch.where(live, g, torch.zeros_like(g))
        w = s["w"][a:e].view(nb, BLOCK)
        m = s["m"][a:e].float().view(nb, BLOCK) * s["m_scale"][blk].unsqueeze(1)
        v = s["v"][a:e].float().view(nb, BLOCK) * s["v_scale"][blk].unsqueeze(1)
        m = b1 * m + (one - b1) * g
        v = b2 * v + (one - b2) * g * g
        w = w - lr * f32(wd) * w - lr * (m * ib1) / (torch.sqrt(v * ib2) + eps)
        fm, fv = _scale_of(m, E4M3), _scale_of(v, E5M2)
        w = torch.where(live, w, torch.zeros_like(w))
        s["w"][a:e] = w.view(-1)
        s["wc"][a:e] = w.view(-1).to(torch.bfloat16)
        s["m"][a:e] = _rounded(m, fm, h >> 16, E4M3).view(-1)
        s["v"][a:e] = _rounded(v, fv, h & 0xFFFF, E5M2).view(-1)
        s["m_scale"][blk], s["v_scale"][blk] = _pow2(fm).view(-1), _pow2(fv).view(-1)
    return {k: s[k] for k in ("w", "wc", "m", "v", "m_scale", "v_scale")}


def _plain_quant(s):
    c, x, out = s["c"], s["x"].float(), {}
    f = _quantized if c["tile"] == 1 else _quantized_square
    if c["straight"]:
        out["q"], out["s"] = f(x, c["fmt"])
    if c["transposed"]:
        out["qt"], out["st"] = f(x.t(), c["fmt"])
    return out


def _wide(q, fmt, k, scales, block, t):
    """The values that a matrix in 8 bits stands for."""
    x = q.view(TORCH8[fmt])[:, :k].to(t)
    full = scales.t().to(t)
    if block > 1:
        full = full.repeat_interleave(block, dim=0)[: x.shape[0]]
    return x * full.repeat_interleave(BLOCK, dim=1)[:, :k]


def _plain_gemm8(s):
    c = s["c"]
    a = _wide(s["a"], c["fa"], c["k"], s["sa"], 1, torch.float32)
    b = _wide(s["b"], c["fb"], c["k"], s["sb"], c["b_block"], torch.float32)
    out = a @ b.t()
    if c["bias"]:
        out = out + s["bias"].float()
    if c["acc"]:
        out = s["out"] + out
        s["out"] = out
    return out.to(s["out"].dtype)


# ---- the framework's calls ----------------------------------------------------------------------------------------

_session = None


def _own(s):
    global _session
    import ctypes
    from paper_2204_06514_b200 import binding as fx, binding_ops as ops
    from paper_2204_06514_b200.state import Session, hparams
    if _session is None:
        _session = Session(0)
    ctx, c = _session.ctx, s["c"]
    P = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else None  # noqa: E731
    prec = fx.FAX_PREC_FP32_VALIDATE if c.get("f32") else fx.FAX_PREC_BF16
    if s["op"] == "emb_fwd":
        ops.fax_op_embedding_forward(ctx, prec, c["n"], c["vocab"], c["d"], P(s["ids"]), P(s["table"]), s["scale"], P(s["out"]))
        return s["out"]
    if s["op"] == "emb_bwd":
        if "scratch" not in s:
            s["scratch"] = _session.arena(ops.fax_op_embedding_backward_scratch_bytes(c["n"], c["vocab"], c["d"]))
        ops.fax_op_embedding_backward(ctx, prec, c["n"], c["vocab"], c["d"], P(s["ids"]), P(s["dout"]), s["scale"], c["acc"], P(s["dtable"]), P(s["scratch"]),
                                      s["scratch"].numel())
        return s["dtable"]
    if s["op"] == "adamw8":
        if "plan" not in s:
            at = lambda t, i: ctypes.c_void_p(t.data_ptr() + i * t.element_size())  # noqa: E731
            plan = [fx.Adamw8Tensor(at(s["w"], a), at(s["m"], a), at(s["v"], a), at(s["m_scale"], a // BLOCK), at(s["v_scale"], a // BLOCK), at(s["g"], a), at(s["wc"], a),
                                         n, wd, seed) for a, n, wd, seed in s["tensors"]]
            s["plan"] = (fx.Adamw8Tensor * len(plan))(*plan)
        fx.fax_adamw8_step(ctx, s["plan"], hparams(grad_is_bf16=int(c["bf16_grad"]), **s["hp"]))
        return {k: s[k] for k in ("w", "wc", "m", "v", "m_scale", "v_scale")}
    if s["op"] == "quant":
        r, k, out = c["rows"], c["cols"], {}
        q, sc, qt, st = (s.get(x) for x in ("q", "s", "qt", "st"))
        ops.fax_op_fp8_quantize(ctx, prec, ops.Fp8QuantizeDesc(r, k, P(s["x"]), k, c["fmt"], c["tile"],
                                                               P(q), 0 if q is None else q.shape[1], P(sc), 0 if sc is None else sc.shape[1],
                                                               P(qt), 0 if qt is None else qt.shape[1], P(st), 0 if st is None else st.shape[1]))
        if q is not None:
            out["q"], out["s"] = q.view(TORCH8[c["fmt"]])[:, :k], sc
        if qt is not None:
            out["qt"], out["st"] = qt.view(TORCH8[c["fmt"]])[:, :r], st
        return out
    ops.fax_op_fp8_gemm(ctx, ops.Fp8GemmDesc(c["m"], c["n"], c["k"], P(s["a"]), s["a"].shape[1], c["fa"], P(s["sa"]), s["sa"].shape[1],
                                             P(s["b"]), s["b"].shape[1], c["fb"], P(s["sb"]), s["sb"].shape[1], c["b_block"],
                                             P(s["out"]), c["n"], int(c["f32"]), int(c["acc"]), P(s["bias"])))
    return s["out"]


def run(s):
    if own:
        return _own(s)
    return {"emb_fwd": _plain_emb_fwd, "emb_bwd": _plain_emb_bwd, "adamw8": _plain_adamw8, "quant": _plain_quant, "gemm8": _plain_gemm8}[s["op"]](s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_scale(amax, fmt):
    """The smallest power of two that brings amax to TOP at most, at least 2^-126; 1 where amax is 0."""
    f, e = torch.frexp(amax / TOP[fmt])                  # amax / TOP = f 2^e, f in [1/2, 1)
    e = torch.where(f == 0.5, e - 1, e).clamp(min=-126)
    return torch.where(amax == 0, torch.ones_like(amax), torch.ldexp(torch.ones_like(amax), e))


def _exact_step(y, fmt):
    """The distance between neighbouring values of the format at |y|."""
    _, e = torch.frexp(y.abs())
    low, digits = ((-6, 3), (-14, 2))[fmt]
    return torch.ldexp(torch.ones_like(y), (e - 1).clamp(min=low) - digits)


def _exact_quant(x, fmt, dims):
    """Nearest values (ties to even) and scales of blocks whose elements lie along `dims`."""
    sc = _exact_scale(x.abs().amax(dim=dims, keepdim=True), fmt)
    y = x / sc
    step = _exact_step(y, fmt)
    return torch.round(y / step) * step, sc


def _blocked(x, tile):
    r, k = x.shape
    rp = _up(r, tile)
    x = torch.nn.functional.pad(x, (0, _up(k, BLOCK) - k, 0, rp - r))
    return x.view(rp // tile, tile, -1, BLOCK)


def _exact_values(x, fmt, tile):
    r, k = x.shape
    q, sc = _exact_quant(_blocked(x, tile), fmt, (1, 3))
    return q.reshape(-1, q.shape[2] * BLOCK)[:r, :k], sc[:, 0, :, 0].t().contiguous()


def _exact_adamw8(s):
    """The definition rounds to float32 after every operation: here each is done in 64 bits and then rounded."""
    hp = s["hp"]
    R = lambda x: x.float().double()  # noqa: E731
    r = lambda x: float(np.float32(x))  # noqa: E731
    lr, b1, b2, eps = (r(hp[k]) for k in ("lr", "beta1", "beta2", "eps"))
    ib1, ib2 = r(1.0 / (1.0 - b1 ** hp["step"])), r(1.0 / (1.0 - b2 ** hp["step"]))
    out = {"w": s["w"].double(), "wc": torch.zeros_like(s["w"], dtype=torch.float64)}
    for name in ("m", "v", "m_scale", "v_scale"):
        out[name] = s[name].double()
    for a, n, wd, seed in s["tensors"]:
        i = torch.arange(n, device=s["dev"])
        x = (seed + hp["step"] * 0x9E3779B9) % 2 ** 32
        for shift, mult in ((16, 0x7FEB352D), (15, 0x846CA68B)):
            x = (x ^ (x >> shift)) * mult % 2 ** 32
        key = x ^ (x >> 16)
        h = (i % 2 ** 32) ^ ((key + (i // 2 ** 32) * 0x85EBCA77) % 2 ** 32)
        for shift, mult in ((16, 0x7FEB352D), (15, 0x846CA68B)):
            h = (((h ^ (h >> shift)) * (mult >> 16) % 2 ** 16 * 2 ** 16) + (h ^ (h >> shift)) * (mult & 0xFFFF)) % 2 ** 32
        h = h ^ (h >> 16)
        g, w = s["g"][a:a + n].double(), out["w"][a:a + n]
        block = i // BLOCK
        m = out["m"][a:a + n] * out["m_scale"][a // BLOCK + block]
        v = out["v"][a:a + n] * out["v_scale"][a // BLOCK + block]
        m = R(R(b1 * m) + R(r(1 - b1) * g))
        v = R(R(b2 * v) + R(R(r(1 - b2) * g) * g))
        upd = R(R(lr * R(m * ib1)) / R(R(torch.sqrt(R(v * ib2))) + eps))
        w = R(R(w - R(r(r(lr) * r(wd)) * w)) - upd)
        out["w"][a:a + n] = w
        out["wc"][a:a + n] = w.float().bfloat16().double()
        for name, t, fmt, u in (("m", m, E4M3, h // 2 ** 16), ("v", v, E5M2, h % 2 ** 16)):
            nb = -(-n // BLOCK)
            amax = torch.nn.functional.pad(t.abs(), (0, nb * BLOCK - n)).view(nb, BLOCK).amax(dim=1)
            sc = _exact_scale(amax, fmt)
            y = t.abs() / sc[block]
            fine = (2.0 ** -29, 2.0 ** -37)[fmt]                    # float32's last digit where the format's smallest values are
            y = torch.where(y < (2.0 ** -6, 2.0 ** -14)[fmt], torch.round(y / fine) * fine, y)
            step = _exact_step(y, fmt)
            q = torch.floor(y / step + (u.double() + 0.5) / 2 ** 16) * step
            q = q.clamp(max=TOP[fmt])
            if fmt == E5M2:
                q = torch.where((t > 0) & (q == 0), torch.full_like(q, 2.0 ** -16), q)
            out[name][a:a + n] = torch.where(t < 0, -q, q)
            out[name + "_scale"][a // BLOCK:a // BLOCK + nb] = sc
    return out


def exact(c, seed):
    s = prepare(c, seed)
    if c["op"] == "emb_fwd":
        ids = s["ids"].long()
        out = torch.zeros((c["n"], c["d"]), dtype=torch.float64, device=s["dev"])
        at = torch.nonzero(ids >= 0).view(-1)
        out[at] = s["table"].double()[ids[at]] * float(np.float32(s["scale"]))
        return out
    if c["op"] == "emb_bwd":
        ids = s["ids"].long()
        at = torch.nonzero(ids >= 0).view(-1)
        out = s["dtable"].double() if c["acc"] else torch.zeros((c["vocab"], c["d"]), dtype=torch.float64, device=s["dev"])
        out.index_add_(0, ids[at], s["dout"][at].double() * float(np.float32(s["scale"])))
        return out
    if c["op"] == "adamw8":
        return _exact_adamw8(s)
    if c["op"] == "quant":
        x, out = s["x"].double(), {}
        if c["straight"]:
            out["q"], out["s"] = _exact_values(x, c["fmt"], c["tile"])
        if c["transposed"]:
            out["qt"], out["st"] = _exact_values(x.t(), c["fmt"], c["tile"])
        return out
    a = _wide(s["a"], c["fa"], c["k"], s["sa"], 1, torch.float64)
    b = _wide(s["b"], c["fb"], c["k"], s["sb"], c["b_block"], torch.float64)
    out = torch.einsum("mk,nk->mn", a, b)
    if c["bias"]:
        out += s["bias"].double()
    if c["acc"]:
        out += s["out"].double()
    return out
