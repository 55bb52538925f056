"""Pieces of a decoder block beyond the dense one, as they are measured: positions by rotation, a gated recurrence in the
place of attention, a feed-forward layer of experts, and dropout on a branch's way back into the residual stream.

  rotary     heads turned by their token's position (and back, for the gradient), in place in a fused q | k | v or not
  dropout    y = resid + kept * x / (1 - p), the kept elements from a counter-based generator
  rec_fwd    h_t = a_t h_{t-1} + b_t with a = sigmoid(f), an output gate and ragged sequences
  rec_train  its forward and backward pass
  ex_out     tokens' choices sorted by expert, their rows laid out expert by expert
  ex_back    sorted, and the experts' rows summed with the router's weights into the residual stream
  ex_grad    sorted, and the gradients of both: of the experts' rows, of the weights and of the tokens' rows

`run` computes them in plain torch operations; where `own` is set, through paper_2204_06514_b200's entry points.
"""
import math

import numpy as np
import torch

own = False

HALVES, PAIRS = 0, 1             # which elements of a head turn together: i and i + rot / 2, or 2 i and 2 i + 1
PLAIN, COMPLEMENT = 0, 1         # what a recurrence adds: x, or (1 - a) x


def listed():
    return [
        # the next tokens of 64 sequences at far positions of their own: latency is all there is
        {"name": "rotary_64_tokens_12x2x64", "op": "rotary", "rows": 64, "heads": 24, "hd": 64, "rot": 64, "layout": HALVES, "extra": 12, "in_place": True, "back": False,
         "seq": 0, "first": 0, "far": 131072, "base": 10000.0, "factor": 1.0, "orig": 0, "amp": 1.0, "f32": False},
        # the 124M model's batch, q and k of the fused projection turned in place
        {"name": "rotary_16384x24x64_in_place", "op": "rotary", "rows": 16384, "heads": 24, "hd": 64, "rot": 64, "layout": HALVES, "extra": 12, "in_place": True, "back": False,
         "seq": 1024, "first": 0, "far": 0, "base": 10000.0, "factor": 1.0, "orig": 0, "amp": 1.0, "f32": False},
        # gradients of 40 heads of 128 turned back on a long context scaled by parts, half of the head, neighbours in pairs
        {"name": "rotary_back_8192x40x128_half_scaled", "op": "rotary", "rows": 8192, "heads": 40, "hd": 128, "rot": 64, "layout": PAIRS, "extra": 0, "in_place": False, "back": True,
         "seq": 8192, "first": 1000003, "far": 0, "base": 500000.0, "factor": 8.0, "orig": 8192, "amp": 1.2079, "f32": False},
        # a branch of the 124M model added to its residual stream
        {"name": "dropout_resid_16384x768", "op": "dropout", "rows": 16384, "cols": 768, "p": 0.1, "resid": True, "f32": False, "pad": 0},
        # the gradient of such a branch at hidden size 4096
        {"name": "dropout_8192x4096", "op": "dropout", "rows": 8192, "cols": 4096, "p": 0.25, "resid": False, "f32": False, "pad": 0},
        # one more token of 256 sequences through a gated recurrence that keeps its state
        {"name": "rec_fwd_256_tokens_1024", "op": "rec_fwd", "n_seq": 256, "seq": 1, "d": 1024, "ragged": 0.0, "input": COMPLEMENT, "gate": True, "fused": False, "f32": False},
        # one long sequence
        {"name": "rec_fwd_1x65536x768", "op": "rec_fwd", "n_seq": 1, "seq": 65536, "d": 768, "ragged": 0.0, "input": COMPLEMENT, "gate": False, "fused": True, "f32": False},
        # the 124M model's batch, trained
        {"name": "rec_train_16x1024x768", "op": "rec_train", "n_seq": 16, "seq": 1024, "d": 768, "ragged": 0.0, "input": COMPLEMENT, "gate": True, "fused": True, "f32": False},
        # 37 sequences of up to 511 tokens packed one after another, hidden size 2047
        {"name": "rec_train_ragged_37x511x2047", "op": "rec_train", "n_seq": 37, "seq": 511, "d": 2047, "ragged": 0.7, "input": PLAIN, "gate": True, "fused": False, "f32": False},
        # the 124M model's batch to two of eight experts of limited capacity
        {"name": "ex_out_16384x768_2of8", "op": "ex_out", "n": 16384, "d": 768, "k": 2, "e": 8, "cap": 5120, "align": 1, "pad": 0.0, "f32": False},
        # sixteen tokens' results from two of eight experts
        {"name": "ex_back_16x4096_2of8", "op": "ex_back", "n": 16, "d": 4096, "k": 2, "e": 8, "cap": 0, "align": 1, "pad": 0.0, "f32": False},
        # a ragged batch, six of sixty-four experts, as many rows as each one has, gradients
        {"name": "ex_grad_8191x2048_6of64", "op": "ex_grad", "n": 8191, "d": 2048, "k": 6, "e": 64, "cap": 0, "align": 128, "pad": 0.05, "f32": False},
    ]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))


def draw(rng):
    op = rng.choice(["rotary", "rotary", "dropout", "rec_fwd", "rec_train", "rec_train", "ex_out", "ex_back", "ex_grad"])
    f32 = rng.random() < 0.25
    if op == "rotary":
        hd = rng.choice([16, 32, 64, 64, 80, 96, 128, 128, 256, 2 * rng.randint(1, 100)])
        heads = _log(rng, 1, 64)
        rows = _log(rng, 1, min(30000, 40000000 // (hd * heads)))
        rot = hd if rng.random() < 0.5 else 2 * rng.randint(1, hd // 2)
        in_place = rng.random() < 0.5
        far = rng.choice([0, 0, 4096, 1000000])
        factor = rng.choice([1.0, 1.0, 4.0, 8.0])
        return {"op": op, "rows": rows, "heads": heads, "hd": hd, "rot": rot, "layout": rng.choice([HALVES, PAIRS]), "extra": rng.choice([0, heads, heads // 2]), "in_place": in_place,
                "back": rng.random() < 0.4, "seq": _log(rng, 1, 4096) if far == 0 else 0, "first": rng.choice([0, 0, 17, 900001]) if far == 0 else 0, "far": far,
                "base": rng.choice([10000.0, 500000.0, 1e6]), "factor": factor, "orig": rng.choice([0, 4096]) if factor > 1 else 0, "amp": 1.0 if in_place else rng.choice([1.0, 1.1386]), "f32": f32}
    if op == "dropout":
        cols = _log(rng, 1, 5000)
        if rng.random() < 0.5:
            cols = (cols + 63) // 64 * 64
        return {"op": op, "rows": _log(rng, 1, 30000000 // cols), "cols": cols, "p": rng.choice([0.0, 0.05, 0.1, 0.1, 0.3, 0.5]), "resid": rng.random() < 0.6, "f32": f32,
                "pad": rng.choice([0, 0, 8, 3])}
    if op in ("rec_fwd", "rec_train"):
        d = _log(rng, 8, 4096)
        if rng.random() < 0.6:
            d = (d + 31) // 32 * 32
        room = 14000000 // d
        n_seq = _log(rng, 1, min(512, room))
        return {"op": op, "n_seq": n_seq, "seq": _log(rng, 1, min(32768, room // n_seq)), "d": d, "ragged": rng.choice([0.0, 0.0, 0.5, 1.0]), "input": rng.choice([PLAIN, COMPLEMENT, COMPLEMENT]),
                "gate": rng.random() < 0.6, "fused": rng.random() < 0.5, "f32": f32}
    d = _log(rng, 8, 4096)
    if rng.random() < 0.7:
        d = (d + 63) // 64 * 64
    e = _log(rng, 2, 256)
    k = min(e, rng.choice([1, 2, 2, 4, 6, 8]))
    n = _log(rng, 1, min(60000, 50000000 // (d * k)))
    return {"op": op, "n": n, "d": d, "k": k, "e": e, "cap": rng.choice([0, -(-n * k // e), -(-5 * n * k // (4 * e))]), "align": rng.choice([1, 16, 128]) if n * k > 64 * e else 1,
            "pad": rng.choice([0.0, 0.0, 0.1]), "f32": f32}


def _slots(c):
    """Rows that hold every expert's tokens, whatever the router chose."""
    if c["cap"]:
        return c["e"] * c["cap"]
    n = c["n"] * c["k"]
    return n + min(c["e"], n) * (c["align"] - 1)


def work(c):
    es = 4 if c["f32"] else 2
    if c["op"] == "rotary":
        moved = c["rot"] if c["in_place"] else c["hd"]
        return {"bytes": 2.0 * c["rows"] * c["heads"] * moved * es + 4.0 * c["rows"] * (c["far"] > 0), "flops": 3.0 * c["rows"] * c["heads"] * c["rot"]}
    if c["op"] == "dropout":
        return {"bytes": (3.0 if c["resid"] else 2.0) * c["rows"] * c["cols"] * es, "flops": 2.0 * c["rows"] * c["cols"]}
    if c["op"] in ("rec_fwd", "rec_train"):
        # half of the ragged lengths' spread is missing on average
        n = c["n_seq"] * c["d"] * max(1.0, c["seq"] * (1 - c["ragged"] / 2))
        states = 8.0 * c["n_seq"] * c["d"]
        forward = (3.0 + c["gate"]) * n * es + states
        if c["op"] == "rec_fwd":
            return {"bytes": forward, "flops": 4.0 * n}
        return {"bytes": forward + (5.0 + 2 * c["gate"]) * n * es + states, "flops": 14.0 * n}
    live = c["n"] * (1 - c["pad"])
    kept = min(live * c["k"], _slots(c))
    plan = 4.0 * (2 * c["n"] * c["k"] + _slots(c) + 2 * c["e"])
    row = c["d"] * es
    if c["op"] == "ex_out":
        return {"bytes": plan + (live + _slots(c)) * row, "flops": 0.0}
    if c["op"] == "ex_back":
        return {"bytes": plan + 4.0 * live * c["k"] + (kept + 2 * c["n"]) * row, "flops": 2.0 * kept * c["d"]}
    return {"bytes": plan + 8.0 * c["n"] * c["k"] + (2 * kept + _slots(c) + 3 * c["n"]) * row, "flops": 4.0 * kept * c["d"]}


# ---- inputs -------------------------------------------------------------------------------------------------------

def _frequencies(c):
    """Radians a position of each turning pair, for contexts scaled by `factor`: all slowed down alike, or (with an
    original length) only the pairs that make few turns in that length, those of 1 to 32 turns in part."""
    i = np.arange(c["rot"] // 2, dtype=np.float64)
    f = c["base"] ** (-2.0 * i / c["rot"])
    if c["factor"] == 1.0:
        return f
    if not c["orig"]:
        return f / c["factor"]
    keep = np.clip((c["orig"] * f / (2 * math.pi) - 1.0) / (32.0 - 1.0), 0.0, 1.0)
    return f * (keep + (1 - keep) / c["factor"])


def _lengths(c, g):
    """Lengths of the sequences, some of them 0 and 1 where they are ragged."""
    if not c["ragged"]:
        return [c["seq"]] * c["n_seq"]
    u = torch.rand(c["n_seq"], generator=g).tolist()
    n = [max(0, int(round(c["seq"] * (1 - c["ragged"] * x)))) for x in u]
    if c["n_seq"] > 1:
        n[u.index(max(u))] = u.index(max(u)) % 2
        n[u.index(min(u))] = c["seq"]
    return n


def prepare(c, seed):
    dev = torch.device("cuda", 0)
    g = torch.Generator(device=dev)
    g.manual_seed(int(seed) * 1009 + 29)
    host = torch.Generator()
    host.manual_seed(int(seed) * 1013 + 31)
    t = torch.float32 if c["f32"] else torch.bfloat16
    normal = lambda *shape: torch.randn(shape, generator=g, device=dev)  # noqa: E731
    s = {"c": c, "dev": dev, "t": t}
    if c["op"] == "rotary":
        s["x"] = normal(c["rows"], (c["heads"] + c["extra"]) * c["hd"]).to(t)
        s["out"] = s["x"] if c["in_place"] else torch.empty((c["rows"], c["heads"] * c["hd"]), dtype=t, device=dev)
        s["pos"] = torch.randint(0, c["far"], (c["rows"],), generator=g, device=dev, dtype=torch.int32) if c["far"] else None
        s["freq"] = torch.as_tensor(_frequencies(c), device=dev)
    elif c["op"] == "dropout":
        pitch = c["cols"] + c["pad"]
        s["x"] = normal(c["rows"], pitch).to(t)
        s["resid"] = normal(c["rows"], pitch).to(t) if c["resid"] else None
        s["out"] = torch.empty((c["rows"], c["cols"]), dtype=t, device=dev)
        s["seed"], s["offset"] = int(seed) * 0x9E3779B97F4A7C15 % 2 ** 64, 7919 * int(seed) + 2 ** 33
    elif c["op"] in ("rec_fwd", "rec_train"):
        n = _lengths(c, host)
        at = np.concatenate([[0], np.cumsum(n)]).astype(np.int64)
        rows, d = c["n_seq"] * c["seq"], c["d"]
        s["at"], s["longest"] = at, max(n)
        s["offsets"] = torch.as_tensor(at.astype(np.int32), device=dev) if c["ragged"] else None
        # where each sequence's first and last row is, of those that have any
        some = [i for i in range(c["n_seq"]) if n[i]]
        s["some"] = torch.as_tensor(some, dtype=torch.int64, device=dev)
        s["begin"], s["end"] = [torch.as_tensor([int(at[i + k]) - k for i in some], dtype=torch.int64, device=dev) for k in (0, 1)]
        parts = 2 + c["gate"]
        if c["fused"]:
            s["proj"] = normal(rows, parts * d).to(t)
            s["dproj"] = torch.zeros_like(s["proj"])
            cut = lambda x: [x[:, i * d:(i + 1) * d] for i in range(parts)]  # noqa: E731
            fxg, dfxg = cut(s["proj"]), cut(s["dproj"])
        else:
            fxg = [normal(rows, d).to(t) for _ in range(parts)]
            dfxg = [torch.zeros((rows, d), dtype=t, device=dev) for _ in range(parts)]
        # channels that forget at once and channels that remember hundreds of tokens
        fxg[0] += (7.0 * torch.rand(d, generator=g, device=dev) - 1.0).to(t)
        s["f"], s["xin"], s["g"] = fxg if c["gate"] else fxg + [None]
        s["df"], s["dx"], s["dg"] = dfxg if c["gate"] else dfxg + [None]
        s["h0"], s["y"], s["h_last"] = normal(c["n_seq"], d), torch.zeros((rows, d), dtype=t, device=dev), torch.empty((c["n_seq"], d), device=dev)
        if c["op"] == "rec_train":
            s["dy"], s["dh_last"], s["dh0"] = normal(rows, d).to(t), normal(c["n_seq"], d), torch.empty((c["n_seq"], d), device=dev)
    else:
        n, k, e, d = c["n"], c["k"], c["e"], c["d"]
        # experts of unequal popularity, a token's choices all different; a share of the tokens is padding
        logits = -0.5 * torch.log(torch.randperm(e, generator=g, device=dev).float() + 3.0) - torch.log(-torch.log(torch.rand((n, e), generator=g, device=dev).clamp(1e-30, 1 - 1e-7)))
        best, ids = logits.topk(k, dim=1)
        live = torch.rand((n, 1), generator=g, device=dev) >= c["pad"]
        s["ids"] = torch.where(live, ids, torch.full_like(ids, -1)).to(torch.int32)
        s["w"] = torch.softmax(best, dim=1)
        slots = _slots(c)
        new = lambda *shape: torch.empty(shape, dtype=torch.int32, device=dev)  # noqa: E731
        s["slot_of"], s["source"], s["offsets"], s["counts"] = new(n, k), new(slots), new(e + 1), new(e)
        if c["op"] == "ex_out":
            s["x"], s["out"] = normal(n, d).to(t), torch.empty((slots, d), dtype=t, device=dev)
        elif c["op"] == "ex_back":
            s["z"], s["resid"], s["out"] = normal(slots, d).to(t), normal(n, d).to(t), torch.empty((n, d), dtype=t, device=dev)
        else:
            s["z"], s["dy"], s["drows"], s["dresid"] = normal(slots, d).to(t), normal(n, d).to(t), normal(slots, d).to(t), normal(n, d).to(t)
            s["dz"], s["dw"], s["dx"] = torch.empty((slots, d), dtype=t, device=dev), torch.empty((n, k), device=dev), torch.empty((n, d), dtype=t, device=dev)
    return s


# ---- plain forms --------------------------------------------------------------------------------------------------

def _positions(s):
    c = s["c"]
    if s["pos"] is not None:
        return s["pos"].long()
    return c["first"] + torch.arange(c["rows"], device=s["dev"]) % c["seq"]


def _plain_rotary(s):
    c = s["c"]
    angle = _positions(s).double().unsqueeze(1) * s["freq"]
    cos, sin = (c["amp"] * torch.cos(angle)).float().unsqueeze(1), (c["amp"] * torch.sin(angle)).float().unsqueeze(1)
    if c["back"]:
        sin = -sin
    x = s["x"][:, :c["heads"] * c["hd"]].view(c["rows"], c["heads"], c["hd"]).float()
    h = c["rot"] // 2
    a, b = (slice(0, h), slice(h, c["rot"])) if c["layout"] == HALVES else (slice(0, c["rot"], 2), slice(1, c["rot"], 2))
    y = x.clone()
    y[..., a] = x[..., a] * cos - x[..., b] * sin
    y[..., b] = x[..., b] * cos + x[..., a] * sin
    s["out"][:, :c["heads"] * c["hd"]] = y.view(c["rows"], -1).to(s["t"])
    return s["out"]


_LOW = 0xFFFFFFFF


def _product(a, m):
    """High and low half of a * m, a of 32 bits held in 64."""
    high = (a * (m >> 16) + (a * (m & 0xFFFF) >> 16)) >> 16
    return high, (a * m) & _LOW


def _draws(c, seed, offset, dev):
    """16 random bits for each element [rows, cols]: Philox4x32-10 (Salmon et al. 2011) of counter (col / 8, row, offset)
    under key `seed`; the words' low halves are the even columns'."""
    groups = -(-c["cols"] // 8)
    x = [torch.arange(groups, device=dev).expand(c["rows"], groups), torch.arange(c["rows"], device=dev).unsqueeze(1).expand(c["rows"], groups),
         torch.tensor(offset & _LOW, device=dev), torch.tensor(offset >> 32, device=dev)]
    k0, k1 = seed & _LOW, seed >> 32
    for _ in range(10):
        h0, l0 = _product(x[0], 0xD2511F53)
        h1, l1 = _product(x[2], 0xCD9E8D57)
        x = [h1 ^ x[1] ^ k0, l1, h0 ^ x[3] ^ k1, l0]
        k0, k1 = (k0 + 0x9E3779B9) & _LOW, (k1 + 0xBB67AE85) & _LOW
    words = torch.stack([w.expand(c["rows"], groups) for w in x], dim=2)
    return torch.stack([words & 0xFFFF, words >> 16], dim=3).view(c["rows"], groups * 8)[:, :c["cols"]]


def _plain_dropout(s):
    c = s["c"]
    limit = int(round(c["p"] * 65536))
    kept = _draws(c, s["seed"], s["offset"], s["dev"]) >= limit
    x = s["x"][:, :c["cols"]].float()
    y = torch.where(kept, x * (65536.0 / (65536 - limit)), torch.zeros_like(x))
    if c["resid"]:
        y = s["resid"][:, :c["cols"]].float() + y
    return y.to(s["t"])


def _scan(a, b, longest):
    """h_i = a_i h_{i-1} + b_i along the rows in both directions' common form: spans double until they cover a sequence."""
    span = 1
    while span < longest:
        b = torch.cat([b[:span], b[span:] + a[span:] * b[:-span]])
        a = torch.cat([a[:span], a[span:] * a[:-span]])
        span *= 2
    return b


def _plain_rec(s):
    c, live = s["c"], int(s["at"][-1])
    f, x = s["f"][:live].float(), s["xin"][:live].float()
    a, ca = torch.sigmoid(f), torch.sigmoid(-f)
    b = x * ca if c["input"] == COMPLEMENT else x
    first = s["h0"][s["some"]]
    left = a.clone()
    left[s["begin"]] = 0.0
    start = b.clone()
    start[s["begin"]] += a[s["begin"]] * first
    h = _scan(left, start, s["longest"])
    out = h
    if c["gate"]:
        g = s["g"][:live].float()
        sg = torch.sigmoid(g)
        out = h * g * sg
    s["y"][:live] = out.to(s["t"])
    s["h_last"].copy_(s["h0"])
    s["h_last"][s["some"]] = h[s["end"]]
    if c["op"] == "rec_fwd":
        return {"y": s["y"], "h_last": s["h_last"]}
    dy = s["dy"][:live].float()
    u = dy * g * sg if c["gate"] else dy.clone()
    u[s["end"]] += s["dh_last"][s["some"]]
    right = torch.cat([a[1:], torch.zeros_like(a[:1])])
    right[s["end"]] = 0.0
    dh = _scan(right.flip(0), u.flip(0), s["longest"]).flip(0)
    before = torch.cat([torch.zeros_like(h[:1]), h[:-1]])
    before[s["begin"]] = first
    if c["input"] == COMPLEMENT:
        s["df"][:live] = (dh * (before - x) * a * ca).to(s["t"])
        s["dx"][:live] = (dh * ca).to(s["t"])
    else:
        s["df"][:live] = (dh * before * a * ca).to(s["t"])
        s["dx"][:live] = dh.to(s["t"])
    if c["gate"]:
        s["dg"][:live] = (dy * h * sg * (1 + g * (1 - sg))).to(s["t"])
    s["dh0"].copy_(s["dh_last"])
    s["dh0"][s["some"]] = (a * dh)[s["begin"]]
    return _rec_outputs(s)


def _rec_outputs(s):
    out = {k: s[k] for k in ("y", "h_last", "dh0")}
    if s["c"]["fused"]:
        out["dproj"] = s["dproj"]
    else:
        out.update({k: s[k] for k in ("df", "dx", "dg") if s[k] is not None})
    return out


def _plain_sort(s):
    c, e = s["c"], s["ids"].view(-1).long()
    total = e.numel()
    key = torch.where((e >= 0) & (e < c["e"]), e, torch.full_like(e, c["e"]))
    order = torch.argsort(key, stable=True)
    counts = torch.zeros(c["e"] + 1, dtype=torch.int64, device=s["dev"]).index_add_(0, key, torch.ones_like(key))[:c["e"]]
    seen = torch.cumsum(counts, 0) - counts
    sorted_key = key[order]
    live = sorted_key < c["e"]
    order, sorted_key = order[live], sorted_key[live]
    rank = torch.arange(order.numel(), device=s["dev"]) - seen[sorted_key]
    if c["cap"]:
        offsets = torch.arange(c["e"] + 1, device=s["dev"]) * c["cap"]
        kept = rank < c["cap"]
        order, sorted_key, rank = order[kept], sorted_key[kept], rank[kept]
    else:
        room = (counts + c["align"] - 1) // c["align"] * c["align"]
        offsets = torch.cat([torch.zeros_like(room[:1]), torch.cumsum(room, 0)])
    slot = offsets[sorted_key] + rank
    slot_of = torch.full((total,), -1, dtype=torch.int64, device=s["dev"])
    slot_of[order] = slot
    source = torch.full((_slots(c),), -1, dtype=torch.int64, device=s["dev"])
    source[slot] = order
    return {"slot_of": slot_of.view(c["n"], c["k"]).int(), "source": source.int(), "offsets": offsets.int(), "counts": counts.int()}


def _plain_experts(s):
    c, out = s["c"], _plain_sort(s)
    slot_of, source = out["slot_of"].long(), out["source"].long()
    has = (source >= 0).unsqueeze(1)
    token = source.clamp(min=0) // c["k"]
    if c["op"] == "ex_out":
        out["rows"] = torch.where(has, s["x"][token], torch.zeros((), dtype=s["t"], device=s["dev"]))
        return out
    kept = slot_of >= 0
    if c["op"] == "ex_back":
        total = torch.zeros((c["n"], c["d"]), device=s["dev"])
        for j in range(c["k"]):
            total += torch.where(kept[:, j:j + 1], s["w"][:, j:j + 1] * s["z"][slot_of[:, j].clamp(min=0)].float(), torch.zeros_like(total))
        out["y"] = (s["resid"].float() + total).to(s["t"])
        return out
    w = s["w"].view(-1)[source.clamp(min=0)].unsqueeze(1)
    dz = w * s["dy"][token].float()
    out["dz"] = torch.where(has, dz, torch.zeros_like(dz)).to(s["t"])
    dw, dx = torch.zeros((c["n"], c["k"]), device=s["dev"]), torch.zeros((c["n"], c["d"]), device=s["dev"])
    for j in range(c["k"]):
        at = slot_of[:, j].clamp(min=0)
        dw[:, j] = torch.where(kept[:, j], (s["z"][at].float() * s["dy"].float()).sum(1), torch.zeros_like(dw[:, j]))
        dx += torch.where(kept[:, j:j + 1], s["drows"][at].float(), torch.zeros_like(dx))
    out["dw"], out["dx"] = dw, (s["dresid"].float() + dx).to(s["t"])
    return out


# ---- the framework's calls ----------------------------------------------------------------------------------------

_session = None


def _own(s):
    global _session
    import ctypes
    from paper_2204_06514_b200 import binding as fx, binding_ops as ops
    from paper_2204_06514_b200.state import Session, rotary_frequencies
    if _session is None:
        _session = Session(0)
    ctx, c = _session.ctx, s["c"]
    P = lambda t: ctypes.c_void_p(t.data_ptr()) if t is not None else None  # noqa: E731
    pitch = lambda t: t.stride(0) if t is not None else 0  # noqa: E731
    prec = fx.FAX_PREC_FP32_VALIDATE if c["f32"] else fx.FAX_PREC_BF16
    if c["op"] == "rotary":
        if "table" not in s:      # the model's table of frequencies, made once
            s["table"] = rotary_frequencies(s["dev"], c["rot"], base=c["base"], factor=c["factor"], original_seq=c["orig"])
        ops.fax_op_rotary(ctx, prec, ops.RotaryDesc(c["rows"], c["heads"], c["hd"], c["rot"], c["layout"], P(s["x"]), pitch(s["x"]), P(s["out"]), pitch(s["out"]),
                                                    P(s["pos"]), c["first"], c["seq"], P(s["table"]), c["amp"], int(c["back"])))
        return s["out"]
    if c["op"] == "dropout":
        ops.fax_op_dropout(ctx, prec, ops.DropoutDesc(c["rows"], c["cols"], P(s["x"]), pitch(s["x"]), P(s["resid"]), pitch(s["resid"]), P(s["out"]), pitch(s["out"]),
                                                      c["p"], s["seed"], s["offset"], None))
        return s["out"]
    if c["op"] in ("rec_fwd", "rec_train"):
        train = c["op"] == "rec_train"
        rows = c["n_seq"] * c["seq"]
        if train and "states" not in s:      # saved activations of the layer
            s["states"] = torch.empty(ops.fax_op_recurrence_states_floats(rows, c["n_seq"], c["d"]), device=s["dev"])
        shape = (rows, c["d"], c["n_seq"], c["seq"], P(s["offsets"]), c["input"], P(s["f"]), pitch(s["f"]), P(s["xin"]), pitch(s["xin"]), P(s["g"]), pitch(s["g"]), P(s["h0"]))
        ops.fax_op_recurrence_forward(ctx, prec, ops.RecurrenceDesc(*shape, P(s["y"]), pitch(s["y"]), P(s["h_last"]), P(s["states"]) if train else None))
        if not train:
            return {"y": s["y"], "h_last": s["h_last"]}
        ops.fax_op_recurrence_backward(ctx, prec, ops.RecurrenceBackwardDesc(*shape, P(s["states"]), P(s["dy"]), pitch(s["dy"]), P(s["dh_last"]), P(s["df"]), pitch(s["df"]),
                                                                             P(s["dx"]), pitch(s["dx"]), P(s["dg"]), pitch(s["dg"]), P(s["dh0"])))
        return _rec_outputs(s)
    n, k, d, slots = c["n"], c["k"], c["d"], _slots(c)
    ops.fax_op_expert_sort(ctx, ops.ExpertSortDesc(n, k, c["e"], c["cap"], c["align"], slots, P(s["ids"]), P(s["slot_of"]), P(s["source"]), P(s["offsets"]), P(s["counts"])))
    out = {x: s[x] for x in ("slot_of", "source", "offsets", "counts")}
    plan = (n, k, d, slots, P(s["slot_of"]), P(s["source"]))
    if c["op"] == "ex_out":
        ops.fax_op_expert_dispatch(ctx, prec, ops.ExpertDispatchDesc(*plan, P(s["x"]), d, P(s["out"]), d))
        out["rows"] = s["out"]
    elif c["op"] == "ex_back":
        ops.fax_op_expert_combine(ctx, prec, ops.ExpertCombineDesc(*plan[:5], P(s["w"]), P(s["z"]), d, P(s["resid"]), d, P(s["out"]), d))
        out["y"] = s["out"]
    else:
        ops.fax_op_expert_combine_backward(ctx, prec, ops.ExpertCombineBackwardDesc(*plan, P(s["w"]), P(s["z"]), d, P(s["dy"]), d, P(s["dz"]), d, P(s["dw"])))
        ops.fax_op_expert_combine(ctx, prec, ops.ExpertCombineDesc(*plan[:5], None, P(s["drows"]), d, P(s["dresid"]), d, P(s["dx"]), d))
        out.update({x: s[x] for x in ("dz", "dw", "dx")})
    return out


def run(s):
    if own:
        return _own(s)
    return {"rotary": _plain_rotary, "dropout": _plain_dropout, "rec_fwd": _plain_rec, "rec_train": _plain_rec}.get(s["c"]["op"], _plain_experts)(s)


# ---- the definitions in 64 bits -----------------------------------------------------------------------------------

def _exact_rotary(s):
    """Pairs as complex numbers, turned by multiplication."""
    c = s["c"]
    x = s["x"][:, :c["heads"] * c["hd"]].double().view(c["rows"], c["heads"], c["hd"])
    head = x[..., :c["rot"]]
    pairs = head.unflatten(2, (2, -1)).transpose(2, 3) if c["layout"] == HALVES else head.unflatten(2, (-1, 2))
    angle = torch.outer(_positions(s).double(), s["freq"])
    turn = torch.polar(torch.full_like(angle, float(np.float32(c["amp"]))), -angle if c["back"] else angle).unsqueeze(1)
    turned = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
    turned = turned.transpose(2, 3) if c["layout"] == HALVES else turned
    y = torch.cat([turned.reshape(c["rows"], c["heads"], c["rot"]), x[..., c["rot"]:]], dim=2).view(c["rows"], -1)
    out = s["x"].double() if c["in_place"] else torch.empty((c["rows"], c["heads"] * c["hd"]), dtype=torch.float64, device=s["dev"])
    out[:, :c["heads"] * c["hd"]] = y
    return out


def _philox(counter, key):
    """The generator in numpy's 64-bit whole numbers."""
    c, (k0, k1) = [np.asarray(x, dtype=np.uint64) for x in counter], key
    low, up = np.uint64(0xFFFFFFFF), np.uint64(32)
    for r in range(10):
        p0, p1 = c[0] * np.uint64(0xD2511F53), c[2] * np.uint64(0xCD9E8D57)
        a, b = np.uint64((k0 + r * 0x9E3779B9) % 2 ** 32), np.uint64((k1 + r * 0xBB67AE85) % 2 ** 32)
        c = [(p1 >> up) ^ c[1] ^ a, p1 & low, (p0 >> up) ^ c[3] ^ b, p0 & low]
    return c


def _exact_dropout(s):
    c, groups = s["c"], -(-s["c"]["cols"] // 8)
    row, group = np.meshgrid(np.arange(c["rows"]), np.arange(groups), indexing="ij")
    o = s["offset"]
    words = _philox((group, row, np.full_like(row, o % 2 ** 32), np.full_like(row, o // 2 ** 32)), (s["seed"] % 2 ** 32, s["seed"] // 2 ** 32))
    bits = np.zeros((c["rows"], groups * 8), dtype=np.int32)
    for j in range(8):
        bits[:, j::8] = words[j // 2] // np.uint64(2 ** (16 * (j % 2))) % np.uint64(2 ** 16)
    limit = round(c["p"] * 65536)
    kept = torch.as_tensor(bits[:, :c["cols"]], device=s["dev"]) >= limit
    y = torch.where(kept, s["x"][:, :c["cols"]].double() / (1 - limit / 65536), 0.0)
    return y + s["resid"][:, :c["cols"]].double() if c["resid"] else y


def _exact_rec(s):
    """Step by step over all sequences at once, the longest ones first."""
    c, at = s["c"], s["at"]
    n = np.diff(at)
    by = np.argsort(-n, kind="stable")
    first = torch.as_tensor(at[:-1][by].copy(), device=s["dev"])
    alive = [int(np.sum(n > t)) for t in range(s["longest"])]
    by = torch.as_tensor(by.copy(), device=s["dev"])
    f, x = s["f"].double(), s["xin"].double()
    a, rest = 1 / (1 + torch.exp(-f)), 1 / (1 + torch.exp(f))
    b = x * rest if c["input"] == COMPLEMENT else x
    gate = slope = None
    if c["gate"]:
        g = s["g"].double()
        sg = 1 / (1 + torch.exp(-g))
        gate, slope = g * sg, sg + g * sg * (1 - sg)
    h, before, hs = s["h0"].double()[by], torch.zeros_like(a), torch.zeros_like(a)
    for t, m in enumerate(alive):
        r = first[:m] + t
        before[r] = h[:m]
        h[:m] = a[r] * h[:m] + b[r]
        hs[r] = h[:m]
    h_last = torch.empty_like(h)
    h_last[by] = h
    live = int(at[-1])
    y = s["y"].double()
    y[:live] = (hs * gate if c["gate"] else hs)[:live]
    if c["op"] == "rec_fwd":
        return {"y": y, "h_last": h_last}
    dy, carry, dh = s["dy"].double(), s["dh_last"].double()[by], torch.zeros_like(a)
    for t in range(s["longest"] - 1, -1, -1):
        r = first[:alive[t]] + t
        now = carry[:alive[t]] + (dy[r] * gate[r] if c["gate"] else dy[r])
        dh[r] = now
        carry[:alive[t]] = a[r] * now
    dh0 = torch.empty_like(carry)
    dh0[by] = carry
    grads = {"df": dh * a * rest * (before - x if c["input"] == COMPLEMENT else before), "dx": dh * rest if c["input"] == COMPLEMENT else dh}
    if c["gate"]:
        grads["dg"] = dy * hs * slope
    out = {"y": y, "h_last": h_last, "dh0": dh0}
    for v in grads.values():
        v[live:] = 0
    if c["fused"]:
        out["dproj"] = torch.cat(list(grads.values()), dim=1)
    else:
        out.update(grads)
    return out


def _exact_experts(s):
    """Token by token on the host for the places, expert by expert for the sums."""
    c = s["c"]
    ids = s["ids"].cpu().numpy().reshape(-1)
    lists = [np.nonzero(ids == e)[0] for e in range(c["e"])]
    counts = np.array([len(x) for x in lists])
    room = np.full(c["e"], c["cap"]) if c["cap"] else -(-counts // c["align"]) * c["align"]
    offsets = np.concatenate([[0], np.cumsum(room)])
    slot_of, source = np.full(len(ids), -1), np.full(_slots(c), -1)
    for e, x in enumerate(lists):
        x = x[:c["cap"]] if c["cap"] else x
        slot_of[x] = offsets[e] + np.arange(len(x))
        source[offsets[e]:offsets[e] + len(x)] = x
    whole = lambda v: torch.as_tensor(v.astype(np.int32), device=s["dev"])  # noqa: E731
    out = {"slot_of": whole(slot_of.reshape(c["n"], c["k"])), "source": whole(source), "offsets": whole(offsets), "counts": whole(counts)}
    at = torch.as_tensor(np.nonzero(source >= 0)[0], device=s["dev"])
    choice = torch.as_tensor(source[source >= 0], device=s["dev"])
    token = choice // c["k"]
    w = s["w"].double().view(-1)
    wide = lambda rows: torch.zeros((rows, c["d"]), dtype=torch.float64, device=s["dev"])  # noqa: E731
    if c["op"] == "ex_out":
        out["rows"] = wide(_slots(c))
        out["rows"][at] = s["x"].double()[token]
    elif c["op"] == "ex_back":
        out["y"] = s["resid"].double().index_add_(0, token, w[choice].unsqueeze(1) * s["z"].double()[at])
    else:
        out["dz"] = wide(_slots(c))
        dy = s["dy"].double()[token]
        out["dz"][at] = w[choice].unsqueeze(1) * dy
        dw = torch.zeros_like(w)
        dw[choice] = torch.einsum("ij,ij->i", s["z"].double()[at], dy)
        out["dw"] = dw.view(c["n"], c["k"])
        out["dx"] = s["dresid"].double().index_add_(0, token, s["drows"].double()[at])
    return out


def exact(c, seed):
    s = prepare(c, seed)
    return {"rotary": _exact_rotary, "dropout": _exact_dropout, "rec_fwd": _exact_rec, "rec_train": _exact_rec}.get(c["op"], _exact_experts)(s)
