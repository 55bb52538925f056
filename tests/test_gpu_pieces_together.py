"""A block made of the pieces, forward and backward through the C ABI, against a float64 autograd model: attention with
rotary positions, a gated recurrence, a feed-forward of experts, dropout on two branches."""
import numpy as np
import pytest
import torch

import pieces_ref as ref
from parity_util import Session, TOL_FP32, TOL_FWD_BF16, TOL_GRAD_BF16, fx, ptr
from paper_2204_06514_b200 import binding_ops as ops
from paper_2204_06514_b200.state import rotary_frequencies

pytestmark = pytest.mark.gpu

B, T, H, HD, E, K, F = 2, 256, 4, 64, 4, 2, 256
D, N = H * HD, B * T
CAP = 256                     # of 256 on average: some choices of the popular experts are dropped
P_DROP, SEED = 0.2, 77
WEIGHTS = {"qkv": (D, 3 * D), "o": (D, D), "proj": (D, 3 * D), "o2": (D, D), **{f"e{e}a": (D, F) for e in range(E)}, **{f"e{e}b": (F, D) for e in range(E)}}


def inputs(prec):
    rng = np.random.default_rng(21)
    r = lambda *s, scale=1.0: ref.rounded(scale * rng.standard_normal(s), prec)  # noqa: E731
    v = {"x": r(N, D), "dy": r(N, D)}
    for k, s in WEIGHTS.items():
        v[k] = r(*s, scale=s[0] ** -0.5)
        v[k + "_bias"] = r(s[1], scale=0.1)
    v["proj_bias"][:D] += ref.rounded(rng.uniform(0, 4, D), prec)      # gates that remember
    v["proj_bias"] = ref.rounded(v["proj_bias"], prec)
    for i in range(3):
        v[f"ln{i}_g"], v[f"ln{i}_b"] = ref.rounded(1 + 0.1 * rng.standard_normal(D), prec), r(D, scale=0.1)
    v["h0"] = rng.standard_normal((B, D)).astype(np.float32).astype(np.float64)
    logits = rng.standard_normal((N, E)) + np.array([1.0, 0.3, 0.0, -0.5])
    v["ids"] = np.argsort(-logits, axis=1)[:, :K]
    w = np.exp(rng.standard_normal((N, K)))
    v["w"] = (w / w.sum(1, keepdims=True)).astype(np.float32).astype(np.float64)
    return v


# ---- float64 model ----

def model(v):
    t = {k: torch.tensor(a, dtype=torch.float64, requires_grad=True) for k, a in v.items() if k != "ids"}
    ln = lambda x, i: torch.nn.functional.layer_norm(x, (D,), t[f"ln{i}_g"], t[f"ln{i}_b"], 1e-5)  # noqa: E731
    lin = lambda x, k: x @ t[k] + t[k + "_bias"]  # noqa: E731
    drop = lambda x, offset: x * torch.tensor(np.where(ref.kept(N, D, P_DROP, SEED, offset)[0], ref.kept(N, D, P_DROP, SEED, offset)[1], 0.0))  # noqa: E731
    angle = torch.tensor(np.arange(T)[:, None] * ref.frequencies(HD)[None, :])

    def turn(x):                                        # [B, T, H, HD]
        c, s = torch.cos(angle)[:, None], torch.sin(angle)[:, None]
        a, b = x[..., :HD // 2], x[..., HD // 2:]
        return torch.cat([a * c - b * s, b * c + a * s], dim=-1)
    q, k, val = (a.reshape(B, T, H, HD) for a in lin(ln(t["x"], 0), "qkv").chunk(3, dim=1))
    q, k = turn(q), turn(k)
    scores = torch.einsum("bthd,bshd->bhts", q, k) * HD ** -0.5
    scores = scores.masked_fill(torch.triu(torch.ones(T, T, dtype=torch.bool), 1), float("-inf"))
    o = torch.einsum("bhts,bshd->bthd", torch.softmax(scores, -1), val).reshape(N, D)
    x1 = t["x"] + drop(lin(o, "o"), 1)
    f, xin, g = (a.reshape(B, T, D) for a in lin(ln(x1, 1), "proj").chunk(3, dim=1))
    a, h, hs = torch.sigmoid(f), t["h0"], []
    for i in range(T):
        h = a[:, i] * h + (1 - a[:, i]) * xin[:, i]
        hs.append(h)
    rec = (torch.stack(hs, 1) * g * torch.sigmoid(g)).reshape(N, D)
    x2 = x1 + drop(lin(rec, "o2"), 2)
    a3, y = ln(x2, 2), x2
    slot_of, _, _, _ = ref.expert_plan(v["ids"], E, CAP, 1, E * CAP)
    for e in range(E):
        for j in range(K):
            tok = np.nonzero((v["ids"][:, j] == e) & (slot_of[:, j] >= 0))[0]
            out = lin(torch.nn.functional.gelu(lin(a3[tok], f"e{e}a"), approximate="tanh"), f"e{e}b")
            y = y.index_add(0, torch.tensor(tok), t["w"][tok, j:j + 1] * out)
    y.backward(torch.tensor(v["dy"]))
    return y.detach().numpy(), {k: a.grad.numpy() for k, a in t.items() if k != "dy"}


# ---- the same through the library ----

class Block:
    def __init__(self, sess, prec, v):
        self.s, self.prec, dev = sess, prec, sess.device
        self.t, self.f32 = ref.DTYPE[prec], lambda *s: torch.full(s, float("nan"), device=dev)
        self.v = {k: torch.as_tensor(a).to(torch.int32 if k == "ids" else torch.float32 if k in ("w", "h0") else self.t).to(dev).contiguous() for k, a in v.items()}
        self.new = lambda *s: torch.full(s, float("nan"), dtype=self.t, device=dev)  # noqa: E731
        self.table = rotary_frequencies(dev, HD)

    def gemm(self, m, n, k, a, b, c, a_mn=0, b_mn=1, epi=0, bias=None, aux=None, f32=0, ldc=None):
        ops.fax_op_gemm(self.s.ctx, self.prec, ops.GemmDesc(m, n, k, ptr(a), m if a_mn else k, a_mn, ptr(b), n if b_mn else k, b_mn, ptr(c), n if ldc is None else ldc, f32, 0, epi, ptr(bias), None, 0,
                                                           ptr(aux), n if aux is not None else 0, 1.0, 0))

    def linear(self, x, key, out, epi=ops.FAX_EPI_BIAS, aux=None, m=N):
        k, n = WEIGHTS[key]
        self.gemm(m, n, k, x, self.v[key], out, epi=epi, bias=self.v[key + "_bias"], aux=aux)

    def linear_back(self, x, key, dout, dx, m=N, epi=0, aux=None):
        """dx = dout W^T (epilogue), dW = x^T dout."""
        k, n = WEIGHTS[key]
        self.gemm(m, k, n, dout, self.v[key], dx, b_mn=0, epi=epi, aux=aux)
        dw = self.f32(k, n)
        self.gemm(k, n, m, x, dout, dw, a_mn=1, b_mn=1, f32=1)
        return dw

    def ln(self, x, i, out):
        mu, rs = self.f32(N), self.f32(N)
        ops.fax_op_layernorm_forward(self.s.ctx, self.prec, N, D, ptr(x), ptr(self.v[f"ln{i}_g"]), ptr(self.v[f"ln{i}_b"]), 1e-5, ptr(out), ptr(mu), ptr(rs))
        return mu, rs

    def ln_back(self, da, x, i, stats, add, dx):
        dg, db = self.f32(D), self.f32(D)
        nb = ops.fax_op_layernorm_backward_scratch_bytes(N, D)
        sc = self.s.arena(nb)
        ops.fax_op_layernorm_backward(self.s.ctx, self.prec, N, D, ptr(da), ptr(x), ptr(stats[0]), ptr(stats[1]), ptr(self.v[f"ln{i}_g"]), ptr(add), ptr(dx), ptr(dg), ptr(db), ptr(sc), nb)
        return dg, db

    def rotary(self, buf, back):
        ops.fax_op_rotary(self.s.ctx, self.prec, ops.RotaryDesc(N, 2 * H, HD, HD, ops.FAX_ROTARY_HALVES, ptr(buf), 3 * D, ptr(buf), 3 * D, None, 0, T, ptr(self.table), 1.0, back))

    def drop(self, x, resid, y, offset):
        ops.fax_op_dropout(self.s.ctx, self.prec, ops.DropoutDesc(N, D, ptr(x), D, ptr(resid), D if resid is not None else 0, ptr(y), D, P_DROP, SEED, offset, None))

    def run(self):
        c, prec, v, new = self.s.ctx, self.prec, self.v, self.new
        out, es = {}, torch.empty((), dtype=self.t).element_size()
        # attention with rotary positions
        a1, qkv, o, br, x1, lse = new(N, D), new(N, 3 * D), new(N, D), new(N, D), new(N, D), self.f32(B, H, T)
        st1 = self.ln(v["x"], 0, a1)
        self.linear(a1, "qkv", qkv)
        self.rotary(qkv, 0)
        ops.fax_op_attention_forward(c, prec, B, T, H, HD, ptr(qkv), ptr(o), ptr(lse))
        self.linear(o, "o", br)
        self.drop(br, v["x"], x1, 1)
        # recurrence, its three inputs columns of one projection
        a2, proj, rec, br2, x2, h_last = new(N, D), new(N, 3 * D), new(N, D), new(N, D), new(N, D), self.f32(B, D)
        st2 = self.ln(x1, 1, a2)
        self.linear(a2, "proj", proj)
        states = self.f32(ops.fax_op_recurrence_states_floats(N, B, D))
        col = lambda t, i: t.data_ptr() + i * D * es  # noqa: E731
        shape = (N, D, B, T, None, ops.FAX_RECURRENCE_COMPLEMENT, col(proj, 0), 3 * D, col(proj, 1), 3 * D, col(proj, 2), 3 * D, ptr(v["h0"]))
        ops.fax_op_recurrence_forward(c, prec, ops.RecurrenceDesc(*shape, ptr(rec), D, ptr(h_last), ptr(states)))
        self.linear(rec, "o2", br2)
        self.drop(br2, x1, x2, 2)
        # experts of a fixed capacity, so that every product's size is known here
        a3, slots = new(N, D), E * CAP
        st3 = self.ln(x2, 2, a3)
        whole = lambda *s: torch.empty(s, dtype=torch.int32, device=self.s.device)  # noqa: E731
        slot_of, source, offsets, counts = whole(N, K), whole(slots), whole(E + 1), whole(E)
        ops.fax_op_expert_sort(c, ops.ExpertSortDesc(N, K, E, CAP, 1, slots, ptr(v["ids"]), ptr(slot_of), ptr(source), ptr(offsets), ptr(counts)))
        xe, hid, act, ye, y = new(slots, D), new(slots, F), new(slots, F), new(slots, D), new(N, D)
        ops.fax_op_expert_dispatch(c, prec, ops.ExpertDispatchDesc(N, K, D, slots, ptr(slot_of), ptr(source), ptr(a3), D, ptr(xe), D))
        rows = lambda t, e: t[e * CAP:(e + 1) * CAP]  # noqa: E731
        for e in range(E):
            self.linear(rows(xe, e), f"e{e}a", rows(hid, e), epi=ops.FAX_EPI_BIAS_GELU, aux=rows(act, e), m=CAP)
            self.linear(rows(act, e), f"e{e}b", rows(ye, e), m=CAP)
        ops.fax_op_expert_combine(c, prec, ops.ExpertCombineDesc(N, K, D, slots, ptr(slot_of), ptr(v["w"]), ptr(ye), D, ptr(x2), D, ptr(y), D))
        out["y"] = y
        # backward
        dye, dw, dxe, dh, da3 = new(slots, D), self.f32(N, K), new(slots, D), new(slots, F), new(N, D)
        ops.fax_op_expert_combine_backward(c, prec, ops.ExpertCombineBackwardDesc(N, K, D, slots, ptr(slot_of), ptr(source), ptr(v["w"]), ptr(ye), D, ptr(v["dy"]), D, ptr(dye), D, ptr(dw)))
        out["w"] = dw
        for e in range(E):
            out[f"e{e}b"] = self.linear_back(rows(act, e), f"e{e}b", rows(dye, e), rows(dh, e), m=CAP, epi=ops.FAX_EPI_DGELU, aux=rows(hid, e))
            out[f"e{e}a"] = self.linear_back(rows(xe, e), f"e{e}a", rows(dh, e), rows(dxe, e), m=CAP)
        ops.fax_op_expert_combine(c, prec, ops.ExpertCombineDesc(N, K, D, slots, ptr(slot_of), None, ptr(dxe), D, None, 0, ptr(da3), D))
        dx2, dbr2, drec, dproj, da2, dh0 = new(N, D), new(N, D), new(N, D), new(N, 3 * D), new(N, D), self.f32(B, D)
        out["ln2_g"], out["ln2_b"] = self.ln_back(da3, x2, 2, st3, v["dy"], dx2)
        self.drop(dx2, None, dbr2, 2)
        out["o2"] = self.linear_back(rec, "o2", dbr2, drec)
        ops.fax_op_recurrence_backward(c, prec, ops.RecurrenceBackwardDesc(*shape, ptr(states), ptr(drec), D, None, col(dproj, 0), 3 * D, col(dproj, 1), 3 * D, col(dproj, 2), 3 * D, ptr(dh0)))
        out["h0"] = dh0
        out["proj"] = self.linear_back(a2, "proj", dproj, da2)
        dx1, dbr, do, dqkv, da1, dx = new(N, D), new(N, D), new(N, D), new(N, 3 * D), new(N, D), new(N, D)
        out["ln1_g"], out["ln1_b"] = self.ln_back(da2, x1, 1, st2, dx2, dx1)
        self.drop(dx1, None, dbr, 1)
        out["o"] = self.linear_back(o, "o", dbr, do)
        nb = ops.fax_op_attention_backward_scratch_bytes(prec, B, T, H, HD)
        sc = self.s.arena(nb)
        ops.fax_op_attention_backward(c, prec, B, T, H, HD, ptr(qkv), ptr(o), ptr(lse), ptr(do), ptr(dqkv), ptr(sc), nb)
        self.rotary(dqkv, 1)
        out["qkv"] = self.linear_back(a1, "qkv", dqkv, da1)
        out["ln0_g"], out["ln0_b"] = self.ln_back(da1, v["x"], 0, st1, dx1, dx)
        out["x"] = dx
        return {k: t.double().cpu().numpy() for k, t in out.items()}


@pytest.mark.parametrize("prec", [fx.FAX_PREC_FP32_VALIDATE, fx.FAX_PREC_BF16])
def test_block_of_the_pieces(prec):
    """Bounds of the library's blocks: 1e-4 of a tensor's largest value in float; in bf16 1e-2 forward, 2e-2 for gradients (every
    stored tensor is rounded by up to 2^-8, some thirty of them one after another, like a random walk)."""
    v = inputs(prec)
    y, grads = model(v)
    sess = Session(0)
    try:
        got = Block(sess, prec, v).run()
        assert fx.fax_check_device_status(sess.ctx)[0] == fx.FAX_OK
    finally:
        sess.close()
    for k, g in got.items():
        want = y if k == "y" else grads[k]
        assert np.isfinite(g).all(), k
        err = np.abs(g - want).max() / np.abs(want).max()
        assert err <= (TOL_FP32 if prec else TOL_FWD_BF16 if k == "y" else TOL_GRAD_BF16), (k, err)
