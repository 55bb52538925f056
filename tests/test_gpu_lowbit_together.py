"""The operators on few bits as a training step uses them, one feeding the next; the language model with its token
table's gradient summed in sorted order; 8-bit moments under the whole model."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import LmRunner, O, Session, TOL_GRAD_BF16, TOL_FP32, fx, host, hparams, ptr, relerr, synth
from paper_2204_06514_b200 import binding_ops as ops
from paper_2204_06514_b200.state import Moments8, ParamSet
from test_gpu_block import lm_case

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    st, detail = fx.fax_check_device_status(s.ctx)
    s.close()
    assert st == fx.FAX_OK, detail


def up(x, a=16):
    return -(-x // a) * a


class Quantized:
    """A matrix in 8 bits as it stands and transposed."""

    def __init__(self, sess, prec, x, fmt, tile):
        r, c = x.shape
        dev = sess.device
        self.q, self.qt = (torch.zeros(s, dtype=torch.uint8, device=dev) for s in ((r, up(c)), (c, up(r))))
        self.s, self.st = (torch.zeros(s, device=dev) for s in ((-(-c // 128), -(-r // tile)), (-(-r // 128), -(-c // tile))))
        self.r, self.c, self.fmt, self.tile = r, c, fmt, tile
        ops.fax_op_fp8_quantize(sess.ctx, prec, ops.Fp8QuantizeDesc(
            r, c, ptr(x), x.stride(0), fmt, tile, ptr(self.q), self.q.shape[1], ptr(self.s), self.s.shape[1],
            ptr(self.qt), self.qt.shape[1], ptr(self.st), self.st.shape[1]))

    def straight(self):
        return self.q, self.s, self.c

    def transposed(self):
        return self.qt, self.st, self.r

    def wide(self, transposed=False):
        q, s, k = self.transposed() if transposed else self.straight()
        return ref.widen(host(q[:, :k].contiguous().view(ref.TORCH8[self.fmt])), host(s), self.tile)


def product(sess, a, b, out, accumulate=False, bias=None):
    (qa, sa, k), (qb, sb, k2), fa, fb, tb = a[0], b[0], a[1].fmt, b[1].fmt, b[1].tile
    assert k == k2
    ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(out.shape[0], out.shape[1], k, ptr(qa), qa.shape[1], fa, ptr(sa), sa.shape[1], ptr(qb), qb.shape[1], fb, ptr(sb),
                                                  sb.shape[1], tb, ptr(out), out.shape[1], int(out.dtype == torch.float32), int(accumulate),
                                                  ptr(bias) if bias is not None else None))


def near(got, want, size, k, bf16):
    tol = (k + 3 * (-(-k // 128)) + 4) * 2.0 ** -23 * size + (2.0 ** -8 * np.abs(want) if bf16 else 0)
    assert np.all(np.abs(got - want) <= tol), np.abs(got - want).max()


@pytest.mark.parametrize("n,vocab,d,f", [(130, 60, 64, 96), (257, 300, 144, 200), (512, 1000, 256, 512)])
def test_two_steps_of_a_projection_on_a_token_table(sess, n, vocab, d, f):
    """y = (scale table[ids]) W in 8 bits, its input and weight gradients, the table's gradient, AdamW on both."""
    rng = np.random.default_rng(n)
    dev = sess.device
    scale = float(np.sqrt(d))
    table = ParamSet(0.02 * rng.standard_normal((vocab, d)).astype(np.float32), fx.FAX_PREC_BF16, dev, 0.1)
    w = ParamSet(0.05 * rng.standard_normal((d, f)).astype(np.float32), fx.FAX_PREC_BF16, dev, 0.1)
    opt = Moments8([table, w], seed=77)
    state = [[host(p.w).ravel(), np.zeros(p.w.numel()), np.ones(-(-p.w.numel() // 128)), np.zeros(p.w.numel()), np.ones(-(-p.w.numel() // 128))] for p in (table, w)]
    scratch = sess.arena(ops.fax_op_embedding_backward_scratch_bytes(n, vocab, d))
    for step in (1, 2):
        ids = rng.integers(-1, vocab, n).astype(np.int32)
        tid = torch.as_tensor(ids).to(dev)
        x = torch.empty((n, d), dtype=torch.bfloat16, device=dev)
        ops.fax_op_embedding_forward(sess.ctx, 0, n, vocab, d, ptr(tid), ptr(table.wc), scale, ptr(x))
        assert torch.equal(x, torch.as_tensor(ref.embedding(ids, host(table.wc), scale)).float().to(torch.bfloat16).to(dev))
        qx, qw = Quantized(sess, 0, x, 0, 1), Quantized(sess, 1, w.w, 0, 128)
        y = torch.empty((n, f), dtype=torch.bfloat16, device=dev)
        product(sess, (qx.straight(), qx), (qw.transposed(), qw), y)                 # rows of x, W transposed
        dy = torch.as_tensor(rng.standard_normal((n, f)).astype(np.float32)).to(torch.bfloat16).to(dev)
        qdy = Quantized(sess, 0, dy, 1, 1)
        dx = torch.empty((n, d), dtype=torch.bfloat16, device=dev)
        product(sess, (qdy.straight(), qdy), (qw.straight(), qw), dx)                # rows of dy, W as stored
        dw = torch.zeros((d, f), device=dev)
        for _ in range(2):                                                           # two halves of a gradient, added
            product(sess, (qx.transposed(), qx), (qdy.transposed(), qdy), dw, accumulate=True)
        w.g.copy_(dw)
        ops.fax_op_embedding_backward(sess.ctx, 0, n, vocab, d, ptr(tid), ptr(dx), scale, 0, ptr(table.g), ptr(scratch), scratch.numel())

        # each against the formulas in 64 bits on what it was given
        ax, aw, ady = qx.wide(), qw.wide(), qdy.wide()
        near(host(y), ax @ aw, np.abs(ax) @ np.abs(aw), d, True)
        near(host(dx), ady @ aw.T, np.abs(ady) @ np.abs(aw).T, f, True)
        bx, bdy = qx.wide(True), qdy.wide(True)
        near(host(dw), 2 * bx @ bdy.T, 2 * np.abs(bx) @ np.abs(bdy).T, 2 * n + 2, False)
        count = np.bincount(ids[ids >= 0], minlength=vocab)[:, None]
        size = ref.embedding_grad(ids, np.abs(host(dx)), vocab, scale)
        assert np.all(np.abs(host(table.g) - ref.embedding_grad(ids, host(dx), vocab, scale)) <= (count + 3) * 2.0 ** -24 * size)

        opt.step(sess.ctx, hparams(step=step, **HP))
        for i, p in enumerate((table, w)):
            old = state[i][0]
            state[i] = list(ref.adamw8(*state[i], host(p.g).ravel(), 0.1, 77 + i, step=step, **HP))
            assert np.array_equal(host(opt.m[i].view(torch.float8_e4m3fn)), state[i][1]) and np.array_equal(host(opt.m_scale[i]), state[i][2])
            assert np.array_equal(host(opt.v[i].view(torch.float8_e5m2)), state[i][3]) and np.array_equal(host(opt.v_scale[i]), state[i][4])
            upd = np.abs(state[i][0] - old) + HP["lr"] * 0.1 * np.abs(old)
            assert np.all(np.abs(host(p.w).ravel() - state[i][0]) <= 6 * 2.0 ** -24 * (np.abs(old) + np.abs(state[i][0])) + 2.0 ** -19 * upd)
            state[i][0] = host(p.w).ravel()
            assert torch.equal(p.wc, p.w.to(torch.bfloat16))


def test_gradients_against_differences(sess):
    """The product is linear in each factor and the lookup in its table: <dy, f(x + h) - f(x)> is <gradient, h> for any h,
    up to the float32 sums on either side."""
    rng = np.random.default_rng(8)
    n, d, f, vocab = 200, 160, 136, 40
    dev = sess.device
    rnd = lambda *s: torch.as_tensor(rng.standard_normal(s).astype(np.float32)).to(dev)  # noqa: E731
    x0, x1, w0, w1, dy = (Quantized(sess, 1, t, 0, 128 if i in (2, 3) else 1) for i, t in enumerate((rnd(n, d), rnd(n, d), rnd(d, f), rnd(d, f), rnd(n, f))))
    ys = []
    for a, b in ((x0, w0), (x1, w0), (x0, w1)):
        y = torch.empty((n, f), device=dev)
        product(sess, (a.straight(), a), (b.transposed(), b), y)
        ys.append(host(y))
    dx = torch.empty((n, d), device=dev)
    product(sess, (dy.straight(), dy), (w0.straight(), w0), dx)
    g = dy.wide()
    total = np.abs(g).sum() * np.abs(ys[0]).max()
    assert abs((g * (ys[1] - ys[0])).sum() - (host(dx) * (x1.wide() - x0.wide())).sum()) <= (d + f) * 2.0 ** -22 * total
    # the weight gradient takes both factors in blocks along the tokens: with those values the identity is the same
    dw = torch.empty((d, f), device=dev)
    product(sess, (x0.transposed(), x0), (dy.transposed(), dy), dw)
    xt, gt = x0.wide(True).T, dy.wide(True).T
    h = w1.wide() - w0.wide()
    assert abs((gt * (xt @ h)).sum() - (host(dw) * h).sum()) <= (n + 8) * 2.0 ** -22 * (np.abs(xt).T @ np.abs(gt) * np.abs(h)).sum()
    # lookup
    ids = torch.as_tensor(rng.integers(-1, vocab, n).astype(np.int32)).to(dev)
    t0, t1, do = rnd(vocab, d), rnd(vocab, d), rnd(n, d)
    outs = []
    for t in (t0, t1):
        o = torch.empty((n, d), device=dev)
        ops.fax_op_embedding_forward(sess.ctx, 1, n, vocab, d, ptr(ids), ptr(t), 3.0, ptr(o))
        outs.append(host(o))
    gt = torch.empty((vocab, d), device=dev)
    s = sess.arena(ops.fax_op_embedding_backward_scratch_bytes(n, vocab, d))
    ops.fax_op_embedding_backward(sess.ctx, 1, n, vocab, d, ptr(ids), ptr(do), 3.0, 0, ptr(gt), ptr(s), s.numel())
    lhs, rhs = (host(do) * (outs[1] - outs[0])).sum(), (host(gt) * (host(t1) - host(t0))).sum()
    assert abs(lhs - rhs) <= (n + 8) * 2.0 ** -23 * (np.abs(host(do)) * (np.abs(outs[0]) + np.abs(outs[1]))).sum()


@pytest.mark.parametrize("prec", [0, 1])
def test_lm_with_sorted_embedding_gradient(sess, prec):
    fx.fax_set_sorted_embedding_gradient(sess.ctx, True)
    try:
        if prec == 0:
            cfg = synth.scaled(synth.CONFIGS["C4"], batch=2, seq=128, n_layers=2)
        else:
            cfg = synth.Config("lm_sorted32", 14, batch=2, seq=5, d_model=8, n_heads=2, head_dim=4, d_ff=16, n_layers=2, vocab=11)
        lm_case(sess, cfg, prec, synth.lm_params(cfg))
    finally:
        fx.fax_set_sorted_embedding_gradient(sess.ctx, False)


def test_lm_step_replayed_with_sorted_embedding_gradient(sess):
    """The switch drops the recorded step graphs, and a replayed step sorts again: new tokens in the same buffers."""
    cfg = synth.Config("lm_replay", 15, batch=2, seq=128, d_model=128, n_heads=2, head_dim=64, d_ff=256, n_layers=1, vocab=256)
    lm = synth.lm_params(cfg)
    ids, tg = synth.lm_tokens(cfg)
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a)).to(sess.device)  # noqa: E731
    runs = []
    rng = np.random.default_rng(3)
    batches = [(ids, tg)] + [tuple(rng.integers(0, cfg.vocab, ids.shape).astype(np.int32) for _ in range(2)) for _ in range(5)]
    for on in (False, True):
        fx.fax_set_sorted_embedding_gradient(sess.ctx, on)
        r = LmRunner(sess, cfg, lm, fx.FAX_PREC_BF16, weight_decay=0.1)
        tid, ttg = dev(ids), dev(tg)
        losses = []
        for step, (a, b) in enumerate(batches, 1):
            tid.copy_(torch.as_tensor(a)); ttg.copy_(torch.as_tensor(b))
            r.step(tid, ttg, hparams(step=step, **HP))
            losses.append(float(r.loss.item()))
        runs.append((losses, host(r.wte.g)))
    fx.fax_set_sorted_embedding_gradient(sess.ctx, False)
    # the same step twice but for the order of float32 additions, which the following steps see through bf16 weights
    assert np.allclose(runs[0][0], runs[1][0], rtol=2e-2)
    assert relerr(runs[1][1], runs[0][1]) <= 2 * TOL_GRAD_BF16


def test_moments8_under_the_language_model(sess):
    """Gradients from fax_lm_accumulate, every tensor of the model updated by one fax_adamw8_step: bit for bit."""
    cfg = synth.Config("lm_adam8", 16, batch=2, seq=128, d_model=128, n_heads=2, head_dim=64, d_ff=256, n_layers=2, vocab=256)
    ids, tg = synth.lm_tokens(cfg)
    r = LmRunner(sess, cfg, synth.lm_params(cfg), fx.FAX_PREC_BF16, weight_decay=0.1)
    dev = lambda a: torch.as_tensor(np.ascontiguousarray(a)).to(sess.device)  # noqa: E731
    params = [p for _, p in r.named_params()]
    opt = Moments8(params, seed=5)
    state = [[host(p.w).ravel(), np.zeros(p.w.numel()), np.ones(-(-p.w.numel() // 128)), np.zeros(p.w.numel()), np.ones(-(-p.w.numel() // 128))] for p in params]
    for step in (1, 2):
        r.accumulate(dev(ids), dev(tg), False, 1.0)
        opt.step(sess.ctx, hparams(step=step, **HP))
        for i, p in enumerate(params):
            state[i] = list(ref.adamw8(*state[i], host(p.g).ravel(), p.weight_decay, 5 + i, step=step, **HP))
            assert np.array_equal(host(opt.m[i].view(torch.float8_e4m3fn)), state[i][1])
            assert np.array_equal(host(opt.v[i].view(torch.float8_e5m2)), state[i][3])
            assert relerr(host(p.w).ravel(), state[i][0]) <= 1e-6
            assert torch.equal(p.wc, p.w.to(torch.bfloat16))
            state[i][0] = host(p.w).ravel()
