"""AdamW with 8-bit moments: the moments bit for bit what the definition gives (its every float32 operation rounded on
its own), the weights within the errors of the hardware's square root and reciprocal."""
import ctypes as C

import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import Session, fx, hparams, host, ptr

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


class State:
    """One tensor with moments in 8 bits; 64 guard bytes behind each buffer."""

    def __init__(self, n, dev, w, wd, seed, copy=True):
        nb = -(-n // 128)
        self.n, self.wd, self.seed = n, wd, seed
        self.w = torch.full((n + 16,), 5.0, device=dev)
        self.w[:n] = torch.as_tensor(w)
        self.m = torch.full((n + 64,), 0x55, dtype=torch.uint8, device=dev)
        self.v = self.m.clone()
        self.m[:n] = 0; self.v[:n] = 0
        self.ms = torch.full((nb + 16,), 5.0, device=dev)
        self.vs = self.ms.clone()
        self.ms[:nb] = 1; self.vs[:nb] = 1
        self.wc = torch.full((n + 32,), 5.0, dtype=torch.bfloat16, device=dev) if copy else None
        # the reference's copy
        self.r = [np.asarray(w, np.float64), np.zeros(n), np.ones(nb), np.zeros(n), np.ones(nb)]
        self.tol = np.zeros(n)

    def struct(self, g):
        return fx.Adamw8Tensor(ptr(self.w), ptr(self.m), ptr(self.v), ptr(self.ms), ptr(self.vs), ptr(g), ptr(self.wc), self.n, self.wd, self.seed)

    def advance(self, g, step, hp):
        old = self.r[0]
        self.r = list(ref.adamw8(*self.r, g.double().cpu().numpy(), self.wd, self.seed, step=step, **hp))
        # weights: three float32 roundings of w on each side (2^-24 each); the update: root and reciprocal within 2 units
        # of the last place (2^-22 each) and six roundings (2^-24 each), below 2^-20 on either side.  Its size is the change
        # of w plus what the decay took.  The moments do not depend on w: the errors of the steps add up
        with np.errstate(invalid="ignore"):
            upd = np.abs(self.r[0] - old) + hp["lr"] * self.wd * np.abs(old)
            self.tol = self.tol + 6 * 2.0 ** -24 * (np.abs(old) + np.abs(self.r[0])) + 2.0 ** -19 * upd

    def check(self):
        n, nb = self.n, -(-self.n // 128)
        w, m, ms, v, vs = self.r
        got = host(self.w[:n])
        fin = np.isfinite(w)
        assert np.array_equal(got[~fin], w[~fin], equal_nan=True)
        assert np.all(np.abs(got[fin] - w[fin]) <= self.tol[fin])
        assert np.array_equal(host(self.m[:n].view(torch.float8_e4m3fn)), m, equal_nan=True)
        assert np.array_equal(host(self.v[:n].view(torch.float8_e5m2)), v, equal_nan=True)
        assert np.array_equal(host(self.ms[:nb]), ms) and np.array_equal(host(self.vs[:nb]), vs)
        assert bool((self.w[n:] == 5).all()) and bool((self.m[n:] == 0x55).all()) and bool((self.v[n:] == 0x55).all())
        assert bool((self.ms[nb:] == 5).all()) and bool((self.vs[nb:] == 5).all())
        if self.wc is not None:
            a, b = self.wc[:n], self.w[:n].to(torch.bfloat16)
            assert torch.equal(a.view(torch.int16)[~torch.isnan(b)], b.view(torch.int16)[~torch.isnan(b)])
            assert bool((self.wc[n:] == 5).all())


def grad(n, rng, dev, bf16=False):
    g = rng.standard_normal(n) * 10.0 ** rng.uniform(-8, 0, n)
    g[rng.random(n) < 0.1] = 0
    t = torch.as_tensor(g.astype(np.float32)).to(dev)
    return t.to(torch.bfloat16) if bf16 else t


@pytest.mark.parametrize("bf16", [0, 1])
@pytest.mark.parametrize("n", [1, 3, 4, 127, 128, 129, 130, 1023, 4096, 4097, 100_003])
def test_steps_bit_for_bit(sess, n, bf16):
    rng = np.random.default_rng(n + bf16)
    s = State(n, sess.device, rng.standard_normal(n).astype(np.float32), 0.1, seed=n)
    for step in (1, 2, 3, 50, 51, 100_000):
        g = grad(n, rng, sess.device, bf16)
        fx.fax_adamw8_step(sess.ctx, [s.struct(g)], hparams(step=step, grad_is_bf16=bf16, **HP))
        s.advance(g, step, HP)
        s.check()


def test_many_tensors_in_one_call(sess):
    """More than one launch's worth, empty ones among them, with and without a bf16 copy: each as if alone."""
    rng = np.random.default_rng(9)
    sizes = [3, 128, 0, 4096, 2049, 77, 640] * 13
    ts = [State(n, sess.device, rng.standard_normal(n).astype(np.float32), 0.1 if i % 2 else 0.0, seed=1000 + i, copy=bool(i % 3)) for i, n in enumerate(sizes)]
    for step in (1, 2):
        gs = [grad(n, rng, sess.device) for n in sizes]
        fx.fax_adamw8_step(sess.ctx, [t.struct(g) for t, g in zip(ts, gs)], hparams(step=step, **HP))
        for t, g in zip(ts, gs):
            t.advance(g, step, HP)
    for t in ts:
        t.check()
    fx.fax_adamw8_step(sess.ctx, [], hparams(step=1, **HP))


def test_extreme_gradients(sess):
    """Infinities and NaN stay with their element; sizes at float32's ends; a block of zeros; no v above 0 becomes 0."""
    n = 640
    w = np.ones(n, np.float32)
    g = np.zeros(n, np.float32)
    g[0:128] = 1e-3; g[3] = np.inf; g[5] = np.nan; g[7] = -np.inf; g[9] = 3e38; g[11] = 1e25
    g[128:256] = np.logspace(-30, 18, 128)
    g[256:384] = 1e-42
    g[384:400] = -2.5
    s = State(n, sess.device, w, 0.0, seed=77)
    t = torch.as_tensor(g).to(sess.device)
    for step in (1, 2, 3):
        fx.fax_adamw8_step(sess.ctx, [s.struct(t)], hparams(step=step, **HP))
        s.advance(t, step, HP)
        s.check()
    v = s.v[:n].view(torch.float8_e5m2).float()
    assert bool(((v > 0) | torch.isnan(v))[128 + 24:256].all())      # far below the block's largest, yet not zero


def test_moments_are_right_on_average(sess):
    """Constant gradients: v tends to g^2 although every step moves it by less than half an 8-bit step, which the
    nearest value would never do.  A rounding that is right on average has a spread of half a step at most: an
    eighth of v (e5m2), a sixteenth of m (e4m3).  A step's noise decays by beta, so its squares add up to
    1 / (1 - beta^2) of one, and the mean of n independent elements has 1 / sqrt(n) of that: six such spreads,
    twice over because v itself varies, and the 16 random bits' own bias of 2^-17 of a step, 1 / (1 - beta) times."""
    n = 1 << 16
    s = State(n, sess.device, np.zeros(n, np.float32), 0.0, seed=5)
    g = torch.full((n,), 0.37, device=sess.device)
    b1, b2, steps = float(np.float32(0.9)), float(np.float32(0.99)), 300
    for step in range(1, steps + 1):
        fx.fax_adamw8_step(sess.ctx, [s.struct(g)], hparams(step=step, **dict(HP, beta2=0.99)))
    v = s.v[:n].view(torch.float8_e5m2).double() * s.vs[:n // 128].double().repeat_interleave(128)
    m = s.m[:n].view(torch.float8_e4m3fn).double() * s.ms[:n // 128].double().repeat_interleave(128)
    for x, b, want, part in ((v, b2, 0.37 ** 2, 4), (m, b1, 0.37, 8)):
        tol = 6 * 2 * (1 / (2 * part)) / np.sqrt((1 - b * b) * n) + 2.0 ** -17 / part / (1 - b) + b ** steps
        assert abs(float(x.mean()) / want - 1) <= tol, (float(x.mean()), want, tol)


def test_replayed_from_a_graph(sess):
    rng = np.random.default_rng(2)
    n = 3000
    st = torch.cuda.Stream(sess.device)
    with torch.cuda.stream(st):
        s2 = Session(0)
        try:
            s = State(n, sess.device, rng.standard_normal(n).astype(np.float32), 0.1, seed=8)
            g = grad(n, rng, sess.device)
            arr = (fx.Adamw8Tensor * 1)(s.struct(g))
            fx.fax_adamw8_step(s2.ctx, arr, hparams(step=4, **HP))
            s.advance(g, 4, HP)
            st.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                fx.fax_adamw8_step(s2.ctx, arr, hparams(step=5, **HP))
            for _ in range(2):
                g.copy_(grad(n, rng, sess.device))
                graph.replay()
                s.advance(g, 5, HP)
            st.synchronize()
            s.check()
            del graph
        finally:
            s2.close()
