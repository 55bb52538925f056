"""The operators on few bits and the token table's under a context's settings, in its profile, and on two streams at once."""
import numpy as np
import pytest
import torch

from parity_util import Session, fx, hparams, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu


class Chain:
    """Lookup -> 8 bits -> product -> table's gradient from the product's -> AdamW: each reads what the one before wrote."""

    def __init__(self, sess, m, n, k, vocab, rng):
        dev = sess.device
        self.s, self.dims = sess, (m, n, k, vocab)
        new = lambda *shape, t=torch.float32: torch.zeros(shape, dtype=t, device=dev)  # noqa: E731
        self.table0 = torch.as_tensor(rng.standard_normal((vocab, k)).astype(np.float32)).to(torch.bfloat16).to(dev)
        self.w = torch.as_tensor(rng.standard_normal((n, k)).astype(np.float32)).to(torch.bfloat16).to(dev)
        self.ids = torch.as_tensor(rng.integers(-1, vocab, m).astype(np.int32)).to(dev)
        self.x, self.y, self.dtable = new(m, k, t=torch.bfloat16), new(m, n), new(vocab, k)
        kb = -(-k // 128)
        self.qx, self.sx, self.qw, self.sw = new(m, k, t=torch.uint8), new(kb, m), new(n, k, t=torch.uint8), new(kb, -(-n // 128))
        self.qy, self.sy, self.qwt, self.swt = new(m, n, t=torch.uint8), new(-(-n // 128), m), new(k, n, t=torch.uint8), new(-(-n // 128), kb)
        self.master, self.table = new(vocab, k), new(vocab, k, t=torch.bfloat16)
        cnt = vocab * k
        self.m8, self.v8, self.ms, self.vs = new(cnt, t=torch.uint8), new(cnt, t=torch.uint8), new(-(-cnt // 128)), new(-(-cnt // 128))
        self.scratch = sess.arena(ops.fax_op_embedding_backward_scratch_bytes(m, vocab, k))
        self.adam = (fx.Adamw8Tensor * 1)(fx.Adamw8Tensor(ptr(self.master), ptr(self.m8), ptr(self.v8), ptr(self.ms), ptr(self.vs), ptr(self.dtable), ptr(self.table), cnt, 0.1, 3))
        self.reset()

    def reset(self):
        self.table.copy_(self.table0)
        self.master.copy_(self.table0)
        for t in (self.m8, self.v8, self.ms, self.vs):
            t.zero_()
        torch.cuda.synchronize()

    def run(self, steps=3):
        c, (m, n, k, vocab) = self.s.ctx, self.dims
        for step in range(1, steps + 1):
            ops.fax_op_embedding_forward(c, 0, m, vocab, k, ptr(self.ids), ptr(self.table), 0.5, ptr(self.x))
            ops.fax_op_fp8_quantize(c, 0, ops.Fp8QuantizeDesc(m, k, ptr(self.x), k, 0, 1, ptr(self.qx), k, ptr(self.sx), m, None, 0, None, 0))
            ops.fax_op_fp8_quantize(c, 0, ops.Fp8QuantizeDesc(n, k, ptr(self.w), k, 0, 128, ptr(self.qw), k, ptr(self.sw), -(-n // 128), ptr(self.qwt), n, ptr(self.swt), -(-k // 128)))
            ops.fax_op_fp8_gemm(c, ops.Fp8GemmDesc(m, n, k, ptr(self.qx), k, 0, ptr(self.sx), m, ptr(self.qw), k, 0, ptr(self.sw), -(-n // 128), 128, ptr(self.y), n, 1, 0, None))
            ops.fax_op_fp8_quantize(c, 1, ops.Fp8QuantizeDesc(m, n, ptr(self.y), n, 1, 1, ptr(self.qy), n, ptr(self.sy), m, None, 0, None, 0))
            ops.fax_op_fp8_gemm(c, ops.Fp8GemmDesc(m, k, n, ptr(self.qy), n, 1, ptr(self.sy), m, ptr(self.qwt), n, 0, ptr(self.swt), -(-k // 128), 128, ptr(self.x), k, 0, 0, None))
            ops.fax_op_embedding_backward(c, 0, m, vocab, k, ptr(self.ids), ptr(self.x), 0.5, 0, ptr(self.dtable), ptr(self.scratch), self.scratch.numel())
            fx.fax_adamw8_step(c, self.adam, hparams(step=step, lr=1e-2, beta1=0.9, beta2=0.95, eps=1e-8))

    def result(self):
        self.s.stream.synchronize()
        return [t.clone() for t in (self.table, self.master, self.m8, self.v8, self.ms, self.vs, self.dtable, self.y)]


def same(a, b):
    return all(torch.equal(x.view(torch.uint8), y.view(torch.uint8)) for x, y in zip(a, b))


DIMS = [(300, 272, 400, 500), (1500, 512, 640, 3000), (16, 1024, 4096, 64)]


@pytest.mark.parametrize("dims", DIMS)
def test_a_contexts_settings_change_no_bit(dims):
    rng = np.random.default_rng(dims[0])
    sess = Session(0)
    try:
        c = Chain(sess, *dims, rng)
        c.run()
        want = c.result()
        assert float(want[7].abs().max()) > 0 and bool(torch.isfinite(want[1]).all())
        for put, back in ((lambda: fx.fax_set_dependent_launch(sess.ctx, False), lambda: fx.fax_set_dependent_launch(sess.ctx, True)),
                          (lambda: fx.fax_set_gemm_l2_budget(sess.ctx, 0), lambda: fx.fax_set_gemm_l2_budget(sess.ctx, 48_000_000)),
                          (lambda: fx.fax_set_gemm_l2_budget(sess.ctx, 1 << 20), lambda: fx.fax_set_gemm_l2_budget(sess.ctx, 48_000_000))):
            c.reset()
            put()
            c.run()
            assert same(c.result(), want)
            back()
        assert fx.fax_check_device_status(sess.ctx)[0] == fx.FAX_OK
    finally:
        sess.close()


def test_tile_order_of_many_tiles_changes_no_bit():
    """More tiles than the SMs hold at once, so that the L2 budget decides an order."""
    m, n, k = 4000, 5000, 256
    sess = Session(0)
    try:
        dev = sess.device
        g = torch.Generator(device=dev).manual_seed(1)
        a, b = (torch.randn((r, k), device=dev, generator=g).to(torch.float8_e4m3fn).view(torch.uint8) for r in (m, n))
        sa, sb = torch.ones((2, m), device=dev), torch.ones((2, n), device=dev)
        outs = []
        for budget in (48_000_000, 0, 100_000, 1 << 40):
            fx.fax_set_gemm_l2_budget(sess.ctx, budget)
            out = torch.full((m, n), float("nan"), device=dev)
            ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(m, n, k, ptr(a), k, 0, ptr(sa), m, ptr(b), k, 0, ptr(sb), n, 1, ptr(out), n, 1, 0, None))
            outs.append(out)
        torch.cuda.synchronize()
        assert bool(torch.isfinite(outs[0]).all()) and all(torch.equal(o, outs[0]) for o in outs)
    finally:
        sess.close()


def test_two_streams_at_once():
    """Two contexts on streams of their own, the chains interleaved from one thread: each has the result it has alone."""
    streams = [torch.cuda.Stream(0), torch.cuda.Stream(0)]
    chains, want = [], []
    try:
        for st, dims in zip(streams, (DIMS[1], (1100, 784, 336, 2000))):
            with torch.cuda.stream(st):
                c = Chain(Session(0), *dims, np.random.default_rng(7))
                chains.append(c)
                c.run()
                want.append(c.result())
                c.reset()
        for rep in range(4):
            for c, st in zip(chains, streams):
                with torch.cuda.stream(st):
                    c.run()
            got = [c.result() for c in chains]
            assert same(got[0], want[0]) and same(got[1], want[1])
            for c in chains:
                c.reset()
        for c in chains:
            assert fx.fax_check_device_status(c.s.ctx)[0] == fx.FAX_OK
    finally:
        torch.cuda.synchronize()
        for c in chains:
            c.s.close()


def test_two_graphs_replayed_at_once():
    """Captured chains with scratch of their own, replayed on two streams."""
    streams = [torch.cuda.Stream(0), torch.cuda.Stream(0)]
    chains, want, graphs = [], [], []
    try:
        for st, dims in zip(streams, (DIMS[0], (900, 144, 208, 100))):
            with torch.cuda.stream(st):
                c = Chain(Session(0), *dims, np.random.default_rng(9))
                chains.append(c)
                c.run()
                want.append(c.result())
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=st):
                    c.run()
                graphs.append(g)
        for rep in range(3):
            for c in chains:
                c.reset()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            got = [c.result() for c in chains]
            assert same(got[0], want[0]) and same(got[1], want[1])
    finally:
        torch.cuda.synchronize()
        graphs.clear()
        for c in chains:
            c.s.close()


def test_profile_names_the_operators():
    sess = Session(0)
    try:
        m, n, k, vocab = 300, 272, 400, 500
        c = Chain(sess, m, n, k, vocab, np.random.default_rng(3))
        c.run(1)
        want = c.result()
        c.reset()
        fx.fax_profile_begin(sess.ctx)
        c.run(1)
        prof = fx.fax_profile_end(sess.ctx)
        assert same(c.result(), want)
        flops = {name: e["flops"] for name, e in prof.items() if e["flops"]}
        assert sum(flops.values()) == 4.0 * m * n * k and len(flops) == 1
        assert sum(e["launches"] for e in prof.values()) == 8 and all(e["ms"] > 0 for e in prof.values())
    finally:
        sess.close()
