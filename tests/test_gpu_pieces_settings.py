"""The pieces under a context's settings, in its profile, on two streams and in two graphs at once."""
import numpy as np
import pytest
import torch

from parity_util import Session, fx, ptr
from paper_2204_06514_b200 import binding_ops as ops
from paper_2204_06514_b200.state import rotary_frequencies

pytestmark = pytest.mark.gpu


class Chain:
    """Rotary -> dropout -> recurrence and back -> experts and back: each reads what the one before wrote, the last one feeds the next step."""

    def __init__(self, sess, rows, d, n_seq, experts, rng):
        dev = sess.device
        self.s, self.dims = sess, (rows, d, n_seq, experts)
        bf = lambda *s: torch.as_tensor(rng.standard_normal(s)).to(torch.bfloat16).to(dev)  # noqa: E731
        self.x0, self.f, self.g = bf(rows, d), bf(rows, d), bf(rows, d)
        new = lambda *s, t=torch.bfloat16: torch.zeros(s, dtype=t, device=dev)  # noqa: E731
        self.x, self.y, self.rec, self.df, self.dx, self.dg, self.out = (new(rows, d) for _ in range(7))
        self.slots = ops.fax_op_expert_slots(rows, 2, experts, 0, 16)
        self.rows_e, self.dz = new(self.slots, d), new(self.slots, d)
        f32 = lambda *s: torch.zeros(s, device=dev)  # noqa: E731
        self.h_last, self.dh0, self.dw = f32(n_seq, d), f32(n_seq, d), f32(rows, 2)
        self.states = f32(ops.fax_op_recurrence_states_floats(rows, n_seq, d))
        i32 = lambda a: torch.as_tensor(np.asarray(a, dtype=np.int32)).to(dev)  # noqa: E731
        cuts = np.sort(rng.integers(0, rows + 1, n_seq - 1))
        self.offsets = i32(np.concatenate([[0], cuts, [rows]]))
        self.longest = int(np.diff(np.concatenate([[0], cuts, [rows]])).max())
        self.ids, self.w = i32(rng.integers(-1, experts, (rows, 2))), torch.as_tensor(rng.random((rows, 2))).float().to(dev)
        self.slot_of, self.source, self.eo, self.counts = i32(np.zeros((rows, 2))), i32(np.zeros(self.slots)), i32(np.zeros(experts + 1)), i32(np.zeros(experts))
        self.table, self.step = rotary_frequencies(dev, 32), torch.zeros(1, dtype=torch.int64, device=dev)
        self.reset()

    def reset(self):
        self.x.copy_(self.x0)
        self.step.zero_()
        torch.cuda.synchronize()

    def run(self, steps=3):
        c, (n, d, n_seq, e) = self.s.ctx, self.dims
        for _ in range(steps):
            ops.fax_op_rotary(c, 0, ops.RotaryDesc(n, d // 32, 32, 32, 1, ptr(self.x), d, ptr(self.x), d, None, 5, 100, ptr(self.table), 1.0, 0))
            ops.fax_op_dropout(c, 0, ops.DropoutDesc(n, d, ptr(self.x), d, ptr(self.x0), d, ptr(self.y), d, 0.3, 11, 0, ptr(self.step)))
            shape = (n, d, n_seq, self.longest, ptr(self.offsets), 1, ptr(self.f), d, ptr(self.y), d, ptr(self.g), d, None)
            ops.fax_op_recurrence_forward(c, 0, ops.RecurrenceDesc(*shape, ptr(self.rec), d, ptr(self.h_last), ptr(self.states)))
            ops.fax_op_recurrence_backward(c, 0, ops.RecurrenceBackwardDesc(*shape, ptr(self.states), ptr(self.rec), d, None, ptr(self.df), d, ptr(self.dx), d, ptr(self.dg), d, ptr(self.dh0)))
            ops.fax_op_expert_sort(c, ops.ExpertSortDesc(n, 2, e, 0, 16, self.slots, ptr(self.ids), ptr(self.slot_of), ptr(self.source), ptr(self.eo), ptr(self.counts)))
            ops.fax_op_expert_dispatch(c, 0, ops.ExpertDispatchDesc(n, 2, d, self.slots, ptr(self.slot_of), ptr(self.source), ptr(self.dx), d, ptr(self.rows_e), d))
            ops.fax_op_expert_combine(c, 0, ops.ExpertCombineDesc(n, 2, d, self.slots, ptr(self.slot_of), ptr(self.w), ptr(self.rows_e), d, ptr(self.y), d, ptr(self.out), d))
            ops.fax_op_expert_combine_backward(c, 0, ops.ExpertCombineBackwardDesc(n, 2, d, self.slots, ptr(self.slot_of), ptr(self.source), ptr(self.w), ptr(self.rows_e), d, ptr(self.df), d,
                                                                                  ptr(self.dz), d, ptr(self.dw)))
            self.step.add_(1)
            self.x.copy_(self.out)

    def result(self):
        self.s.stream.synchronize()
        return [t.clone() for t in (self.x, self.rec, self.df, self.dx, self.dg, self.h_last, self.dh0, self.slot_of, self.source, self.dz, self.dw)]


def same(a, b):
    return all(torch.equal(x.contiguous().view(torch.uint8), y.contiguous().view(torch.uint8)) for x, y in zip(a, b))


DIMS = [(1000, 64, 3, 4), (6000, 256, 2, 8), (300, 96, 40, 100)]


@pytest.mark.parametrize("dims", DIMS)
def test_dependent_launch_changes_no_bit(dims):
    sess = Session(0)
    try:
        c = Chain(sess, *dims, np.random.default_rng(1))
        c.run()
        want = c.result()
        assert all(bool(torch.isfinite(t.float()).all()) for t in want) and float(want[0].float().abs().max()) > 0
        for on in (False, True):
            fx.fax_set_dependent_launch(sess.ctx, on)
            c.reset()
            c.run()
            assert same(c.result(), want)
        assert fx.fax_check_device_status(sess.ctx)[0] == fx.FAX_OK
    finally:
        sess.close()


def test_two_streams_at_once():
    streams, chains, want = [torch.cuda.Stream(0), torch.cuda.Stream(0)], [], []
    try:
        for st, dims in zip(streams, DIMS):
            with torch.cuda.stream(st):
                c = Chain(Session(0), *dims, np.random.default_rng(2))
                chains.append(c)
                c.run()
                want.append(c.result())
                c.reset()
        for _ in range(4):
            for c, st in zip(chains, streams):
                with torch.cuda.stream(st):
                    c.run()
            for c, w in zip(chains, want):
                assert same(c.result(), w)
                c.reset()
        assert all(fx.fax_check_device_status(c.s.ctx)[0] == fx.FAX_OK for c in chains)
    finally:
        torch.cuda.synchronize()
        for c in chains:
            c.s.close()


def test_two_graphs_replayed_at_once():
    streams, chains, want, graphs = [torch.cuda.Stream(0), torch.cuda.Stream(0)], [], [], []
    try:
        for st, dims in zip(streams, DIMS[1:]):
            with torch.cuda.stream(st):
                c = Chain(Session(0), *dims, np.random.default_rng(3))
                chains.append(c)
                c.run()
                want.append(c.result())
                g = torch.cuda.CUDAGraph()
                with torch.cuda.graph(g, stream=st):
                    c.run()
                graphs.append(g)
        for _ in range(3):
            for c in chains:
                c.reset()
            for g, st in zip(graphs, streams):
                with torch.cuda.stream(st):
                    g.replay()
            for c, w in zip(chains, want):
                assert same(c.result(), w)
    finally:
        torch.cuda.synchronize()
        graphs.clear()
        for c in chains:
            c.s.close()


def test_profile_names_the_operators():
    sess = Session(0)
    try:
        c = Chain(sess, *DIMS[0], np.random.default_rng(4))
        c.run(1)
        want = c.result()
        c.reset()
        before = sess.launches()
        fx.fax_profile_begin(sess.ctx)
        c.run(1)
        prof = fx.fax_profile_end(sess.ctx)
        assert same(c.result(), want)
        assert {k: e["launches"] for k, e in prof.items()} == {"rotary": 1, "dropout": 1, "recurrence": 2, "expert": 4}
        assert all(e["ms"] > 0 and e["bytes"] > 0 for e in prof.values()) and sess.launches() - before == 8
    finally:
        sess.close()
