"""The gated recurrence, forward and backward, against the 64-bit definition token by token."""
import numpy as np
import pytest
import torch

import pieces_ref as ref
from parity_util import Session, fx, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


class Layer:
    """Inputs of one call on the device, as columns of a fused buffer or by themselves."""

    def __init__(self, sess, prec, lengths, d, gated, mode, seed, fused=False, pad=0, rows=None, uniform=False, h0=True, dh_last=True):
        rng = np.random.default_rng(seed)
        self.sess, self.prec, self.d, self.mode, self.gated, self.uniform = sess, prec, d, mode, gated, uniform
        self.at = np.concatenate([[0], np.cumsum(lengths)]).astype(np.int64)
        self.n_seq, self.seq = len(lengths), int(max(lengths, default=0))
        self.rows = int(self.at[-1]) if rows is None else rows
        t, dev, n = ref.DTYPE[prec], sess.device, 2 + gated
        vals = [ref.rounded(rng.standard_normal((self.rows, d)), prec) for _ in range(4)]
        vals[0] = ref.rounded(vals[0] + rng.uniform(-1, 7, d), prec)
        self.f, self.x, self.g, self.dy = vals
        width = n * d if fused else d

        def place(values, copy=True):
            if fused:
                buf = torch.full((self.rows, width + pad), 7.0, dtype=t, device=dev)
                views = [buf[:, i * d:(i + 1) * d] for i in range(n)]
            else:
                views = [torch.full((self.rows, d + pad), 7.0, dtype=t, device=dev)[:, :d] for _ in range(n)]
            if copy:
                for v, a in zip(views, values):
                    v.copy_(torch.as_tensor(a))
            return views + [None] * (3 - n)
        self.tf, self.tx, self.tg = place(vals)
        self.df, self.dx, self.dg = place(vals, copy=False)
        self.y = torch.full((self.rows, d), 7.0, dtype=t, device=dev)
        self.tdy = torch.as_tensor(self.dy).to(t).to(dev)
        f32 = lambda a: torch.as_tensor(a).float().to(dev)  # noqa: E731
        self.h0 = rng.standard_normal((self.n_seq, d)).astype(np.float32).astype(np.float64) if h0 else np.zeros((self.n_seq, d))
        self.dh_last = rng.standard_normal((self.n_seq, d)).astype(np.float32).astype(np.float64) if dh_last else np.zeros((self.n_seq, d))
        self.th0, self.tdh_last = f32(self.h0) if h0 else None, f32(self.dh_last) if dh_last else None
        self.h_last, self.dh0 = (torch.full((self.n_seq, d), 7.0, device=dev) for _ in range(2))
        self.offsets = None if uniform else torch.as_tensor(self.at.astype(np.int32), device=dev)
        self.states = torch.full((ops.fax_op_recurrence_states_floats(self.rows, self.n_seq, d),), 7.0, device=dev)

    def shape(self):
        ld = lambda t: t.stride(0) if t is not None else 0  # noqa: E731
        return (self.rows, self.d, self.n_seq, self.seq, ptr(self.offsets), self.mode, ptr(self.tf), ld(self.tf), ptr(self.tx), ld(self.tx), ptr(self.tg), ld(self.tg), ptr(self.th0))

    def forward(self, keep=True):
        ops.fax_op_recurrence_forward(self.sess.ctx, self.prec, ops.RecurrenceDesc(*self.shape(), ptr(self.y), self.y.stride(0), ptr(self.h_last), ptr(self.states) if keep else None))

    def backward(self):
        ld = lambda t: t.stride(0) if t is not None else 0  # noqa: E731
        ops.fax_op_recurrence_backward(self.sess.ctx, self.prec, ops.RecurrenceBackwardDesc(
            *self.shape(), ptr(self.states), ptr(self.tdy), ld(self.tdy), ptr(self.tdh_last), ptr(self.df), ld(self.df), ptr(self.dx), ld(self.dx), ptr(self.dg), ld(self.dg), ptr(self.dh0)))

    def reference(self):
        g = self.g if self.gated else None
        fwd = ref.recurrence(self.f, self.x, g, self.h0, self.at, self.mode)
        return fwd, ref.recurrence_backward(self.f, self.x, g, self.h0, self.at, self.mode, self.dy, self.dh_last, fwd)

    def check(self, backward=True):
        fwd, grads = self.reference()
        live, u = int(self.at[-1]), ref.UNIT[self.prec]
        num = lambda t: t.double().cpu().numpy()  # noqa: E731

        def near(name, got, want, bound, unit):
            # (2^-126: what float flushes)
            bad = ~(np.abs(got - want) <= bound + unit * (np.abs(want) + bound) + 2.0 ** -126)
            assert not bad.any(), (name, int(bad.sum()), np.argwhere(bad)[0], got[bad][0], want[bad][0])
        near("y", num(self.y)[:live], fwd["y"][:live], fwd["e_y"][:live], u)
        assert (num(self.y)[live:] == 7).all()
        last = np.zeros_like(self.h0)
        for s in range(self.n_seq):
            if self.at[s + 1] > self.at[s]:
                last[s] = fwd["e_h"][self.at[s + 1] - 1]
        near("h_last", num(self.h_last), fwd["h_last"], last, ref.F32)
        if backward:
            for name, t in (("df", self.df), ("dx", self.dx), ("dg", self.dg)):
                if t is not None:
                    near(name, num(t)[:live], grads[name][0][:live], grads[name][1][:live], u)
                    assert (num(t)[live:] == 7).all()
            near("dh0", num(self.dh0), *grads["dh0"], ref.F32)


LENGTHS = {"one token": [1], "tokens of many": [1] * 70, "a stretch": [16, 16], "a stretch and one": [17], "one CTA": [128, 100], "one CTA, two rounds' worth": [129], "clusters": [500, 300, 1000],
           "rounds of a cluster": [2500], "ragged": [0, 1, 37, 0, 16, 300, 15, 33, 0], "all empty": [0, 0, 0], "many short": [3, 0, 9, 16, 1] * 60}


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("gated,mode", [(False, ref.PLAIN), (True, ref.PLAIN), (False, ref.COMPLEMENT), (True, ref.COMPLEMENT)])
@pytest.mark.parametrize("lengths", list(LENGTHS))
def test_sequences(sess, lengths, gated, mode, prec):
    n = LENGTHS[lengths]
    # rows in boxes (72 and 136: pitches of whole 16 bytes, a last tile of 8 channels), pairs or single channels (70, 33)
    for d, fused, pad in ((70, True, 0), (33, False, 3), (72, True, 0), (136, False, 8)):
        layer = Layer(sess, prec, n, d, gated, mode, len(n) + d, fused=fused, pad=pad, uniform=len(set(n)) == 1 and fused, rows=None if fused else sum(n) + 5)
        if layer.uniform:
            layer.rows = layer.n_seq * layer.seq
        layer.forward()
        layer.backward()
        layer.check()


@pytest.mark.parametrize("d,pad", [(1, 0), (2, 0), (31, 1), (64, 64), (65, 0), (128, 2), (200, 1)])
def test_widths_and_pitches(sess, d, pad):
    for fused in (False, True):
        layer = Layer(sess, 0, [40, 200], d, True, ref.COMPLEMENT, d, fused=fused, pad=pad)
        layer.forward()
        layer.backward()
        layer.check()


def test_channels_and_sequences_that_fill_the_gpu(sess):
    """So many that each warp takes a whole sequence; long ones among short ones."""
    rng = np.random.default_rng(0)
    layer = Layer(sess, 0, list(rng.integers(0, 60, 640)), 130, True, ref.COMPLEMENT, 1)
    layer.forward()
    layer.backward()
    layer.check()


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("lengths", [[1] * 40, [2, 0, 1, 2, 0], [1]])
def test_a_token_or_two(sess, lengths, prec):
    """Widths of whole 16-byte vectors and others, sequences of 0 to 2 tokens, and longer ones than the caller says."""
    for d, gated, mode, uniform in ((64, True, ref.COMPLEMENT, True), (8, False, ref.PLAIN, False), (24, True, ref.PLAIN, False), (1032, False, ref.COMPLEMENT, False), (12, True, ref.COMPLEMENT, True)):
        layer = Layer(sess, prec, lengths, d, gated, mode, d, uniform=uniform and len(set(lengths)) == 1)
        layer.forward()
        layer.backward()
        layer.check()
    layer = Layer(sess, prec, [40, 17], 64, True, ref.COMPLEMENT, 5)
    layer.seq = 1
    layer.forward()
    layer.backward()
    layer.check()


def test_without_states_gate_or_initial_values(sess):
    layer = Layer(sess, 0, [100, 50], 64, False, ref.PLAIN, 2, h0=False, dh_last=False)
    layer.forward(keep=False)
    assert bool((layer.states == 7).all())
    y = layer.y.clone()
    layer.forward()
    assert torch.equal(y, layer.y)
    layer.backward()
    layer.check()


@pytest.mark.parametrize("prec", [0, 1])
def test_a_sequence_continued(sess, prec):
    """In pieces, a token at a time too, with the state handed on in place: the state as in one call, but for its roundings."""
    whole = Layer(sess, prec, [150], 48, True, ref.COMPLEMENT, 4)
    whole.forward()
    state = whole.th0.clone()
    y = torch.empty_like(whole.y)
    e = whole.y.element_size() * 48
    at = 0
    for n in [1, 1, 1, 17, 100, 1, 29]:
        off = lambda t: t.data_ptr() + at * e  # noqa: E731
        ops.fax_op_recurrence_forward(sess.ctx, prec, ops.RecurrenceDesc(n, 48, 1, n, None, 1, off(whole.tf), 48, off(whole.tx), 48, off(whole.tg), 48, ptr(state), off(y), 48, ptr(state), None))
        at += n
    whole.y, whole.h_last = y, state
    whole.check(backward=False)


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("d", [64, 65])
@pytest.mark.parametrize("said", [0, 1, 16, 17, 20, 100000])
def test_the_longest_length_is_only_a_hint(sess, d, said, prec):
    layer = Layer(sess, prec, [300, 5, 700], d, True, ref.COMPLEMENT, 17)
    layer.seq = said
    layer.forward()
    layer.backward()
    layer.check()


@pytest.mark.parametrize("d", [64, 63])
def test_what_lies_behind_a_sequence_is_not_looked_at(sess, d):
    """A sequence's last rows share boxes with its neighbour's: NaN there, and in rows of no sequence, change nothing."""
    clean, dirty = (Layer(sess, 0, [37, 16, 40], d, True, ref.PLAIN, 18, rows=100) for _ in range(2))
    for t in (dirty.tf, dirty.tx, dirty.tg, dirty.tdy):
        t[37:53] = float("nan")
        t[93:] = float("nan")
    for layer in (clean, dirty):
        layer.forward()
        layer.backward()
    for a, b in ((clean.y, dirty.y), (clean.df, dirty.df), (clean.dx, dirty.dx), (clean.dg, dirty.dg)):
        assert torch.equal(a[:37], b[:37]) and torch.equal(a[53:93], b[53:93]) and bool((b[93:] == 7).all())


def test_gradients_in_place_of_their_inputs(sess):
    a, b = (Layer(sess, 0, [300, 20], 64, True, ref.COMPLEMENT, 6, fused=True) for _ in range(2))
    a.forward()
    a.backward()
    b.forward()
    b.df, b.dx, b.dg = b.tf, b.tx, b.tg
    b.dh0 = b.tdh_last
    b.backward()
    for x, y in ((a.df, b.df), (a.dx, b.dx), (a.dg, b.dg), (a.dh0, b.dh0)):
        assert torch.equal(x, y)


@pytest.mark.parametrize("d", [64, 63, 129])
def test_states_in_place_where_a_cluster_shares_a_sequence(sess, d):
    """h_last in the place of h0, dh0 in that of dh_last, with many CTAs a sequence, a short and an empty sequence among them."""
    for seed in range(4):
        a, b = (Layer(sess, 0, [5000, 3, 0, 2100], d, True, ref.COMPLEMENT, 30 + seed) for _ in range(2))
        b.h_last, b.dh0 = b.th0, b.tdh_last
        for layer in (a, b):
            layer.forward()
            layer.backward()
        for x, y in ((a.y, b.y), (a.h_last, b.h_last), (a.df, b.df), (a.dx, b.dx), (a.dg, b.dg), (a.dh0, b.dh0)):
            assert torch.equal(x, y)


@pytest.mark.parametrize("value", [np.nan, np.inf, -np.inf])
@pytest.mark.parametrize("d", [66, 64])
@pytest.mark.parametrize("prec", [0, 1])
def test_values_that_are_not_finite_stay_in_their_sequence_and_channel(sess, value, d, prec):
    for name in ("f", "x", "g"):
        clean, dirty = (Layer(sess, prec, [200, 40, 1], d, True, ref.COMPLEMENT, 9) for _ in range(2))
        getattr(dirty, "t" + name)[90, 5] = value
        for layer in (clean, dirty):
            layer.forward()
            layer.backward()
        for x, y in ((clean.y, dirty.y), (clean.df, dirty.df), (clean.dx, dirty.dx), (clean.dg, dirty.dg)):
            x[:200, 5] = 0
            y[:200, 5] = 0
            assert torch.equal(x, y)
        clean.h_last[0, 5] = dirty.h_last[0, 5] = 0
        assert torch.equal(clean.h_last, dirty.h_last)


def test_gates_that_are_shut_or_open(sess):
    """f of +-inf and of +-1000: a is exactly 1 or 0; with a = 0 the state before is forgotten, with a = 1 kept."""
    layer = Layer(sess, 1, [40], 8, False, ref.COMPLEMENT, 3)
    f = np.zeros((40, 8))
    f[:, 0:2], f[:, 2:4], f[:, 4], f[:, 5] = 1000.0, -1000.0, np.inf, -np.inf
    layer.f = f
    layer.tf.copy_(torch.as_tensor(f))
    layer.forward()
    y = layer.y.double().cpu().numpy()
    for c in (0, 1, 4):
        assert np.array_equal(y[:, c], np.full(40, layer.h0[0, c]))
    for c in (2, 3, 5):
        assert np.array_equal(y[:, c], layer.x[:, c])


def test_offsets_out_of_range_touch_nothing_else(sess):
    """Offsets beyond the rows, negative ones and falling ones are cut off, as documented."""
    layer = Layer(sess, 0, [20, 30, 10], 64, True, ref.PLAIN, 12)
    good = layer.at.copy()
    layer.offsets = torch.tensor([-5, 20, 10, 10**9], dtype=torch.int32, device=sess.device)
    layer.at = np.array([0, 20, 10, 60])
    layer.forward()
    layer.backward()
    assert good[-1] == 60
    # sequence 0: rows 0 to 19, 1: none, 2: rows 10 to 59 (which overlaps 0 in the outputs' rows 10 to 19)
    assert torch.equal(layer.h_last[1], layer.th0[1]) and torch.equal(layer.dh0[1], layer.tdh_last[1])
    alone = Layer(sess, 0, [20, 30, 10], 64, True, ref.PLAIN, 12)
    alone.offsets = torch.tensor([0, 20, 20, 20], dtype=torch.int32, device=sess.device)
    alone.forward()
    assert torch.equal(alone.y[:10], layer.y[:10]) and bool((alone.y[20:] == 7).all())
    assert torch.equal(alone.h_last[0], layer.h_last[0])


def test_the_same_bits_every_time(sess):
    layer = Layer(sess, 0, [3000, 700], 128, True, ref.COMPLEMENT, 13)
    layer.forward()
    layer.backward()
    first = [t.clone() for t in (layer.y, layer.df, layer.dx, layer.dg, layer.dh0, layer.h_last)]
    for _ in range(5):
        layer.forward()
        layer.backward()
        for a, b in zip(first, (layer.y, layer.df, layer.dx, layer.dg, layer.dh0, layer.h_last)):
            assert torch.equal(a, b)


def test_rows_behind_two_to_the_31_elements(sess):
    rows, pitch, d = 140000, 16000, 64
    dev = sess.device
    small = Layer(sess, 0, [45], d, False, ref.COMPLEMENT, 14)
    small.forward()
    small.backward()
    bufs = [torch.zeros((rows, pitch), dtype=torch.bfloat16, device=dev) for _ in range(3)]
    lo = rows - 45
    for b, t in zip(bufs, (small.tf, small.tx, small.tdy)):
        b[lo:, :d] = t
    off = torch.tensor([lo, rows], dtype=torch.int32, device=dev)
    states = torch.empty(ops.fax_op_recurrence_states_floats(rows, 1, d), device=dev)
    h_last, dh0 = torch.empty((1, d), device=dev), torch.empty((1, d), device=dev)
    y = torch.zeros((rows, pitch), dtype=torch.bfloat16, device=dev)
    shape = (rows, d, 1, 45, ptr(off), 1, ptr(bufs[0]), pitch, ptr(bufs[1]), pitch, None, 0, ptr(small.th0))
    ops.fax_op_recurrence_forward(sess.ctx, 0, ops.RecurrenceDesc(*shape, ptr(y), pitch, ptr(h_last), ptr(states)))
    assert torch.equal(y[lo:, :d], small.y) and torch.equal(h_last, small.h_last)
    # df over f, dx into y
    ops.fax_op_recurrence_backward(sess.ctx, 0, ops.RecurrenceBackwardDesc(*shape, ptr(states), ptr(bufs[2]), pitch, ptr(small.tdh_last), ptr(bufs[0]), pitch, ptr(y), pitch, None, 0, ptr(dh0)))
    assert torch.equal(bufs[0][lo:, :d], small.df) and torch.equal(y[lo:, :d], small.dx) and torch.equal(dh0, small.dh0)
    assert float(y[:lo, :d].abs().max()) == 0 and float(y[:, d:d + 64].abs().max()) == 0


@pytest.mark.parametrize("d", [64, 40, 31])
def test_pitches_of_their_own(sess, d):
    """Every matrix with a pitch of its own, whole 16 bytes or not: the same bits as without gaps where the rows come in alike, values in the bounds everywhere."""
    for pads in ([8, 16, 24, 32, 40, 8, 16, 48], [1, 2, 3, 4, 5, 6, 7, 9]):
        layer = Layer(sess, 0, [50, 0, 130], d, True, ref.COMPLEMENT, 21)
        t = {}
        for i, name in enumerate(("tf", "tx", "tg", "tdy", "y", "df", "dx", "dg")):
            old = getattr(layer, name)
            wide = torch.full((old.shape[0], d + pads[i]), 7.0, dtype=old.dtype, device=sess.device)
            wide[:, :d] = old
            t[name] = wide
            setattr(layer, name, wide[:, :d])
        layer.forward()
        layer.backward()
        layer.check()
        for name, wide in t.items():
            assert bool((wide[:, d:] == 7).all()), name


def test_nothing_to_do(sess):
    """No rows: the states pass through; no sequences: nothing is touched."""
    for prec in (0, 1):
        layer = Layer(sess, prec, [0, 0], 24, True, ref.PLAIN, 3)
        layer.forward()
        layer.backward()
        assert torch.equal(layer.h_last, layer.th0) and torch.equal(layer.dh0, layer.tdh_last)
        ops.fax_op_recurrence_forward(sess.ctx, prec, ops.RecurrenceDesc(0, 24, 0, 0, None, 0, None, 24, None, 24, None, 0, None, None, 24, None, None))
