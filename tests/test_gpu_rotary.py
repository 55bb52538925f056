"""Rotary positions against the 64-bit definition."""
import numpy as np
import pytest
import torch

import pieces_ref as ref
from parity_util import Session, fx, ptr
from paper_2204_06514_b200 import binding_ops as ops
from paper_2204_06514_b200.state import rotary_frequencies

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


def rotate(sess, prec, x, heads, hd, rot, layout, positions=None, first=0, seq=0, scaling=(1e4, 1.0, 0), amplitude=1.0, back=False, in_place=False, lead=0, pad=0):
    """x [rows, heads, hd] of numbers T holds.  Rows have `lead` foreign elements before and `pad` behind; checks that they stay.  Returns y."""
    rows, width = x.shape[0], heads * hd
    buf = torch.full((rows, lead + width + pad), 7.0, dtype=ref.DTYPE[prec], device=sess.device)
    buf[:, lead:lead + width] = torch.as_tensor(x.reshape(rows, width)).to(buf)
    out = buf if in_place else torch.full_like(buf, 7.0)
    pos = None if positions is None else torch.as_tensor(positions.astype(np.int32), device=sess.device)
    table = rotary_frequencies(sess.device, rot, *scaling)
    at = lambda t: t.data_ptr() + lead * t.element_size()  # noqa: E731
    ops.fax_op_rotary(sess.ctx, prec, ops.RotaryDesc(rows, heads, hd, rot, layout, at(buf), buf.stride(0), at(out), out.stride(0), ptr(pos), first, seq, ptr(table), amplitude, int(back)))
    got = out.double().cpu().numpy()
    assert (got[:, :lead] == 7).all() and (got[:, lead + width:] == 7).all()
    return got[:, lead:lead + width].reshape(rows, heads, hd)


def check(got, want, bound, prec):
    assert np.all(np.abs(got - want) <= bound + ref.UNIT[prec] * (np.abs(want) + bound) + 1e-38)


SHAPES = [  # rows, heads, head_dim, rot_dim, lead, pad
    (1, 1, 2, 2, 0, 0), (1, 24, 64, 64, 0, 768), (37, 3, 64, 32, 0, 0), (300, 5, 80, 40, 8, 16), (129, 2, 96, 96, 4, 4), (64, 7, 66, 66, 0, 0), (50, 3, 128, 20, 1, 2), (1000, 1, 256, 256, 0, 0),
    (3, 64, 128, 128, 0, 0), (2, 2, 1024, 1024, 0, 0), (5, 1, 1024, 6, 3, 0), (11, 300, 40, 40, 0, 0),
]


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("layout", [ref.HALVES, ref.PAIRS])
@pytest.mark.parametrize("shape", SHAPES)
def test_rotation_of_many_shapes(sess, shape, layout, prec):
    rows, heads, hd, rot, lead, pad = shape
    rng = np.random.default_rng(rows * 7 + hd)
    x = ref.rounded(rng.standard_normal((rows, heads, hd)), prec)
    for back, in_place in ((False, False), (True, True)):
        want, bound = ref.rotary(x, np.arange(rows) % 13 + 40, ref.frequencies(rot), rot, layout, 1.25, back)
        check(rotate(sess, prec, x, heads, hd, rot, layout, None, 40, 13, amplitude=1.25, back=back, in_place=in_place, lead=lead, pad=pad), want, bound, prec)


@pytest.mark.parametrize("scaling", [(1e4, 1.0, 0), (5e5, 8.0, 0), (1e6, 16.0, 4096)])
def test_far_positions_and_scaled_contexts(sess, scaling):
    rng = np.random.default_rng(11)
    p = np.concatenate([[0, 1, -1, 2**31 - 1, -2**31, 10**6, 123456789], rng.integers(-2**31, 2**31, 50)])
    x = rng.standard_normal((len(p), 2, 64)).astype(np.float32).astype(np.float64)
    want, bound = ref.rotary(x, p, ref.frequencies(64, *scaling), 64, ref.HALVES)
    check(rotate(sess, 1, x, 2, 64, 64, ref.HALVES, p, scaling=scaling), want, bound, 1)


def test_first_position_passes_32_bits(sess):
    x = np.random.default_rng(2).standard_normal((6, 1, 16)).astype(np.float32).astype(np.float64)
    first = 2**31 - 3
    want, bound = ref.rotary(x, first + np.arange(6), ref.frequencies(16), 16, ref.PAIRS)
    check(rotate(sess, 1, x, 1, 16, 16, ref.PAIRS, None, first, 0), want, bound, 1)


def test_gradient_is_the_transpose(sess):
    """<R x, dy> = <x, R' dy> in float, up to the roundings of both sides' elements."""
    rng = np.random.default_rng(5)
    x, dy = (rng.standard_normal((200, 4, 64)).astype(np.float32).astype(np.float64) for _ in range(2))
    p = rng.integers(0, 10**5, 200)
    y = rotate(sess, 1, x, 4, 64, 48, ref.PAIRS, p, amplitude=1.2)
    dx = rotate(sess, 1, dy, 4, 64, 48, ref.PAIRS, p, amplitude=1.2, back=True)
    _, by = ref.rotary(x, p, ref.frequencies(48), 48, ref.PAIRS, 1.2)
    _, bx = ref.rotary(dy, p, ref.frequencies(48), 48, ref.PAIRS, 1.2, back=True)
    slack = np.sum((by + ref.F32 * np.abs(y)) * np.abs(dy)) + np.sum((bx + ref.F32 * np.abs(dx)) * np.abs(x))
    assert abs(np.sum(y * dy) - np.sum(x * dx)) <= slack


def test_values_that_are_not_finite_stay_in_their_pair(sess):
    x = np.ones((4, 2, 32))
    x[1, 0, 3], x[2, 1, 20] = np.nan, np.inf
    y = rotate(sess, 0, x, 2, 32, 32, ref.HALVES, np.array([0, 5, 6, 7]))
    bad = ~np.isfinite(y)
    assert sorted(zip(*np.nonzero(bad))) == [(1, 0, 3), (1, 0, 19), (2, 1, 4), (2, 1, 20)]


def test_rows_behind_two_to_the_31_elements(sess):
    rows, pitch, width = 140000, 16000, 64
    x = torch.zeros((rows, pitch), dtype=torch.bfloat16, device=sess.device)
    v = torch.randn((rows, width), device=sess.device).to(torch.bfloat16)
    x[:, 100:100 + width] = v
    table = rotary_frequencies(sess.device, 64)
    ops.fax_op_rotary(sess.ctx, 0, ops.RotaryDesc(rows, 1, 64, 64, 0, x.data_ptr() + 200, pitch, x.data_ptr() + 200, pitch, None, 0, 0, ptr(table), 1.0, 0))
    last = slice(rows - 50, rows)
    want, bound = ref.rotary(v[last].double().cpu().numpy().reshape(50, 1, 64), np.arange(rows)[last], ref.frequencies(64), 64, ref.HALVES)
    check(x[last, 100:164].double().cpu().numpy().reshape(50, 1, 64), want, bound, 0)
    assert float(x[:, :100].abs().max()) == 0 and float(x[:, 164:300].abs().max()) == 0


@pytest.mark.parametrize("layout", [ref.HALVES, ref.PAIRS])
@pytest.mark.parametrize("pitches", [(128, 200), (131, 128), (136, 129)])
def test_pitches_of_their_own(sess, pitches, layout):
    """x and y with pitches (and so alignments) that differ, the rest of a head copied."""
    rng = np.random.default_rng(6)
    x = ref.rounded(rng.standard_normal((77, 2, 64)), 0)
    bx, by = (torch.full((77, p), 7.0, dtype=torch.bfloat16, device=sess.device) for p in pitches)
    bx[:, :128] = torch.as_tensor(x.reshape(77, 128)).to(bx)
    table = rotary_frequencies(sess.device, 32)
    ops.fax_op_rotary(sess.ctx, 0, ops.RotaryDesc(77, 2, 64, 32, layout, ptr(bx), pitches[0], ptr(by), pitches[1], None, 3, 0, ptr(table), 0.5, 0))
    want, bound = ref.rotary(x, 3 + np.arange(77), ref.frequencies(32), 32, layout, 0.5)
    check(by[:, :128].double().cpu().numpy().reshape(77, 2, 64), want, bound, 0)
    assert bool((by[:, 128:] == 7).all()) and np.array_equal(by[:, :128].double().cpu().numpy().reshape(77, 2, 64)[..., 32:], x[..., 32:])


def test_more_pairs_than_31_bits_count(sess):
    """2^29 rows of four pairs, single elements because the rows begin at odd ones: several launches, one count of positions."""
    rows, dev = 2**29 + 100, sess.device
    buf = torch.zeros(rows * 8 + 1, dtype=torch.bfloat16, device=dev)
    x = buf[1:].view(rows, 8)
    spots = torch.tensor([0, 1, 2**29 - 64 - 1, 2**29 - 64, 2**29 - 1, 2**29 + 99], device=dev)
    v = torch.randn((len(spots), 8), device=dev).to(torch.bfloat16)
    x[spots] = v
    table = rotary_frequencies(dev, 8)
    for seq in (0, 1000):
        x[spots] = v
        ops.fax_op_rotary(sess.ctx, 0, ops.RotaryDesc(rows, 1, 8, 8, 0, x.data_ptr(), 8, x.data_ptr(), 8, None, 5, seq, ptr(table), 1.0, 0))
        p = spots.cpu().numpy()
        want, bound = ref.rotary(v.double().cpu().numpy().reshape(-1, 1, 8), 5 + (p % seq if seq else p), ref.frequencies(8), 8, ref.HALVES)
        check(x[spots].double().cpu().numpy().reshape(-1, 1, 8), want, bound, 0)
        assert float(x[2**29 - 5000:2**29 - 100].abs().max()) == 0
