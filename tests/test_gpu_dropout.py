"""Dropout: its mask bit for bit, its values against 64 bits."""
import numpy as np
import pytest
import torch

import pieces_ref as ref
from parity_util import Session, fx, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu
SEED, OFFSET = 0x0123456789ABCDEF, 0xFEDCBA9876543210


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


def drop(sess, prec, x, resid, p, seed=SEED, offset=OFFSET, pads=(0, 0, 0), alias=None, offset_device=None):
    """x, resid [rows, cols] as T holds them; pads: foreign columns behind x, resid and y, which have to stay.  alias: y is "x" or "resid"."""
    rows, cols = x.shape
    bufs = []
    for a, pad in zip((x, resid, np.full_like(x, 7.0)), pads):
        b = torch.full((rows, cols + pad), 7.0, dtype=ref.DTYPE[prec], device=sess.device)
        b[:, :cols] = torch.as_tensor(a if a is not None else np.zeros_like(x)).to(b)
        bufs.append(b)
    bx, br, by = bufs
    by = {"x": bx, "resid": br}.get(alias, by)
    r = br if resid is not None else None
    ops.fax_op_dropout(sess.ctx, prec, ops.DropoutDesc(rows, cols, ptr(bx), bx.stride(0), ptr(r), br.stride(0), ptr(by), by.stride(0), p, seed, offset, ptr(offset_device)))
    got = by.double().cpu().numpy()
    assert (got[:, cols:] == 7).all()
    return got[:, :cols]


def check(got, x, resid, p, prec, seed=SEED, offset=OFFSET):
    keep, scale = ref.kept(*x.shape, p, seed, offset)
    want = np.where(keep, x * scale, 0.0)
    # the scale's rounding and the fused product and sum's, then T's
    bound = ref.F32 * np.abs(want)
    if resid is not None:
        want = want + resid
        bound = bound + ref.F32 * np.abs(want)
    assert np.all(np.abs(got - want) <= bound + ref.UNIT[prec] * (np.abs(want) + bound))
    if resid is None:
        assert np.all((got == 0) | keep)
    return keep


SHAPES = [(1, 1, (0, 0, 0)), (1, 8, (0, 0, 0)), (3, 7, (0, 0, 0)), (100, 250, (0, 0, 0)), (33, 768, (8, 16, 8)), (70, 64, (3, 0, 1)), (257, 33, (7, 15, 23)), (2, 5000, (0, 0, 0)), (2000, 16, (0, 0, 0)),
          (129, 20, (4, 4, 4)), (1, 100003, (0, 0, 0))]


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("shape", SHAPES)
def test_values_and_mask(sess, shape, prec):
    rows, cols, pads = shape
    rng = np.random.default_rng(cols)
    x, r = (ref.rounded(rng.standard_normal((rows, cols)), prec) for _ in range(2))
    for p, resid, alias in ((0.1, r, None), (0.5, None, None), (0.25, r, "resid"), (0.3, None, "x"), (0.4, r, "x")):
        check(drop(sess, prec, x, resid, p, pads=pads, alias=alias), x, resid, p, prec)


@pytest.mark.parametrize("p", [0.0, 1.0, 2.0 ** -16, 1e-6, 1 - 2.0 ** -16, 0.9999999])
def test_extreme_probabilities(sess, p):
    x = np.ones((50, 4096))
    got = drop(sess, 1, x, None, p)
    keep = check(got, x, None, p, 1)
    if p == 0.0 or p == 1e-6:
        assert keep.all() and np.array_equal(got, x)
    if p in (1.0, 0.9999999):
        assert not keep.any()
        r = np.random.default_rng(0).standard_normal((50, 4096)).astype(np.float32).astype(np.float64)
        assert np.array_equal(drop(sess, 1, x, r, p), r)


def test_dropped_elements_are_not_looked_at(sess):
    rng = np.random.default_rng(1)
    x = rng.choice([np.nan, np.inf, -np.inf], (40, 96))
    keep, _ = ref.kept(40, 96, 0.5, SEED, OFFSET)
    for resid in (None, np.full((40, 96), 3.0)):
        got = drop(sess, 0, x, resid, 0.5)
        assert np.all(got[~keep] == (0.0 if resid is None else 3.0)) and not np.isfinite(got[keep]).any()


def test_offsets_and_seeds_draw_anew(sess):
    x = np.ones((64, 512))
    masks = [drop(sess, 1, x, None, 0.5, s, o) != 0 for s, o in ((1, 0), (1, 1), (1, 2**32), (2, 0), (1 + 2**32, 0))]
    for i, a in enumerate(masks):
        for b in masks[:i]:
            # 32768 fair coins agree: 0.5 +- 6 standard deviations of 0.0028
            assert abs(np.mean(a == b) - 0.5) < 0.017
    assert np.array_equal(masks[0], drop(sess, 1, x, None, 0.5, 1, 0) != 0)


def test_share_that_is_kept(sess):
    n = 1024 * 4096
    for p in (0.1, 0.37):
        share = float(np.mean(drop(sess, 1, np.ones((1024, 4096)), None, p) != 0))
        assert abs(share - (1 - p)) < 6 * np.sqrt(p * (1 - p) / n) + 2.0 ** -17


def test_offset_on_the_device_is_added_when_the_kernel_runs(sess):
    """A captured call draws anew at each replay, as the eager calls with these offsets do."""
    x = np.ones((20, 128))
    add = torch.tensor([5], dtype=torch.int64, device=sess.device)
    assert np.array_equal(drop(sess, 0, x, None, 0.5, 9, 2**64 - 3, offset_device=add), drop(sess, 0, x, None, 0.5, 9, 2))
    side = torch.cuda.Stream()
    with torch.cuda.stream(side):
        s2 = Session(0)
    try:
        bx = torch.ones((20, 128), dtype=torch.bfloat16, device=sess.device)
        by = torch.empty_like(bx)
        desc = ops.DropoutDesc(20, 128, ptr(bx), 128, None, 0, ptr(by), 128, 0.5, 9, 100, ptr(add))
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=side):
            ops.fax_op_dropout(s2.ctx, 0, desc)
            add.add_(1)
        for k in range(3):
            add_now = int(add.item())
            graph.replay()
            torch.cuda.synchronize()
            assert np.array_equal(by.double().cpu().numpy(), drop(sess, 0, x, None, 0.5, 9, 100 + add_now))
        del graph
    finally:
        s2.close()


def test_gradient_is_the_same_mask(sess):
    """dx of sum(dy * y): the forward call's kept elements, scaled."""
    rng = np.random.default_rng(8)
    x, dy, r = (ref.rounded(rng.standard_normal((31, 72)), 1) for _ in range(3))
    y = drop(sess, 1, x, r, 0.2)
    step = ref.rounded(x + 0.25, 1)
    dx = drop(sess, 1, dy, None, 0.2)
    # y is linear in x: the quotient of differences is dx / dy but for roundings of y (|y| < 8, twice 2^-24 of it over a step of 0.25)
    slope = (drop(sess, 1, step, r, 0.2) - y) / (step - x)
    assert np.all(np.abs(slope * dy - dx) <= np.abs(dy) * 2 * 8 * ref.F32 / 0.25 + 4 * ref.F32 * np.abs(dx))


def test_rows_behind_two_to_the_31_elements(sess):
    rows, cols, pitch = 140000, 16, 16000
    x = torch.ones((rows, pitch), dtype=torch.bfloat16, device=sess.device)
    ops.fax_op_dropout(sess.ctx, 0, ops.DropoutDesc(rows, cols, ptr(x), pitch, None, 0, ptr(x), pitch, 0.5, 3, 4, None))
    keep, _ = ref.kept(rows, cols, 0.5, 3, 4)
    assert np.array_equal(x[:, :cols].float().cpu().numpy(), np.where(keep, 2.0, 0.0)) and bool((x[:, cols:cols + 64] == 1).all())
