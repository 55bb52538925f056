"""Tokens to their experts and back: the plan exactly, the rows against 64 bits."""
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


def sort(sess, ids, n_experts, capacity=0, align=1, extra=0):
    n, k = ids.shape
    slots = ops.fax_op_expert_slots(n, k, n_experts, capacity, align) + extra
    new = lambda *shape: torch.full(shape, 12345, dtype=torch.int32, device=sess.device)  # noqa: E731
    slot_of, source, offsets, counts = new(n, k), new(slots), new(n_experts + 1), new(n_experts)
    t = torch.as_tensor(ids.astype(np.int32), device=sess.device)
    ops.fax_op_expert_sort(sess.ctx, ops.ExpertSortDesc(n, k, n_experts, capacity, align, slots, ptr(t), ptr(slot_of), ptr(source), ptr(offsets), ptr(counts)))
    return slot_of, source, offsets, counts


def choices(rng, n, k, e, pad=0.1):
    ids = rng.zipf(1.3, (n, k)) % e
    ids[rng.random((n, k)) < pad] = -1
    return ids


PLANS = [  # tokens, choices, experts, capacity, align, more slots
    (1, 1, 1, 0, 1, 0), (1, 2, 8, 0, 128, 0), (5, 3, 2, 2, 1, 3), (100, 1, 1024, 0, 16, 0), (333, 2, 8, 40, 1, 0), (2048, 2, 8, 0, 128, 0), (2049, 2, 7, 0, 1, 100), (5000, 8, 64, 0, 128, 0),
    (16384, 2, 8, 5120, 1, 0), (9999, 3, 1024, 11, 1, 5), (4097, 1, 1, 0, 7, 0), (60001, 4, 256, 0, 64, 0), (0, 2, 4, 0, 8, 0), (0, 2, 4, 3, 1, 2),
]


@pytest.mark.parametrize("plan", PLANS)
def test_plan(sess, plan):
    n, k, e, capacity, align, extra = plan
    ids = choices(np.random.default_rng(n), n, k, e)
    if n > 10:
        ids[3], ids[4] = e, -2**31                      # outside, from either end
    got = sort(sess, ids, e, capacity, align, extra)
    for g, w in zip(got, ref.expert_plan(ids, e, capacity, align, got[1].numel())):
        assert np.array_equal(g.cpu().numpy(), w)


@pytest.mark.parametrize("n,k,e", [(3000, 2, 5), (40000, 1, 3)])
def test_all_tokens_to_one_expert_or_to_none(sess, n, k, e):
    for value in (e - 1, 0, -1):
        for capacity in (0, 100, n * k):
            ids = np.full((n, k), value)
            got = sort(sess, ids, e, capacity, 1)
            for g, w in zip(got, ref.expert_plan(ids, e, capacity, 1, got[1].numel())):
                assert np.array_equal(g.cpu().numpy(), w)


def test_a_capacity_of_two_to_the_30(sess):
    got = sort(sess, np.zeros((26, 1), dtype=np.int64), 1, 1 << 30)
    assert int(got[2][1]) == 1 << 30 and int(got[3][0]) == 26
    assert torch.equal(got[1][:26].cpu(), torch.arange(26, dtype=torch.int32)) and bool((got[1][26:] == -1).all())


def pitched(sess, a, prec, pad):
    b = torch.full((a.shape[0], a.shape[1] + pad), 7.0, dtype=ref.DTYPE[prec], device=sess.device)
    b[:, :a.shape[1]] = torch.as_tensor(a).to(b)
    return b


ROWS = [  # tokens, choices, experts, capacity, align, width, pitch's rest
    (1, 1, 1, 0, 1, 1, 0), (7, 2, 4, 0, 16, 64, 0), (16, 2, 8, 0, 1, 4096, 0), (100, 3, 5, 30, 1, 40, 8), (50, 8, 9, 0, 1, 33, 0), (2000, 2, 8, 400, 1, 24, 3), (30, 11, 16, 0, 4, 300, 4), (9, 20, 32, 0, 1, 2056, 0),
    (1300, 1, 3, 0, 128, 272, 0),
]


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("case", ROWS)
def test_rows_there_and_back(sess, case, prec):
    n, k, e, capacity, align, d, pad = case
    rng = np.random.default_rng(n + d)
    ids = choices(rng, n, k, e)
    slot_t, source_t, _, _ = sort(sess, ids, e, capacity, align, 2)
    slots = source_t.numel()
    slot_of, source = slot_t.cpu().numpy(), source_t.cpu().numpy()
    data = lambda rows: ref.rounded(rng.standard_normal((rows, d)), prec)  # noqa: E731
    x, z, resid, dy, w = data(n), data(slots), data(n), data(n), rng.standard_normal((n, k)).astype(np.float32).astype(np.float64)
    empty = source < 0
    z[empty] = np.nan                                   # empty slots are nobody's
    tx, tz, tr, tdy = (pitched(sess, a, prec, pad) for a in (x, z, resid, dy))
    tw = torch.as_tensor(w).float().to(sess.device)
    num = lambda t: t.double().cpu().numpy()  # noqa: E731
    u = ref.UNIT[prec]

    def near(t, want, bound):
        got = num(t)
        assert (got[:, d:] == 7).all()
        assert np.all(np.abs(got[:, :d] - want) <= bound + u * (np.abs(want) + bound))

    out = pitched(sess, np.full((slots, d), 7.0), prec, pad)
    ops.fax_op_expert_dispatch(sess.ctx, prec, ops.ExpertDispatchDesc(n, k, d, slots, ptr(slot_t), ptr(source_t), ptr(tx), d + pad, ptr(out), d + pad))
    near(out, np.where(empty[:, None], 0.0, x[np.maximum(source, 0) // k]), 0.0)

    y = pitched(sess, np.full((n, d), 7.0), prec, pad)
    for weights, r in ((w, resid), (None, None), (w, None), (None, resid)):
        ops.fax_op_expert_combine(sess.ctx, prec, ops.ExpertCombineDesc(n, k, d, slots, ptr(slot_t), ptr(tw) if weights is not None else None, ptr(tz), d + pad,
                                                                       ptr(tr) if r is not None else None, d + pad if r is not None else 0, ptr(y), d + pad))
        near(y, *ref.combine(slot_of, weights, z, r))
    ops.fax_op_expert_combine(sess.ctx, prec, ops.ExpertCombineDesc(n, k, d, slots, ptr(slot_t), ptr(tw), ptr(tz), d + pad, ptr(tr), d + pad, ptr(tr), d + pad))
    near(tr, *ref.combine(slot_of, w, z, resid))

    want_dz = np.zeros((slots, d))
    want_dz[~empty] = w.reshape(-1)[source[~empty]][:, None] * dy[source[~empty] // k]
    want_dw, size = np.zeros(n * k), np.zeros(n * k)
    prods = z[~empty] * dy[source[~empty] // k]
    want_dw[source[~empty]], size[source[~empty]] = prods.sum(1), np.abs(prods).sum(1)
    for dw in (True, False):
        dz, tdw = pitched(sess, np.full((slots, d), 7.0), prec, pad), torch.full((n, k), 7.0, device=sess.device)
        ops.fax_op_expert_combine_backward(sess.ctx, prec, ops.ExpertCombineBackwardDesc(n, k, d, slots, ptr(slot_t), ptr(source_t), ptr(tw), ptr(tz) if dw else None, d + pad, ptr(tdy), d + pad,
                                                                                        ptr(dz), d + pad, ptr(tdw) if dw else None))
        near(dz, want_dz, ref.F32 * np.abs(want_dz))
        if dw:
            # d products and additions, in whatever order
            assert np.all(np.abs(num(tdw).reshape(-1) - want_dw) <= (d + 1) * ref.F32 * size)
        else:
            assert bool((tdw == 7).all())
    # dz in place of z: every row written, the same bits
    ops.fax_op_expert_combine_backward(sess.ctx, prec, ops.ExpertCombineBackwardDesc(n, k, d, slots, ptr(slot_t), ptr(source_t), ptr(tw), ptr(tz), d + pad, ptr(tdy), d + pad, ptr(tz), d + pad, ptr(tdw)))
    assert torch.equal(tz, dz)


def test_gradients_are_the_differences(sess):
    """Combine is linear in z and in w: differences of its outputs are its gradients, but for float's roundings."""
    rng = np.random.default_rng(3)
    n, k, e, d = 20, 2, 4, 16
    slot_t, source_t, _, _ = sort(sess, choices(rng, n, k, e, 0.2), e)
    slots = source_t.numel()
    z, w, dy = (rng.standard_normal(s).astype(np.float32).astype(np.float64) for s in ((slots, d), (n, k), (n, d)))
    dev = sess.device
    put = lambda a: torch.as_tensor(a).float().to(dev)  # noqa: E731

    def loss(z, w):
        y = torch.empty((n, d), device=dev)
        tz, tw = put(z), put(w)
        ops.fax_op_expert_combine(sess.ctx, 1, ops.ExpertCombineDesc(n, k, d, slots, ptr(slot_t), ptr(tw), ptr(tz), d, None, 0, ptr(y), d))
        return float((y.double().cpu().numpy() * dy).sum())
    dz, dw, tz, tw, tdy = torch.empty((slots, d), device=dev), torch.empty((n, k), device=dev), put(z), put(w), put(dy)
    ops.fax_op_expert_combine_backward(sess.ctx, 1, ops.ExpertCombineBackwardDesc(n, k, d, slots, ptr(slot_t), ptr(source_t), ptr(tw), ptr(tz), d, ptr(tdy), d, ptr(dz), d, ptr(dw)))
    base = loss(z, w)
    # a step of 1 in one element changes y by at most 5; every y (below 32 in size) is rounded twice in each loss, sum |dy| < 512
    slack = 4 * 32 * ref.F32 * 512
    for a, grad in ((z, dz), (w, dw)):
        for at in [tuple(rng.integers(0, s) for s in a.shape) for _ in range(12)]:
            a[at] += 1.0
            assert abs(loss(z, w) - base - float(grad[at])) <= slack
            a[at] -= 1.0


def test_plans_that_are_wrong_read_and_write_nothing_outside(sess):
    """Slots outside the buffer count as none (documented)."""
    n, k, d, slots = 6, 2, 32, 8
    dev = sess.device
    slot_of = torch.tensor([[0, 8], [1, -7], [2, 2**31 - 1], [-2**31, 3], [4, 100], [5, 6]], dtype=torch.int32, device=dev)
    source = torch.tensor([0, 2, 4, 7, 8, 10, 11, -1], dtype=torch.int32, device=dev)
    x = torch.randn((n, d), device=dev)
    out = torch.full((slots, d), 7.0, device=dev)
    ops.fax_op_expert_dispatch(sess.ctx, 1, ops.ExpertDispatchDesc(n, k, d, slots, ptr(slot_of), ptr(source), ptr(x), d, ptr(out), d))
    want = torch.stack([x[0], x[1], x[2], x[3], x[4], x[5], x[5], torch.zeros(d, device=dev)])
    assert torch.equal(out, want)
    y = torch.empty((n, d), device=dev)
    ops.fax_op_expert_combine(sess.ctx, 1, ops.ExpertCombineDesc(n, k, d, slots, ptr(slot_of), None, ptr(out), d, None, 0, ptr(y), d))
    assert torch.equal(y[:5], x[:5]) and torch.equal(y[5], x[5] + x[5])


def test_rows_behind_two_to_the_31_elements(sess):
    n, d = 140000, 16000
    dev = sess.device
    x = torch.zeros((n, d), dtype=torch.bfloat16, device=dev)
    x[-64:] = torch.randn((64, d), device=dev).to(torch.bfloat16)
    ids = torch.zeros((n, 1), dtype=torch.int32, device=dev)
    ids[::2] = 1
    new = lambda *s: torch.empty(s, dtype=torch.int32, device=dev)  # noqa: E731
    slot_of, source, offsets, counts = new(n, 1), new(n), new(3), new(2)
    ops.fax_op_expert_sort(sess.ctx, ops.ExpertSortDesc(n, 1, 2, 0, 1, n, ptr(ids), ptr(slot_of), ptr(source), ptr(offsets), ptr(counts)))
    out, back = torch.empty_like(x), torch.empty_like(x)
    ops.fax_op_expert_dispatch(sess.ctx, 0, ops.ExpertDispatchDesc(n, 1, d, n, ptr(slot_of), ptr(source), ptr(x), d, ptr(out), d))
    assert torch.equal(out[n // 2 - 32:n // 2], x[-63::2]) and torch.equal(out[-32:], x[-64::2])
    ops.fax_op_expert_combine(sess.ctx, 0, ops.ExpertCombineDesc(n, 1, d, n, ptr(slot_of), None, ptr(out), d, None, 0, ptr(back), d))
    assert torch.equal(back, x)


@pytest.mark.parametrize("d", [64, 63])
def test_pitches_of_their_own(sess, d):
    """Every matrix with a pitch of its own: the same values as without gaps."""
    rng = np.random.default_rng(8)
    n, k, e = 37, 2, 3
    slot_t, source_t, _, _ = sort(sess, choices(rng, n, k, e), e, 0, 8)
    slots = source_t.numel()
    w = torch.as_tensor(rng.random((n, k))).float().to(sess.device)

    def run(pads):
        make = lambda rows, i: pitched(sess, ref.rounded(np.random.default_rng(100 + i).standard_normal((rows, d)), 0), 0, pads[i])  # noqa: E731
        x, z, r, dy, out, y, dz = make(n, 0), make(slots, 1), make(n, 2), make(n, 3), make(slots, 4), make(n, 5), make(slots, 6)
        dw = torch.empty((n, k), device=sess.device)
        ld = lambda t: t.stride(0)  # noqa: E731
        ops.fax_op_expert_dispatch(sess.ctx, 0, ops.ExpertDispatchDesc(n, k, d, slots, ptr(slot_t), ptr(source_t), ptr(x), ld(x), ptr(out), ld(out)))
        ops.fax_op_expert_combine(sess.ctx, 0, ops.ExpertCombineDesc(n, k, d, slots, ptr(slot_t), ptr(w), ptr(z), ld(z), ptr(r), ld(r), ptr(y), ld(y)))
        ops.fax_op_expert_combine_backward(sess.ctx, 0, ops.ExpertCombineBackwardDesc(n, k, d, slots, ptr(slot_t), ptr(source_t), ptr(w), ptr(z), ld(z), ptr(dy), ld(dy), ptr(dz), ld(dz), ptr(dw)))
        for t, p in zip((out, y, dz), (pads[4], pads[5], pads[6])):
            assert p == 0 or bool((t[:, d:] == 7).all())
        return out[:, :d].clone(), y[:, :d].clone(), dz[:, :d].clone(), dw
    a, b = run([0] * 7), run([8, 16, 1, 8, 24, 3, 8])
    c = run([8, 16, 24, 8, 24, 8, 40])
    for x, y, z in zip(a[:3], b[:3], c[:3]):
        assert torch.equal(x, y) and torch.equal(x, z)
    # (the sums of dw run in another order where vectors are single elements)
    assert float((a[3] - c[3]).abs().max()) <= 64 * 2.0 ** -24 * 64 and float((a[3] - b[3]).abs().max()) <= 64 * 2.0 ** -24 * 64
