"""Token table lookup and its gradient by sorted tokens against 64-bit references, through the C ABI."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import Session, fx, host, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


DT = (torch.bfloat16, torch.float32)


def ids_for(kind, n, vocab, rng):
    if kind == "zipf":
        return np.minimum(np.exp(rng.random(n) * np.log(vocab + 1)).astype(np.int64), vocab).astype(np.int32) - 1
    if kind == "same":
        return np.full(n, vocab // 2, np.int32)
    if kind == "pad":
        i = rng.integers(0, vocab, n).astype(np.int32)
        i[rng.random(n) < 0.5] = -1
        i[rng.random(n) < 0.1] = vocab
        i[rng.random(n) < 0.05] = np.iinfo(np.int32).max
        return i
    if kind == "none":
        return np.full(n, -1, np.int32)
    return rng.integers(0, vocab, n).astype(np.int32)


def backward(sess, prec, ids, dout, vocab, scale, acc, dtable, scratch=None):
    n, d = dout.shape
    nb = ops.fax_op_embedding_backward_scratch_bytes(n, vocab, d)
    if scratch is None:
        scratch = sess.arena(nb).fill_(0xA5)
    ops.fax_op_embedding_backward(sess.ctx, prec, n, vocab, d, ptr(ids), ptr(dout), scale, acc, ptr(dtable), ptr(scratch), nb)
    return scratch


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("n,vocab,d", [(1, 1, 1), (1, 50, 64), (7, 3, 33), (128, 1000, 256), (33, 500, 1032), (300, 70000, 130), (64, 40, 4096)])
@pytest.mark.parametrize("kind", ["uniform", "pad"])
def test_lookup(sess, prec, n, vocab, d, kind):
    rng = np.random.default_rng(n * 31 + d)
    ids = ids_for(kind, n, vocab, rng)
    table = torch.as_tensor(rng.standard_normal((vocab, d)).astype(np.float32)).to(DT[prec])
    out = torch.full((n + 1, d), 7.0, dtype=DT[prec], device=sess.device)
    t, i = table.to(sess.device), torch.as_tensor(ids).to(sess.device)
    ops.fax_op_embedding_forward(sess.ctx, prec, n, vocab, d, ptr(i), ptr(t), 11.3, ptr(out))
    want = torch.as_tensor(ref.embedding(ids, table.double().numpy(), 11.3))
    # one float32 product and, in bf16, a second rounding: a float32 half step and a bf16 half step
    tol = (2.0 ** -8 + 2.0 ** -24) if prec == 0 else 2.0 ** -24
    got = out[:n].double().cpu()
    assert bool(((got - want).abs() <= tol * want.abs()).all())
    assert bool((out[n] == 7).all())                                 # nothing behind the last row


SHAPES = [(1, 1, 1), (1, 9, 64), (5, 2, 7), (31, 31, 8), (32, 400, 16), (33, 7, 1000), (511, 100, 24), (513, 255, 520), (513, 256, 40),
          (1000, 65535, 64), (1025, 65536, 8), (4099, 300, 96), (3000, 70000, 33),
          (512, 1, 1024), (512, 40000, 520), (513, 9, 256), (512, 70, 519), (37, 3000, 1032), (300, 1, 513), (512, 33, 2), (1024, 5, 256), (1024, 40000, 1032), (700, 90, 513), (1037, 1, 40), (2048, 255, 24), (5000, 7, 1), (1700, 256, 2056), (1100, 3000, 1025)]


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("n,vocab,d", SHAPES)
@pytest.mark.parametrize("kind", ["zipf", "pad", "same", "none"])
@pytest.mark.parametrize("acc", [0, 1])
def test_gradient(sess, prec, n, vocab, d, kind, acc):
    rng = np.random.default_rng(n * 7 + d * 3 + vocab)
    ids = ids_for(kind, n, vocab, rng)
    dout = torch.as_tensor(rng.standard_normal((n, d)).astype(np.float32)).to(DT[prec])
    old = torch.as_tensor(rng.standard_normal((vocab, d)).astype(np.float32))
    guard = torch.full((vocab + 1, d), 7.0, device=sess.device)
    dt = guard[:vocab]
    dt.copy_(old)
    i, g = torch.as_tensor(ids).to(sess.device), dout.to(sess.device)
    scale = 1.7
    backward(sess, prec, i, g, vocab, scale, acc, dt)
    x = dout.double().numpy()
    want = ref.embedding_grad(ids, x, vocab, scale) + (old.double().numpy() if acc else 0)
    # k additions of float32 round k times, each by half a step of a partial sum at most; the scale and the old value two more
    count = np.bincount(ids[(ids >= 0) & (ids < vocab)], minlength=vocab)[:, None]
    size = ref.embedding_grad(ids, np.abs(x), vocab, scale) + (np.abs(old.double().numpy()) if acc else 0)
    got = host(dt)
    assert np.all(np.abs(got - want) <= (count + 3) * 2.0 ** -24 * size)
    if acc:                                                          # rows without tokens keep their bits
        assert np.array_equal(got[count[:, 0] == 0], old.double().numpy()[count[:, 0] == 0])
    assert bool((guard[vocab] == 7).all())


@pytest.mark.parametrize("n,vocab,d", [(40000, 50304, 64), (140000, 1 << 20, 8), (200000, 12, 16)])
def test_gradient_of_long_batches(sess, n, vocab, d):
    """Several tiles of the sort per block of counts, three digits, runs over many chunks."""
    rng = np.random.default_rng(n)
    ids = ids_for("zipf", n, vocab, rng)
    dout = torch.as_tensor(rng.integers(-3, 4, (n, d)).astype(np.float32)).to(torch.bfloat16)      # whole numbers: sums are exact
    dt = torch.full((vocab, d), float("nan"), device=sess.device)
    i, g = torch.as_tensor(ids).to(sess.device), dout.to(sess.device)
    backward(sess, 0, i, g, vocab, 0.5, 0, dt)
    want = torch.zeros((vocab, d), dtype=torch.float64, device=sess.device).index_add_(0, i.long(), g.double()) * 0.5
    assert torch.equal(dt.double(), want)


def test_gradient_is_the_same_bits_and_order(sess):
    """Twice the same call: the same bits, also with the scratch as another call left it, and for unaligned buffers."""
    rng = np.random.default_rng(3)
    for n, vocab, d in ((6000, 50, 72), (900, 20, 72), (500, 20, 72), (512, 3, 1024), (100, 2, 4100), (300, 40, 33)):
        same_bits(sess, rng, n, vocab, d)


def same_bits(sess, rng, n, vocab, d):
    i = torch.as_tensor(ids_for("zipf", n, vocab, rng)).to(sess.device)
    g = torch.as_tensor((rng.standard_normal((n, d)) * 10.0 ** rng.uniform(-4, 4, (n, 1))).astype(np.float32)).to(sess.device)
    a, b = torch.empty((vocab, d), device=sess.device), torch.empty((vocab, d), device=sess.device)
    s = backward(sess, 1, i, g, vocab, 1.0, 0, a)
    backward(sess, 1, i.flip(0).contiguous(), g, vocab, 1.0, 0, b, s)
    backward(sess, 1, i, g, vocab, 1.0, 0, b, s)
    assert torch.equal(a, b)
    flat = torch.empty(vocab * d + 1, device=sess.device)
    off = flat[1:].view(vocab, d)                                    # not 16-byte aligned: one element at a time, the same order
    backward(sess, 1, i, g, vocab, 1.0, 0, off, s)
    assert torch.equal(a, off)


def test_gradient_replayed_from_a_graph(sess):
    """Captured with its launches and replayed on other ids: nothing is kept from the first run."""
    rng = np.random.default_rng(5)
    for n in (700, 1500, 300):
        replayed(sess, rng, n, 90, 48)


def replayed(sess, rng, n, vocab, d):
    st = torch.cuda.Stream(sess.device)
    with torch.cuda.stream(st):
        s2 = Session(0)
        try:
            i = torch.as_tensor(ids_for("zipf", n, vocab, rng)).to(sess.device)
            g = torch.as_tensor(rng.integers(-3, 4, (n, d)).astype(np.float32)).to(sess.device)
            dt = torch.empty((vocab, d), device=sess.device)
            scratch = backward(s2, 1, i, g, vocab, 1.0, 0, dt)
            st.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                backward(s2, 1, i, g, vocab, 1.0, 0, dt, scratch)
            for _ in range(3):
                i.copy_(torch.as_tensor(ids_for("pad", n, vocab, rng)))
                dt.fill_(float("nan"))
                graph.replay()
                st.synchronize()
                ids = i.cpu().numpy()
                assert np.array_equal(host(dt), ref.embedding_grad(ids, g.double().cpu().numpy(), vocab, 1.0))
            del graph
        finally:
            s2.close()


def test_no_tokens(sess):
    dt = torch.full((5, 12), 3.0, device=sess.device)
    empty = torch.empty((0, 12), device=sess.device)
    ops.fax_op_embedding_forward(sess.ctx, 1, 0, 5, 12, None, None, 1.0, None)
    nb = ops.fax_op_embedding_backward_scratch_bytes(0, 5, 12)
    s = sess.arena(nb)
    ops.fax_op_embedding_backward(sess.ctx, 1, 0, 5, 12, None, ptr(empty), 1.0, 1, ptr(dt), ptr(s), nb)
    assert bool((dt == 3).all())
    ops.fax_op_embedding_backward(sess.ctx, 1, 0, 5, 12, None, ptr(empty), 1.0, 0, ptr(dt), ptr(s), nb)
    assert bool((dt == 0).all())
