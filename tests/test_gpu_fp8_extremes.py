"""The 8-bit product and what is added in memory at the ends of float32's range."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import Session, fx, host, ptr
from paper_2204_06514_b200 import binding_ops as ops
from test_gpu_fp8_routes import Matrix, call

pytestmark = pytest.mark.gpu
SMALLEST, LARGEST = 2.0 ** -126, (2 - 2.0 ** -23) * 2.0 ** 127


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    st, detail = fx.fax_check_device_status(s.ctx)
    s.close()
    assert st == fx.FAX_OK, detail


@pytest.mark.parametrize("m,n,k,f32", [(254, 254, 128, 1), (254, 254, 384, 1), (254, 254, 128, 0), (254, 254, 2100, 1)])
@pytest.mark.parametrize("positive", [True, False])
def test_every_scale(sess, m, n, k, f32, positive):
    """Row i of A has the scale 2^(i - 126), row j of B 2^(126 - j): every pair of them.  What float32 holds is right; beyond
    its largest number infinite (or the largest, or NaN where infinities of both signs meet), below its smallest at most
    the smallest normal number off for each of the sums' additions."""
    g = torch.Generator(device=sess.device)
    g.manual_seed(k)
    a, b = Matrix(sess, m, k, 0, 1, g, positive=positive), Matrix(sess, n, k, 0, 1, g, positive=positive)
    a.s[:, :m] = torch.exp2(torch.arange(m, device=sess.device).double() - 126).float()
    b.s[:, :n] = torch.exp2(126 - torch.arange(n, device=sess.device).double()).float()
    out = torch.empty((m, n), dtype=torch.float32 if f32 else torch.bfloat16, device=sess.device)
    call(sess, a, b, out, n)
    wa, wb = a.wide(), b.wide()
    want, size = wa @ wb.t(), wa.abs() @ wb.abs().t()
    got = out.double()
    safe = size < LARGEST / 2                                        # no partial sum can pass the largest number
    tol = (k + 3 * (-(-k // 128)) + 4) * (2.0 ** -23 * size + SMALLEST) + (0 if f32 else 2.0 ** -8 * want.abs())
    bad = safe & ~((got - want).abs() <= tol)
    assert not bool(bad.any()), (int(bad.sum()), torch.argwhere(bad)[:5].tolist(), got[bad][:5].tolist(), want[bad][:5].tolist())
    over = want.abs() > 2 * LARGEST
    if positive:
        assert bool((got[over] >= LARGEST).all()) and bool(over.any())
    assert bool(safe.any())


@pytest.mark.parametrize("n,shift", [(64, 0), (61, 1)])
def test_product_added_to_small_numbers(sess, n, shift):
    """Additions in memory take subnormal numbers for 0 (as documented): off by the smallest normal number for each."""
    m, k = 64, 128
    g = torch.Generator(device=sess.device)
    g.manual_seed(n)
    a, b = Matrix(sess, m, k, 0, 1, g), Matrix(sess, n, k, 0, 1, g)
    a.s.fill_(2.0 ** -80); b.s.fill_(2.0 ** -60)
    flat = torch.randn(m * n + shift, generator=g, device=sess.device) * 2.0 ** -126
    out = flat[shift:].view(m, n)
    old = out.double().clone()
    call(sess, a, b, out, n, acc=1)
    wa, wb = a.wide(), b.wide()
    want, size = old + wa @ wb.t(), old.abs() + wa.abs() @ wb.abs().t()
    assert bool(((out.double() - want).abs() <= (k + 8) * 2.0 ** -23 * size + 2 * SMALLEST).all())


@pytest.mark.parametrize("n", [100, 3000])
@pytest.mark.parametrize("d", [32, 33])
def test_table_gradient_added_to_small_numbers(sess, n, d):
    vocab = 50
    rng = np.random.default_rng(n + d)
    ids = rng.integers(0, vocab, n).astype(np.int32)
    tid = torch.as_tensor(ids).to(sess.device)
    g = torch.as_tensor((rng.standard_normal((n, d)) * 2.0 ** -127).astype(np.float32)).to(sess.device)
    out = torch.as_tensor((rng.standard_normal((vocab, d)) * 2.0 ** -126).astype(np.float32)).to(sess.device)
    old = host64(out)
    nb = ops.fax_op_embedding_backward_scratch_bytes(n, vocab, d)
    s = sess.arena(nb)
    ops.fax_op_embedding_backward(sess.ctx, 1, n, vocab, d, ptr(tid), ptr(g), 1.0, 1, ptr(out), ptr(s), nb)
    want = old + ref.embedding_grad(ids, host64(g), vocab, 1.0)
    size = np.abs(old) + ref.embedding_grad(ids, np.abs(host64(g)), vocab, 1.0)
    count = np.bincount(ids, minlength=vocab)[:, None]
    assert np.all(np.abs(host64(out) - want) <= (count + 3) * 2.0 ** -24 * size + 2 * SMALLEST)


def host64(t):
    return t.double().cpu().numpy()
