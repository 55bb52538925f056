"""The operators on few bits and the token table's on matrices whose positions pass 31 and 32 bits: looked at where they
end, where a wrapped position would write, and as a whole where that is quick."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import Session, fx, hparams, host, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu


@pytest.fixture
def sess():
    torch.cuda.empty_cache()
    if torch.cuda.mem_get_info(0)[0] < 80 * 2 ** 30:
        pytest.skip("too little device memory is free")
    s = Session(0)
    yield s
    st, detail = fx.fax_check_device_status(s.ctx)
    s.close()
    torch.cuda.empty_cache()
    assert st == fx.FAX_OK, detail


def gen(sess, seed):
    g = torch.Generator(device=sess.device)
    g.manual_seed(seed)
    return g


def test_lookup(sess):
    """A table and an output of more than 2^31 elements each."""
    vocab, d, n = (1 << 21) + 5, 1032, (1 << 21) + 77
    g = gen(sess, 1)
    table = torch.randn((vocab, d), generator=g, device=sess.device, dtype=torch.bfloat16)
    ids = torch.randint(0, vocab, (n,), generator=g, device=sess.device, dtype=torch.int32)
    ids[:3] = torch.tensor([vocab - 1, 0, vocab], dtype=torch.int32)
    ids[-3:] = torch.tensor([vocab - 2, -1, vocab - 1], dtype=torch.int32)
    out = torch.full((n, d), 9.0, device=sess.device, dtype=torch.bfloat16)
    ops.fax_op_embedding_forward(sess.ctx, 0, n, vocab, d, ptr(ids), ptr(table), 0.5, ptr(out))
    for lo in range(0, n, 1 << 18):
        i = ids[lo:lo + (1 << 18)].long()
        ok = ((i >= 0) & (i < vocab)).unsqueeze(1)
        want = table[i.clamp(0, vocab - 1)] * 0.5                    # exact
        assert torch.equal(out[lo:lo + (1 << 18)], torch.where(ok, want, torch.zeros_like(want)))


@pytest.mark.parametrize("n,vocab,d", [(3000, (1 << 21) + 5, 1032), (300, (1 << 21) + 5, 1032), (700, (1 << 21) + 5, 1033), ((1 << 21) + 77, 1000, 1032)])
@pytest.mark.parametrize("accumulate", [0, 1])
def test_table_gradient(sess, n, vocab, d, accumulate):
    """A table, or a batch, of more than 2^31 elements; whole numbers, so that sums are exact."""
    g = gen(sess, n)
    ids = torch.randint(0, vocab, (n,), generator=g, device=sess.device, dtype=torch.int32)
    ids[:2] = torch.tensor([vocab - 1, 0], dtype=torch.int32)
    ids[-2:] = torch.tensor([vocab - 1, -1], dtype=torch.int32)
    dout = torch.randint(-3, 4, (n, d), generator=g, device=sess.device, dtype=torch.int8).to(torch.bfloat16)
    table = torch.full((vocab, d), 2.0 if accumulate else float("nan"), device=sess.device)
    nb = ops.fax_op_embedding_backward_scratch_bytes(n, vocab, d)
    s = sess.arena(nb)
    ops.fax_op_embedding_backward(sess.ctx, 0, n, vocab, d, ptr(ids), ptr(dout), 0.5, accumulate, ptr(table), ptr(s), nb)
    ids[-1] = 0
    dout[-1] = 0
    rows, where = ids.long().unique(return_inverse=True)
    want = torch.zeros((rows.numel(), d), device=sess.device)
    for lo in range(0, n, 1 << 18):
        want.index_add_(0, where[lo:lo + (1 << 18)], dout[lo:lo + (1 << 18)].float())
    assert torch.equal(table[rows], 0.5 * want + (2.0 if accumulate else 0.0))
    table[rows] = 2.0 if accumulate else 0.0                         # the others are as they have to be
    assert all(bool((table[lo:lo + (1 << 17)] == (2.0 if accumulate else 0.0)).all()) for lo in range(0, vocab, 1 << 17))


def test_adamw8(sess):
    """2^32 + 300 elements in one tensor: blocks at both ends and around 2^31 and 2^32 against the definition, whose random
    bits take in the position's upper half."""
    n, seed, step = (1 << 32) + 300, 11, 3
    dev = sess.device
    hp = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)
    w = torch.zeros(n + 4, device=dev)
    g = torch.zeros(n + 4, device=dev, dtype=torch.bfloat16)
    m, v = (torch.zeros(n + 4, dtype=torch.uint8, device=dev) for _ in range(2))
    nb = -(-n // 128)
    ms, vs = (torch.zeros(nb + 1, device=dev) for _ in range(2))
    rng = np.random.default_rng(0)
    spans = [(0, 256), ((1 << 31) - 128, (1 << 31) + 128), ((1 << 32) - 256, n)]
    start = {}
    for lo, hi in spans:
        x = torch.as_tensor(rng.standard_normal(hi - lo).astype(np.float32))
        y = torch.as_tensor((rng.standard_normal(hi - lo) * 10.0 ** rng.uniform(-6, 0, hi - lo)).astype(np.float32)).to(torch.bfloat16)
        w[lo:hi], g[lo:hi] = x.to(dev), y.to(dev)
        start[lo] = (x.double().numpy(), y.double().numpy())
    t = fx.Adamw8Tensor(ptr(w), ptr(m), ptr(v), ptr(ms), ptr(vs), ptr(g), None, n, 0.1, seed)
    fx.fax_adamw8_step(sess.ctx, [t], hparams(step=step, grad_is_bf16=1, **hp))
    key = ref.mix32((seed + step * 0x9E3779B9) & 0xFFFFFFFF)
    for lo, hi in spans:
        x, y = start[lo]
        k = hi - lo
        zero, one = np.zeros(k), np.zeros(-(-k // 128))
        want = ref.adamw8(x, zero, one, zero, one, y, 0.1, seed, step=step, **hp)[0]
        assert np.abs(host(w[lo:hi]) - want).max() <= 1e-6
        # the moments before they are rounded, in the definition's float32 steps, and the bits of these positions
        f = lambda a: np.asarray(a, np.float64).astype(np.float32).astype(np.float64)  # noqa: E731
        o1, o2 = float(f(1 - float(np.float32(0.9)))), float(f(1 - float(np.float32(0.95))))
        i = np.arange(lo, hi, dtype=np.uint64)
        h = ref.mix32((i & np.uint64(0xFFFFFFFF)) ^ ((key + (i >> np.uint64(32)) * np.uint64(0x85EBCA77)) & np.uint64(0xFFFFFFFF)))
        qm, sm = ref.round_moment(f(o1 * y), 0, (h >> np.uint64(16)).astype(np.float64))
        qv, sv = ref.round_moment(f(f(o2 * y) * y), 1, (h & np.uint64(0xFFFF)).astype(np.float64))
        assert np.array_equal(host(m[lo:hi].view(torch.float8_e4m3fn)), qm) and np.array_equal(host(v[lo:hi].view(torch.float8_e5m2)), qv)
        b = lo // 128
        assert np.array_equal(host(ms[b:b + len(sm)]), sm) and np.array_equal(host(vs[b:b + len(sv)]), sv)
    assert not bool(w[n:].any()) and not bool(m[n:].any()) and float(ms[nb]) == 0
    assert bool((ms[2:(1 << 24) - 1] == 1).all()) and not bool(m[256:(1 << 31) - 128].any())


def test_quantize(sess):
    """70000 x 70000 both ways: 4.9e9 elements."""
    n = 70000
    g = gen(sess, 5)
    x = torch.randn((n, n), generator=g, device=sess.device, dtype=torch.bfloat16)
    q, qt = (torch.zeros((n, n), dtype=torch.uint8, device=sess.device) for _ in range(2))
    kb = -(-n // 128)
    s, st = (torch.zeros((kb, n), device=sess.device) for _ in range(2))
    ops.fax_op_fp8_quantize(sess.ctx, 0, ops.Fp8QuantizeDesc(n, n, ptr(x), n, 0, 1, ptr(q), n, ptr(s), n, ptr(qt), n, ptr(st), n))
    for lo in (0, 30720, n - 100):                                   # 30720 rows are 2^31 elements and more; a multiple of 128
        for mat, codes, scales in ((x[lo:lo + 100], q, s), (x[:, lo:lo + 100].t(), qt, st)):
            want, ws = ref.quantize(mat.double().cpu().numpy(), 0, 1)
            assert np.array_equal(host(codes[lo:lo + 100].view(torch.float8_e4m3fn)), want)
            assert np.array_equal(host(scales[:, lo:lo + 100]), ws)


def codes(sess, rows, k, g):
    """Small whole numbers, exact in e4m3, with scales of 1: products are exact."""
    x = torch.randint(-3, 4, (rows, k), generator=g, device=sess.device, dtype=torch.int8)
    return x.to(torch.float8_e4m3fn), torch.ones((-(-k // 128), rows), device=sess.device)


@pytest.mark.parametrize("m,n,k,f32,acc", [(50000, 50001, 160, 1, 0), (50000, 50004, 160, 1, 1), (50000, 50001, 160, 1, 1), (40000, 65544, 160, 0, 0), (70000, 64, 70000, 1, 0)])
def test_product(sess, m, n, k, f32, acc):
    """Outputs and a left factor of more than 2^31 elements, at pitches that a tensor map can and cannot describe."""
    g = gen(sess, 6)
    (a, sa), (b, sb) = codes(sess, m, k, g), codes(sess, n, k, g)
    out = torch.full((m, n), 5.0, dtype=torch.float32 if f32 else torch.bfloat16, device=sess.device)
    ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(m, n, k, ptr(a), k, 0, ptr(sa), m, ptr(b), k, 0, ptr(sb), n, 1, ptr(out), n, f32, acc, None))
    b32 = b.float().t().contiguous()
    step = max(1, (1 << 28) // max(n, k))
    for lo in range(0, m, step):
        want = torch.mm(a[lo:lo + step].float(), b32) + (5.0 if acc else 0.0)      # whole numbers below 2^24: exact
        assert torch.equal(out[lo:lo + step], want.to(out.dtype)), lo
