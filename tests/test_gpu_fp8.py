"""Quantisation in blocks and products of matrices in 8-bit floating point against 64-bit references."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import Session, fx, host, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu
DT = (torch.bfloat16, torch.float32)


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    st, detail = fx.fax_check_device_status(s.ctx)
    s.close()
    assert st == fx.FAX_OK, detail


def up(x, a):
    return -(-x // a) * a


def values(r, c, rng):
    x = rng.standard_normal((r, c)) * 10.0 ** rng.uniform(-3, 3, (r, 1)) * 10.0 ** rng.uniform(-2, 2, (1, c))
    x[rng.random((r, c)) < 0.05] = 0
    return x.astype(np.float32)


def quantize(sess, prec, x, r, c, ldx, fmt, tile, straight, transposed, extra=0):
    """Returns {name: (bytes, scales)}, buffers pre-filled with 0x55 / 7 beyond what is written."""
    dev = sess.device
    q = torch.full((r, up(c, 16) + extra), 0x55, dtype=torch.uint8, device=dev) if straight else None
    s = torch.full((-(-c // 128), -(-r // tile) + 1), 7.0, device=dev) if straight else None
    qt = torch.full((c, up(r, 16) + extra), 0x55, dtype=torch.uint8, device=dev) if transposed else None
    st = torch.full((-(-r // 128), -(-c // tile) + 1), 7.0, device=dev) if transposed else None
    P = lambda t: (ptr(t), t.shape[1]) if t is not None else (None, 0)  # noqa: E731
    ops.fax_op_fp8_quantize(sess.ctx, prec, ops.Fp8QuantizeDesc(r, c, ptr(x), ldx, fmt, tile, *P(q), *P(s), *P(qt), *P(st)))
    return q, s, qt, st


def check(q, s, x, r, c, fmt, tile):
    want, ws = ref.quantize(x, fmt, tile)
    got = host(q[:, :c].contiguous().view(ref.TORCH8[fmt]))
    assert np.array_equal(got, want, equal_nan=True)
    assert np.array_equal(host(s[:, :-1]), ws)
    assert bool((q[:, c:] == 0x55).all()) and bool((s[:, -1] == 7).all())


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("tile", [1, 128])
@pytest.mark.parametrize("r,c", [(1, 1), (1, 300), (17, 128), (128, 16), (129, 257), (250, 130), (300, 1000), (64, 4096)])
def test_quantize_bit_for_bit(sess, prec, fmt, tile, r, c):
    rng = np.random.default_rng(r * 1000 + c)
    for straight, transposed, pad, shift in ((1, 1, 0, 0), (1, 0, 8, 0), (0, 1, 3, 0), (1, 1, 5, 1)):
        ldx = c + pad
        flat = torch.full((r * ldx + 1,), float("nan"), dtype=DT[prec], device=sess.device)
        x = flat[shift:shift + r * ldx].view(r, ldx)                 # also from an address that is not 16-byte aligned
        x[:, :c] = torch.as_tensor(values(r, c, rng)).to(DT[prec])
        q, s, qt, st = quantize(sess, prec, x, r, c, ldx, fmt, tile, straight, transposed, extra=16)
        x64 = x[:, :c].double().cpu().numpy()
        if straight:
            check(q, s, x64, r, c, fmt, tile)
        if transposed:
            check(qt, st, x64.T, c, r, fmt, tile)


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("fmt", [0, 1])
@pytest.mark.parametrize("tile", [1, 128])
def test_quantize_extremes(sess, prec, fmt, tile):
    """Blocks of zeros, the smallest and largest numbers, values at and next to the binade's end, infinities and NaN."""
    r, c = 256, 256
    x = np.zeros((r, c), np.float32)
    top = ref.TOP[fmt]
    x[0, :4] = [top, -top, 0.5, 0.25]
    x[1, :4] = [top * (1 + 2.0 ** -7), 1, -1, 0.5]
    x[2, :3] = [3e38, 1e-30, -3e38]
    x[3, :3] = [1e-44, -1e-41, 1e-38]
    x[4, :5] = [np.inf, 1, -2, np.nan, -np.inf]
    x[5, 128:] = np.inf
    x[6, :128] = np.linspace(-top, top, 128)
    x[7, :128] = top * 2.0 ** -np.arange(128).astype(np.float32)
    x[128:, 128:] = 1e-3
    t = torch.as_tensor(x).to(sess.device).to(DT[prec])
    q, s, qt, st = quantize(sess, prec, t, r, c, c, fmt, tile, True, True)
    x64 = t.double().cpu().numpy()
    check(q, s, x64, r, c, fmt, tile)
    check(qt, st, x64.T, c, r, fmt, tile)


# ---- products ----

def operands(m, n, k, fa, fb, b_tile, rng):
    a, sa = ref.quantize(values(m, k, rng).astype(np.float64), fa, 1)
    b, sb = ref.quantize(values(n, k, rng).astype(np.float64), fb, b_tile)
    return a, sa, b, sb


def to_dev(sess, q, s, fmt, pad_k, pad_s):
    """Bytes with a pitch past K (NaN codes there, which must not be read as data) and scales with a pitch past the rows (NaN)."""
    b = ref.bytes_of(q, fmt, up(q.shape[1], 16) + pad_k, fill=0x7F).to(sess.device)
    t = torch.full((s.shape[0], s.shape[1] + pad_s), float("nan"))
    t[:, :s.shape[1]] = torch.as_tensor(s).float()
    return b, t.to(sess.device)


def product(sess, m, n, k, fa, fb, b_tile, f32, acc, bias, rng, pad=0, out_pad=0, shift=0):
    a, sa, b, sb = operands(m, n, k, fa, fb, b_tile, rng)
    ta, tsa = to_dev(sess, a, sa, fa, 16 * pad, pad)
    tb, tsb = to_dev(sess, b, sb, fb, 32 * pad, pad)
    dt = torch.float32 if f32 else torch.bfloat16
    ldc = n + out_pad
    flat = torch.full((m * ldc + shift,), 7.0, dtype=dt, device=sess.device)
    out = flat[shift:].view(m, ldc)
    old = rng.standard_normal((m, n)) * 10 if acc else np.zeros((m, n))
    if acc:
        out[:, :n] = torch.as_tensor(old).float()
        old = host(out[:, :n])
    tbias = torch.as_tensor(rng.standard_normal(n).astype(np.float32)).to(torch.bfloat16).to(sess.device) if bias else None
    ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(m, n, k, ptr(ta), ta.shape[1], fa, ptr(tsa), tsa.shape[1], ptr(tb), tb.shape[1], fb, ptr(tsb),
                                                  tsb.shape[1], b_tile, ptr(out), ldc, int(f32), int(acc), ptr(tbias) if bias else None))
    wa, wb = ref.widen(a, sa, 1), ref.widen(b, sb, b_tile)
    want, size = wa @ wb.T, np.abs(wa) @ np.abs(wb).T
    extra = host(tbias)[None, :] if bias else 0.0
    want = want + extra + old
    size = size + np.abs(extra) + np.abs(old)
    got = host(out[:, :n])
    st, detail = fx.fax_check_device_status(sess.ctx)
    assert st == fx.FAX_OK, detail
    # every partial sum is at most `size`: K additions on the tensor cores, one product and one addition per block of
    # 128, bias and old value, each off by one float32 step at most; a bf16 result is rounded once more
    tol = (k + 3 * (-(-k // 128)) + 4) * 2.0 ** -23 * size + (0 if f32 else 2.0 ** -8 * np.abs(want))
    bad = np.abs(got - want) > tol
    assert not bad.any(), (int(bad.sum()), np.argwhere(bad)[:4], got[bad][:4], want[bad][:4])
    if out_pad:
        assert bool((out[:, n:] == 7).all())
    return got


@pytest.mark.parametrize("m,n,k", [(1, 1, 1), (1, 8, 16), (2, 128, 128), (16, 256, 130), (127, 129, 127), (128, 64, 512), (129, 257, 385), (256, 256, 128),
                                   (255, 300, 1000), (300, 520, 640), (1, 4096, 1024), (700, 40, 2048)])
@pytest.mark.parametrize("b_tile", [1, 128])
@pytest.mark.parametrize("f32,acc,bias", [(0, 0, 0), (0, 0, 1), (1, 0, 0), (1, 1, 0), (1, 1, 1)])
def test_product(sess, m, n, k, b_tile, f32, acc, bias):
    rng = np.random.default_rng(m * 3 + n * 5 + k)
    product(sess, m, n, k, 0, 0, b_tile, f32, acc, bias, rng)


@pytest.mark.parametrize("fa,fb", [(0, 1), (1, 0), (1, 1)])
@pytest.mark.parametrize("m,n,k", [(16, 40, 200), (130, 260, 300)])
@pytest.mark.parametrize("b_tile", [1, 128])
def test_product_formats(sess, fa, fb, m, n, k, b_tile):
    rng = np.random.default_rng(m + n + k + fa)
    product(sess, m, n, k, fa, fb, b_tile, 1, 0, 0, rng)


@pytest.mark.parametrize("m,n,k", [(5, 9, 100), (130, 300, 260), (200, 256, 384)])
@pytest.mark.parametrize("b_tile", [1, 128])
@pytest.mark.parametrize("f32", [0, 1])
def test_product_pitches(sess, m, n, k, b_tile, f32):
    """Pitches past every matrix, NaN between the rows of A, B and the scales, a C that is not aligned: untouched around."""
    rng = np.random.default_rng(m + n)
    for out_pad, shift in ((16, 0), (3, 0), (5, 1)):
        product(sess, m, n, k, 0, 0, b_tile, f32, 0, 1, rng, pad=3, out_pad=out_pad, shift=shift)


@pytest.mark.parametrize("m,n,k", [(1, 512, 2048), (16, 1024, 4096), (33, 200, 3000), (64, 300, 1111), (97, 129, 2500), (128, 64, 8192), (200, 130, 4100), (300, 260, 1920)])
@pytest.mark.parametrize("b_tile", [1, 128])
@pytest.mark.parametrize("f32,acc,bias,pad", [(0, 0, 1, 0), (1, 1, 0, 0), (1, 0, 0, 3)])
def test_product_of_few_tiles_and_long_k(sess, m, n, k, b_tile, f32, acc, bias, pad):
    """Slices of K on a cluster of CTAs, joined by the first: one to four groups of 32 rows, ragged last slices."""
    rng = np.random.default_rng(m + n * 2 + k)
    product(sess, m, n, k, 0, 1, b_tile, f32, acc, bias, rng, out_pad=pad)


def test_product_is_the_same_bits_every_time(sess):
    rng = np.random.default_rng(12)
    for m, n, k in ((16, 1024, 4096), (300, 500, 2000)):
        a, sa, b, sb = operands(m, n, k, 0, 0, 128, rng)
        (ta, tsa), (tb, tsb) = to_dev(sess, a, sa, 0, 0, 0), to_dev(sess, b, sb, 0, 0, 0)
        outs = []
        for _ in range(4):
            out = torch.full((m, n), float("nan"), device=sess.device)
            ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(m, n, k, ptr(ta), ta.shape[1], 0, ptr(tsa), m, ptr(tb), tb.shape[1], 0, ptr(tsb), tsb.shape[1], 128, ptr(out), n, 1, 0, None))
            outs.append(out)
        assert all(torch.equal(o, outs[0]) for o in outs)


def test_product_of_many_tiles(sess):
    """More tiles than pairs of SMs, ragged on every side; against a product in 64 bits on the GPU."""
    m, n, k = 5100, 4200, 900
    rng = np.random.default_rng(0)
    for b_tile in (1, 128):
        product(sess, m, n, k, 0, 1, b_tile, 1, 1, 1, rng)


def test_product_with_nan(sess):
    """A NaN element of A reaches its row and nothing else; one of B its column."""
    rng = np.random.default_rng(4)
    m, n, k = 140, 150, 300
    a, sa, b, sb = operands(m, n, k, 0, 0, 1, rng)
    a[17, 200] = np.nan
    b[33, 5] = np.nan
    ta, tsa = to_dev(sess, a, sa, 0, 0, 0)
    tb, tsb = to_dev(sess, b, sb, 0, 0, 0)
    out = torch.zeros((m, n), device=sess.device)
    ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(m, n, k, ptr(ta), ta.shape[1], 0, ptr(tsa), m, ptr(tb), tb.shape[1], 0, ptr(tsb), n, 1, ptr(out), n, 1, 0, None))
    nan = np.zeros((m, n), bool)
    nan[17, :] = True
    nan[:, 33] = True
    assert np.array_equal(torch.isnan(out).cpu().numpy(), nan)


def test_quantize_and_product_in_a_graph(sess):
    """Captured together and replayed on other inputs."""
    rng = np.random.default_rng(6)
    m, n, k = 200, 144, 272
    st = torch.cuda.Stream(sess.device)
    with torch.cuda.stream(st):
        s2 = Session(0)
        try:
            x = torch.zeros((m, k), dtype=torch.bfloat16, device=sess.device)
            w = torch.as_tensor(values(k, n, rng)).to(sess.device)
            qx = torch.zeros((m, k), dtype=torch.uint8, device=sess.device)
            sx = torch.zeros((3, m), device=sess.device)
            qw = torch.zeros((n, k), dtype=torch.uint8, device=sess.device)
            sw = torch.zeros((3, 2), device=sess.device)
            y = torch.zeros((m, n), device=sess.device)

            def go():
                ops.fax_op_fp8_quantize(s2.ctx, 0, ops.Fp8QuantizeDesc(m, k, ptr(x), k, 0, 1, ptr(qx), k, ptr(sx), m, None, 0, None, 0))
                ops.fax_op_fp8_quantize(s2.ctx, 1, ops.Fp8QuantizeDesc(k, n, ptr(w), n, 0, 128, None, 0, None, 0, ptr(qw), k, ptr(sw), 2))
                ops.fax_op_fp8_gemm(s2.ctx, ops.Fp8GemmDesc(m, n, k, ptr(qx), k, 0, ptr(sx), m, ptr(qw), k, 0, ptr(sw), 2, 128, ptr(y), n, 1, 0, None))
            go()
            st.synchronize()
            graph = torch.cuda.CUDAGraph()
            with torch.cuda.graph(graph, stream=st):
                go()
            for _ in range(3):
                x.copy_(torch.as_tensor(values(m, k, rng)).to(torch.bfloat16))
                w.copy_(torch.as_tensor(values(k, n, rng)))
                graph.replay()
                st.synchronize()
                a = ref.widen(*ref.quantize(x.double().cpu().numpy(), 0, 1), 1)
                b = ref.widen(*ref.quantize(w.double().cpu().numpy().T, 0, 128), 128)
                size = np.abs(a) @ np.abs(b).T
                assert np.all(np.abs(host(y) - a @ b.T) <= (k + 13) * 2.0 ** -23 * size)
            del graph
        finally:
            s2.close()


@pytest.mark.parametrize("tall", [0, 1])
def test_quantize_of_the_longest_rows(sess, tall):
    """2^31 - 1 columns (rows for the transposed output): the last vector is cut, and positions pass 32 bits."""
    big, tail = 2 ** 31 - 1, 400
    dev = sess.device
    if torch.cuda.mem_get_info(dev)[0] < 40 * 2 ** 30:
        pytest.skip("too little device memory is free")
    x = torch.zeros(big + 25, dtype=torch.bfloat16, device=dev)
    end = torch.as_tensor(values(1, tail, np.random.default_rng(1))[0]).to(torch.bfloat16)
    x[big - tail:big] = end.to(dev)
    x[big:] = float("inf")                                           # not part of the matrix
    q = torch.full((big + 1,), 0x55, dtype=torch.uint8, device=dev)
    s = torch.full((2 ** 24 + 1,), 7.0, device=dev)
    wide = (ptr(q), big + 1, ptr(s), 1)
    none = (None, 0, None, 0)
    if tall:
        d = ops.Fp8QuantizeDesc(big, 1, ptr(x), 1, 0, 1, *none, *wide)
    else:
        d = ops.Fp8QuantizeDesc(1, big, ptr(x), big + 9, 0, 1, *wide, *none)
    ops.fax_op_fp8_quantize(sess.ctx, 0, d)
    lead = 128 - (big - tail) % 128                                  # the tail's first element stands inside a block
    want, ws = ref.quantize(np.concatenate([np.zeros(128 - lead), end.double().numpy()])[None], 0, 1)
    got = host(q[big - tail - (128 - lead):big].view(ref.TORCH8[0]))
    assert np.array_equal(got, want[0]) and np.array_equal(host(s[2 ** 24 - ws.shape[0]:2 ** 24]), ws[:, 0])
    assert int(q[big]) == 0x55 and float(s[2 ** 24]) == 7 and not bool(q[:big - tail].any()) and bool((s[:2 ** 24 - ws.shape[0]] == 1).all())


@pytest.mark.parametrize("m,n,k", [(300, 260, 600), (256, 512, 128), (5100, 1300, 200)])
@pytest.mark.parametrize("f32,acc,bias", [(0, 0, 1), (1, 1, 0)])
def test_product_on_single_sms(sess, m, n, k, f32, acc, bias):
    """With pairs of SMs switched off."""
    fx.fax_set_gemm_two_cta(sess.ctx, False)
    try:
        product(sess, m, n, k, 0, 0, 128, f32, acc, bias, np.random.default_rng(m))
    finally:
        fx.fax_set_gemm_two_cta(sess.ctx, True)
