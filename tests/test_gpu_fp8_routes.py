"""The 8-bit product on each of its kernels, pairs of SMs above all: every test names the tile it runs on and asks for it."""
import ctypes as C

import numpy as np
import pytest
import torch

from parity_util import Session, fx, ptr
from paper_2204_06514_b200 import binding_ops as ops

T8 = (torch.float8_e4m3fn, torch.float8_e5m2)


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    st, detail = fx.fax_check_device_status(s.ctx)
    s.close()
    assert st == fx.FAX_OK, detail


def up(x, a):
    return -(-x // a) * a


class Matrix:
    """rows x k codes of a format, both signs (or none), with scales 2^-6 .. 2^6 for 1 x 128 or 128 x 128 of them.  Behind
    column k and behind the last scale of a row of scales there is NaN."""

    def __init__(self, sess, rows, k, fmt, tile, g, positive=False, pad=0):
        dev = sess.device
        self.fmt, self.tile, self.k = fmt, tile, k
        top = (0x7E, 0x7B)[fmt]                                      # the largest finite code
        low = (0x20, 0x30)[fmt]                                      # magnitudes of 2^-3 .. TOP
        code = torch.randint(low, top + 1, (rows, k), generator=g, device=dev, dtype=torch.int32)
        if not positive:
            code |= torch.randint(0, 2, (rows, k), generator=g, device=dev, dtype=torch.int32) << 7
            code[torch.rand((rows, k), generator=g, device=dev) < 0.05] = 0
        self.q = torch.full((rows, up(k, 16) + 16 * pad), 0x7F, dtype=torch.uint8, device=dev)
        self.q[:, :k] = code.to(torch.uint8)
        sr = -(-rows // tile)
        self.s = torch.full((-(-k // 128), sr + pad), float("nan"), device=dev)
        self.s[:, :sr] = torch.exp2(torch.randint(-6, 7, (self.s.shape[0], sr), generator=g, device=dev).float())

    def wide(self):
        rows = self.q.shape[0]
        s = self.s[:, :-(-rows // self.tile)].double().t()
        s = s.repeat_interleave(self.tile, dim=0)[:rows].repeat_interleave(128, dim=1)[:, :self.k]
        return self.q.view(T8[self.fmt])[:, :self.k].double() * s

    def args(self):
        return ptr(self.q), self.q.shape[1], self.fmt, ptr(self.s), self.s.shape[1]


def call(sess, a, b, out, n, acc=0, bias=None):
    ops.fax_op_fp8_gemm(sess.ctx, ops.Fp8GemmDesc(a.q.shape[0], n, a.k, *a.args(), *b.args(), b.tile, ptr(out), out.stride(0), int(out.dtype == torch.float32), acc, ptr(bias)))


def tolerance(k, size, want, f32):
    """Every partial sum is at most `size`: K additions on the tensor cores, one product and one addition per block of 128,
    bias and old value, each off by one float32 step at most; a bf16 result is rounded once more."""
    return (k + 3 * (-(-k // 128)) + 4) * 2.0 ** -23 * size + (0 if f32 else 2.0 ** -8 * want.abs())


def check(sess, m, n, k, fa, fb, b_tile, f32, acc, bias, seed, pad=0, out_pad=0, shift=0):
    g = torch.Generator(device=sess.device)
    g.manual_seed(seed)
    a, b = Matrix(sess, m, k, fa, 1, g, pad=pad), Matrix(sess, n, k, fb, b_tile, g, pad=2 * pad)
    dt = torch.float32 if f32 else torch.bfloat16
    ldc = n + out_pad
    flat = torch.full((shift + m * ldc + 4 * ldc,), 7.0, dtype=dt, device=sess.device)         # four rows behind the last one
    out = flat[shift:shift + m * ldc].view(m, ldc)
    old = torch.zeros((m, n), dtype=torch.float64, device=sess.device)
    if acc:
        out[:, :n] = 1e4 * torch.randn((m, n), generator=g, device=sess.device)
        old = out[:, :n].double()
    tb = torch.randn(n, generator=g, device=sess.device).mul(1e3).to(torch.bfloat16) if bias else None
    call(sess, a, b, out, n, acc, tb)
    wa, wb = a.wide(), b.wide()
    extra = old + (tb.double() if bias else 0.0)
    want, size = wa @ wb.t() + extra, wa.abs() @ wb.abs().t() + old.abs() + (tb.double().abs() if bias else 0.0)
    err = (out[:, :n].double() - want).abs()
    st, detail = fx.fax_check_device_status(sess.ctx)
    assert st == fx.FAX_OK, detail
    bad = err > tolerance(k, size, want, f32)
    assert not bool(bad.any()), (int(bad.sum()), torch.argwhere(bad)[:4].tolist(), err[bad][:4].tolist(), want[bad][:4].tolist())
    assert bool((out[:, n:] == 7).all()) and bool((flat[:shift] == 7).all()) and bool((flat[shift + m * ldc:] == 7).all())
    return a, b, out


# Rows: a last pair of tiles whose second SM has all (4096), some (900, 3000, 3500) or none (the others) of its 128 rows; columns
# that end anywhere in a tile; K that ends anywhere in a block, a word of four scales, or a segment of 512.  4100 x 4099 and
# 4100 x 4104 have several tiles for each pair, so that both accumulators are used again.
PAIRS = [
    (520, 5000, 3900, 0, (2, 256, 1)), (900, 3500, 3900, 0, (2, 256, 1)), (4096, 770, 3900, 0, (2, 256, 1)), (4100, 4104, 2100, 0, (2, 256, 1)),
    (1300, 5000, 3900, 1, (2, 256, 1)), (1900, 3500, 3900, 1, (2, 256, 1)), (1100, 6010, 3900, 1, (2, 256, 1)), (4100, 4099, 4000, 1, (2, 256, 1)),
    (1300, 3500, 600, 0, (2, 192, 1)), (3500, 1283, 600, 0, (2, 192, 1)), (776, 6010, 700, 0, (2, 192, 1)), (1900, 5000, 500, 0, (2, 192, 1)),
    (900, 2500, 900, 1, (2, 192, 1)), (3000, 770, 1030, 1, (2, 192, 1)), (776, 6010, 712, 1, (2, 192, 1)), (1900, 5001, 500, 1, (2, 192, 1)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,f32,tile", PAIRS)
@pytest.mark.parametrize("fa,fb,b_tile", [(0, 0, 128), (0, 1, 1), (1, 0, 128), (1, 1, 1)])
def test_pairs(sess, m, n, k, f32, tile, fa, fb, b_tile):
    assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32) == tile
    for acc, bias in ((0, 1), (1, 0)) if f32 else ((0, 0), (0, 1)):
        check(sess, m, n, k, fa, fb, b_tile, f32, acc, bias, seed=m + n + k + acc)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,f32,tile", [PAIRS[i] for i in (0, 1, 5, 6, 8, 9, 12, 15)])
@pytest.mark.parametrize("b_tile", [1, 128])
def test_pairs_with_pitches(sess, m, n, k, f32, tile, b_tile):
    """NaN behind every matrix's rows and scales; C at pitches that a tensor map can and cannot describe, and unaligned."""
    assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32) == tile
    for out_pad, shift, acc in ((up(n, 8) + 8 - n, 0, f32), (3, 0, 0), (5, 1, f32)):
        check(sess, m, n, k, 0, 1, b_tile, f32, acc, 1, seed=n + out_pad, pad=3, out_pad=out_pad, shift=shift)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,f32,tile", [PAIRS[i] for i in (0, 3, 4, 7, 9, 13)])
def test_pairs_and_single_sms_agree(sess, m, n, k, f32, tile):
    """The same call with pairs off: no other kernel runs in their place unasked, and both are right."""
    assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32) == tile
    a, b, out = check(sess, m, n, k, 0, 1, 128, f32, 0, 1, seed=5)
    fx.fax_set_gemm_two_cta(sess.ctx, False)
    try:
        assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32)[0] == 1
        a1, b1, out1 = check(sess, m, n, k, 0, 1, 128, f32, 0, 1, seed=5)
    finally:
        fx.fax_set_gemm_two_cta(sess.ctx, True)
    assert torch.equal(a.q, a1.q) and torch.equal(b.s, b1.s)
    size = a.wide().abs() @ b.wide().abs().t() + 1e4
    assert bool(((out.double() - out1.double()).abs() <= 2 * tolerance(k, size, torch.maximum(out.double().abs(), out1.double().abs()), f32)).all())


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,f32,tile", [PAIRS[i] for i in (0, 4, 9, 13)])
def test_pairs_with_nan(sess, m, n, k, f32, tile):
    """A NaN element or scale of A reaches its row and nothing else; one of B its column (its 128 columns)."""
    assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32) == tile
    g = torch.Generator(device=sess.device)
    g.manual_seed(1)
    a, b = Matrix(sess, m, k, 0, 1, g), Matrix(sess, n, k, 0, 128, g)
    a.q[m - 1, k - 1] = 0x7F
    a.q[140, 3] = 0xFF
    a.s[1, 7] = float("nan")
    b.q[n - 1, 0] = 0x7F
    b.s[0, 2] = float("nan")
    out = torch.zeros((m, n), dtype=torch.float32 if f32 else torch.bfloat16, device=sess.device)
    call(sess, a, b, out, n)
    nan = torch.zeros((m, n), dtype=torch.bool, device=sess.device)
    nan[[m - 1, 140, 7]] = True
    nan[:, n - 1] = True
    nan[:, 256:384] = True
    assert torch.equal(torch.isnan(out), nan)


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,f32,tile", [PAIRS[i] for i in (1, 3, 5, 10, 14)])
def test_pairs_give_the_same_bits_every_time(sess, m, n, k, f32, tile):
    assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32) == tile
    g = torch.Generator(device=sess.device)
    g.manual_seed(2)
    a, b = Matrix(sess, m, k, 0, 1, g), Matrix(sess, n, k, 0, 1, g)
    first = None
    for _ in range(5):
        out = torch.full((m, n), float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device=sess.device)
        call(sess, a, b, out, n)
        first = out if first is None else first
        assert torch.equal(out, first)


# ---- the single-SM tiles ----

SINGLE = [
    (300, 200, 600, 0, (1, 64, 1)), (520, 200, 900, 1, (1, 64, 1)), (300, 500, 2100, 0, (1, 64, 2)), (776, 200, 2100, 1, (1, 64, 2)),
    (900, 1283, 600, 0, (1, 128, 1)), (776, 1500, 600, 1, (1, 128, 1)), (900, 1283, 100, 1, (1, 128, 1)), (16, 4096, 4096, 0, (1, 128, 4)),
    (1900, 1283, 600, 0, (1, 256, 1)), (900, 2500, 600, 1, (1, 256, 1)), (4100, 4099, 300, 0, (1, 256, 1)), (4100, 4099, 300, 1, (1, 256, 1)),
]


@pytest.mark.gpu
@pytest.mark.parametrize("m,n,k,f32,tile", SINGLE)
@pytest.mark.parametrize("fa,fb,b_tile", [(0, 0, 128), (1, 0, 1)])
def test_single_sms(sess, m, n, k, f32, tile, fa, fb, b_tile):
    assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, f32) == tile
    check(sess, m, n, k, fa, fb, b_tile, f32, f32, 1, seed=m, pad=1, out_pad=8)


# ---- how far float sums over a long K are off ----

@pytest.mark.gpu
@pytest.mark.parametrize("m,n,pairs,tile", [(300, 200, 1, (1, 64, 2)), (1900, 1283, 0, (1, 256, 1)), (1900, 1283, 1, (2, 192, 1)), (1300, 5000, 1, (2, 256, 1))])
def test_float_sums_do_not_drift_over_a_long_k(sess, m, n, pairs, tile):
    """All operands positive, so that what an accumulator cuts off adds up.  Float outputs are summed in segments of 512 k:
    16 additions of 32 products each, off by two float32 steps of the segment's sum at most (the products are aligned to the
    largest of them, then the sum is cut off): 32 * 2^-23 of it.  The segments are added to nearest: half a step of each
    partial sum, which grow evenly: (S + 1) / 2 * 2^-24 in all for S of them, and 2^-24 for each slice of K.
    One sum over all of K would be off by a quarter to a half of a step of each of K / 32 partial sums: 2e-5 and more."""
    k = 40000
    fx.fax_set_gemm_two_cta(sess.ctx, bool(pairs))
    try:
        assert ops.fax_op_fp8_gemm_tile(sess.ctx, m, n, k, 1) == tile
        g = torch.Generator(device=sess.device)
        g.manual_seed(3)
        a, b = Matrix(sess, m, k, 0, 1, g, positive=True), Matrix(sess, n, k, 0, 128, g, positive=True)
        for x in (a, b):
            x.s.fill_(1.0)
        out = torch.empty((m, n), device=sess.device)
        call(sess, a, b, out, n)
    finally:
        fx.fax_set_gemm_two_cta(sess.ctx, True)
    want = a.wide() @ b.wide().t()
    rel = (out.double() - want) / want
    bound = 32 * 2.0 ** -23 + ((-(-k // 512) + 1) / 2 + tile[2]) * 2.0 ** -24
    assert float(rel.abs().max()) <= bound, (float(rel.abs().max()), float(rel.mean()), bound)


# ---- the query's refusals: no GPU is needed ----

def test_tile_refusals():
    from paper_2204_06514_b200 import build, binding
    build.build()
    lib = binding.load_library()
    ctx = C.cast((C.c_char * 8192)(), C.c_void_p)
    o = [C.byref(C.c_int32()) for _ in range(3)]
    f = lib.fax_op_fp8_gemm_tile
    assert f(None, 1, 1, 1, 0, *o) == -1
    for i in range(3):
        p = list(o)
        p[i] = None
        assert f(ctx, 1, 1, 1, 0, *p) == -1
    for bad in ((0, 1, 1), (1, -1, 1), (1, 1, 0)):
        assert f(ctx, *bad, 0, *o) == -1
    for bad in ((0x7fffffff, 1, 1), (1, 0x7fffffff, 1), (1, 1, 0x7fffffff)):
        assert f(ctx, *bad, 0, *o) == -2
