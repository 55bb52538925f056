"""What the operators on few bits and the token table's refuse, checked before any CUDA call: no GPU is needed.
The context is a block of zeros that a refused call never looks into."""
import ctypes as C

import numpy as np
import pytest
import torch

import lowbit_ref as ref

INV, SHAPE, SMALL = -1, -2, -3
P = 1 << 20            # a well aligned address that no refused call touches


@pytest.fixture(scope="module")
def lib():
    from paper_2204_06514_b200 import build, binding
    build.build()
    return binding.load_library()


@pytest.fixture
def ctx():
    return C.cast((C.c_char * 8192)(), C.c_void_p)


def test_embedding_refusals(lib, ctx):
    fwd = lambda prec=0, n=4, v=5, d=8, ids=P, t=P, o=P, c=ctx: lib.fax_op_embedding_forward(c, prec, n, v, d, ids, t, 1.0, o)  # noqa: E731
    for bad in (dict(c=None), dict(prec=2), dict(n=-1), dict(v=0), dict(d=0), dict(ids=None), dict(t=None), dict(o=None), dict(ids=P + 2), dict(t=P + 1), dict(o=P + 1),
                dict(prec=1, t=P + 2)):
        assert fwd(**bad) == INV, bad
    assert fwd(n=(1 << 30) + 1) == SHAPE
    assert fwd(n=0, ids=None, t=None, o=None) == 0
    nb = C.c_size_t()
    sb = lib.fax_op_embedding_backward_scratch_bytes
    assert sb(4, 5, 8, None) == INV and sb(-1, 5, 8, C.byref(nb)) == INV and sb(4, 0, 8, C.byref(nb)) == INV and sb(4, 5, 0, C.byref(nb)) == INV
    assert sb(1000, 50, 8, C.byref(nb)) == 0
    need = nb.value

    def bwd(prec=0, n=1000, v=50, d=8, ids=P, g=P, o=P, s=P, size=need, c=ctx):
        return lib.fax_op_embedding_backward(c, prec, n, v, d, ids, g, 1.0, 0, o, s, size)
    for bad in (dict(c=None), dict(prec=-1), dict(n=-1), dict(v=0), dict(d=-3), dict(ids=None), dict(g=None), dict(o=None), dict(s=None), dict(s=P + 16), dict(o=P + 2),
                dict(ids=P + 1), dict(prec=1, g=P + 2)):
        assert bwd(**bad) == INV, bad
    assert bwd(size=need - 1) == SMALL
    assert bwd(n=(1 << 30) + 1) == SHAPE


def test_scratch_grows_with_the_batch(lib):
    from paper_2204_06514_b200 import binding_ops as ops
    a = [ops.fax_op_embedding_backward_scratch_bytes(n, 50304, 768) for n in (0, 1, 1000, 16384, 1 << 20, 1 << 30)]
    assert a == sorted(a) and a[-1] >= 16 * (1 << 30)


def test_adamw8_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding as fx

    def call(c=ctx, hp=None, arr=True, **kw):
        f = dict(w=P, m=P, v=P, m_scale=P, v_scale=P, g=P, w_compute=None, n=1000, weight_decay=0.1, seed=1)
        f.update(kw)
        h = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, step=1, grad_is_bf16=0)
        h.update(hp or {})
        t = fx.Adamw8Tensor(*(f[k] for k in ("w", "m", "v", "m_scale", "v_scale", "g", "w_compute", "n", "weight_decay", "seed")))
        return lib.fax_adamw8_step(c, C.byref(t) if arr else None, 1, C.byref(fx.AdamwHparams(*h.values())))
    for bad in (dict(c=None), dict(arr=False), dict(w=None), dict(m=None), dict(v=None), dict(m_scale=None), dict(v_scale=None), dict(g=None), dict(w=P + 4), dict(g=P + 8),
                dict(m=P + 2), dict(v=P + 1), dict(m_scale=P + 2), dict(v_scale=P + 1), dict(w_compute=P + 4), dict(hp=dict(step=0)), dict(hp=dict(beta1=1.0)),
                dict(hp=dict(beta2=-0.1)), dict(hp=dict(eps=-1.0)), dict(hp=dict(lr=float("nan"))), dict(hp=dict(eps=float("inf")))):
        assert call(**bad) == INV, bad
    t = fx.Adamw8Tensor()
    assert lib.fax_adamw8_step(ctx, C.byref(t), -1, C.byref(fx.AdamwHparams(1e-3, 0.9, 0.95, 1e-8, 1, 0))) == INV
    assert lib.fax_adamw8_step(ctx, C.byref(t), 1, None) == INV
    assert lib.fax_adamw8_step(ctx, C.byref(t), 1, C.byref(fx.AdamwHparams(1e-3, 0.9, 0.95, 1e-8, 1, 0))) == 0     # nothing but an empty tensor


def test_quantize_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding_ops as ops
    names = [f for f, _ in ops.Fp8QuantizeDesc._fields_]
    good = dict(rows=200, cols=300, x=P, ldx=300, format=0, tile=1, q=P, ldq=304, s=P, lds=200, qt=P, ldqt=208, st=P, ldst=300)

    def call(prec=0, c=ctx, **kw):
        f = dict(good, **kw)
        return lib.fax_op_fp8_quantize(c, prec, C.byref(ops.Fp8QuantizeDesc(*(f[k] for k in names))))
    for bad in (dict(c=None), dict(prec=3), dict(x=None), dict(q=None, qt=None), dict(format=2), dict(format=-1), dict(tile=64), dict(tile=0), dict(rows=0), dict(cols=-1),
                dict(ldx=299), dict(x=P + 1), dict(prec=1, x=P + 2), dict(s=None), dict(st=None), dict(ldq=288), dict(ldq=301), dict(ldqt=192), dict(ldqt=209), dict(q=P + 8),
                dict(qt=P + 4), dict(s=P + 2), dict(st=P + 1), dict(lds=199), dict(ldst=299), dict(tile=128, lds=1), dict(tile=128, ldst=2)):
        assert call(**bad) == INV, bad
    assert lib.fax_op_fp8_quantize(ctx, 0, None) == INV
    assert call(rows=0x7fffffff, cols=0x7fffffff, ldx=1 << 31, ldq=1 << 31, lds=1 << 31, ldqt=1 << 31, ldst=1 << 31) == SHAPE


def test_product_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding_ops as ops
    names = [f for f, _ in ops.Fp8GemmDesc._fields_]
    good = dict(M=200, N=300, K=400, A=P, lda=400, a_format=0, a_scale=P, a_scale_ld=200, B=P, ldb=400, b_format=1, b_scale=P, b_scale_ld=300, b_tile=1,
                C=P, ldc=300, c_f32=1, accumulate=1, bias=None)

    def call(c=ctx, **kw):
        f = dict(good, **kw)
        return lib.fax_op_fp8_gemm(c, C.byref(ops.Fp8GemmDesc(*(f[k] for k in names))))
    for bad in (dict(c=None), dict(A=None), dict(B=None), dict(C=None), dict(a_scale=None), dict(b_scale=None), dict(M=0), dict(N=-1), dict(K=0), dict(a_format=2), dict(b_format=-1),
                dict(b_tile=64), dict(c_f32=0), dict(lda=384), dict(lda=408), dict(ldb=392), dict(ldb=401), dict(ldc=299), dict(a_scale_ld=199), dict(b_scale_ld=299),
                dict(b_tile=128, b_scale_ld=2), dict(A=P + 8), dict(B=P + 1), dict(C=P + 2), dict(a_scale=P + 2), dict(b_scale=P + 1), dict(bias=P + 1)):
        assert call(**bad) == INV, bad
    assert lib.fax_op_fp8_gemm(ctx, None) == INV
    assert call(lda=1 << 40) == SHAPE


# ---- the references themselves ----

@pytest.mark.parametrize("fmt", [0, 1])
def test_reference_rounding_is_the_formats(fmt):
    """Every value of the format is a fixed point, and rounding to nearest agrees with torch's conversion."""
    codes = torch.arange(256, dtype=torch.uint8).view(ref.TORCH8[fmt]).double().numpy()
    codes = codes[np.isfinite(codes)]
    step = ref.step_at(codes, fmt)
    assert np.array_equal(np.round(codes / step) * step, codes)
    rng = np.random.default_rng(fmt)
    x = rng.standard_normal((64, 300)) * 10.0 ** rng.uniform(-5, 5, (64, 1))
    q, s = ref.quantize(x, fmt, 1)
    y = (x / np.repeat(s.T, 128, axis=1)[:, :300])
    assert np.array_equal(torch.as_tensor(y).to(ref.TORCH8[fmt]).double().numpy(), q)
    assert np.abs(q).max() <= ref.TOP[fmt] and np.all(np.log2(s) == np.round(np.log2(s)))


def test_reference_moments():
    rng = np.random.default_rng(0)
    x = rng.standard_normal(1000) * 10.0 ** rng.uniform(-6, 0, 1000)
    for fmt, y in ((0, x), (1, x * x)):
        low, s = ref.round_moment(y, fmt, np.zeros(1000))
        high, _ = ref.round_moment(y, fmt, np.full(1000, 65535.0))
        t = np.repeat(s, 128)[:1000]
        assert np.all(np.abs(low) <= np.abs(high)) and np.all(np.abs(low * t - y) <= ref.step_at(y / t, fmt) * t * (1 + 1e-6))
        assert np.array_equal(torch.as_tensor(low).to(ref.TORCH8[fmt]).double().numpy(), low)


def test_embedding_refuses_rows_past_its_positions(lib, ctx):
    nb = C.c_size_t()
    for d in ((1 << 30) + 1, 0x7fffffff):
        assert lib.fax_op_embedding_forward(ctx, 0, 1, 2, d, P, P, 1.0, P) == SHAPE
        assert lib.fax_op_embedding_backward_scratch_bytes(1, 2, d, C.byref(nb)) == SHAPE
        assert lib.fax_op_embedding_backward(ctx, 0, 1, 2, d, P, P, 1.0, 0, P, P, 1 << 40) == SHAPE
    assert lib.fax_op_embedding_backward_scratch_bytes(1, 2, 1 << 30, C.byref(nb)) == 0


@pytest.mark.parametrize("n", [2, 40, 41, 300])
def test_adamw8_refuses_the_same_weights_twice(lib, ctx, n):
    from paper_2204_06514_b200 import binding as fx
    t = [fx.Adamw8Tensor(P * (i + 1), P, P, P, P, P, None, 64, 0.0, 1) for i in range(n)]
    t[-1].w = t[n // 2 - 1].w
    arr = (fx.Adamw8Tensor * n)(*t)
    hp = C.byref(fx.AdamwHparams(1e-3, 0.9, 0.95, 1e-8, 1, 0))
    assert lib.fax_adamw8_step(ctx, arr, n, hp) == INV
    for x in arr:                                                    # empty tensors share whatever they like
        x.n = 0
    assert lib.fax_adamw8_step(ctx, arr, n, hp) == 0
