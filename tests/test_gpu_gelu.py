"""GELU in the epilogues of a product and on its own, element by element: where 1 + tanh cancels as well."""
import numpy as np
import pytest
import torch

from parity_util import Session, fx, host, ptr
from paper_2204_06514_b200 import binding_ops as ops

pytestmark = pytest.mark.gpu
M, N, K = 256, 256, 128


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


def every_h(dev):
    """65536 bf16 numbers: every one with |h| in [2^-8, 8), both signs, some of them twice."""
    bits = torch.arange(0x3B80, 0x4100, dtype=torch.int32)
    h = torch.cat([bits, bits | 0x8000])
    h = h.repeat(-(-M * N // h.numel()))[:M * N]
    return torch.where(h >= 0x8000, h - 0x10000, h).to(torch.int16).view(torch.bfloat16).view(M, N).to(dev)


def gemm(sess, epi, a, b, c, bias=None, aux=None, two_cta=True):
    fx.fax_set_gemm_two_cta(sess.ctx, two_cta)
    try:
        ops.fax_op_gemm(sess.ctx, 0, ops.GemmDesc(M, N, K, ptr(a), K, 0, ptr(b), K, 0, ptr(c), N, 0, 0, epi, ptr(bias), None, 0, ptr(aux), N, 1.0, 0))
    finally:
        fx.fax_set_gemm_two_cta(sess.ctx, True)


def terms(x):
    """u' and (1 + tanh u) / 2, (1 - tanh u) / 2 without the cancellation that leaves 0 of 1 + tanh u below u = -19."""
    u = np.sqrt(2 / np.pi) * (x + 0.044715 * x ** 3)
    return np.sqrt(2 / np.pi) * (1 + 3 * 0.044715 * x * x), 1 / (1 + np.exp(-2 * u)), 1 / (1 + np.exp(2 * u))


# u = sqrt(2/pi) (h + 0.044715 h^3) in float32: below 2^-21 of |u| off, |u| <= 25, so exp(-2u) is off by a relative
# 2 * 25 * 2^-21, and 1 / (1 + exp(-2u)) by no more; the approximations of exp2 and the reciprocal add 2^-21 at most,
# the products around them 2^-21: below 2^-15 of the value in all.  Then half a bf16 step (and 2^-133 for bf16's
# smallest numbers).
REL = 2.0 ** -15


@pytest.mark.parametrize("two_cta", [True, False])
def test_gelu_of_every_number(sess, two_cta):
    """h = H times the unit matrix: exact, so GELU is all that rounds."""
    h = every_h(sess.device)
    eye = torch.zeros((N, K), device=sess.device, dtype=torch.bfloat16)
    eye[:K] = torch.eye(K, dtype=torch.bfloat16)
    bias = torch.zeros(N, dtype=torch.bfloat16, device=sess.device)
    for half in (0, 1):                                              # 128 columns of h at a time, in the first 128 of C
        a = h[:, half * K:(half + 1) * K].contiguous()
        c, g = (torch.empty((M, N), dtype=torch.bfloat16, device=sess.device) for _ in range(2))
        gemm(sess, ops.FAX_EPI_BIAS_GELU, a, eye, c, bias, g, two_cta)
        assert torch.equal(c[:, :K], a)
        want = host(a) * terms(host(a))[1]
        err = np.abs(host(g[:, :K]) - want)
        assert np.all(err <= (REL + 2.0 ** -8) * np.abs(want) + 2.0 ** -133), (err / np.abs(want)).max()


@pytest.mark.parametrize("two_cta", [True, False])
def test_gelu_derivative_of_every_number(sess, two_cta):
    """A product of 1 everywhere times the derivative.  It is s + 2 h s (1 - s) u' with s = 1 / (1 + exp(-2u)): each term
    within REL of its size, and 1 - s within 2^-22."""
    h = every_h(sess.device)
    a = torch.zeros((M, K), dtype=torch.bfloat16, device=sess.device); a[:, 0] = 1
    b = torch.zeros((N, K), dtype=torch.bfloat16, device=sess.device); b[:, 0] = 1
    c = torch.empty((M, N), dtype=torch.bfloat16, device=sess.device)
    gemm(sess, ops.FAX_EPI_DGELU, a, b, c, aux=h, two_cta=two_cta)
    x = host(h)
    du, s, rest = terms(x)
    want = s + 2 * x * s * rest * du
    size = s + 2 * np.abs(x) * s * (rest + 2.0 ** -7) * du            # REL times 2^-7 is 2^-22
    err = np.abs(host(c) - want)
    assert np.all(err <= 2.0 ** -8 * np.abs(want) + 2 * REL * size + 2.0 ** -133), (err / np.abs(want)).max()
