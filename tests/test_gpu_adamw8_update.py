"""The update of the weights under 8-bit moments: its root and its quotient where they can go wrong."""
import numpy as np
import pytest
import torch

from parity_util import Session, fx, hparams, host, ptr

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    s.close()


def first_step(sess, g, lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8, w=0.0):
    """Weights after step 1 from moments of zero, without decay."""
    n, dev = g.numel(), sess.device
    wt = torch.full((n,), w, device=dev)
    m, v = (torch.zeros(n, dtype=torch.uint8, device=dev) for _ in range(2))
    ms, vs = (torch.zeros(-(-n // 128), device=dev) for _ in range(2))
    t = fx.Adamw8Tensor(ptr(wt), ptr(m), ptr(v), ptr(ms), ptr(vs), ptr(g), None, n, 0.0, 3)
    fx.fax_adamw8_step(sess.ctx, [t], hparams(step=1, lr=lr, beta1=beta1, beta2=beta2, eps=eps))
    return wt


@pytest.mark.parametrize("what", [float("inf"), float("-inf"), float("nan"), 3e38, 1e25])
def test_one_element_out_of_range_leaves_its_neighbours(sess, what):
    """With eps = 0 a gradient and moments of zero give 0 / 2^-63 = 0 (the root is taken of at least 2^-126), whatever
    stands beside them in the block of 128."""
    g = torch.zeros(384, device=sess.device)
    g[1] = 1e-25                                                     # g^2 is 0 in float32: over the smallest root
    g[2] = -3e-3
    g[128:256] = g[:128]
    g[128 + 77] = what
    w = first_step(sess, g, eps=0.0, w=0.5)
    others = torch.arange(128, device=sess.device) != 77
    assert torch.equal(w[128:256][others], w[:128][others]) and bool((w[256:] == 0.5).all())
    assert bool((w[3:128] == 0.5).all())
