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


@pytest.mark.parametrize("order", ["sorted", "mixed"])
@pytest.mark.parametrize("eps", [0.0, 1e-8, 1e-3])
@pytest.mark.parametrize("lr,beta1,beta2", [(1e-3, 0.9, 0.95), (1.0, 0.0, 0.999), (3e-4, 0.9, 0.0)])
def test_root_and_quotient_within_a_unit_of_the_last_place(sess, order, eps, lr, beta1, beta2):
    """From weights and moments of zero a step leaves minus the update: lr m c1 / (sqrt(v c2) + eps), the root taken of at
    least 2^-126.  Root and quotient are each off by one unit of the last place at most, 2^-23 of the value, and the sum
    with eps by half a unit.  Gradients of 1e-30 to 1e18, sorted (blocks beyond 2^96 take the library's root and quotient,
    the others the approximations) and mixed within blocks; whole binades of consecutive ones among them."""
    rng = np.random.default_rng(7)
    g = np.concatenate([10.0 ** rng.uniform(-30, 18, 1 << 19), np.arange(1 << 23, 1 << 24, 37) * 2.0 ** -23, np.arange(1 << 23, 1 << 24, 37) * 2.0 ** -33]).astype(np.float32)
    g *= rng.choice([-1, 1], g.size).astype(np.float32)
    g = g[np.argsort(np.abs(g))] if order == "sorted" else rng.permutation(g)
    w = host(first_step(sess, torch.as_tensor(g).to(sess.device), lr, beta1, beta2, eps))

    f = lambda x: np.asarray(x, np.float64).astype(np.float32).astype(np.float64)  # noqa: E731
    lr, b1, b2, eps = (float(np.float32(x)) for x in (lr, beta1, beta2, eps))
    c1, c2, g = float(f(1 / (1 - b1))), float(f(1 / (1 - b2))), g.astype(np.float64)
    m, v = f(float(f(1 - b1)) * g), f(f(float(f(1 - b2)) * g) * g)
    a, x = f(lr * f(m * c1)), np.maximum(f(v * c2), 2.0 ** -126)
    want = -a / (np.sqrt(x) + eps)
    bound = (2 * 2.0 ** -23 + (2.0 ** -24 if eps else 0)) * (1 + 2.0 ** -20) * np.abs(want) + 2.0 ** -149
    err = np.abs(w - want)
    assert np.all(err <= bound), (int((err > bound).sum()), float((err / np.abs(want)).max() * 2 ** 23), g[np.argmax(err / bound)])
