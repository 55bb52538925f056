"""The recurrence's gates over the whole range of their inputs: what a shut gate lets through is nothing, whatever stands before or behind it."""
import numpy as np
import pytest
import torch

import pieces_ref as ref
from test_gpu_recurrence import Layer, sess  # noqa: F401

pytestmark = pytest.mark.gpu

# a token or two; one stretch; CTAs that share a sequence; the same without boxes
SHAPES = [([1, 2, 1], 64), ([16, 9], 64), ([100, 300], 64), ([100, 300], 63), ([37], 62)]


def shut(prec):
    """Where exp(-|v|) is below every float32 number."""
    return [float(torch.finfo(ref.DTYPE[prec]).min), -1e30, -1000.0, -200.0]


def fill(layer, name, values):
    """Channel c has values[c % len(values)] in every row."""
    v = np.tile(np.resize(ref.rounded(values, layer.prec), layer.d), (layer.rows, 1))
    setattr(layer, name, v)
    getattr(layer, "t" + name).copy_(torch.as_tensor(v))


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("mode", [ref.PLAIN, ref.COMPLEMENT])
@pytest.mark.parametrize("lengths,d", SHAPES)
def test_a_shut_output_gate(sess, lengths, d, mode, prec):  # noqa: F811
    """g sigmoid(g) and its derivative are 0 for a g this low: no output, and no gradient but dh_last's."""
    layer = Layer(sess, prec, lengths, d, True, mode, 1, dh_last=False)
    fill(layer, "g", shut(prec))
    layer.forward()
    layer.backward()
    for t in (layer.y, layer.df, layer.dx, layer.dg, layer.dh0):
        assert float(t.abs().max()) == 0


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("lengths,d", SHAPES)
def test_a_state_that_is_forgotten(sess, lengths, d, prec):  # noqa: F811
    """a is 0: a large state leaves nothing behind, a large gradient hands nothing back."""
    layer = Layer(sess, prec, lengths, d, False, ref.PLAIN, 2)
    fill(layer, "f", shut(prec) + [-np.inf])
    layer.th0.fill_(1e38)
    layer.tdh_last.fill_(1.0)
    layer.forward()
    layer.backward()
    assert torch.equal(layer.y.float(), layer.tx.float())
    ends = torch.as_tensor(layer.at[1:] - 1, device=sess.device)
    assert torch.equal(layer.h_last, layer.tx.float()[ends])
    assert float(layer.df.abs().max()) == 0 and float(layer.dh0.abs().max()) == 0
    layer.th0.fill_(1.0)
    layer.tdh_last.fill_(1e38)
    layer.forward()
    layer.backward()
    assert float(layer.dh0.abs().max()) == 0


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("lengths,d", SHAPES)
def test_a_shut_output_gate_beside_a_large_state(sess, lengths, d, prec):  # noqa: F811
    """The products of a large state with a large gradient pass float's range; what the gate's derivative, 0, makes of them does not."""
    layer = Layer(sess, prec, lengths, d, True, ref.PLAIN, 1, dh_last=False)
    fill(layer, "g", shut(prec))
    fill(layer, "f", [np.inf])
    layer.tx.zero_()
    layer.th0.fill_(1e38)
    layer.tdy.fill_(10.0)
    layer.forward()
    layer.backward()
    assert bool((layer.h_last == layer.th0).all())
    for t in (layer.y, layer.df, layer.dx, layer.dg, layer.dh0):
        assert float(t.abs().max()) == 0


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("length", [1, 5])
def test_gates_along_their_range(sess, length, prec):  # noqa: F811
    """sigmoid(f) and 1 - sigmoid(f) of a token from -100 to 100: within their relative error, and 2^-126, below which a float is flushed."""
    f = ref.rounded(np.linspace(-100, 100, 1001), prec)
    for mode, h0, x in ((ref.PLAIN, 1.0, 0.0), (ref.COMPLEMENT, 0.0, 1.0)):
        # the gates are the last token's; the ones before it keep the state (f = inf), and add nothing
        layer = Layer(sess, prec, [length], len(f), False, mode, 3)
        v = np.full((length, len(f)), np.inf)
        v[-1] = f
        layer.tf.copy_(torch.as_tensor(v))
        layer.tx.fill_(0.0)
        layer.tx[-1] = x
        layer.th0.fill_(h0)
        layer.forward()
        want = ref.sigmoid(f) if mode == ref.PLAIN else ref.sigmoid(-f)
        got = layer.h_last[0].double().cpu().numpy()
        assert np.all(np.abs(got - want) <= (ref.gate_error(f) + 8 * ref.F32) * want + 2.0 ** -126)
