"""The recurrence where channels and sequences alone fill the GPU, so that each warp takes whole sequences: every way rows come in,
both types, with and without a gate, on both sides of the numbers of sequences at which the backward pass takes larger CTAs."""
import numpy as np
import pytest

import pieces_ref as ref
from test_gpu_recurrence import Layer, sess  # noqa: F401

pytestmark = pytest.mark.gpu

# units (sequences times tiles of 64 channels) by the SMs: from 12 an SM on a warp has a sequence by itself; up to 16, and
# from 24 to 32, the backward pass takes CTAs of 16 warps (where sequences have more than two stretches)
UNITS = {"12": (12, 0), "12 and one": (12, 1), "13": (13, 0), "16": (16, 0), "16 and one": (16, 1), "24 and one": (24, 1), "32": (32, 0)}


@pytest.mark.parametrize("prec", [0, 1])
@pytest.mark.parametrize("gated", [False, True])
@pytest.mark.parametrize("d", [64, 62, 63], ids=["boxes", "pairs", "singles"])
@pytest.mark.parametrize("units", list(UNITS))
def test_a_sequence_a_warp(sess, units, d, gated, prec):  # noqa: F811
    import torch
    an_sm, more = UNITS[units]
    n = an_sm * torch.cuda.get_device_properties(0).multi_processor_count + more
    rng = np.random.default_rng(n + d)
    lengths = rng.integers(0, 4, n)
    lengths[rng.integers(0, n, 20)] = rng.integers(33, 60, 20)
    layer = Layer(sess, prec, list(lengths), d, gated, ref.PLAIN if d == 62 else ref.COMPLEMENT, d)
    assert layer.seq > 32
    layer.forward()
    layer.backward()
    layer.check()
