"""The 8-bit product on pairs of SMs: captured and replayed, on two streams at once, and without programmatic launches."""
import pytest
import torch

from parity_util import Session, fx
from paper_2204_06514_b200 import binding_ops as ops
from test_gpu_fp8_routes import Matrix, call

pytestmark = pytest.mark.gpu
SHAPES = [(900, 3500, 3900, 0), (1300, 5000, 3900, 1), (1300, 3500, 600, 0), (3000, 770, 1030, 1)]


class Products:
    """The four shapes' operands and outputs on one stream."""

    def __init__(self, seed):
        self.stream = torch.cuda.Stream(0)
        with torch.cuda.stream(self.stream):
            self.s = Session(0)
            g = torch.Generator(device=self.s.device)
            g.manual_seed(seed)
            self.ops = []
            for m, n, k, f32 in SHAPES:
                assert ops.fax_op_fp8_gemm_tile(self.s.ctx, m, n, k, f32)[0] == 2
                a, b = Matrix(self.s, m, k, 0, 1, g), Matrix(self.s, n, k, 1, 128, g)
                out = torch.full((m, n), float("nan"), dtype=torch.float32 if f32 else torch.bfloat16, device=self.s.device)
                self.ops.append((a, b, out, n))
        self.stream.synchronize()

    def run(self):
        for a, b, out, n in self.ops:
            call(self.s, a, b, out, n)

    def results(self):
        self.stream.synchronize()
        return [out.clone() for _, _, out, _ in self.ops]

    def clear(self):
        with torch.cuda.stream(self.stream):
            for o in self.ops:
                o[2].fill_(float("nan"))
        self.stream.synchronize()

    def close(self):
        self.stream.synchronize()
        st, detail = fx.fax_check_device_status(self.s.ctx)
        self.s.close()
        assert st == fx.FAX_OK, detail


@pytest.fixture
def two():
    p = [Products(1), Products(2)]
    yield p
    for x in p:
        x.close()


def same(a, b):
    return all(torch.equal(x, y) for x, y in zip(a, b))


def alone(two):
    want = []
    for p in two:
        p.run()
        want.append(p.results())
        p.clear()
    assert not same(*want)
    return want


def test_on_two_streams_at_once(two):
    want = alone(two)
    for _ in range(10):
        for p in two:
            p.run()
    assert all(same(p.results(), w) for p, w in zip(two, want))


def test_two_graphs_replayed_at_once(two):
    want = alone(two)
    graphs = []
    for p in two:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, stream=p.stream):
            for _ in range(3):
                p.run()
        graphs.append(g)
        p.clear()
    for _ in range(5):
        for p, g in zip(two, graphs):
            with torch.cuda.stream(p.stream):
                g.replay()
    assert all(same(p.results(), w) for p, w in zip(two, want))
    # other numbers in the same buffers
    for p, g in zip(two, graphs):
        for a, b, _, _ in p.ops:
            with torch.cuda.stream(p.stream):
                a.q ^= 0x80                                          # every sign of A
        with torch.cuda.stream(p.stream):
            g.replay()
    got = [p.results() for p in two]
    for p in two:
        p.clear()
    assert all(same(x, y) for x, y in zip(got, alone(two))) and not same(got[0], want[0])
    del graphs


def test_without_programmatic_launches(two):
    want = alone(two)
    for p in two:
        fx.fax_set_dependent_launch(p.s.ctx, False)
        p.run()
    assert all(same(p.results(), w) for p, w in zip(two, want))
