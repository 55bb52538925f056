"""Scratch of the token table's gradient: what serves a batch serves every shorter one, a smaller table and fewer columns."""
import pytest

N = [0, 1, 2, 15, 16, 17, 300, 511, 512, 513, 1000, 4095, 16000, 16383, 16384, 16385, 16400, 20000, 32768, 32769, 60000, 65537, 131071, 131072, 131073, 131584, 131585,
     200000, 262144, 262145, 524289, 1 << 20, (1 << 20) + 1, 3 << 20, (1 << 24) - 1, 1 << 24, (1 << 24) + 513, 1 << 30]


@pytest.fixture(scope="module")
def need():
    from paper_2204_06514_b200 import build, binding_ops as ops
    build.build()
    return ops.fax_op_embedding_backward_scratch_bytes


@pytest.mark.parametrize("vocab,d", [(1, 1), (2, 8), (255, 64), (256, 768), (50304, 768), (50304, 4096), (1 << 24, 16), ((1 << 31) - 1, 3)])
def test_scratch_never_shrinks_with_more_tokens(need, vocab, d):
    sizes = [need(n, vocab, d) for n in N]
    assert sizes == sorted(sizes), [(N[i], sizes[i], N[i + 1], sizes[i + 1]) for i in range(len(N) - 1) if sizes[i] > sizes[i + 1]]


@pytest.mark.parametrize("n", [1, 513, 16384, 131073])
def test_scratch_never_shrinks_with_the_table(need, n):
    for d in (1, 8, 768):
        sizes = [need(n, v, d) for v in (1, 2, 127, 255, 256, 65535, 65536, 50304 * 4, 1 << 24, (1 << 31) - 1)]
        assert sizes == sorted(sizes), d
    sizes = [need(n, 1000, d) for d in (1, 3, 4, 7, 8, 768, 4096)]
    assert sizes == sorted(sizes)


@pytest.mark.gpu
@pytest.mark.parametrize("accumulate", [0, 1])
def test_scratch_of_the_longest_batch_serves_the_shorter(accumulate):
    import numpy as np
    import torch
    import lowbit_ref as ref
    from parity_util import Session, host, ptr
    from paper_2204_06514_b200 import binding_ops as ops
    longest, vocab, d = 16385, 300, 24
    s = Session(0)
    try:
        nb = ops.fax_op_embedding_backward_scratch_bytes(longest, vocab, d)
        scratch = torch.full((nb + 4096,), 0x55, dtype=torch.uint8, device=s.device)
        rng = np.random.default_rng(1)
        for n in (longest, 16384, 16000, 8193, 600, 1):
            ids = rng.integers(-1, vocab, n).astype(np.int32)
            tid, g = torch.as_tensor(ids).to(s.device), torch.as_tensor(rng.standard_normal((n, d)).astype(np.float32)).to(s.device)
            out = torch.ones((vocab, d), device=s.device)
            ops.fax_op_embedding_backward(s.ctx, 1, n, vocab, d, ptr(tid), ptr(g), 0.5, accumulate, ptr(out), ptr(scratch), nb)
            want, size = ref.embedding_grad(ids, host(g), vocab, 0.5), ref.embedding_grad(ids, np.abs(host(g)), vocab, 0.5)
            # one rounding an addition, of a sum that is at most `size`; the scale and the old value once each
            count = np.bincount(ids[ids >= 0], minlength=vocab)[:, None]
            assert np.all(np.abs(host(out) - want - accumulate) <= (count + 3) * 2.0 ** -24 * (size + accumulate)), n
        assert bool((scratch[nb:] == 0x55).all())
    finally:
        s.close()
