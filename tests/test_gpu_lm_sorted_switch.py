"""The switch between float atomics and sorted sums for the language model's token table gradient."""
import numpy as np
import pytest
import torch

from parity_util import LmRunner, Session, fx, hparams, synth

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


@pytest.fixture
def sess():
    s = Session(0)
    yield s
    s.close()


def tokens(sess, cfg):
    return [torch.as_tensor(np.ascontiguousarray(a)).to(sess.device) for a in synth.lm_tokens(cfg)]


@pytest.mark.parametrize("batch", [2, 8])
def test_arena_without_the_sorts_part(sess, batch):
    """A vocabulary so small that the sort's scratch does not fit the logits' buffer: the arena that ends behind row_loss
    serves every call while the switch is off, and is refused while it is on."""
    cfg = synth.Config("lm_small_vocab", 17, batch=batch, seq=128, d_model=1024, n_heads=16, head_dim=64, d_ff=1024, n_layers=1, vocab=128)
    r = LmRunner(sess, cfg, synth.lm_params(cfg), fx.FAX_PREC_BF16, weight_decay=0.1)
    ids, tg = tokens(sess, cfg)
    short = (fx.fax_lm_arena_layout(r.lcfg)["row_loss"] + 4 * cfg.tokens + 255) // 256 * 256
    assert short < r.scratch_bytes
    r.scratch[short:] = 0x55
    r.state.scratch_bytes = short
    r.forward_backward(ids, tg)
    r.accumulate(ids, tg, True, 0.5)
    loss = r.step(ids, tg, hparams(step=1, **HP), want_host_loss=True)
    assert 0 < loss < 20 and bool((r.scratch[short:] == 0x55).all())
    fx.fax_set_sorted_embedding_gradient(sess.ctx, True)
    for call in (lambda: r.forward_backward(ids, tg), lambda: r.accumulate(ids, tg, True, 0.5), lambda: r.step(ids, tg, hparams(step=2, **HP))):
        with pytest.raises(fx.FaxError):
            call()
    r.state.scratch_bytes = short + 256
    with pytest.raises(fx.FaxError):
        r.forward_backward(ids, tg)
    r.state.scratch_bytes = r.scratch_bytes
    r.step(ids, tg, hparams(step=2, **HP))
    torch.cuda.synchronize()
    assert bool((r.scratch[short:] == 0x55).all()) == (cfg.tokens <= 512)      # so few tokens are not sorted


def test_switch_drops_the_recorded_steps(sess):
    """One model, the same buffers: steps recorded under one setting are not replayed under the other.  1024 tokens of 256
    ids take five launches sorted (count, two digits, sums, runs over chunk edges) where the atomics take one."""
    cfg = synth.Config("lm_switch", 18, batch=4, seq=256, d_model=128, n_heads=2, head_dim=64, d_ff=256, n_layers=1, vocab=256)
    r = LmRunner(sess, cfg, synth.lm_params(cfg), fx.FAX_PREC_BF16, weight_decay=0.1)
    ids, tg = tokens(sess, cfg)
    step, counts = 0, []
    for on in (False, True, False, True):
        fx.fax_set_sorted_embedding_gradient(sess.ctx, on)
        for _ in range(4):                                           # as it is, recorded, replayed twice
            step += 1
            before = sess.launches()
            r.step(ids, tg, hparams(step=step, **HP))
            counts.append(sess.launches() - before)
    n = counts[0]
    assert counts == [n] * 4 + [n + 4] * 4 + [n] * 4 + [n + 4] * 4


def test_sorted_gradient_is_the_same_bits_every_time(sess):
    """In float32 the order of the token table's additions is all that could change from run to run."""
    cfg = synth.Config("lm_bits", 19, batch=4, seq=256, d_model=64, n_heads=2, head_dim=32, d_ff=64, n_layers=1, vocab=11)
    r = LmRunner(sess, cfg, synth.lm_params(cfg), fx.FAX_PREC_FP32_VALIDATE)
    ids, tg = tokens(sess, cfg)
    fx.fax_set_sorted_embedding_gradient(sess.ctx, True)
    first = None
    for _ in range(6):
        r.forward_backward(ids, tg)
        if first is None:
            first = r.wte.g.clone()
        assert torch.equal(r.wte.g, first) and bool(first.any())
