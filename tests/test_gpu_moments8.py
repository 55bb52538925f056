"""8-bit moments in place of the float32 ones: what they take, and a model and a block without any others."""
import numpy as np
import pytest
import torch

import lowbit_ref as ref
from parity_util import BlockRunner, LmRunner, Session, fx, host, hparams, synth
from paper_2204_06514_b200.state import Moments8, ParamSet

pytestmark = pytest.mark.gpu
HP = dict(lr=1e-3, beta1=0.9, beta2=0.95, eps=1e-8)


@pytest.fixture(scope="module")
def sess():
    s = Session(0)
    yield s
    st, detail = fx.fax_check_device_status(s.ctx)
    s.close()
    assert st == fx.FAX_OK, detail


def held(make):
    torch.cuda.synchronize()
    before = torch.cuda.memory_allocated()
    keep = make()
    return torch.cuda.memory_allocated() - before, keep


def test_optimizer_state_is_two_bytes_a_parameter(sess):
    """Beside weights, bf16 copy and gradient (10 bytes): 8 bytes of float32 moments, or 2 and two scales for each 128."""
    n = 1 << 22
    w = np.zeros(n, np.float32)
    plain, a = held(lambda: ParamSet(w, fx.FAX_PREC_BF16, sess.device, 0.1))
    bare, b = held(lambda: ParamSet(w, fx.FAX_PREC_BF16, sess.device, 0.1, moments=False))
    eight, c = held(lambda: Moments8([b]))
    assert plain == 18 * n and bare == 10 * n and eight == 2 * n + 8 * (n // 128)


def step_against_reference(sess, params, opt, state, seed, step):
    opt.step(sess.ctx, hparams(step=step, **HP))
    for i, p in enumerate(params):
        state[i] = list(ref.adamw8(*state[i], host(p.g).ravel(), p.weight_decay, seed + i, step=step, **HP))
        assert np.array_equal(host(opt.m[i].view(torch.float8_e4m3fn)), state[i][1])
        assert np.array_equal(host(opt.v[i].view(torch.float8_e5m2)), state[i][3])
        assert np.abs(host(p.w).ravel() - state[i][0]).max() <= 1e-6 * np.abs(state[i][0]).max()
        state[i][0] = host(p.w).ravel()
        assert torch.equal(p.wc, p.w.to(torch.bfloat16)) and bool(p.g.any())


def zero_state(params):
    blocks = lambda p: -(-p.w.numel() // 128)  # noqa: E731
    return [[host(p.w).ravel(), np.zeros(p.w.numel()), np.ones(blocks(p)), np.zeros(p.w.numel()), np.ones(blocks(p))] for p in params]


@pytest.mark.parametrize("sorted_sums", [0, 1])
def test_language_model_without_float32_moments(sess, sorted_sums):
    cfg = synth.Config("lm_m8", 20, batch=2, seq=128, d_model=128, n_heads=2, head_dim=64, d_ff=256, n_layers=2, vocab=256)
    r = LmRunner(sess, cfg, synth.lm_params(cfg), fx.FAX_PREC_BF16, weight_decay=0.1, moments=False)
    ids, tg = (torch.as_tensor(np.ascontiguousarray(a)).to(sess.device) for a in synth.lm_tokens(cfg))
    params = [p for _, p in r.named_params()]
    assert all(p.m is None and p.v is None for p in params)
    opt, state = Moments8(params, seed=5), zero_state(params)
    fx.fax_set_sorted_embedding_gradient(sess.ctx, bool(sorted_sums))
    try:
        losses = []
        for step in (1, 2, 3):
            r.accumulate(ids, tg, False, 0.5)
            r.accumulate(ids, tg, True, 0.5)
            step_against_reference(sess, params, opt, state, 5, step)
            losses.append(float(r.loss.item()))
        r.forward_backward(ids, tg)
        assert np.all(np.isfinite(losses)) and bool(r.wte.g.any())
    finally:
        fx.fax_set_sorted_embedding_gradient(sess.ctx, False)
    # what would update weights by float32 moments says so, before anything is changed
    w = r.wte.w.clone()
    cpu = lambda t: t.cpu().pin_memory()  # noqa: E731
    for call in (lambda: r.step(ids, tg, hparams(step=4, **HP)), lambda: r.apply_adamw(hparams(step=4, **HP)), lambda: r.step_host(cpu(ids), cpu(tg), hparams(step=4, **HP))):
        with pytest.raises(fx.FaxError) as e:
            call()
        assert e.value.status == fx.FAX_ERR_INVALID_ARG
    assert torch.equal(r.wte.w, w)


def test_block_without_float32_moments(sess):
    cfg = synth.Config("block_m8", 21, batch=1, seq=128, d_model=128, n_heads=2, head_dim=64, d_ff=256)
    r = BlockRunner(sess, cfg, synth.block_params(cfg), fx.FAX_PREC_BF16, moments=False)
    x, dy = (r.to_device(a) for a in synth.block_inputs(cfg))
    params = list(r.p.values())
    opt, state = Moments8(params, seed=9), zero_state(params)
    for step in (1, 2):
        r.forward(x)
        r.backward(dy)
        step_against_reference(sess, params, opt, state, 9, step)
    for call in (lambda: r.step(x, dy, hparams(step=3, **HP)), lambda: r.adamw(hparams(step=3, **HP))):
        with pytest.raises(fx.FaxError) as e:
            call()
        assert e.value.status == fx.FAX_ERR_INVALID_ARG


def test_gradients_of_the_sets_are_float32(sess):
    """A step asked for with bf16 gradients reads the sets' own all the same, as fax_lm_step does."""
    rng = np.random.default_rng(2)
    p = ParamSet(rng.standard_normal(1000).astype(np.float32), fx.FAX_PREC_BF16, sess.device, 0.1)
    p.g.copy_(torch.as_tensor(rng.standard_normal(1000).astype(np.float32)))
    opt, state = Moments8([p], seed=4), zero_state([p])
    opt.step(sess.ctx, hparams(step=1, grad_is_bf16=1, **HP))
    want = ref.adamw8(*state[0], host(p.g), 0.1, 4, step=1, **HP)
    assert np.array_equal(host(opt.m[0].view(torch.float8_e4m3fn)), want[1]) and np.abs(host(p.w) - want[0]).max() <= 1e-6
