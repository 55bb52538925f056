"""What the rotary positions, the dropout, the gated recurrence and the routing to experts refuse, checked before any CUDA
call (the context is a block of zeros that a refused call never looks into), the host-side tables, and the references themselves."""
import ctypes as C
import math
import os
import subprocess

import numpy as np
import pytest

import pieces_ref as ref

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


def caller(lib, name, struct, good, prec=True):
    fields = [f for f, _ in struct._fields_]
    assert sorted(fields) == sorted(good)

    def call(c, prec_value=0, **kw):
        f = dict(good, **kw)
        args = (c, prec_value) if prec else (c,)
        return getattr(lib, name)(*args, C.byref(struct(*(f[k] for k in fields))))
    return call


def test_rotary_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding_ops as ops
    call = caller(lib, "fax_op_rotary", ops.RotaryDesc, dict(rows=10, heads=4, head_dim=64, rot_dim=32, layout=0, x=P, ldx=256, y=2 * P, ldy=256, positions=None, first=0,
                                                             seq=10, frequencies=P, amplitude=1.0, backward=0))
    for bad in (dict(rows=-1), dict(heads=0), dict(head_dim=1), dict(rot_dim=31), dict(rot_dim=66), dict(rot_dim=0), dict(layout=2), dict(layout=-1), dict(seq=-1), dict(ldx=255),
                dict(ldy=255), dict(x=None), dict(y=None), dict(frequencies=None), dict(frequencies=P + 4), dict(positions=P + 2), dict(x=P + 1), dict(y=P + 1), dict(y=P, ldy=264)):
        assert call(ctx, **bad) == INV, bad
    assert call(None) == INV and call(ctx, 2) == INV and call(ctx, -1) == INV and call(ctx, 1, x=P + 2) == INV
    assert lib.fax_op_rotary(ctx, 0, None) == INV
    assert call(ctx, head_dim=1026, ldx=1 << 14, ldy=1 << 14) == SHAPE
    assert call(ctx, head_dim=65, ldx=260, ldy=260) == SHAPE
    assert call(ctx, rows=(1 << 30) + 1) == SHAPE
    assert call(ctx, rows=0, x=None, y=None, frequencies=None) == 0


def test_rotary_frequency_refusals_and_values(lib):
    from paper_2204_06514_b200 import binding_ops as ops
    f = lib.fax_rotary_frequencies
    out = (C.c_uint64 * 512)()
    for bad in ((0, 1e4, 1.0, 0, 1.0, 32.0), (63, 1e4, 1.0, 0, 1.0, 32.0), (1026, 1e4, 1.0, 0, 1.0, 32.0), (64, 0.5, 1.0, 0, 1.0, 32.0), (64, math.nan, 1.0, 0, 1.0, 32.0), (64, math.inf, 1.0, 0, 1.0, 32.0),
                (64, 1e4, 0.5, 0, 1.0, 32.0), (64, 1e4, math.nan, 0, 1.0, 32.0), (64, 1e4, 2.0, -1, 1.0, 32.0), (64, 1e4, 2.0, 4096, 32.0, 32.0), (64, 1e4, 2.0, 4096, math.nan, 32.0),
                (64, 1e4, 2.0, 4096, 1.0, math.inf)):
        assert f(*bad, out) == INV, bad
    assert f(64, 1e4, 1.0, 0, 1.0, 32.0, None) == INV
    for rot, base, factor, original in ((2, 1e4, 1.0, 0), (64, 1e4, 1.0, 0), (128, 5e5, 8.0, 8192), (96, 1e6, 4.0, 0), (1024, 1.0, 1.0, 0), (64, 1e4, 32.0, 1)):
        got = np.array(ops.fax_rotary_frequencies(rot, base, factor, original), dtype=np.float64) / 2.0 ** 64 * 2 * math.pi
        # both sides: a power, a quotient by 2 pi, and four more products at most, of 53 bits; the words' own step is 2^-64 of a turn
        np.testing.assert_allclose(got, ref.frequencies(rot, base, factor, original), rtol=16 * 2.0 ** -53, atol=2 * math.pi * 2.0 ** -65)


def test_dropout_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding_ops as ops
    call = caller(lib, "fax_op_dropout", ops.DropoutDesc, dict(rows=10, cols=64, x=P, ldx=64, resid=2 * P, ldr=64, y=3 * P, ldy=64, p=0.1, seed=1, offset=2, offset_device=None))
    for bad in (dict(rows=-1), dict(cols=0), dict(p=-0.01), dict(p=1.01), dict(p=math.nan), dict(ldx=63), dict(ldr=63), dict(ldy=63), dict(x=None), dict(y=None), dict(x=P + 1), dict(y=P + 1),
                dict(resid=P + 1), dict(offset_device=P + 4), dict(y=P, ldy=72), dict(y=2 * P, ldy=72)):
        assert call(ctx, **bad) == INV, bad
    assert call(None) == INV and call(ctx, 2) == INV and call(ctx, 1, y=P + 2) == INV
    assert lib.fax_op_dropout(ctx, 0, None) == INV
    wide = (1 << 30) + 1
    assert call(ctx, cols=wide, ldx=wide, ldr=wide, ldy=wide) == SHAPE
    assert call(ctx, rows=0x7fffffff, cols=1 << 20, ldx=1 << 20, ldr=1 << 20, ldy=1 << 20) == SHAPE
    assert call(ctx, rows=0, x=None, y=None) == 0


SHAPE_FIELDS = dict(rows=100, d=64, n_seq=10, seq=10, offsets=None, input=1, f=P, ldf=64, x=P, ldx=64, g=P, ldg=64, h0=None)


def test_recurrence_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding_ops as ops
    fwd = caller(lib, "fax_op_recurrence_forward", ops.RecurrenceDesc, dict(SHAPE_FIELDS, y=P, ldy=64, h_last=None, states=None))
    bwd = caller(lib, "fax_op_recurrence_backward", ops.RecurrenceBackwardDesc,
                 dict(SHAPE_FIELDS, states=P, dy=P, lddy=64, dh_last=None, df=2 * P, lddf=64, dx=2 * P, lddx=64, dg=2 * P, lddg=64, dh0=None))
    shared = (dict(rows=-1), dict(d=0), dict(n_seq=-1), dict(seq=-1), dict(input=2), dict(input=-1), dict(rows=99), dict(ldf=63), dict(ldx=63), dict(ldg=63), dict(f=None), dict(x=None), dict(f=P + 1),
              dict(x=P + 1), dict(g=P + 1), dict(offsets=P + 2), dict(h0=P + 2), dict(states=P + 1))
    for bad in shared + (dict(y=None), dict(ldy=63), dict(y=P + 1), dict(h_last=P + 2)):
        assert fwd(ctx, **bad) == INV, bad
    for bad in shared + (dict(states=None), dict(dy=None), dict(df=None), dict(dx=None), dict(dg=None), dict(lddy=63), dict(lddf=63), dict(lddx=63), dict(lddg=63), dict(dy=P + 1), dict(df=P + 1),
                         dict(dx=P + 1), dict(dg=P + 1), dict(dh_last=P + 2), dict(dh0=P + 2), dict(df=P, lddf=72), dict(dx=P, lddx=72), dict(dg=P, lddg=72)):
        assert bwd(ctx, **bad) == INV, bad
    for call, name in ((fwd, "forward"), (bwd, "backward")):
        assert call(None) == INV and call(ctx, 2) == INV and call(ctx, 1, f=P + 2) == INV
        assert getattr(lib, "fax_op_recurrence_" + name)(ctx, 0, None) == INV
        assert call(ctx, rows=(1 << 30) + 1, offsets=P) == SHAPE
        assert call(ctx, rows=0, n_seq=0, seq=0) == 0
    n = C.c_size_t()
    q = lib.fax_op_recurrence_states_floats
    assert q(10, 1, 4, None) == INV and q(-1, 1, 4, C.byref(n)) == INV and q(10, -1, 4, C.byref(n)) == INV and q(10, 1, 0, C.byref(n)) == INV
    assert q(160, 10, 8, C.byref(n)) == 0 and n.value == 20 * 8
    assert q(1 << 30, 1 << 20, 1 << 20, C.byref(n)) == 0 and n.value == ((1 << 26) + (1 << 20)) << 20


def test_every_sequence_has_its_own_kept_states(lib):
    """The states of sequence s begin at block offsets[s] / 16 + s: no two sequences share one, and all are within the size asked for."""
    rng = np.random.default_rng(5)
    for _ in range(200):
        lengths = rng.integers(0, 70, rng.integers(1, 30))
        at = np.concatenate([[0], np.cumsum(lengths)])
        end = 0
        for s, n in enumerate(lengths):
            first = at[s] // 16 + s
            assert first >= end
            end = first + -(-n // 16)
        assert end <= at[-1] // 16 + len(lengths)


def test_expert_refusals(lib, ctx):
    from paper_2204_06514_b200 import binding_ops as ops
    n = C.c_int32()
    q = lib.fax_op_expert_slots
    for bad in ((-1, 2, 8, 0, 1), (4, 0, 8, 0, 1), (4, 2, 0, 0, 1), (4, 2, 8, -1, 1), (4, 2, 8, 0, 0)):
        assert q(*bad, C.byref(n)) == INV, bad
    assert q(4, 2, 8, 0, 1, None) == INV
    assert q(4, 2, 1025, 0, 1, C.byref(n)) == SHAPE and q(1 << 30, 2, 8, 0, 1, C.byref(n)) == SHAPE and q(4, 2, 1024, 1 << 22, 1, C.byref(n)) == SHAPE
    assert q(100, 2, 8, 0, 128, C.byref(n)) == 0 and n.value == 200 + 8 * 127
    assert q(3, 1, 8, 0, 128, C.byref(n)) == 0 and n.value == 3 + 3 * 127
    assert q(100, 2, 8, 40, 0, C.byref(n)) == 0 and n.value == 320
    sort = caller(lib, "fax_op_expert_sort", ops.ExpertSortDesc, dict(n_tokens=10, top_k=2, n_experts=4, capacity=0, align=1, slots=20, ids=P, slot_of=P, source=P, offsets=P, counts=P), prec=False)
    for bad in (dict(n_tokens=-1), dict(top_k=0), dict(n_experts=0), dict(capacity=-1), dict(align=0), dict(ids=None), dict(slot_of=None), dict(source=None), dict(offsets=None), dict(counts=None),
                dict(ids=P + 2), dict(slot_of=P + 1), dict(source=P + 2), dict(offsets=P + 2), dict(counts=P + 3)):
        assert sort(ctx, **bad) == INV, bad
    assert sort(None) == INV and lib.fax_op_expert_sort(ctx, None) == INV
    assert sort(ctx, slots=19) == SMALL and sort(ctx, capacity=6, slots=23) == SMALL
    assert sort(ctx, n_experts=1025) == SHAPE
    rows = dict(n_tokens=10, top_k=2, d=64, slots=20, slot_of=P)
    dispatch = caller(lib, "fax_op_expert_dispatch", ops.ExpertDispatchDesc, dict(rows, source=P, x=P, ldx=64, out=P, ldo=64))
    combine = caller(lib, "fax_op_expert_combine", ops.ExpertCombineDesc, dict(rows, weights=P, z=P, ldz=64, resid=P, ldr=64, y=2 * P, ldy=64))
    back = caller(lib, "fax_op_expert_combine_backward", ops.ExpertCombineBackwardDesc, dict(rows, source=P, weights=P, z=P, ldz=64, dy=P, lddy=64, dz=2 * P, lddz=64, dw=P))
    shared = (dict(n_tokens=-1), dict(top_k=0), dict(d=0), dict(slots=-1), dict(slot_of=None), dict(slot_of=P + 2))
    for call, more in ((dispatch, (dict(source=None), dict(x=None), dict(out=None), dict(ldx=63), dict(ldo=63), dict(source=P + 1), dict(x=P + 1), dict(out=P + 1))),
                       (combine, (dict(z=None), dict(y=None), dict(ldz=63), dict(ldr=63), dict(ldy=63), dict(weights=P + 2), dict(z=P + 1), dict(resid=P + 1), dict(y=P + 1), dict(y=P, ldy=72))),
                       (back, (dict(source=None), dict(weights=None), dict(z=None), dict(dy=None), dict(dz=None), dict(ldz=63), dict(lddy=63), dict(lddz=63), dict(source=P + 1), dict(weights=P + 2),
                               dict(z=P + 1), dict(dy=P + 1), dict(dz=P + 1), dict(dw=P + 2), dict(dz=P, lddz=72)))):
        for bad in shared + more:
            assert call(ctx, **bad) == INV, bad
        assert call(None) == INV and call(ctx, 2) == INV
        assert call(ctx, n_tokens=1 << 30) == SHAPE
        assert call(ctx, n_tokens=0, slots=0) == 0
    for name in ("dispatch", "combine", "combine_backward"):
        assert getattr(lib, "fax_op_expert_" + name)(ctx, 0, None) == INV


def test_descriptors_lie_as_the_header_s(tmp_path):
    """Sizes and places of the fields, as a C compiler has them."""
    from paper_2204_06514_b200 import binding_ops as ops
    names = {"RotaryDesc": "rotary", "DropoutDesc": "dropout", "RecurrenceDesc": "recurrence", "RecurrenceBackwardDesc": "recurrence_backward", "ExpertSortDesc": "expert_sort",
             "ExpertDispatchDesc": "expert_dispatch", "ExpertCombineDesc": "expert_combine", "ExpertCombineBackwardDesc": "expert_combine_backward"}
    lines, want = [], []
    for py, c in names.items():
        struct = getattr(ops, py)
        lines.append(f'printf("%zu\\n", sizeof(fax_{c}_desc));')
        want.append(C.sizeof(struct))
        for field, _ in struct._fields_:
            lines.append(f'printf("%zu\\n", offsetof(fax_{c}_desc, {field}));')
            want.append(getattr(struct, field).offset)
    src = tmp_path / "sizes.c"
    src.write_text('#include <stdio.h>\n#include <stddef.h>\n#include "fax_ops.h"\nint main(void) {\n' + "\n".join(lines) + "\nreturn 0; }\n")
    include = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "include")
    subprocess.check_call(["gcc", "-std=c99", "-I", include, str(src), "-o", str(tmp_path / "sizes")])
    got = [int(x) for x in subprocess.check_output([str(tmp_path / "sizes")], text=True).split()]
    assert got == want


# ---- the references themselves ----

def test_generator_gives_the_published_vectors():
    """Known answers of Philox4x32-10, published with it."""
    ones = 0xFFFFFFFF
    for counter, key, want in (((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
                               ((ones,) * 4, (ones,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
                               ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0), (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))):
        assert tuple(int(w) for w in ref.philox(counter, key)) == want


@pytest.mark.parametrize("mode", [ref.PLAIN, ref.COMPLEMENT])
@pytest.mark.parametrize("gated", [False, True])
def test_reference_gradients_are_the_differences(mode, gated):
    rng = np.random.default_rng(3)
    offsets, d = np.array([0, 5, 5, 6, 13]), 3
    f, x, g, dy = (rng.standard_normal((14, d)) for _ in range(4))
    h0, dh_last = rng.standard_normal((4, d)), rng.standard_normal((4, d))

    def loss(f, x, g, h0):
        r = ref.recurrence(f, x, g if gated else None, h0, offsets, mode)
        return float(np.sum(r["y"][:13] * dy[:13]) + np.sum(r["h_last"] * dh_last))
    fwd = ref.recurrence(f, x, g if gated else None, h0, offsets, mode)
    grads = ref.recurrence_backward(f, x, g if gated else None, h0, offsets, mode, dy, dh_last, fwd)
    args = {"df": f, "dx": x, "dh0": h0, **({"dg": g} if gated else {})}
    for name, a in args.items():
        for at in np.ndindex(a.shape):
            keep, step = a[at], 1e-5
            a[at] = keep + step
            up = loss(f, x, g, h0)
            a[at] = keep - step
            down = loss(f, x, g, h0)
            a[at] = keep
            # third derivatives of order 10 at most times step^2, and 1e-16 of a loss of order 10 over the step
            assert abs((up - down) / (2 * step) - (grads[name][0][at] if name == "dh0" or at[0] < 13 else 0)) < 1e-8 + 1e-9, (name, at)


@pytest.mark.parametrize("layout", [ref.HALVES, ref.PAIRS])
def test_reference_rotation_and_its_gradient(layout):
    rng = np.random.default_rng(4)
    x, dy = rng.standard_normal((6, 2, 10)), rng.standard_normal((6, 2, 10))
    p, freq = np.arange(6) * 1000, ref.frequencies(6)
    y, _ = ref.rotary(x, p, freq, 6, layout, 1.3)
    dx, _ = ref.rotary(dy, p, freq, 6, layout, 1.3, back=True)
    assert abs(np.sum(y * dy) - np.sum(x * dx)) < 1e-12
    np.testing.assert_allclose(np.linalg.norm(y[..., :6], axis=2), 1.3 * np.linalg.norm(x[..., :6], axis=2), rtol=1e-13)
    assert np.array_equal(y[..., 6:], x[..., 6:])
