"""Rotary forms on the host: the angles a form is made with, and every refusal (nothing is launched: the addresses are never followed)."""
import ctypes as C
import math

import numpy as np
import pytest

from paper_2602_07529_b200 import binding as B
from test_step_refusals import INVALID, OK, P, UNSUPPORTED, WORKSPACE, tables


def form(layout=0, first=0, rotary_dim=128, base=1e4, scaling=0, factor=1.0, length=4096.0, slow=1.0, fast=32.0, amplitude=1.0):
    f = B._RopeForm()
    return B.lib.mv_rope_form_init(C.byref(f), layout, first, rotary_dim, base, scaling, factor, length, slow, fast, amplitude), f


@pytest.mark.parametrize("rd", [16, 48, 64, 128])
@pytest.mark.parametrize("base", [1.0, 1e4, 5e5])
def test_angles(rd, base):
    """Against the formulas in 80 bits; a double power and a product or two: a few units in the last place."""
    i = np.arange(rd // 2, dtype=np.longdouble)
    plain = np.longdouble(base) ** (-2 * i / rd)
    turns = np.longdouble(4096) * plain / (2 * np.longdouble(np.pi))
    w = np.clip((turns - 1) / 31, 0, 1)
    want = {0: plain, 1: plain / 8, 2: (np.longdouble(base) * np.longdouble(8) ** (np.longdouble(rd) / (rd - 2))) ** (-2 * i / rd), 3: w * plain + (1 - w) * plain / 8}
    for scaling, theta in want.items():
        st, f = form(rotary_dim=rd, base=base, scaling=scaling, factor=8.0)
        assert st == OK and f.rotary_dim == rd and f.amplitude == 1.0
        assert np.abs(np.asarray(f.theta[:rd // 2]) / theta.astype(float) - 1).max() < 2.0 ** -46
        assert not any(f.theta[rd // 2:])
    # the slowest pair of the enlarged base is stretched by the factor, the fastest by nothing
    f = form(rotary_dim=rd, base=base, scaling=2, factor=8.0)[1]
    assert f.theta[0] == 1.0 and math.isclose(f.theta[rd // 2 - 1] * 8.0, float(plain[-1]), rel_tol=1e-12)


def test_form_refuses():
    assert B.lib.mv_rope_form_init(None, 0, 0, 64, 1e4, 0, 1.0, 1.0, 0.0, 1.0, 1.0) == INVALID
    for kw in ({"layout": 2}, {"layout": -1}, {"scaling": 4}, {"scaling": -1}, {"base": 0.5}, {"base": math.nan}, {"base": math.inf}, {"amplitude": 0.0},
               {"amplitude": -1.0}, {"amplitude": math.nan}, {"amplitude": 2000.0}, {"scaling": 1, "factor": 0.5}, {"scaling": 3, "factor": math.inf},
               {"scaling": 3, "length": 0.0}, {"scaling": 3, "slow": 4.0, "fast": 4.0}, {"scaling": 3, "slow": -1.0}, {"scaling": 3, "fast": math.inf}):
        assert form(**kw)[0] == INVALID, kw
    for kw in ({"first": 8}, {"first": -16}, {"first": 128}, {"rotary_dim": 0}, {"rotary_dim": 24}, {"rotary_dim": 144}):
        assert form(**kw)[0] == UNSUPPORTED, kw
    assert form(scaling=0, factor=0.0, length=-1.0, slow=9.0, fast=0.0)[0] == OK   # what a scaling does not read is not looked at


def rotate(f, g, pos=P, n=8, backward=0, q=P, qs=1024, k=P, ks=256, qo=P, qos=1024, ko=P, kos=256):
    return B.lib.mv_rope_rotate(C.byref(f) if f else None, C.byref(g) if g else None, pos, n, backward, q, qs, k, ks, qo, qos, ko, kos, None)


def bad_forms(d):
    out = []
    for kw in ({"layout": 3}, {"first": 4}, {"first": -16}, {"first": d}, {"rotary_dim": 8}, {"rotary_dim": 0}, {"rotary_dim": d + 16}, {"amplitude": 0.0},
               {"amplitude": math.nan}):
        f = form(rotary_dim=min(d, 128))[1]
        for k, v in kw.items():
            setattr(f, k, v)
        out.append(f)
    for x in (math.nan, 1.5, -1.5, math.inf):
        f = form(rotary_dim=d)[1]
        f.theta[d // 2 - 1] = x
        out.append(f)
    f = form(rotary_dim=d)[1]
    f.first = 16          # reaches past the head
    return out + [f]


def test_rotate_refuses():
    g = B.make_geom(8, 2, 128, 0, "bf16")
    f = form()[1]
    assert rotate(f, g, n=0) == OK and rotate(f, g, q=None, qo=None, k=None, ko=None) == OK
    assert rotate(None, g) == INVALID and rotate(f, None) == INVALID
    for kw in ({"n": -1}, {"backward": 2}, {"pos": None}, {"pos": P + 2}, {"q": None}, {"qo": None}, {"k": None}, {"ko": None}, {"q": P + 8}, {"ko": P + 2},
               {"qs": 1016}, {"qs": 1028}, {"ks": 128}, {"qos": 1023}, {"kos": 260}, {"qs": 2048}, {"qs": 1 << 61, "qos": 1 << 61},
               {"k": P, "ko": P, "ks": 512}):
        assert rotate(f, g, **kw) == INVALID, kw
    assert rotate(f, g, n=1 << 31) == UNSUPPORTED
    for dtype, d in (("bf16", 64), ("bf16", 128), ("f32", 128)):
        for x in bad_forms(d):
            assert rotate(x, B.make_geom(8, 2, d, 0, dtype)) == INVALID
    assert rotate(f, B.make_geom(8, 2, 64, 0, "bf16")) == INVALID     # a form of 128 elements on heads of 64
    assert rotate(f, B.make_geom(8, 3, 128, 0, "bf16")) == UNSUPPORTED
    assert rotate(f, B.make_geom(8, 2, 96, 0, "bf16")) == UNSUPPORTED


def test_writes_refuse_forms():
    ref = C.byref
    for d in (64, 128):
        g = B.make_geom(8, 2, d, 100, "bf16")
        t = tables()
        for x in bad_forms(d):
            assert B.lib.mv_rope_write_kv_fp8_blk_form(ref(t), ref(g), ref(x), P, P, P, P, P, P, P, P, None) == INVALID
            assert B.lib.mv_rope_write_kv_form(None, ref(g), ref(x), *[P] * 7, None) == INVALID
        ok = form(rotary_dim=d)[1]
        assert B.lib.mv_rope_write_kv_fp8_blk_form(ref(t), ref(g), None, P, P, P, P, P, P, P, P, None) == INVALID
        assert B.lib.mv_rope_write_kv_fp8_blk_form(ref(t), ref(g), ref(ok), P, None, P, P, P, P, P, P, None) == INVALID
        assert B.lib.mv_rope_write_kv_fp8_blk_form(ref(t), ref(g), ref(ok), P + 8, P, P, P, P, P, P, P, None) == INVALID
        assert B.lib.mv_rope_write_kv_fp8_blk_form(ref(tables(max_rows=0)), ref(g), ref(ok), *[P] * 8, None) == OK
        assert B.lib.mv_rope_write_kv_form(None, ref(g), ref(ok), *[P] * 7, None) == INVALID
        assert B.lib.mv_rope_write_kv_form(None, ref(g), ref(ok), P, P + 4, *[P] * 5, None) == INVALID
    g32 = B.make_geom(8, 2, 128, 100, "f32")
    assert B.lib.mv_rope_write_kv_fp8_blk_form(ref(tables()), ref(g32), ref(form()[1]), *[P] * 8, None) == UNSUPPORTED


def test_positions_of_a_plan():
    out = C.c_void_p()
    assert B.lib.mv_plan_positions(None, C.byref(out)) == INVALID
    from paper_2602_07529_b200 import synth
    plan = B.Plan(synth.config1().batch)
    assert B.lib.mv_plan_positions(plan.handle, None) == INVALID
    assert B.lib.mv_plan_positions(plan.handle, C.byref(out)) == WORKSPACE     # not uploaded


def test_form_object():
    f = B.RopeForm(B.ROPE_PAIRS, 32, first=64, theta=np.linspace(1, 0, 16))
    assert np.array_equal(f.theta, np.linspace(1, 0, 16)) and f.c_form.layout == 1 and f.c_form.first == 64
    with pytest.raises(ValueError, match="16 angles"):
        B.RopeForm(0, 32, theta=[1.0])
    with pytest.raises(B.MvError):
        B.RopeForm(0, 24)
    with pytest.raises(KeyError):
        B.RopeForm(0, 32, scaling="else")
