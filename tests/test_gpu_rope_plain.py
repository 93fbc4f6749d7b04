"""A form of whole heads in halves with a base is the rotation of the calls without one, forward and in the gradients.

The angles are the same doubles.  The 16-bit and f32 write and the rotation by itself round every product and sum in the same places: the
same bits.  The block-scaled write without a form fuses b cos + a sin the other way round for k (q is alike): of the products and the sum of
a pair of length L two are rounded on either side, each by at most 2^-24 L, so the two floats x, y differ by at most 2^-22 L.
  k_rot   each is rounded to bf16, off by at most 2^-8 of itself: |X - Y| <= 2^-22 L + 2^-8 (|x| + |y|), and |x| <= |X| / (1 - 2^-8)
  bytes   each is off by at most 2^-4 of itself or 2^-10 of the scale s: |X - Y| <= 2^-22 L + 2^-4 (|x| + |y|) + 2^-9 s, |x| <= |X| / (1 - 2^-4) + 2^-10 s
  scales, and all of q and V: equal, since the rule of the K scale looks at k before its rotation."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2602_07529_b200 import synth

pytestmark = pytest.mark.gpu


def _mods():
    from paper_2602_07529_b200 import binding as B, runtime
    return B, runtime


def drawn(shape, seed, dtype):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("base", [1e4, 5e5])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("prefix", [40, 2500])   # one token and four tokens to a CTA
def test_paged_write(prefix, dtype, d, base):
    B, runtime = _mods()
    tokens = [[([], 0, prefix), ([0], 0, 130), ([0], 0, 41), ([1, 2], 0, 300)]]
    b = synth.build_batch(tokens, rng=np.random.default_rng(2))
    g = synth.Geometry(6, 3, d, dtype=dtype)
    pod = runtime.PlanOnDevice(b, geom=g)
    n, dt = pod.stats()["n_new_tokens"], runtime.torch_dtype(g)
    geom = B.make_geom(6, 3, d, b.num_pages, dtype, rope_base=base)
    q, k, v = drawn((n, 6, d), 1, dt), drawn((n, 3, d), 2, dt), drawn((n, 3, d), 3, dt)
    form = B.RopeForm(B.ROPE_HALVES, d, base=base)
    outs = []
    for call in (lambda *a: B.mv_rope_write_kv(pod.plan, geom, *a), lambda *a: B.mv_rope_write_kv_form(pod.plan, geom, form, *a)):
        out = [torch.zeros_like(q), torch.zeros_like(k)] + [torch.zeros(runtime.pool_shape(b.num_pages, g), dtype=dt, device="cuda") for _ in range(2)]
        call(q, k, v, *out)
        outs.append(out)
    assert all(torch.equal(x, y) for x, y in zip(*outs))
    # and of the rotation by itself
    alone = [torch.zeros_like(q), torch.zeros_like(k)]
    B.mv_rope_rotate(form, geom, pod.plan, q, k, *alone)
    assert torch.equal(alone[0], outs[0][0]) and torch.equal(alone[1], outs[0][1])


@pytest.mark.parametrize("base", [1e4, 5e5])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("rows", [60, 2100])     # one row and eight rows to a CTA
def test_block_scaled_write(rows, d, base):
    B, runtime = _mods()
    b = synth.build_batch([[([], 33, 20), ([0], 5, rows - 20)]], rng=np.random.default_rng(3))
    steps = runtime.StepOnDevice(b, 2, blocks=False)
    t = steps.build()
    geom = B.make_geom(6, 3, d, b.num_pages, "bf16", rope_base=base)
    q, k, v = (drawn((rows, h, d), i, torch.bfloat16) for i, h in enumerate((6, 3, 3)))
    form = B.RopeForm(B.ROPE_HALVES, d, base=base)
    outs = []
    for call in (lambda *a: B.mv_rope_write_kv_fp8_blk(t, geom, *a), lambda *a: B.mv_rope_write_kv_fp8_blk_form(t, geom, form, *a)):
        out = [torch.zeros_like(q), torch.zeros_like(k)] + [torch.full((b.num_pages, 3, 16, d), 0x38, dtype=torch.uint8, device="cuda") for _ in range(2)]
        out.append(torch.full((b.num_pages, 3, 2), 2.0 ** -9, device="cuda"))
        call(q, k, v, *out)
        outs.append(out)
    assert steps.read_status() == 0
    (q0, k0, k8, v8, s0), (q1, k1, k9, v9, s1) = outs
    assert torch.equal(q0, q1) and torch.equal(v8, v9) and torch.equal(s0, s1)
    half = k.double()[..., :d // 2], k.double()[..., d // 2:]
    length = torch.hypot(*half).repeat(1, 1, 2)
    x, y = k0.double(), k1.double()
    assert ((x - y).abs() <= 2.0 ** -22 * length + 2.0 ** -8 / (1 - 2.0 ** -8) * (x.abs() + y.abs())).all()
    slot = steps.t["slot"][:rows]
    s = s0[slot // 16, :, 0].double()[..., None]
    x, y = (p[slot // 16, :, slot % 16].view(torch.float8_e4m3fn).double() * s for p in (k8, k9))
    assert ((x - y).abs() <= 2.0 ** -22 * length + 2.0 ** -4 / (1 - 2.0 ** -4) * (x.abs() + y.abs()) + 2.0 ** -9 * s * (1 + 2.0 ** -4)).all()


def test_raw_gradients_without_a_form():
    """The geometry's own rotation turned back is that of a form with its base; a base that no form takes is refused before anything runs."""
    B, runtime = _mods()
    wl = dataclasses.replace(synth.config4(prefix=300), batch=synth.build_batch([[([], 0, 70), ([0], 0, 130)]], rng=np.random.default_rng(1)), geom=synth.Geometry(4, 2, 128))
    dout = drawn((200, 4, 128), 4, torch.bfloat16)
    form = B.RopeForm(B.ROPE_HALVES, 128, base=wl.geom.rope_base)
    a, c = (runtime.PrefillState(wl, form=f) for f in (None, form))
    assert all(torch.equal(x, y) for x, y in zip(a.forward_backward(dout, raw=True), c.forward_backward(dout, raw=True)))
    low = runtime.PrefillState(dataclasses.replace(wl, geom=dataclasses.replace(wl.geom, rope_base=0.5)))
    low.out.fill_(7.0)
    with pytest.raises(B.MvError, match="INVALID"):
        low.forward_backward(dout, raw=True)
    torch.cuda.synchronize()
    assert (low.out == 7).all()
    low.forward_backward(dout)      # the rotated tensors' gradients need no form
