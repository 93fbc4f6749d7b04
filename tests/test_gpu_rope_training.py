"""The prompt's attention with its rotation, forward and backward, against torch autograd in 64 bits on a chain of nodes.

Tolerance: that of the backward kernels' own tests (P, dS and the outputs are rounded to bf16): relative L2 of 1e-2 per gradient; the way back through
the rotation adds one rounding to bf16, 2^-8 of a value, well inside."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2602_07529_b200 import synth
from helpers import rel_l2
from test_gpu_rope_form import FORMS, make, turned

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("which", [None, 1, 4, 6])
def test_gradients_of_raw_q_and_k(which):
    from paper_2602_07529_b200 import binding as B, runtime
    b = synth.build_batch([[([], 0, 70), ([0], 0, 130), ([1], 0, 41)]], rng=np.random.default_rng(1))
    wl = dataclasses.replace(synth.config4(prefix=300), batch=b, geom=synth.Geometry(4, 2, 128))
    form = None if which is None else make(*FORMS[which], 128)
    st = runtime.PrefillState(wl, form=form)
    g = torch.Generator(device="cuda").manual_seed(3)
    for x in (st.q, st.k, st.v):
        x.copy_(torch.randn(x.shape, generator=g, device="cuda"))
    dout = torch.randn(st.q.shape, generator=g, device="cuda").bfloat16()
    out, dq, dk, dv = st.forward_backward(dout, raw=True)
    used = form if form is not None else B.RopeForm(0, 128, base=wl.geom.rope_base)
    c, n = used.c_form, st.q.shape[0]
    pos = torch.arange(n, dtype=torch.float64)
    assert np.array_equal(st.plan.table("pos_id"), np.arange(n))
    angle = pos[:, None] * torch.from_numpy(used.theta)
    cos, sin = (f(angle)[:, None] * float(c.amplitude) for f in (torch.cos, torch.sin))
    h = c.rotary_dim // 2
    lo, hi = ((torch.arange(h) + c.first, torch.arange(h) + c.first + h) if c.layout == 0 else (c.first + 2 * torch.arange(h), c.first + 2 * torch.arange(h) + 1))

    def rotate(x):
        y = x.clone()
        y[..., lo], y[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., hi] * cos + x[..., lo] * sin
        return y

    q, k, v = (x.double().cpu().requires_grad_() for x in (st.q, st.k, st.v))
    kk, vv = (x.repeat_interleave(2, 1) for x in (rotate(k), v))
    score = torch.einsum("ihd,jhd->hij", rotate(q), kk) * 128 ** -0.5
    score = score.masked_fill(torch.ones(n, n, dtype=torch.bool).triu(1), -torch.inf)
    ref = torch.einsum("hij,jhd->ihd", torch.softmax(score, -1), vv)
    ref.backward(dout.double().cpu())
    assert rel_l2(out.double().cpu(), ref.detach()) <= 1e-2
    for got, x in ((dq, q), (dk, k), (dv, v)):
        assert rel_l2(got.double().cpu(), x.grad) <= 1e-2
