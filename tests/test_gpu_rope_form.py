"""Rotary forms on the GPU against 80-bit arithmetic on the host, and the writes that take them.

Tolerances, fixed before the first run, per element of a pair of length L = |(a, b)| with amplitude A:
  rounding of the result: 2^-8 of it in bf16, 2^-24 in float;
  angle: pos * theta and its reduction as doubles: under 2^-27 for the angles drawn here (below 2^25); cosine and sine as floats within two
  units in the last place, 2^-22; their product with A rounded once more, 2^-24; two products and a difference, 2^-23 L A: together under 2^-20 L A.
A stored 8-bit value is off by at most half a step, 2^-4 of it (or 2^-10 among the subnormals) times the scale, plus the same 2^-20 L A."""
import math

import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu

FORMS = [  # layout, rotary part, first element, angles
    (0, 128, 0, {}), (1, 128, 0, {"base": 5e5}), (0, 64, 0, {"scaling": "linear", "factor": 4.0}), (1, 64, 64, {"scaling": "base", "factor": 8.0}),
    (0, 16, 112, {"scaling": "ramp", "factor": 16.0, "length": 4096, "amplitude": 1.2772589}), (1, 48, 32, {"amplitude": 0.75}),
    (1, 96, 16, {"scaling": "ramp", "factor": 32.0, "length": 8192, "slow": 1.0, "fast": 4.0, "amplitude": 1.5}),
    (0, 80, 48, {"theta": "own"}),
]


def make(layout, part, first, kw, d):
    from paper_2602_07529_b200 import binding as B
    kw = dict(kw)
    part = min(part, d)
    first = min(first, d - part)
    if kw.get("theta") == "own":
        kw["theta"] = np.random.default_rng(1).uniform(-1, 1, part // 2)
    return B.RopeForm(layout, part, first=first, **kw)


def turned(form, pos, x, backward=False):
    """(y, length of the pairs) in float64 (angles in 80 bits), x [n][heads][d]."""
    c = form.c_form
    a = np.asarray(pos, np.longdouble)[:, None] * np.asarray(form.theta, np.longdouble)
    A = float(c.amplitude)
    cos, sin = (np.cos(a) * A).astype(float)[:, None], (np.sin(a) * A * (-1 if backward else 1)).astype(float)[:, None]
    f, h = c.first, c.rotary_dim // 2
    lo, hi = (slice(f, f + h), slice(f + h, f + 2 * h)) if c.layout == 0 else (slice(f, f + 2 * h, 2), slice(f + 1, f + 2 * h, 2))
    x = x.double().cpu().numpy()
    y, length = x.copy(), np.zeros_like(x)
    y[..., lo], y[..., hi] = x[..., lo] * cos - x[..., hi] * sin, x[..., hi] * cos + x[..., lo] * sin
    length[..., lo] = length[..., hi] = np.hypot(x[..., lo], x[..., hi]) * A
    return y, length


def close(got, form, pos, x, backward=False):
    y, length = turned(form, pos, x, backward)
    eps = 2.0 ** -8 if got.dtype == torch.bfloat16 else 2.0 ** -24
    err = np.abs(got.double().cpu().numpy() - y)
    assert (err <= eps * np.abs(y) + 2.0 ** -20 * length).all(), err.max()
    plain = torch.from_numpy(length == 0)
    assert torch.equal(got.cpu()[plain], x.cpu().to(got.dtype)[plain])    # what is not turned is the same


def normal(shape, seed, dtype=torch.bfloat16):
    return torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda").to(dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", range(len(FORMS)))
def test_rotate(which, d, dtype):
    from paper_2602_07529_b200 import binding as B
    form = make(*FORMS[which], d)
    rng = np.random.default_rng(which)
    dt = torch.bfloat16 if dtype == "bf16" else torch.float32
    for n, hq, hkv in ((1, 4, 1), (7, 5, 5), (129, 32, 8), (2051, 6, 2)):
        pos = rng.integers(-100, 1 << 24, n).astype(np.int32)
        p = torch.from_numpy(pos).cuda()
        geom = B.make_geom(hq, hkv, d, 0, dtype)
        q, k = normal((n, hq, d), n, dt), normal((n, hkv, d), n + 1, dt)
        qo, ko = torch.full_like(q, float("nan")), torch.full_like(k, float("nan"))
        B.mv_rope_rotate(form, geom, p, q, k, qo, ko)
        close(qo, form, pos, q)
        close(ko, form, pos, k)
        # in place, one tensor, backward
        q2 = q.clone()
        B.mv_rope_rotate(form, geom, p, q2, None, q2, None, backward=True)
        close(q2, form, pos, q, True)
        k2 = k.clone()
        B.mv_rope_rotate(form, geom, p, None, k2, None, k2)
        assert torch.equal(k2, ko)


def test_rows_of_one_projection():
    """q, k and v side by side: token strides, in and out; what lies between stays as it was."""
    from paper_2602_07529_b200 import binding as B
    n, hq, hkv, d = 301, 8, 2, 128
    form = make(1, 64, 32, {}, d)
    geom = B.make_geom(hq, hkv, d, 0, "bf16")
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 37
    x = normal((n, hq + 2 * hkv, d), 1)
    a, b = x[:, :hq], x[:, hq:hq + hkv]
    qo, ko = torch.zeros(n, hq, d, dtype=torch.bfloat16, device="cuda"), torch.zeros(n, hkv, d, dtype=torch.bfloat16, device="cuda")
    B.mv_rope_rotate(form, geom, pos, a, b, qo, ko)
    close(qo, form, pos.cpu().numpy(), a)
    close(ko, form, pos.cpu().numpy(), b)
    y = x.clone()
    B.mv_rope_rotate(form, geom, pos, y[:, :hq], y[:, hq:hq + hkv], y[:, :hq], y[:, hq:hq + hkv])
    assert torch.equal(y[:, :hq], qo) and torch.equal(y[:, hq:hq + hkv], ko) and torch.equal(y[:, hq + hkv:], x[:, hq + hkv:])
    z = torch.full((n, hq + 2 * hkv, d), 3.0, dtype=torch.bfloat16, device="cuda")
    B.mv_rope_rotate(form, geom, pos, qo, None, z[:, 2:2 + hq], None, backward=True)
    assert (z[:, :2] == 3).all() and (z[:, 2 + hq:] == 3).all()
    close(z[:, 2:2 + hq], form, pos.cpu().numpy(), qo, True)
    for bad in (x[:, :hq, ::2], x.transpose(0, 1)[:hq], x[:, :hq].float(), x[:, :hq - 1], x[:, :hq].cpu()):
        with pytest.raises(ValueError):
            B.mv_rope_rotate(form, geom, pos, bad, None, qo, None)
    with pytest.raises(ValueError):
        B.mv_rope_rotate(form, geom, pos[:-1], a, b, qo, ko)
    with pytest.raises(ValueError):
        B.mv_rope_rotate(form, geom, pos, None, None, None, None)


def test_not_finite_stays_in_its_pair():
    from paper_2602_07529_b200 import binding as B
    form, geom = make(1, 64, 0, {}, 128), B.make_geom(2, 1, 128, 0, "f32")
    q = normal((5, 2, 128), 3, torch.float32)
    clean = q.clone()
    q[2, 1, 10], q[3, 0, 100] = float("inf"), float("nan")
    pos = torch.arange(5, dtype=torch.int32, device="cuda")
    out, ref = torch.empty_like(q), torch.empty_like(q)
    B.mv_rope_rotate(form, geom, pos, q, None, out, None)
    B.mv_rope_rotate(form, geom, pos, clean, None, ref, None)
    off = ~(out == ref)
    assert sorted(map(tuple, off.nonzero().tolist())) == [(2, 1, 10), (2, 1, 11), (3, 0, 100)]


def test_gradient():
    """<R x, y> = <x, R^T y> exactly in the formula; and differences of a scalar function of the rotated tensors."""
    from paper_2602_07529_b200 import binding as B
    n, hq, d = 9, 3, 64
    form, geom = make(0, 48, 16, {"amplitude": 1.3}, d), B.make_geom(hq, hq, d, 0, "f32")
    pos = torch.arange(n, dtype=torch.int32, device="cuda") * 1001
    x, w = normal((n, hq, d), 1, torch.float32), normal((n, hq, d), 2, torch.float32)

    def f(x):  # sum(w * sin(R x))
        y = torch.empty_like(x)
        B.mv_rope_rotate(form, geom, pos, x, None, y, None)
        return float((w.double() * y.double().sin()).sum()), y

    _, y = f(x)
    dy = (w.double() * y.double().cos()).float()
    dx = torch.empty_like(x)
    B.mv_rope_rotate(form, geom, pos, None, dy, None, dx, backward=True)
    close(dx, form, pos.cpu().numpy(), dy, True)
    for i, step in enumerate((2.0 ** -7,) * 3):
        u = normal(x.shape, 10 + i, torch.float32)
        u /= u.norm()
        slope = (f(x + step * u)[0] - f(x - step * u)[0]) / (2 * step)
        # third derivative: |w| A^3 |u_i|^3 summed, below max|w| A^3; times step^2 / 6; and 2^-22 of sum |w y| over the step by rounding
        tol = float(w.abs().max()) * 1.3 ** 3 * step ** 2 / 6 + 2.0 ** -22 * float((w * y).abs().sum()) / step
        assert abs(slope - float((dx.double() * u.double()).sum())) <= tol


@pytest.mark.parametrize("dtype,d", [("bf16", 128), ("bf16", 64), ("f32", 128), ("f32", 64)])
@pytest.mark.parametrize("which", [1, 4, 6])
def test_paged_write(which, dtype, d):
    """mv_rope_write_kv_form: pools, rotated q and k, through a plan; the plan's positions feed mv_rope_rotate."""
    import dataclasses
    from paper_2602_07529_b200 import binding as B, runtime, synth
    form = make(*FORMS[which], d)
    for wl in (synth.config1(), synth.config4(prefix=700) if "prefix" in synth.config4.__code__.co_varnames else synth.config1()):
        b = wl.batch
        g = dataclasses.replace(wl.geom, dtype=dtype, head_dim=d)
        pod = runtime.PlanOnDevice(b, geom=g)
        n, pos = pod.stats()["n_new_tokens"], pod.plan.table("pos_id")
        dt = runtime.torch_dtype(g)
        geom = B.make_geom(g.n_q_heads, g.n_kv_heads, d, b.num_pages, dtype)
        q, k, v = normal((n, g.n_q_heads, d), 1, dt), normal((n, g.n_kv_heads, d), 2, dt), normal((n, g.n_kv_heads, d), 3, dt)
        kp, vp = (torch.full(runtime.pool_shape(b.num_pages, g), float("nan"), dtype=dt, device="cuda") for _ in range(2))
        qr, kr = torch.empty_like(q), torch.empty_like(k)
        B.mv_rope_write_kv_form(pod.plan, geom, form, q, k, v, qr, kr, kp, vp)
        close(qr, form, pos, q)
        close(kr, form, pos, k)
        slot = torch.from_numpy(pod.plan.table("slot")).cuda()
        assert torch.equal(runtime.pool_tokens(kp, slot), kr) and torch.equal(runtime.pool_tokens(vp, slot), v)
        assert int((~torch.isnan(kp)).sum()) == kr.numel()        # nothing else was written
        qo, ko = torch.empty_like(q), torch.empty_like(k)
        B.mv_rope_rotate(form, geom, pod.plan, q, k, qo, ko)
        assert torch.equal(qo, qr) and torch.equal(ko, kr)
        with pytest.raises(ValueError):
            B.mv_rope_rotate(form, geom, pod.plan, q[1:], None, qo[1:], None)


def test_plain_form_is_the_old_call():
    """A form of the whole head in halves with plain angles gives what the calls without one give, bit for bit."""
    from paper_2602_07529_b200 import binding as B, runtime, synth
    wl = synth.config2(n_req=2, prefix=40, branches=3, branch_len=21)
    st = runtime.DecodeStateFP8Blk(wl)
    t = st.steps.build()
    # the angles as those calls compute them: 2^(i c), c = -2 log2(base) / 128
    form = B.RopeForm(0, 128, theta=[math.exp2(i * (-2.0 * math.log2(wl.geom.rope_base) / 128)) for i in range(64)])
    outs = []
    for call in (lambda *a: B.mv_rope_write_kv_fp8_blk(t, st.geom, *a), lambda *a: B.mv_rope_write_kv_fp8_blk_form(t, st.geom, form, *a)):
        pools = [st.k_pages.clone(), st.v_pages.clone(), st.kv_scale.clone()]
        q_rot, k_rot = torch.zeros_like(st.q), torch.zeros_like(st.k)
        call(st.q, st.k, st.v, q_rot, k_rot, *pools)
        outs.append(pools + [q_rot, k_rot])
    assert all(torch.equal(a, b) for a, b in zip(*outs))


@pytest.mark.parametrize("rows", [40, 2100])
@pytest.mark.parametrize("which,d", [(0, 128), (1, 64), (3, 128), (4, 128), (5, 64), (6, 128), (7, 64)])
def test_block_scaled_write(which, d, rows):
    """Runs of a few tokens in pages of their own, some pages partly filled: bytes, scales, q and k."""
    from paper_2602_07529_b200 import binding as B
    form = make(*FORMS[which], d)
    A = max(1.0, float(form.c_form.amplitude))
    hq, hkv = 6, 2
    rng = np.random.default_rng([which, d, rows])
    slot, page = [], 0
    while len(slot) < rows - 3:
        off = int(rng.integers(0, 16))
        n = min(int(rng.integers(1, 17 - off)), rows - 3 - len(slot))
        slot += [page * 16 + off + i for i in range(n)]
        page += 1
    n, pages = len(slot), page + 2
    slot = np.asarray(slot)
    pos = rng.integers(0, 1 << 20, n)
    t = B.StepTables(torch.zeros(rows, dtype=torch.int32, device="cuda"), torch.full((rows,), -1, dtype=torch.int64, device="cuda"), torch.zeros(8, dtype=torch.int32, device="cuda"))
    t._keep[0][:n], t._keep[1][:n] = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(slot).cuda()
    geom = B.make_geom(hq, hkv, d, pages, "bf16")
    q, k, v = normal((rows, hq, d), 1), normal((rows, hkv, d), 2), normal((rows, hkv, d), 3)
    k *= torch.exp2(torch.randint(-12, 12, (rows, 1, 1), generator=torch.Generator(device="cuda").manual_seed(4), device="cuda")).bfloat16()
    old8 = [torch.randint(0, 120, (pages, hkv, 16, d), dtype=torch.uint8, device="cuda") for _ in range(2)]
    old_s = torch.exp2(torch.randint(-8, 3, (pages, hkv, 2), device="cuda").float())
    kp, vp, sc = old8[0].clone(), old8[1].clone(), old_s.clone()
    qr, kr = torch.full_like(q, 7.0), torch.full_like(k, 7.0)
    B.mv_rope_write_kv_fp8_blk_form(t, geom, form, q, k, v, qr, kr, kp, vp, sc)
    assert B.mv_step_tables_read_status(t) == 0
    close(qr[:n], form, pos, q[:n])
    close(kr[:n], form, pos, k[:n])
    assert (qr[n:] == 7).all() and (kr[n:] == 7).all()
    want_k, len_k = turned(form, pos, k[:n])
    pg = torch.from_numpy(slot // 16)
    for which_pool, (pool, x, length, raw, top) in enumerate(((kp, want_k, len_k, k[:n].float().cpu() * A, 316.0),
                                                              (vp, v[:n].double().cpu().numpy(), np.zeros((n, hkv, d)), v[:n].float().cpu(), 448.0))):
        got_s, was = sc[..., which_pool].cpu(), old_s[..., which_pool].cpu()
        stored = pool.view(torch.float8_e4m3fn).float().double().cpu().numpy()
        for p in range(pages):
            at = (pg == p).nonzero()[:, 0].numpy()
            if len(at) == 0:
                assert torch.equal(got_s[p], was[p]) and torch.equal(pool[p].cpu(), old8[which_pool][p].cpu())
                continue
            amax = raw[at].abs().amax((0, 2)).double()
            need = torch.exp2(torch.ceil(torch.log2(amax / top)).clamp(-60, 40))
            first = int(slot[at[0]] % 16)
            held = was[p].double() if first else torch.zeros_like(need)
            bound = torch.frexp(amax / top)[0] == 0.5     # exactly at the bound of a scale: that one or the next
            s = got_s[p].double()
            assert ((s == torch.maximum(need, held)) | (bound & ((s == torch.maximum(2 * need, held)) | (s == torch.maximum(need / 2, held))))).all()
            val = stored[p][:, slot[at] % 16].transpose(1, 0, 2) * s.numpy()[None, :, None]
            err = np.abs(val - x[at])
            assert (err <= np.maximum(2.0 ** -4 * np.abs(x[at]), 2.0 ** -10 * s.numpy()[None, :, None]) + 2.0 ** -20 * length[at]).all()
            assert (np.abs(x[at]) <= 448.0 * s.numpy()[None, :, None] * (1 + 2.0 ** -20)).all()       # nothing had to be cut off
            # tokens that were there have moved to the scale: exact but for subnormals
            before = old8[which_pool][p, :, :first].view(torch.float8_e4m3fn).float().double().cpu().numpy() * was[p].numpy()[:, None, None]
            now = stored[p][:, :first] * s.numpy()[:, None, None]
            assert (np.abs(now - before) <= 2.0 ** -10 * s.numpy()[:, None, None]).all()


def test_capture_and_streams():
    """Captured and replayed after the inputs change; on a stream that is not the current one."""
    from paper_2602_07529_b200 import binding as B
    n, form, geom = 65, make(1, 64, 0, {}, 128), B.make_geom(4, 2, 128, 0, "bf16")
    pos = torch.arange(n, dtype=torch.int32, device="cuda")
    q, k = normal((n, 4, 128), 1), normal((n, 2, 128), 2)
    qo, ko = torch.empty_like(q), torch.empty_like(k)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.mv_rope_rotate(form, geom, pos, q, k, qo, ko, stream=side)
    side.synchronize()
    close(qo, form, pos.cpu().numpy(), q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mv_rope_rotate(form, geom, pos, q, k, qo, ko)
    q.copy_(normal((n, 4, 128), 9))
    pos += 1000
    graph.replay()
    torch.cuda.synchronize()
    close(qo, form, pos.cpu().numpy(), q)
    close(ko, form, pos.cpu().numpy(), k)
