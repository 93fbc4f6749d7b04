"""Decode attention over the block-scaled 8-bit cache where its arithmetic is strained: scores that leap, scales far apart, weights far
apart, magnitudes that differ inside a group; with many streams of several tiles each, so that a share holds tiles of which the later
ones move what the first ones set.

Bound of an element, before the first run (64-bit reference; p softmax weights, w_j = p_j * scale of V's block, v_j stored values):
  2^-8 |out|                                     bf16 rounds by half a step
  (2^-8 + 2^-12) sum_j w_j |v_j|                 a weight as two 8-bit floats, exp2 and the joins of partial results
  2^-19 max_j w_j * sum_j |v_j|                  what a weight loses below the smallest 8-bit float
  1.1 (sum_j w_j |v_j| ds_j + (sum_j p_j ds_j) sum_j w_j |v_j|)   scores off by ds_j, the tenth for the second order:
      ds_j = sm_scale (2^-17 max |q| sum_d |K_jd| + 2^-20 sum_d |q_d K_jd|) + 2^-22 max_j |s_j|
      (q as two 8-bit floats; 128 products summed in 32 bits; scores against a reference in 32 bits)
"""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from paper_2602_07529_b200 import synth
from test_gpu_fp8_blk import _batch_of, _mods, pools_of

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def elementwise(q, k8, v8, scale, t, group, sm_scale, weight=2.0 ** -8 + 2.0 ** -12, floor=2.0 ** -19, own_q=False):
    """(row, out, bound) of every row of the step.  own_q: q's rounding counts from the row's own largest element, else from its group's."""
    d, hkv = q.shape[2], k8.shape[1]
    ro, eo, ent, counts = (t[k].cpu() for k in ("group_row_off", "group_ent_off", "entries", "counts"))
    kd = k8.view(torch.float8_e4m3fn).double() * scale[:, :, 0].double()[:, :, None, None]
    vb, se = v8.view(torch.float8_e4m3fn).double(), scale[:, :, 1].double()
    for g in range(int(counts[1])):
        e = ent[int(eo[g]):int(eo[g + 1])].long()
        r0, r1 = int(ro[g]), int(ro[g + 1])
        qabs = q[r0:r1].double().abs().view(r1 - r0, hkv, group, d)
        most = qabs.amax((0, 2, 3))[:, None].expand(hkv, group)
        for r in range(r0, r1):
            b = r - r0
            sel = e[((e[:, 2 + b // 32] >> (b % 32)) & 1) > 0]
            tok = (torch.arange(16) < sel[:, 1:2]).reshape(-1).nonzero()[:, 0].to(q.device)
            page = sel[:, 0].to(q.device)
            kk, vv = (x[page].transpose(1, 2).reshape(-1, hkv, d)[tok] for x in (kd, vb))
            sv = se[page][:, None, :].expand(-1, 16, -1).reshape(-1, hkv)[tok]
            qq = q[r].double().view(hkv, group, d)
            s = torch.einsum("hgd,nhd->hgn", qq, kk) * sm_scale
            qm = qabs[b].amax(-1) if own_q else most
            ds = (torch.einsum("hg,nh->hgn", qm * 2.0 ** -17, kk.abs().sum(2)) + 2.0 ** -20 * torch.einsum("hgd,nhd->hgn", qq.abs(), kk.abs())) * sm_scale
            ds = ds + 2.0 ** -22 * s.abs().amax(-1, keepdim=True)
            p = torch.softmax(s, -1)
            w = p * sv.t()[:, None, :]
            va = vv.abs()
            ref, a = torch.einsum("hgn,nhd->hgd", w, vv), torch.einsum("hgn,nhd->hgd", w, va)
            moved = torch.einsum("hgn,nhd->hgd", w * ds, va) + a * (p * ds).sum(-1)[..., None]
            tol = 2.0 ** -8 * ref.abs() + weight * a + 1.1 * moved + floor * w.amax(-1)[..., None] * va.sum(0)[:, None, :] + 1e-30
            yield r, ref.reshape(-1, d), tol.reshape(-1, d)


def attend(batch, hq, hkv, d, q, pools, sm_scale=0.0):
    B, runtime = _mods()
    step = runtime.StepOnDevice(batch, hq // hkv)
    step.build()
    geom = B.make_geom(hq, hkv, d, batch.num_pages, "bf16", sm_scale=sm_scale)
    ws = torch.full((B.mv_decode_fp8_blk_workspace_bytes(geom),), 255, dtype=torch.uint8, device="cuda")
    out = torch.full_like(q, 7.0)
    B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, *pools, out, ws)
    assert step.read_status() == 0
    return out, step


def check(batch, hq, hkv, d, q, pools, sm_scale=0.0, **kw):
    out, step = attend(batch, hq, hkv, d, q, pools, sm_scale)
    worst = 0.0
    for r, ref, tol in elementwise(q, *pools, step.t, hq // hkv, sm_scale or d ** -0.5, **kw):
        err = (out[r].double() - ref).abs()
        assert not torch.isnan(err).any(), r
        worst = max(worst, float((err / tol).max()))
    assert worst <= 1.0, worst
    return out, step


def streams(n_req=40, prefix=2000, branches=2, seed=5):
    """Streams that hold enough tiles for segments of many tiles: a prompt, and branches of a few tokens each with one new one."""
    return _batch_of([[([], prefix + 3 * r, 0)] + [([0], 5 * b, 1) for b in range(branches)] for r in range(n_req)], seed)


def of_prompt(batch, values):
    """Per slot of the pool [pages, 16]: values[request][token] for the prompts' tokens, 0 elsewhere."""
    x = np.zeros((batch.num_pages, 16), np.float32)
    for r in range(batch.n_req):
        v = int(batch.node_off[r])
        n = int(batch.node_len[v])
        t = np.arange(n)
        x[batch.page_idx[batch.page_off[v] + t // 16], t % 16] = values(r, n)
    return torch.from_numpy(x).cuda()


def keyed(batch, hkv, d, col0):
    """A cache whose keys have one element besides zeros, so that q = (1, 0, 0, ...) makes it the score; random V."""
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, 3)
    k = torch.zeros(batch.num_pages, hkv, 16, d, device="cuda")
    k[..., 0] = col0[:, None, :]
    sc[..., 0] = 1.0
    return k.to(torch.float8_e4m3fn).view(torch.uint8).contiguous(), v8, sc


def unit_q(batch, hq, d):
    q = torch.zeros(int(batch.node_new.sum()), hq, d, device="cuda").bfloat16()
    q[..., 0] = 1.0
    return q


# (query heads, KV heads, branches): 2, 16, 32 and 64 q-vectors in a stream
SHAPES = [(8, 8, 2), (32, 8, 4), (64, 8, 4), (64, 8, 8)]


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES)
@pytest.mark.parametrize("leap", [60, 86, 88, 200])
def test_one_score_leaps(hq, hkv, branches, d, leap):
    """All scores are 0 but one, deep in the history: the answer is that token's V.  The references move by up to 288 powers of two."""
    batch = streams(branches=branches)
    col0 = of_prompt(batch, lambda r, n: np.where(np.arange(n) == 700 + 23 * r, 64.0, 0.0))
    check(batch, hq, hkv, d, unit_q(batch, hq, d), keyed(batch, hkv, d, col0), sm_scale=leap / 64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES)
@pytest.mark.parametrize("leap,at", [(10, 900), (60, 900), (48, 330), (52, 330), (60, 330)])
def test_one_score_leaps_behind_blocks_of_zeros(hq, hkv, branches, d, leap, at):
    """The history begins with V = 0, whose blocks have the lowest scale: its exponent counts in the references, which move by 54 powers
    of two where the zeros end (token 320), together with the score's leap or before it."""
    batch = streams(branches=branches)
    col0 = of_prompt(batch, lambda r, n: np.where(np.arange(n) == at + r, 64.0, 0.0))
    k8, v8, sc = keyed(batch, hkv, d, col0)
    for r in range(batch.n_req):
        v = int(batch.node_off[r])
        pages = torch.from_numpy(batch.page_idx[batch.page_off[v]:batch.page_off[v] + 20].astype(np.int64)).cuda()
        v8[pages] = 0
        sc[pages, :, 1] = 2.0 ** -60
    check(batch, hq, hkv, d, unit_q(batch, hq, d), (k8, v8, sc), sm_scale=leap / 64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES)
@pytest.mark.parametrize("name", ["ramp up", "ramp down", "stairs", "late sink"])
def test_references_move_along_the_history(hq, hkv, branches, d, name):
    batch = streams(branches=branches)
    fn = {"ramp up": lambda r, n: np.linspace(-200, 250, n), "ramp down": lambda r, n: np.linspace(250, -200, n),
          "stairs": lambda r, n: 16.0 * (np.arange(n) // (128 + r)), "late sink": lambda r, n: np.where(np.arange(n) == n - 2, 30.0, (np.arange(n) * 37 % 64) / 32.0)}[name]
    q = unit_q(batch, hq, d)
    q[..., 0] *= torch.linspace(-1.0, 2.0, hq, device="cuda").bfloat16()[None]    # heads that see it rise, fall and stand still
    check(batch, hq, hkv, d, q, keyed(batch, hkv, d, of_prompt(batch, fn)), sm_scale=0.5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES)
def test_scores_of_a_wide_spread(hq, hkv, branches, d):
    """Random scores of about a dozen units, V's scales up to 2^16 apart: every few tiles something moves."""
    batch = streams(branches=branches)
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, 11, spread=8)
    sc[..., 0] = 2.0 ** -6
    q = torch.randn(int(batch.node_new.sum()), hq, d, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    check(batch, hq, hkv, d, q, (k8, v8, sc), sm_scale=1.0)


def test_tables_of_every_size_around_the_plain_shared_memory_limit():
    """The first build of a process, for request sizes at which the kernel's shared memory passes what a launch gets without asking."""
    code = """
import sys
sys.path[:0] = ["tests", "."]
from test_gpu_fp8_blk import _batch_of, _mods, check_tables
for n in (800, 815, 816, 817, 818):
    batch = _batch_of([[([], 1, 0)] + [([v], 0, int(v == n - 2)) for v in range(n - 1)]])
    step = _mods()[1].StepOnDevice(batch, 4)
    step.build()
    check_tables(step, batch)
"""
    r = subprocess.run([sys.executable, "-c", code], cwd=ROOT, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-2000:]


@pytest.mark.parametrize("what,at,value", [("group_tile_off", 2, 2 ** 29 + 5), ("group_tile_off", 2, -(2 ** 31)), ("group_tile_off", 2, 2), ("group_ent_off", 2, 5000), ("group_ent_off", 2, -7),
                                           ("group_ent_off", 2, 2 ** 31 - 1), ("group_row_off", 2, 2 ** 31 - 1), ("group_row_off", 2, -(2 ** 31)), ("group_row_off", 2, 400)])
def test_tables_of_the_callers_own_with_offsets_that_do_not_fit(what, at, value):
    """Groups whose rows or entries leave the arrays, or whose tiles do not follow from their entries, are reported and skipped;
    the groups around them keep their results."""
    B, _ = _mods()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    t = {"pos_id": i32(*[0] * 9), "slot": torch.full((9,), -1, dtype=torch.int64, device="cuda"), "counts": i32(8, 4, 40, 7, 0, 0, 0, 0),
         "group_row_off": i32(0, 2, 4, 6, 8, 8), "group_ent_off": i32(0, 9, 18, 30, 40, 40), "group_tile_off": i32(0, 2, 4, 6, 8, 8),
         "entries": torch.stack([torch.arange(44) % 23, torch.full((44,), 16), torch.full((44,), 3), torch.zeros(44)], 1).int().cuda()}
    d, geom = 128, B.make_geom(8, 2, 128, 23, "bf16")
    pools = pools_of(23, 2, d, 3)
    q = torch.randn(9, 8, d, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    ws = torch.zeros(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    outs = []
    for spoilt in (False, True):
        if spoilt:
            t[what][at] = value
        tables = B.StepTables(**t, rows_per_group=16)
        out = torch.full_like(q, 7.0)
        B.mv_dag_decode_attn_fp8_blk(tables, geom, q, *pools, out, ws)
        assert B.mv_step_tables_read_status(tables) == (1 if spoilt else 0)
        outs.append(out)
    good, out = outs
    assert not (good[:8] == 7.0).all(-1).any() and (good[8] == 7.0).all()
    assert torch.equal(out[:2], good[:2]) and torch.equal(out[6:], good[6:])
    assert (out[2:6] == 7.0).all()     # both groups that share the offset


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES)
@pytest.mark.parametrize("pages", [3, 20, 1000])
def test_scales_of_zero(hq, hkv, branches, d, pages):
    """The first blocks of the history, or all of them, have scales of zero: they weigh like any other and their values are zero."""
    batch = streams(branches=branches)
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, 17)
    first = np.concatenate([batch.page_idx[batch.page_off[v]:min(batch.page_off[v] + pages, batch.page_off[v + 1])]
                            for r in range(batch.n_req) for v in range(batch.node_off[r], batch.node_off[r + 1])])
    first = torch.from_numpy(first.astype(np.int64)).cuda()
    v8[first] = 0
    sc[first] = 0.0
    q = torch.randn(int(batch.node_new.sum()), hq, d, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda").bfloat16()
    out, _ = check(batch, hq, hkv, d, q, (k8, v8, sc))
    assert pages < 1000 or (out == 0).all()


# Weights in three 8-bit floats: off by at most 1.5 * 2^-10 of themselves (2^-11 for exp2, joins and sums on top makes less than 2^-9), or 2^-29
# of the row's largest (2^-28 with the half-precision number's own last step).
FINE = {"weight": 2.0 ** -9, "floor": 2.0 ** -28}


def with_sink(batch, hq, hkv, d, mass, sink_value):
    """q and a cache whose first token takes ``mass`` of every row, before a tail of scores of spread one and V of mean 1/2."""
    rng = np.random.default_rng(1)
    n = int(max(batch.node_len))
    tail = torch.from_numpy((8 * rng.standard_normal(n)).astype(np.float32)).to(torch.float8_e4m3fn).float().numpy()
    k8, v8, sc = keyed(batch, hkv, d, of_prompt(batch, lambda r, m: np.concatenate([[0.0], tail[1:m]])))
    score = float(np.log(np.exp(tail[1:] / 8.0).sum() * mass / (1.0 - mass)))
    k, v = k8.view(torch.float8_e4m3fn).float(), v8.view(torch.float8_e4m3fn).float() + 32.0
    first = torch.from_numpy(batch.page_idx[batch.page_off[batch.node_off[:-1]]].astype(np.int64)).cuda()
    k[first, :, 0, 1] = 32.0
    v[first, :, 0] = sink_value
    q = torch.zeros(int(batch.node_new.sum()), hq, d, device="cuda")
    q[..., 0], q[..., 1] = 0.125, score / 32.0
    f8 = lambda x: x.to(torch.float8_e4m3fn).view(torch.uint8).contiguous()
    return q.bfloat16(), (f8(k), f8(v), sc)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES)
@pytest.mark.parametrize("mass", [0.9, 0.97, 0.999])
@pytest.mark.parametrize("sink_value", [0.0, 64.0])
def test_a_sink_leaves_the_tail_its_share(hq, hkv, branches, d, mass, sink_value):
    """A first token that takes nearly all of a row, its own V zero or not, and 16K others that share the rest."""
    batch = streams(10, 16000, branches)
    q, pools = with_sink(batch, hq, hkv, d, mass, sink_value)
    check(batch, hq, hkv, d, q, pools, 1.0, **FINE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("sink_value", [0.0, 64.0])
def test_a_sink_before_64k_tokens(d, sink_value):
    batch = streams(6, 65000, 4)
    q, pools = with_sink(batch, 16, 4, d, 0.97, sink_value)
    check(batch, 16, 4, d, q, pools, 1.0, **FINE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,requests,length,branches", [
    (8, 2, 1, 40000, 2), (4, 1, 1, 60000, 1), (2, 2, 1, 9000, 1), (40, 8, 60, 1900, 3), (8, 8, 90, 700, 1), (7, 1, 3, 20000, 9), (64, 8, 8, 5000, 8)])
def test_long_and_cut_streams_element_by_element(hq, hkv, requests, length, branches, d):
    """Flat random scores over long histories: every weight is small, so that a part lost on the way, or counted twice, shows."""
    batch = _batch_of([[([], length + 13 * r, 0)] + [([0], 5 * b, 1) for b in range(branches)] for r in range(requests)])
    q = torch.randn(int(batch.node_new.sum()), hq, d, generator=torch.Generator(device="cuda").manual_seed(26), device="cuda").bfloat16()
    out, step = check(batch, hq, hkv, d, q, pools_of(batch.num_pages, hkv, d, 25), **FINE)
    # and the bound tells: zeros fail it everywhere, a result without a 64th of the history somewhere
    r, ref, tol = next(elementwise(q, *pools_of(batch.num_pages, hkv, d, 25), step.t, hq // hkv, d ** -0.5, **FINE))
    assert (ref.abs() > tol).float().mean() > 0.5


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,branches", SHAPES[1:])
@pytest.mark.parametrize("power", [6, 12, 16, 60])
@pytest.mark.parametrize("large", ["heads", "rows"])
def test_rows_and_heads_of_one_stream_differ_in_magnitude(hq, hkv, branches, d, power, large):
    """Some heads, or some rows, have one element of 2^power, in a channel where every key is zero; the others of their group and
    KV head are of ordinary size and keep the accuracy that their own elements give."""
    batch = streams(12, 700, branches)
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, 13)
    k8[..., 0] = 0
    n = int(batch.node_new.sum())
    q = torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    spike = torch.zeros(n, hq, d, device="cuda")
    spike[..., 0] = 2.0 ** power
    which = (torch.arange(hq, device="cuda") % 4 == 1)[None, :, None] if large == "heads" else (torch.arange(n, device="cuda") % branches == 2)[:, None, None]
    check(batch, hq, hkv, d, torch.where(which, spike, q).bfloat16(), (k8, v8, sc), own_q=True, **FINE)


@pytest.mark.parametrize("d", [64, 128])
def test_q_of_every_magnitude(d):
    """q-vectors from 2^-100 to 2^20 in one stream, zeros among them: tiny ones average, large ones pick."""
    batch = streams(6, 700, 8)
    k8, v8, sc = pools_of(batch.num_pages, 4, d, 14)
    n = int(batch.node_new.sum())
    q = torch.zeros(n, 32, d, device="cuda")
    power = (torch.arange(n * 32, device="cuda") * 29 % 121 - 100).view(n, 32).double()
    # one element each, so that a score is one product: exact in 8-bit floats
    at = torch.arange(n * 32, device="cuda").view(n, 32) % d
    q.scatter_(2, at[..., None], torch.exp2(power).float()[..., None])
    q[3] = 0
    check(batch, 32, 4, d, q.bfloat16(), (k8, v8, sc), own_q=True, **FINE)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv", [(32, 4), (16, 8), (15, 3), (64, 1)])
@pytest.mark.parametrize("spread", [0, 8])
def test_streams_of_all_widths_follow_one_another(hq, hkv, d, spread):
    """Groups of few and of many q-vectors in turn, short and long, so that a share goes from one width to another; what lies behind
    the tokens of a page is NaN, and some rows see a part of their group's pages only."""
    group = hq // hkv
    most = max(1, 64 // group)
    rng = np.random.default_rng(hq + d)
    rows = [1 + (5 * r) % most for r in range(120)]
    batch = _batch_of([[([], int(rng.integers(1, 1800)), 0)] + [([0], int(rng.integers(0, 200)), 1) for _ in range(n)] for n in rows])
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, 33, spread=spread)
    if spread:
        sc[..., 0] = 2.0 ** -5
    used = torch.zeros(batch.num_pages, 16, dtype=torch.bool)
    for node in range(batch.n_nodes):
        n = int(batch.node_len[node] + batch.node_new[node])
        for p in range((n + 15) // 16):
            used[int(batch.page_idx[batch.page_off[node] + p]), :min(16, n - 16 * p)] = True
    q = torch.randn(int(batch.node_new.sum()), hq, d, generator=torch.Generator(device="cuda").manual_seed(8), device="cuda").bfloat16()
    clean, _ = check(batch, hq, hkv, d, q, (k8, v8, sc), own_q=True, **FINE)
    hole = (~used).cuda()[:, None, :, None].expand_as(k8)
    k8[hole], v8[hole] = 0x7F, 0xFF
    dirty, _ = attend(batch, hq, hkv, d, q, (k8, v8, sc))
    assert torch.equal(clean, dirty)
