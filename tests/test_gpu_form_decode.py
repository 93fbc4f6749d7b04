"""Decode steps of the runtime with a rotary form: history and new tokens rotated by it, and attention over what was written.

Tolerances: rotation as in the tests of the forms (a rounding to bf16 and 2^-20 of a pair's length); attention as in those of the decode calls,
relative L2 of 1e-2 (bf16 weights or 8-bit pieces, results in bf16)."""
import numpy as np
import pytest
import torch

from paper_2602_07529_b200 import synth
from helpers import rel_l2
from test_gpu_fp8_blk import visible_counts
from test_gpu_rope_form import close

pytestmark = pytest.mark.gpu


def _mods():
    from paper_2602_07529_b200 import binding as B, runtime
    return B, runtime


def workload():
    return synth.config2(n_req=3, prefix=100, branches=3, branch_len=40)


def forms(B):
    return [B.RopeForm(B.ROPE_PAIRS, 64, first=32, base=5e5), B.RopeForm(B.ROPE_HALVES, 128, scaling="ramp", factor=8.0, length=64, amplitude=1.25)]


def attention(st, seen, load):
    """Softmax attention of every row in 64 bits over the pages it sees; load(pages, which) -> [pages][KV heads][16][head_dim]."""
    g = st.wl.geom
    out = []
    for r, (_, pages) in enumerate(seen):
        page = torch.tensor(list(pages), device="cuda")
        there = (torch.arange(16, device="cuda") < torch.tensor(list(pages.values()), device="cuda")[:, None]).flatten()
        k, v = (load(page, w).double().permute(1, 0, 2, 3).reshape(g.n_kv_heads, -1, g.head_dim)[:, there] for w in (0, 1))
        q = st.q_rot[r].double().view(g.n_kv_heads, g.group, g.head_dim)
        p = torch.softmax(torch.einsum("hgd,hkd->hgk", q, k) * g.head_dim ** -0.5, -1)
        out.append(torch.einsum("hgk,hkd->hgd", p, v).reshape(g.n_q_heads, g.head_dim))
    return torch.stack(out)


@pytest.mark.parametrize("which", [0, 1])
def test_bf16_cache(which):
    B, runtime = _mods()
    wl = workload()
    form = forms(B)[which]
    st = runtime.DecodeState(wl, form=form, n_pool_copies=2)
    hist = synth.DagBatch(wl.batch.n_req, wl.batch.node_off, np.zeros_like(wl.batch.node_len), wl.batch.node_len, wl.batch.parent_off, wl.batch.parent_idx,
                          wl.batch.page_off, wl.batch.page_idx, 16, wl.batch.num_pages)
    plan = B.Plan(hist)
    _, kh, _ = runtime._stack_values(wl, "history", "cuda")
    for pool in (0, 1):
        out = st.step(pool).clone()
        kp, vp = st.pools[pool]
        close(runtime.pool_tokens(kp, torch.from_numpy(plan.table("slot")).cuda()), form, plan.table("pos_id"), kh)
        close(runtime.pool_tokens(kp, torch.from_numpy(st.plan.table("slot")).cuda()), form, st.plan.table("pos_id"), st.k)
        close(st.q_rot, form, st.plan.table("pos_id"), st.q)
        load = lambda page, w: (kp, vp)[w][page].permute(0, 1, 3, 2, 4).reshape(len(page), wl.geom.n_kv_heads, 16, 128)
        assert rel_l2(out.double().cpu(), attention(st, visible_counts(wl.batch), load).cpu()) <= 1e-2


@pytest.mark.parametrize("which", [0, 1])
def test_block_scaled_cache(which):
    """Against the definition, and the cache and queries against those of the chunk call's state on the same step."""
    B, runtime = _mods()
    wl = workload()
    form = forms(B)[which]
    st, chunk = runtime.DecodeStateFP8Blk(wl, form=form), runtime.ChunkStateFP8Blk(wl, form=form)
    out, other = st.step(), chunk.step()
    assert st.steps.read_status() == 0 and chunk.chunk.read_status() == 0
    close(st.q_rot, form, st.steps.t["pos_id"].cpu().numpy(), st.q)
    for a, c in ((st.q_rot, chunk.q_rot), (st.k_pages, chunk.k_pages), (st.v_pages, chunk.v_pages), (st.kv_scale, chunk.kv_scale)):
        assert torch.equal(a, c)
    pools = st.k_pages, st.v_pages
    load = lambda page, w: pools[w][page].view(torch.float8_e4m3fn).double() * st.kv_scale[page][..., w].double()[..., None, None]
    ref = attention(st, visible_counts(wl.batch), load).cpu()
    assert rel_l2(out.double().cpu(), ref) <= 1e-2 and rel_l2(other.double().cpu(), ref) <= 1e-2
    plain = runtime.DecodeStateFP8Blk(wl)
    plain.step()
    assert not torch.equal(plain.q_rot, st.q_rot) and not torch.equal(plain.k_pages, st.k_pages)


def test_decode_over_pools_written_elsewhere():
    """Pools that the caller has written with the form, decoded further by the state: the bits of its own pools."""
    B, runtime = _mods()
    form = forms(B)[0]
    wl = workload()
    st = runtime.DecodeState(wl, form=form)
    want = st.step().clone()
    b = wl.batch
    hist = synth.DagBatch(b.n_req, b.node_off, np.zeros_like(b.node_len), b.node_len, b.parent_off, b.parent_idx, b.page_off, b.page_idx, 16, b.num_pages)
    _, kh, vh = runtime._stack_values(wl, "history", "cuda")
    pod = runtime.PlanOnDevice(hist, geom=wl.geom)
    kp, vp = (torch.zeros_like(x) for x in st.pools[0])
    k_rot = torch.empty_like(kh)
    B.mv_rope_write_kv_form(pod.plan, st.geom, form, None, kh, vh, None, k_rot, kp, vp)
    st.pools.append((kp, vp))
    assert torch.equal(st.step(1), want)
