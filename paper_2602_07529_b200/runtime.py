"""Device-side set-up around the C ABI: allocates pools and buffers with PyTorch, moves the seeded
synthetic values to the GPU and sequences the library calls.  No arithmetic of the method lives here;
every step of the path (planning, RoPE + cache write, attention) is a call into the library.
"""
from __future__ import annotations

import dataclasses

import numpy as np
import torch

from . import binding as B
from . import synth


def torch_dtype(geom: synth.Geometry):
    return torch.bfloat16 if geom.dtype == "bf16" else torch.float32


def pool_shape(num_pages: int, geom: synth.Geometry):
    """Shape of a K (or V) page pool: [pages][KV heads][head_dim / 64][page_size][64]."""
    return (num_pages, geom.n_kv_heads, geom.head_dim // 64, geom.page_size, 64)


def pool_tokens(pool, slot):
    """Head vectors [n, KV heads, head_dim] stored at the pool slots ``slot`` (int64 tensor): a view-only gather that
    undoes the 64-element column blocking of the pool."""
    ps = pool.shape[3]
    x = pool[slot // ps, :, :, slot % ps, :]            # [n, Hkv, head_dim / 64, 64]
    return x.reshape(x.shape[0], x.shape[1], -1)


def copy_pages(pools, src, dst, stream=None):
    """Copies pages in every pool, from lists on the host (what ``Scheduler.clone_request`` and ``Scheduler.compact`` return)."""
    dev = pools[0].device
    lists = [torch.from_numpy(np.asarray(x, dtype=np.int32).copy()).to(dev) for x in (src, dst)]
    B.mv_pages_copy(B.PagePools(pools), *lists, stream=stream)
    if stream is not None:  # the lists' memory may be handed out again only when that stream is through
        for x in lists:
            x.record_stream(torch.cuda.ExternalStream(stream, dev) if isinstance(stream, int) else stream)


def _dev_bytes(n: int, device):
    """256-byte aligned uint8 scratch of at least n bytes (torch's caching allocator aligns to 512)."""
    return torch.empty(max(int(n), 256), dtype=torch.uint8, device=device)


class PlanOnDevice:
    """A plan plus the caller-owned device buffer its kernel tables were uploaded to."""

    def __init__(self, batch, device="cuda", chunk_tokens: int = 0, stream=None, geom: synth.Geometry | None = None):
        hints = (geom.n_kv_heads, geom.group) if geom is not None else (0, 0)
        self.plan = B.Plan(batch, chunk_tokens, *hints)
        self.tables = _dev_bytes(self.plan.device_bytes(), device)
        self.plan.upload(self.tables, stream)

    def stats(self):
        return self.plan.stats()


def _stack_values(wl: synth.Workload, which: str, device, heads=None):
    """Concatenate per-request raw values on the device.  which = 'history' (tokens already in the pool),
    'new' (this step's tokens) or 'all' (every token, for prefill).  ``heads`` = (first query head, query heads, first
    KV head, KV heads) keeps only that head slice (sharding by KV head: the values are drawn for the whole geometry)."""
    dt = torch_dtype(wl.geom)
    b = wl.batch
    qs, ks, vs = [], [], []
    for r in range(b.n_req):
        vals = synth.request_values(wl, r)
        lo = int(b.node_off[r])
        off = vals["node_tok_off"]
        idx = []
        for n in b.request_nodes(r):
            a = int(off[n - lo])
            ln, nw = int(b.node_len[n]), int(b.node_new[n])
            if which == "history":
                idx.append(np.arange(a, a + ln))
            elif which == "new":
                idx.append(np.arange(a + ln, a + ln + nw))
            else:
                idx.append(np.arange(a, a + ln + nw))
        idx = np.concatenate(idx) if idx else np.zeros(0, np.int64)
        ks.append(torch.from_numpy(vals["k"][idx]).to(dt))
        vs.append(torch.from_numpy(vals["v"][idx]).to(dt))
        if which != "history":
            qs.append(torch.from_numpy(vals["q"]).to(dt))
    g = wl.geom
    if heads is not None:
        q0, nq, k0, nk = heads
        qs = [x[:, q0:q0 + nq].contiguous() for x in qs]
        ks = [x[:, k0:k0 + nk].contiguous() for x in ks]
        vs = [x[:, k0:k0 + nk].contiguous() for x in vs]
    hq, hkv = (g.n_q_heads, g.n_kv_heads) if heads is None else (heads[1], heads[3])
    cat = lambda xs, h: (torch.cat(xs, 0) if xs else torch.zeros(0, h, g.head_dim, dtype=dt)).to(device)
    q = cat(qs, hq) if which != "history" else None
    return q, cat(ks, hkv), cat(vs, hkv)


def _write_kv(plan, geom, form, q, k, v, q_rot, k_rot, k_pages, v_pages, stream=None):
    """The plan's rotation and cache write, by a rotary form where there is one."""
    args = (q, k, v, q_rot, k_rot, k_pages, v_pages, stream)
    if form is None:
        B.mv_rope_write_kv(plan, geom, *args)
    else:
        B.mv_rope_write_kv_form(plan, geom, form, *args)


def _write_kv_fp8_blk(tables, geom, form, q, k, v, q_rot, k_pages, v_pages, kv_scale, stream=None):
    """The same into the block-scaled 8-bit cache, from a step's tables."""
    args = (q, k, v, q_rot, None, k_pages, v_pages, kv_scale, stream)
    if form is None:
        B.mv_rope_write_kv_fp8_blk(tables, geom, *args)
    else:
        B.mv_rope_write_kv_fp8_blk_form(tables, geom, form, *args)


class DecodeState:
    """Pools holding the history of a decode workload, plus this step's inputs, plan and workspace.  ``form``: a rotary form in place of the
    geometry's own, in history and step."""

    def __init__(self, wl: synth.Workload, device="cuda", chunk_tokens: int = 0, canary: bool = False,
                 n_pool_copies: int = 1, heads=None, form=None):
        assert wl.kind == "decode"
        self.wl, self.device, self.form = wl, device, form
        g, b = wl.geom, wl.batch
        if heads is not None:   # this process owns a slice of the KV heads, their query heads and their pools
            g = dataclasses.replace(g, n_q_heads=heads[1], n_kv_heads=heads[3])
        self.local_geom = g
        self.geom = B.make_geom(g.n_q_heads, g.n_kv_heads, g.head_dim, b.num_pages, g.dtype, g.page_size, 0.0, g.rope_base)
        dt = torch_dtype(g)
        shape = pool_shape(b.num_pages, g)
        fill = float("nan") if canary else 0.0
        self.pools = [(torch.full(shape, fill, dtype=dt, device=device), torch.full(shape, fill, dtype=dt, device=device))
                      for _ in range(n_pool_copies)]
        # history -> pools through the library's own RoPE + cache-write call
        hist = synth.DagBatch(b.n_req, b.node_off, np.zeros_like(b.node_len), b.node_len, b.parent_off, b.parent_idx,
                              b.page_off, b.page_idx, b.page_size, b.num_pages, b.vis_mode, b.pos_mode)
        _, kh, vh = _stack_values(wl, "history", device, heads)
        hp = PlanOnDevice(hist, device, geom=g)
        for kp, vp in self.pools:
            _write_kv(hp.plan, self.geom, form, None, kh, vh, None, None, kp, vp)
        torch.cuda.synchronize()
        del kh, vh, hp
        self.q, self.k, self.v = _stack_values(wl, "new", device, heads)
        self.pod = PlanOnDevice(b, device, chunk_tokens, geom=g)
        self.plan = self.pod.plan
        self.q_rot = torch.empty_like(self.q)
        self.out = torch.empty_like(self.q)
        self.workspace = _dev_bytes(self.plan.workspace_bytes(self.geom, B.OP_DECODE_ATTN), device)

    def step(self, pool: int = 0, stream=None):
        kp, vp = self.pools[pool]
        _write_kv(self.plan, self.geom, self.form, self.q, self.k, self.v, self.q_rot, None, kp, vp, stream)
        B.mv_dag_decode_attn(self.plan, self.geom, self.q_rot, kp, vp, self.out, self.workspace, stream)
        return self.out


class DecodeStateFP8(DecodeState):
    """The same decode workload with the KV history in FP8 pools (8-bit floats, one scale per KV head).  No rotary forms: the write into these
    pools knows the geometry's own rotation only."""

    def __init__(self, wl: synth.Workload, device="cuda", n_pool_copies: int = 1):
        assert wl.kind == "decode" and wl.geom.dtype == "bf16" and wl.geom.head_dim == 128
        self.wl, self.device = wl, device
        g, b = wl.geom, wl.batch
        self.local_geom = g
        self.geom = B.make_geom(g.n_q_heads, g.n_kv_heads, g.head_dim, b.num_pages, g.dtype, g.page_size, 0.0, g.rope_base)
        ks, vs = synth.fp8_scales(g)
        self.kv_scale = torch.from_numpy(np.concatenate([ks, vs])).to(device)
        shape = (b.num_pages, g.n_kv_heads, g.page_size, g.head_dim)
        self.pools = [(torch.zeros(shape, dtype=torch.uint8, device=device), torch.zeros(shape, dtype=torch.uint8, device=device))
                      for _ in range(n_pool_copies)]
        hist = synth.DagBatch(b.n_req, b.node_off, np.zeros_like(b.node_len), b.node_len, b.parent_off, b.parent_idx,
                              b.page_off, b.page_idx, b.page_size, b.num_pages, b.vis_mode, b.pos_mode)
        _, kh, vh = _stack_values(wl, "history", device)
        hp = PlanOnDevice(hist, device, geom=g)
        for kp, vp in self.pools:
            B.mv_rope_write_kv_fp8(hp.plan, self.geom, None, kh, vh, None, kp, vp, self.kv_scale)
        torch.cuda.synchronize()
        del kh, vh, hp
        self.q, self.k, self.v = _stack_values(wl, "new", device)
        self.pod = PlanOnDevice(b, device, 0, geom=g)
        self.plan = self.pod.plan
        self.q_rot = torch.empty_like(self.q)
        self.out = torch.empty_like(self.q)
        self.workspace = _dev_bytes(self.plan.workspace_bytes(self.geom, B.OP_DECODE_ATTN), device)

    def step(self, pool: int = 0, stream=None):
        kp, vp = self.pools[pool]
        B.mv_rope_write_kv_fp8(self.plan, self.geom, self.q, self.k, self.v, self.q_rot, kp, vp, self.kv_scale, stream)
        B.mv_dag_decode_attn_fp8(self.plan, self.geom, self.q_rot, kp, vp, self.kv_scale, self.out, self.workspace, stream)
        return self.out


class StepOnDevice:
    """A step planned on the device: the batch's arrays as CUDA tensors, the tables built from them, and their workspace.
    ``build()`` may be called (or replayed) again after the tensors in ``self.arrays`` have changed; the capacities are
    those of the batch given here unless stated.  ``blocks=False``: positions and slots only."""

    ARRAYS = ("node_off", "node_len", "node_new", "parent_off", "parent_idx", "page_off", "page_idx")

    def __init__(self, batch, group: int, device="cuda", blocks: bool = True, max_rows: int | None = None,
                 max_groups: int | None = None, max_entries: int | None = None):
        i32 = lambda x: torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(device)
        self.arrays = {n: i32(getattr(batch, n)) for n in self.ARRAYS}
        per = max(1, 64 // group)
        off, new = np.asarray(batch.node_off), np.asarray(batch.node_new)
        rows = np.asarray([int(new[off[r]:off[r + 1]].sum()) for r in range(batch.n_req)], np.int64)
        groups = (rows + per - 1) // per
        if max_rows is None:
            max_rows = int(rows.sum())
        if max_groups is None:
            max_groups = max(1, int(groups.sum()))
        if max_entries is None:   # every page once per group, and at most one more entry for every new token
            pages = np.asarray(batch.page_off)[off[1:]] - np.asarray(batch.page_off)[off[:-1]]
            max_entries = int((pages * groups).sum() + rows.sum())
        empty = lambda n, dt: torch.zeros(int(n), dtype=dt, device=device)
        t = {"pos_id": empty(max_rows, torch.int32), "slot": empty(max_rows, torch.int64), "counts": empty(8, torch.int32)}
        if blocks:
            t.update({n: empty(max_groups + 1, torch.int32) for n in ("group_row_off", "group_ent_off", "group_tile_off")})
            t["entries"] = empty(4 * max(1, max_entries), torch.int32).view(-1, 4)
        self.t = t
        self.batch = B.DeviceBatch(batch.n_req, **self.arrays, num_pages=batch.num_pages, vis_mode=batch.vis_mode,
                                   max_req_nodes=max(1, int(np.diff(off).max()) if batch.n_req else 1), pos_mode=batch.pos_mode)
        self.tables = B.StepTables(**t, rows_per_group=per)
        self.workspace = _dev_bytes(B.mv_step_tables_workspace_bytes(self.batch), device)

    def build(self, stream=None):
        B.mv_step_tables_build(self.batch, self.tables, self.workspace, stream)
        return self.tables

    def read_status(self, stream=None) -> int:
        return B.mv_step_tables_read_status(self.tables, stream)


class ChunkOnDevice:
    """A step with any number of new tokens per node, planned on the device: positions and slots (``self.steps``, a StepOnDevice) and
    the query tiles and page lists of the chunk attention.  ``build()`` may be called (or replayed) again after the tensors in
    ``self.arrays`` have changed; the capacities are those of the batch given here unless stated."""

    def __init__(self, batch, group: int, device="cuda", max_rows: int | None = None, max_tiles: int | None = None, max_entries: int | None = None):
        self.steps = StepOnDevice(batch, group, device, blocks=False, max_rows=max_rows)
        self.arrays, self.batch = self.steps.arrays, self.steps.batch
        per = 2 * (128 // group)
        new, off = np.asarray(batch.node_new, np.int64), np.asarray(batch.node_off)
        page_off = np.asarray(batch.page_off, np.int64)
        if max_tiles is None:
            max_tiles = int(((new + per - 1) // per).sum())
        if max_entries is None:   # every page of the request for each of its receiving nodes
            max_entries = sum(int((new[lo:hi] > 0).sum()) * int(page_off[hi] - page_off[lo]) for lo, hi in zip(off[:-1], off[1:]))
        empty = lambda *n: torch.zeros(*n, dtype=torch.int32, device=device)
        self.t = {"tiles": empty(max(1, max_tiles), 8), "entries": empty(max(1, max_entries), 2), "counts": empty(8)}
        self.tables = B.ChunkTables(**self.t, max_rows=self.steps.tables.max_rows, rows_per_tile=per)
        self.workspace = _dev_bytes(B.mv_chunk_tables_workspace_bytes(self.batch), device)

    def build(self, stream=None):
        self.steps.build(stream)
        B.mv_chunk_tables_build(self.batch, self.tables, self.workspace, stream)
        return self.tables

    def read_status(self, stream=None) -> int:
        return max(self.steps.read_status(stream), B.mv_chunk_tables_read_status(self.tables, stream))


class ChunkStateFP8Blk:
    """A step that writes its new tokens (any number per node) into the block-scaled 8-bit cache and attends over it.  ``form``: a rotary form in
    place of the geometry's own."""

    def __init__(self, wl: synth.Workload, device="cuda", form=None):
        assert wl.geom.dtype == "bf16"
        self.wl, self.device, self.form = wl, device, form
        g, b = wl.geom, wl.batch
        self.geom = B.make_geom(g.n_q_heads, g.n_kv_heads, g.head_dim, b.num_pages, g.dtype, g.page_size, 0.0, g.rope_base)
        shape = (b.num_pages, g.n_kv_heads, g.page_size, g.head_dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
        self.kv_scale = torch.zeros(b.num_pages, g.n_kv_heads, 2, dtype=torch.float32, device=device)
        if int(np.asarray(b.node_len).sum()) > 0:
            hist = synth.DagBatch(b.n_req, b.node_off, np.zeros_like(b.node_len), b.node_len, b.parent_off, b.parent_idx,
                                  b.page_off, b.page_idx, b.page_size, b.num_pages, b.vis_mode, b.pos_mode)
            _, kh, vh = _stack_values(wl, "history", device)
            hs = StepOnDevice(hist, g.group, device, blocks=False)
            _write_kv_fp8_blk(hs.build(), self.geom, form, None, kh, vh, None, self.k_pages, self.v_pages, self.kv_scale)
            torch.cuda.synchronize()
            assert hs.read_status() == 0
            del kh, vh, hs
        self.q, self.k, self.v = _stack_values(wl, "new" if wl.kind == "decode" else "all", device)
        self.chunk = ChunkOnDevice(b, g.group, device)
        self.q_rot = torch.empty_like(self.q)
        self.out = torch.empty_like(self.q)
        self.workspace = _dev_bytes(B.mv_chunk_attn_workspace_bytes(self.geom), device)

    def step(self, stream=None):
        t = self.chunk.build(stream)
        _write_kv_fp8_blk(self.chunk.steps.tables, self.geom, self.form, self.q, self.k, self.v, self.q_rot, self.k_pages, self.v_pages, self.kv_scale, stream)
        B.mv_dag_chunk_attn_fp8_blk(t, self.geom, self.q_rot, self.k_pages, self.v_pages, self.kv_scale, self.out, self.workspace, stream)
        return self.out


class DecodeStateFP8Blk(DecodeState):
    """The same decode workload planned on the device, with the KV history in FP8 pools that carry a scale per (page, KV head).  ``form``: a
    rotary form in place of the geometry's own."""

    def __init__(self, wl: synth.Workload, device="cuda", form=None):
        assert wl.kind == "decode" and wl.geom.dtype == "bf16"
        self.wl, self.device, self.form = wl, device, form
        g, b = wl.geom, wl.batch
        self.local_geom = g
        self.geom = B.make_geom(g.n_q_heads, g.n_kv_heads, g.head_dim, b.num_pages, g.dtype, g.page_size, 0.0, g.rope_base)
        shape = (b.num_pages, g.n_kv_heads, g.page_size, g.head_dim)
        self.k_pages, self.v_pages = (torch.zeros(shape, dtype=torch.uint8, device=device) for _ in range(2))
        self.kv_scale = torch.zeros(b.num_pages, g.n_kv_heads, 2, dtype=torch.float32, device=device)
        hist = synth.DagBatch(b.n_req, b.node_off, np.zeros_like(b.node_len), b.node_len, b.parent_off, b.parent_idx,
                              b.page_off, b.page_idx, b.page_size, b.num_pages, b.vis_mode, b.pos_mode)
        _, kh, vh = _stack_values(wl, "history", device)
        hs = StepOnDevice(hist, g.group, device, blocks=False)
        _write_kv_fp8_blk(hs.build(), self.geom, form, None, kh, vh, None, self.k_pages, self.v_pages, self.kv_scale)
        torch.cuda.synchronize()
        assert hs.read_status() == 0
        del kh, vh, hs
        self.q, self.k, self.v = _stack_values(wl, "new", device)
        self.steps = StepOnDevice(b, g.group, device)
        self.q_rot = torch.empty_like(self.q)
        self.out = torch.empty_like(self.q)
        self.workspace = _dev_bytes(B.mv_decode_fp8_blk_workspace_bytes(self.geom), device)

    def step(self, stream=None):
        t = self.steps.build(stream)
        _write_kv_fp8_blk(t, self.geom, self.form, self.q, self.k, self.v, self.q_rot, self.k_pages, self.v_pages, self.kv_scale, stream)
        B.mv_dag_decode_attn_fp8_blk(t, self.geom, self.q_rot, self.k_pages, self.v_pages, self.kv_scale, self.out, self.workspace, stream)
        return self.out


class PrefillState:
    """A prompt's rotation, cache write and attention, and its backward pass.  ``form``: a rotary form in place of the geometry's own."""

    def __init__(self, wl: synth.Workload, device="cuda", with_pool: bool = True, form=None):
        assert wl.kind == "prefill"
        self.wl, self.device, self.with_pool, self.form = wl, device, with_pool, form
        g, b = wl.geom, wl.batch
        self.geom = B.geom_of(wl)
        dt = torch_dtype(g)
        self.q, self.k, self.v = _stack_values(wl, "all", device)
        self.pod = PlanOnDevice(b, device, geom=g)
        self.plan = self.pod.plan
        shape = pool_shape(b.num_pages, g)
        self.k_pages = torch.zeros(shape, dtype=dt, device=device)
        self.v_pages = torch.zeros(shape, dtype=dt, device=device)
        self.q_rot = torch.empty_like(self.q)
        self.k_rot = torch.empty_like(self.k)
        self.out = torch.empty_like(self.q)

    def step(self, stream=None, lse=None):
        pools = (self.k_pages, self.v_pages) if self.with_pool else (None, None)
        _write_kv(self.plan, self.geom, self.form, self.q, self.k, self.v, self.q_rot, self.k_rot, *pools, stream)
        B.mv_dag_prefill_attn(self.plan, self.geom, self.q_rot, self.k_rot, self.v, self.out, lse, stream)
        return self.out

    def forward_backward(self, dout, stream=None, raw: bool = False):
        """Forward with the rows' log-sum-exp kept, then mv_dag_prefill_attn_bwd.  Returns (out, dq_rot, dk_rot, dv), or with ``raw`` the
        gradients of q and k themselves: those of the rotated ones turned back (a geometry's own rotation needs a rope_base of at least 1
        for that)."""
        if raw:  # a form of the geometry's own rotation has the forward call's angles; refused before anything is launched
            turn = self.form if self.form is not None else B.RopeForm(B.ROPE_HALVES, self.wl.geom.head_dim, base=self.wl.geom.rope_base)
        if not hasattr(self, "lse"):
            self.lse = _dev_bytes(self.plan.workspace_bytes(self.geom, B.OP_PREFILL_ATTN), self.device)
            self.bwd_ws = _dev_bytes(self.plan.workspace_bytes(self.geom, B.OP_PREFILL_ATTN_BWD), self.device)
            self.dq, self.dk, self.dv = torch.empty_like(self.q), torch.empty_like(self.k), torch.empty_like(self.v)
        self.step(stream, self.lse)
        B.mv_dag_prefill_attn_bwd(self.plan, self.geom, self.q_rot, self.k_rot, self.v, self.out, dout, self.lse, self.dq, self.dk,
                                  self.dv, self.bwd_ws, stream)
        if raw:
            B.mv_rope_rotate(turn, self.geom, self.plan, self.dq, self.dk, self.dq, self.dk, backward=True, stream=stream)
        return self.out, self.dq, self.dk, self.dv
