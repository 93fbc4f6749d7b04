"""The device-planned decode path over the block-scaled 8-bit cache, each operator against its definition in 64 bits.

Tolerances, fixed before the first run:
  tables   whole numbers: equal.
  scales   powers of two: equal; where a block's largest magnitude lies exactly at the bound of a scale, the next one is
           right as well (the header says so).
  bytes    a stored value is the nearest 8-bit float of x / scale: off by at most half a step of the format at that
           value (2^-4 of it, or 2^-10 among the subnormals), plus what float arithmetic can move a rotated element
           (cos, sin and two products: under 2^-21 of the pair's length).
  q_rot    bf16: 2^-8 of the value, plus the same.
  out      bf16 rounds by at most 2^-8 of the value.  Weights carry at most 2^-8 each (8-bit floats as value plus
           remainder), which moves an output by at most 2^-8 * A in the numerator, A = sum_j p_j |V_j| / sum_j p_j; scores
           are sums of 128 products in 32 bits, off by far less than 2^-12 in the exponent for the magnitudes drawn here, another 2^-12 A.  Small
           weights as 8-bit floats: remainders have a quantum of 2^-9 / 16, the largest weight is kept at 2^5 or more, so a
           weight is off by at most half a quantum, 2^-14 / 2^5 = 2^-19 of the largest: at most N * 2^-19 A's scale for N tokens.
"""
import numpy as np
import pytest
import torch

from oracle import medverse_oracle as O
from paper_2602_07529_b200 import synth
from helpers import batch_dict

pytestmark = pytest.mark.gpu


def _mods():
    from paper_2602_07529_b200 import binding as B, runtime
    return B, runtime


# ------------------------------------------------------------------------------------------------ definitions

def visible_counts(batch):
    """Per row, in row order: (request, {page id: tokens of it the row sees}), straight from the definition."""
    b = batch_dict(batch)
    out = []
    for r in range(batch.n_req):
        lo, hi, parents = O._req_parents(b, r)
        layer = O.node_layers(parents)
        vis = O.visible_sets(parents, layer, batch.vis_mode)
        for v in range(hi - lo):
            for j in range(int(batch.node_new[lo + v])):
                seen = {}
                for u in vis[v]:
                    n = int(batch.node_len[lo + u]) + (j + 1 if u == v else int(batch.node_new[lo + u]))
                    for p in range((n + 15) // 16):
                        seen[int(batch.page_idx[batch.page_off[lo + u] + p])] = min(16, n - 16 * p)
                out.append((r, seen))
    return out


def check_tables(step, batch):
    """The built tables against the oracle's canonical tables and the rows' visible pages."""
    t = {k: v.cpu().numpy() for k, v in step.t.items()}
    want = O.plan_tables(batch_dict(batch))
    n = len(want["pos_id"])
    rows, groups, ents, tiles, status = (int(x) for x in t["counts"][:5])
    assert status == 0 and rows == n and list(t["counts"][5:]) == [0, 0, 0]
    assert np.array_equal(t["pos_id"][:n], want["pos_id"]) and np.array_equal(t["slot"][:n], want["slot"])
    assert (t["slot"][n:] == -1).all() and (t["pos_id"][n:] == 0).all()
    if "entries" not in t:
        return
    seen = visible_counts(batch)
    ro, eo, to = t["group_row_off"], t["group_ent_off"], t["group_tile_off"]
    assert (ro[groups:] == rows).all() and (eo[groups:] == ents).all() and (to[groups:] == tiles).all()
    per = step.tables.c_tables.rows_per_group
    assert ro[0] == 0 and eo[0] == 0 and to[0] == 0
    expect_groups = 0
    for r in range(batch.n_req):
        expect_groups += -(-sum(1 for q, _ in seen if q == r) // per)
    assert groups == expect_groups
    for g in range(groups):
        e = t["entries"][eo[g]:eo[g + 1]]
        assert to[g + 1] - to[g] == -(-len(e) // 8)
        assert len({seen[i][0] for i in range(ro[g], ro[g + 1])}) == 1 and 0 < ro[g + 1] - ro[g] <= per
        mask = e[:, 2].view(np.uint32).astype(np.uint64) | (e[:, 3].view(np.uint32).astype(np.uint64) << np.uint64(32))
        assert (mask != 0).all()
        keys = [(int(p), int(c)) for p, c in e[:, :2]]
        assert len(set(keys)) == len(keys)
        for i in range(ro[g], ro[g + 1]):
            mine = {int(p): int(c) for (p, c), m in zip(keys, mask) if (int(m) >> int(i - ro[g])) & 1}
            assert mine == seen[i][1]
            assert sum(1 for m in mask if (int(m) >> int(i - ro[g])) & 1) == len(mine)     # each page once per row
    return t


def attend64(q, k8, v8, scale, t, group, sm_scale=None):
    """(out, A) in float64 from the tables' entries, row by row; rows outside the step are None."""
    d = q.shape[2]
    hkv = k8.shape[1]
    sm_scale = d ** -0.5 if sm_scale is None else sm_scale
    ro, eo, ent, counts = (t[k].cpu() for k in ("group_row_off", "group_ent_off", "entries", "counts"))
    out = [None] * q.shape[0]
    kd, vd = (p.view(torch.float8_e4m3fn).double() * scale[:, :, w].double()[:, :, None, None] for w, p in enumerate((k8, v8)))
    for g in range(int(counts[1])):
        e = ent[int(eo[g]):int(eo[g + 1])].long()
        for r in range(int(ro[g]), int(ro[g + 1])):
            b = r - int(ro[g])
            sel = e[((e[:, 2 + b // 32] >> (b % 32)) & 1) > 0]
            tok = (torch.arange(16) < sel[:, 1:2]).reshape(-1).nonzero()[:, 0].to(q.device)
            if tok.numel() == 0:
                out[r] = (torch.zeros(q.shape[1], d, dtype=torch.float64, device=q.device),) * 2
                continue
            page = sel[:, 0].to(q.device)
            kk = kd[page].transpose(1, 2).reshape(-1, hkv, d)[tok]
            vv = vd[page].transpose(1, 2).reshape(-1, hkv, d)[tok]
            qq = q[r].double().view(hkv, group, d)
            s = torch.einsum("hgd,nhd->hgn", qq, kk) * sm_scale
            p = torch.softmax(s, -1)
            out[r] = (torch.einsum("hgn,nhd->hgd", p, vv).reshape(-1, d), torch.einsum("hgn,nhd->hgd", p, vv.abs()).reshape(-1, d))
    return out


def check_out(got, want, tokens=4096):
    for r, w in enumerate(want):
        if w is None:
            continue
        ref, a = w
        bad = torch.isnan(ref)
        assert torch.equal(torch.isnan(got[r].double()), bad), r
        tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12 + tokens * 2.0 ** -19) * a + 1e-30
        err = (got[r].double() - ref).abs()
        over = (err > tol) & ~bad
        assert not over.any(), (r, over.nonzero()[:4].tolist(), float((err / tol)[~bad].max()))


def pools_of(n_pages, hkv, d, seed, scales=None, spread=0):
    """A cache of random contents: bytes at scales that differ from block to block by up to 2^spread."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    x = torch.randn(2, n_pages, hkv, 16, d, generator=g, device="cuda")
    e = torch.randint(-spread, spread + 1, (n_pages, hkv, 2), generator=g, device="cuda").float() if spread else torch.zeros(n_pages, hkv, 2, device="cuda")
    scale = torch.exp2(e - 6.0)
    k8 = (x[0] * 64).to(torch.float8_e4m3fn).view(torch.uint8)
    v8 = (x[1] * 64).to(torch.float8_e4m3fn).view(torch.uint8)
    return k8.contiguous(), v8.contiguous(), scale


# ------------------------------------------------------------------------------------------------ tables

def _dag(seed, **kw):
    geom = synth.Geometry(kw.pop("hq", 8), kw.pop("hkv", 2), kw.pop("d", 128), 16, "bf16")
    return synth.random_dag_workload(seed, "decode", geom=geom, **kw)


@pytest.mark.parametrize("vis", [0, 1])
@pytest.mark.parametrize("pos", [0, 1])
@pytest.mark.parametrize("seed,max_new,group", [(0, 1, 4), (1, 1, 1), (2, 7, 8), (3, 40, 16), (4, 100, 64), (5, 256, 4), (6, 40, 1), (7, 17, 2)])
def test_tables_random_dags(vis, pos, seed, max_new, group):
    _, runtime = _mods()
    wl = _dag(seed, n_req=5, max_nodes=12, max_len=90, max_new=max_new, vis_mode=vis, pos_mode=pos)
    step = runtime.StepOnDevice(wl.batch, group, max_rows=int(wl.batch.node_new.sum()) + 3)
    step.build()
    check_tables(step, wl.batch)


def _batch_of(requests, seed=0, **kw):
    return synth.build_batch(requests, rng=np.random.default_rng(seed), **kw)


@pytest.mark.parametrize("name", ["empty", "empty requests", "no new tokens", "one token", "chain", "wide join", "repeated parent", "inner nodes receive"])
def test_tables_odd_batches(name):
    _, runtime = _mods()
    reqs = {"empty": [],
            "empty requests": [[], [([], 5, 1)], [], []],
            "no new tokens": [[([], 40, 0), ([0], 3, 0)]],
            "one token": [[([], 0, 1)]],
            "chain": [[([], 1, 0)] + [([v], 3, 1 if v == 1998 else 0) for v in range(1999)]],
            "wide join": [[([], 17, 0)] + [([0], 15 + v % 4, 0) for v in range(700)] + [(list(range(1, 701)), 0, 1)]],
            "repeated parent": [[([], 17, 0), ([0, 0, 0], 2, 1), ([1, 0, 1], 0, 3)]],
            "inner nodes receive": [[([], 30, 5), ([0], 16, 2), ([0, 1], 1, 17), ([0], 0, 4)]]}[name]
    batch = _batch_of(reqs)
    step = runtime.StepOnDevice(batch, 4, max_rows=40, max_groups=9)
    step.build()
    check_tables(step, batch)


def test_tables_positions_only_and_long_prompt():
    _, runtime = _mods()
    batch = _batch_of([[([], 0, 5000), ([0], 0, 333)], [([], 0, 1)]])
    step = runtime.StepOnDevice(batch, 4, blocks=False)
    step.build()
    check_tables(step, batch)


@pytest.mark.parametrize("what,status", [("parent after child", 2), ("parent negative", 2), ("pages too few", 3), ("page beyond the pool", 1),
                                         ("page negative", 1), ("negative length", 1), ("offsets fall", 1), ("offset beyond the list", 1),
                                         ("too many rows", 5), ("too many groups", 5), ("too many entries", 5), ("too many nodes", 4), ("too many new", 4)])
def test_tables_bad_contents_give_an_empty_step(what, status):
    B, runtime = _mods()
    batch = _batch_of([[([], 40, 0), ([0], 20, 1), ([0], 7, 1)], [([], 300, 0), ([0], 9, 280 if what == "too many new" else 2)]])
    kw = {"too many rows": {"max_rows": 3}, "too many groups": {"max_groups": 1}, "too many entries": {"max_entries": 20}}.get(what, {})
    kw = {"max_rows": 290, "max_groups": 40, "max_entries": 900, **kw}
    step = runtime.StepOnDevice(batch, 4, **kw)
    a = step.arrays
    if what == "parent after child": a["parent_idx"][0] = 1
    if what == "parent negative": a["parent_idx"][1] = -1
    if what == "pages too few": a["node_len"][1] = 33
    if what == "page beyond the pool": a["page_idx"][4] = batch.num_pages
    if what == "page negative": a["page_idx"][4] = -1
    if what == "negative length": a["node_len"][2] = -1
    if what == "offsets fall": a["page_off"][2] = 0
    if what == "offset beyond the list": a["parent_off"][5] = 1000
    if what == "too many nodes":
        step.batch.c_shape.max_req_nodes = 2
    for k, v in step.t.items():
        v.fill_(7)
    step.build()
    assert step.read_status() == status
    t = {k: v.cpu().numpy() for k, v in step.t.items()}
    assert list(t["counts"]) == [0, 0, 0, 0, status, 0, 0, 0]
    assert (t["slot"] == -1).all() and (t["pos_id"] == 0).all()
    assert (t["group_row_off"] == 0).all() and (t["group_ent_off"] == 0).all() and (t["group_tile_off"] == 0).all()
    assert (t["entries"] == 7).all()
    # and the calls behind it touch nothing
    geom = B.make_geom(8, 2, 128, batch.num_pages, "bf16")
    q = torch.randn(kw["max_rows"], 8, 128, device="cuda").bfloat16()
    out, q_rot = torch.full_like(q, 3.0), torch.full_like(q, 3.0)
    k8, v8, sc = pools_of(batch.num_pages, 2, 128, 1)
    before = [x.clone() for x in (k8, v8, sc)]
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    kv = q[:, :2].contiguous()
    B.mv_rope_write_kv_fp8_blk(step.tables, geom, q, kv, kv, q_rot, None, k8, v8, sc)
    B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, k8, v8, sc, out, ws)
    assert (out == 3.0).all() and (q_rot == 3.0).all()
    for x, y in zip(before, (k8, v8, sc)):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------ cache write

def write64(batch_tabs, k, v, k8, v8, scale, base=10000.0):
    """The write by its definition: (values of K and V, scales, slack, tie, slots that belong to the block's tokens) after it, from the pools before it; values in
    float64, unrounded for the new tokens and for stored tokens that moved."""
    pos, slot = batch_tabs
    pools = [p.cpu().view(torch.float8_e4m3fn).double().numpy() for p in (k8, v8)]
    sc = scale.cpu().double().numpy().copy()
    rot = O.rope_rotate(k, pos, base)
    pair = np.sqrt(k[..., :k.shape[-1] // 2] ** 2 + k[..., k.shape[-1] // 2:] ** 2)
    pair = np.concatenate([pair, pair], -1)
    slack = [np.zeros_like(pools[0]), np.zeros_like(pools[1])]
    tie = np.zeros(sc.shape, bool)
    held = np.zeros((sc.shape[0], 16), bool)
    order = {}
    for i, s in enumerate(slot):
        order.setdefault(int(s) // 16, []).append(i)
    for page, rows in order.items():
        off = int(slot[rows[0]]) % 16
        held[page, :off + len(rows)] = True
        for w, (raw, x, top) in enumerate(((k, rot, 316.0), (v, v, 448.0))):
            for h in range(k.shape[1]):
                amax = np.abs(raw[rows, h]).max()
                ok = np.isfinite(amax)
                e = -60.0
                if ok and amax > 0:
                    m, ex = np.frexp(amax / top)          # amax / top = m 2^ex, 1/2 <= m < 1: exact, both are multiples of few bits
                    e = float(np.clip(ex - 1 if m == 0.5 else ex, -60, 40))
                    tie[page, h, w] = m == 0.5
                new = 2.0 ** e
                if off:
                    old = sc[page, h, w]
                    ok = ok and np.isfinite(old)
                    if ok:
                        new = max(new, old)
                        pools[w][page, h, :off] *= old / new
                sc[page, h, w] = new if ok else np.nan
                for i in rows:
                    o = int(slot[i]) % 16
                    pools[w][page, h, o] = x[i, h] / new if ok else 0.0
                    slack[w][page, h, o] = pair[i, h] * 2.0 ** -21 / new if w == 0 and ok else 0.0
    return pools, sc, slack, tie, held


def check_write(state, tabs, before, k, v):
    k8, v8, sc = state
    pools, want_sc, slack, tie, held = write64(tabs, k.cpu().double().numpy(), v.cpu().double().numpy(), *before)
    got_sc = sc.cpu().double().numpy()
    same = (got_sc == want_sc) | (np.isnan(got_sc) & np.isnan(want_sc))
    assert (same | (tie & (got_sc == 2 * want_sc))).all()
    for w, p in enumerate((k8, v8)):
        got = p.cpu().view(torch.float8_e4m3fn).double().numpy()
        assert np.isfinite(got).all()
        lost = np.isnan(got_sc[..., w])
        factor = np.where(lost, 1.0, got_sc[..., w] / np.where(lost, 1.0, want_sc[..., w]))[..., None, None]   # a tie resolved upwards
        ref = pools[w] / np.where(held[:, None, :, None], factor, 1.0)   # (slots behind the tokens stay as they were)
        tol = np.maximum(np.abs(ref) * 2.0 ** -4, 2.0 ** -10) + slack[w]
        err = np.abs(got - np.clip(ref, -448, 448))
        err[lost] = 0.0
        assert (err <= tol).all(), (w, float((err / tol).max()))


def _write_case(requests, hq, hkv, d, seed, scale_of=lambda n: 1.0, max_rows=None, spoil=None, k_rot=True):
    B, runtime = _mods()
    batch = _batch_of(requests, seed)
    step = runtime.StepOnDevice(batch, hq // hkv, blocks=False, max_rows=max_rows)
    step.build()
    n = step.tables.max_rows
    live = int(batch.node_new.sum())
    g = torch.Generator(device="cuda").manual_seed(seed)
    q, k, v = (torch.randn(n, h, d, generator=g, device="cuda") for h in (hq, hkv, hkv))
    mult = torch.tensor([scale_of(i) for i in range(n)], device="cuda")[:, None, None]
    q, k, v = q.bfloat16(), (k * mult).bfloat16(), (v * mult).bfloat16()
    if spoil:
        spoil(k, v)
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, seed, spread=2)
    before = [x.clone() for x in (k8, v8, sc)]
    geom = B.make_geom(hq, hkv, d, batch.num_pages, "bf16")
    q_rot = torch.full_like(q, 5.0)
    k_out = torch.full_like(k, 5.0) if k_rot else None
    B.mv_rope_write_kv_fp8_blk(step.tables, geom, q, k, v, q_rot, k_out, k8, v8, sc)
    assert step.read_status() == 0
    want = O.plan_tables(batch_dict(batch))
    tabs = (want["pos_id"], want["slot"])
    check_write((k8, v8, sc), tabs, before, k[:live], v[:live])
    for got, x in ((q_rot, q), (k_out, k)):
        if got is None:
            continue
        assert (got[live:] == 5.0).all()
        raw = x[:live].cpu().double().numpy()
        ref = O.rope_rotate(raw, tabs[0])
        pair = np.sqrt(raw[..., :d // 2] ** 2 + raw[..., d // 2:] ** 2)
        tol = np.abs(ref) * 2.0 ** -8 + np.concatenate([pair, pair], -1) * 2.0 ** -21
        ok = np.isfinite(ref)
        assert (np.abs(got[:live].cpu().double().numpy() - ref) <= tol)[ok].all()
    # writing the same step again changes nothing: the blocks already have their scales
    again = [x.clone() for x in (k8, v8, sc)]
    B.mv_rope_write_kv_fp8_blk(step.tables, geom, None, k, v, None, None, k8, v8, sc)
    for x, y in zip(again, (k8, v8, sc)):
        assert torch.equal(torch.nan_to_num(x), torch.nan_to_num(y)) if x.is_floating_point() else torch.equal(x, y)
    return k8, v8, sc, before, tabs


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64), (4, 4, 128), (24, 1, 64), (64, 8, 128)])
@pytest.mark.parametrize("new", [1, 5, 33])
def test_write_runs(hq, hkv, d, new):
    reqs = [[([], 3 + 7 * r, 0), ([0], r, new), ([0], 16 - r, 1), ([0], 15, new + r)] for r in range(5)]
    _write_case(reqs, hq, hkv, d, 11 * new + d, max_rows=sum(x[2] for r in reqs for x in r) + 6)


@pytest.mark.parametrize("d", [64, 128])
def test_write_scales_grow_and_shrink(d):
    # magnitudes from far below the smallest scale to far above the largest, tokens one by one into filled pages
    reqs = [[([], r % 16, 1)] for r in range(64)]
    _write_case(reqs, 4, 2, d, 5, scale_of=lambda i: 2.0 ** ((i * 37) % 140 - 80))
    _write_case(reqs, 4, 2, d, 6, scale_of=lambda i: 0.0)
    _write_case([[([], 0, 40), ([0], 0, 7)]], 4, 2, d, 7, scale_of=lambda i: 4.0 ** (i % 9 - 4))


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_write_non_finite(bad):
    def spoil(k, v):
        k[1, 0, 5] = bad
        v[2, 1, 100] = bad
    _, _, sc, _, tabs = _write_case([[([], 20, 3), ([0], 15, 3)]], 4, 2, 128, 9, spoil=spoil)
    page = lambda i: int(tabs[1][i]) // 16
    assert torch.isnan(sc[page(1), 0, 0]) and torch.isnan(sc[page(2), 1, 1])
    assert int(torch.isnan(sc).sum()) == 2


def test_write_prompt_of_many_chunks():
    _write_case([[([], 0, 2100), ([0], 0, 777), ([0], 0, 1), ([1, 2], 0, 15)]], 8, 2, 128, 13, max_rows=3000)
    _write_case([[([], 9, 2100), ([0], 7, 33)]], 4, 2, 64, 14)


def test_write_in_place():
    B, runtime = _mods()
    batch = _batch_of([[([], 9, 0), ([0], 5, 4)]])
    step = runtime.StepOnDevice(batch, 4, blocks=False)
    step.build()
    g = torch.Generator(device="cuda").manual_seed(1)
    q, k, v = (torch.randn(4, h, 128, generator=g, device="cuda").bfloat16() for h in (8, 2, 2))
    geom = B.make_geom(8, 2, 128, batch.num_pages, "bf16")
    res = []
    for alias in (False, True):
        k8, v8, sc = pools_of(batch.num_pages, 2, 128, 3)
        q1, k1 = q.clone(), k.clone()
        qr, kr = (q1, k1) if alias else (torch.empty_like(q), torch.empty_like(k))
        B.mv_rope_write_kv_fp8_blk(step.tables, geom, q1, k1, v, qr, kr, k8, v8, sc)
        res.append((qr, kr, k8, v8, sc))
    for x, y in zip(*res):
        assert torch.equal(x, y)


# ------------------------------------------------------------------------------------------------ attention

def _attend(batch, hq, hkv, d, seed, pools=None, q=None, max_rows=None, sm_scale=0.0, tokens=4096, group_tables=None, check=True):
    B, runtime = _mods()
    step = runtime.StepOnDevice(batch, hq // hkv, max_rows=max_rows)
    step.build()
    assert step.read_status() == 0
    geom = B.make_geom(hq, hkv, d, batch.num_pages, "bf16", sm_scale=sm_scale)
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, seed) if pools is None else pools
    n = step.tables.max_rows
    if q is None:
        q = torch.randn(n, hq, d, generator=torch.Generator(device="cuda").manual_seed(seed + 1), device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    ws = torch.full((B.mv_decode_fp8_blk_workspace_bytes(geom),), 255, dtype=torch.uint8, device="cuda")  # NaN, were it read unwritten
    B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, k8, v8, sc, out, ws)
    assert step.read_status() == 0
    live = int(batch.node_new.sum())
    assert (out[live:] == 7.0).all()
    if check:
        check_out(out, attend64(q, k8, v8, sc, step.t, hq // hkv, sm_scale or None), tokens)
    return out, step, (k8, v8, sc), q, geom, ws


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (8, 2, 64), (4, 4, 128), (3, 3, 64), (24, 1, 128), (40, 8, 128), (64, 1, 128), (64, 1, 64), (16, 2, 64)])
@pytest.mark.parametrize("seed,max_new", [(0, 1), (1, 1), (2, 9), (3, 40)])
def test_attention_random_dags(hq, hkv, d, seed, max_new):
    wl = _dag(seed, n_req=4, max_nodes=9, max_len=150, max_new=max_new, hq=hq, hkv=hkv, d=d)
    _attend(wl.batch, hq, hkv, d, seed, max_rows=int(wl.batch.node_new.sum()) + 2)


@pytest.mark.parametrize("vis", [0, 1])
def test_attention_other_visibility_and_scale(vis):
    wl = _dag(17, n_req=3, max_nodes=10, max_len=100, vis_mode=vis)
    _attend(wl.batch, 8, 2, 128, 17, sm_scale=0.31)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("length", [0, 1, 15, 16, 17, 127, 128, 129, 255, 1000])
def test_attention_one_row_of_any_length(d, length):
    _attend(_batch_of([[([], length, 1)]]), 4, 2, d, length)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_long_history_is_split(d):
    _attend(_batch_of([[([], 40000, 0), ([0], 333, 1), ([0], 1, 2)]]), 8, 2, d, 21, tokens=41000)


@pytest.mark.parametrize("hq,hkv,d", [(8, 2, 128), (64, 8, 128), (8, 2, 64)])
def test_attention_many_requests(hq, hkv, d):
    rng = np.random.default_rng(3)
    reqs = [[([], int(rng.integers(1, 400)), 0)] + [([0], int(rng.integers(0, 60)), 1) for _ in range(int(rng.integers(1, 9)))] for _ in range(150)]
    _attend(_batch_of(reqs), hq, hkv, d, 23)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("hq,hkv,requests,length,branches", [
    (4, 1, 1, 60000, 1),    # one stream in every share
    (2, 2, 1, 9000, 1),     # one q-vector per stream
    (40, 8, 60, 1900, 3),   # more cut q-vectors than warps that join them, an odd number in each stream
    (8, 8, 90, 700, 1),     # the same with one
    (7, 1, 3, 20000, 9),    # 63 q-vectors in each of few streams
])
def test_attention_joins_cut_streams(hq, hkv, requests, length, branches, d):
    reqs = [[([], length + 13 * r, 0)] + [([0], 5 * b, 1) for b in range(branches)] for r in range(requests)]
    _attend(_batch_of(reqs), hq, hkv, d, 25, tokens=length + 13 * requests + 64)


def test_attention_over_a_pool_without_pages():
    """No page id is valid then: every row gets zeros, and the bad entry is reported."""
    B, _ = _mods()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    t = {"pos_id": i32(0, 0), "slot": torch.full((2,), -1, dtype=torch.int64, device="cuda"), "counts": i32(2, 1, 1, 1, 0, 0, 0, 0),
         "group_row_off": i32(0, 2), "group_ent_off": i32(0, 1), "group_tile_off": i32(0, 1), "entries": i32(0, 16, 3, 0).view(1, 4)}
    tables = B.StepTables(**t, rows_per_group=16)
    geom = B.make_geom(8, 2, 128, 0, "bf16")
    k8, v8, sc = pools_of(1, 2, 128, 5)
    q = torch.randn(2, 8, 128, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    B.mv_dag_decode_attn_fp8_blk(tables, geom, q, k8, v8, sc, out, ws)
    assert B.mv_step_tables_read_status(tables) == 1 and (out == 0).all()


@pytest.mark.parametrize("d", [64, 128])
def test_attention_scales_differ_from_page_to_page(d):
    """Blocks whose scales lie up to 2^16 apart: scores decide through K, the numerator through V."""
    batch = _batch_of([[([], 700, 0), ([0], 40, 1), ([0], 90, 1)] for _ in range(3)])
    k8, v8, sc = pools_of(batch.num_pages, 2, d, 31, spread=8)
    sc[..., 0] = 2.0 ** -6          # scores of ordinary size ...
    _attend(batch, 8, 2, d, 31, pools=(k8, v8, sc))
    sc[::3, :, 0] = 2.0 ** -8       # ... and K scales that differ too
    sc[..., 1] = torch.where(torch.arange(batch.num_pages, device="cuda")[:, None] % 2 == 0, 2.0 ** 40, 2.0 ** -60)
    _attend(batch, 8, 2, d, 31, pools=(k8, v8, sc))
    sc[..., 1] = 2.0 ** -60
    _attend(batch, 8, 2, d, 31, pools=(k8, v8, sc))


def bound64(q, k8, v8, scale, t, group):
    """(row, out, bound) in float64, element by element, where one token may dominate a row and have values near zero itself: the
    second term of the weights' rounding then belongs to the row's largest weight, not to A.  With w_j = p_j * scale of V:
      2^-8 |out| (bf16) + (2^-8 + 2^-12) sum_j w_j |v_j|  +  2^-19 max_j w_j * sum_j |v_j|
      + what q's rounding (2^-17 of the group's largest element) moves the scores: ds_j = 2^-17 max |q| sum |K_j| * sm_scale,
        sum_j w_j |v_j| ds_j + (sum_j p_j ds_j) sum_j w_j |v_j|, and a tenth of it for the second order."""
    d, hkv = q.shape[2], k8.shape[1]
    ro, eo, ent, counts = (t[k].cpu() for k in ("group_row_off", "group_ent_off", "entries", "counts"))
    kd = k8.view(torch.float8_e4m3fn).double() * scale[:, :, 0].double()[:, :, None, None]
    vb, se = v8.view(torch.float8_e4m3fn).double(), scale[:, :, 1].double()
    for g in range(int(counts[1])):
        e = ent[int(eo[g]):int(eo[g + 1])].long()
        r0, r1 = int(ro[g]), int(ro[g + 1])
        qmax = q[r0:r1].double().abs().view(r1 - r0, hkv, group * d).amax((0, 2))
        for r in range(r0, r1):
            b = r - r0
            sel = e[((e[:, 2 + b // 32] >> (b % 32)) & 1) > 0]
            tok = (torch.arange(16) < sel[:, 1:2]).reshape(-1).nonzero()[:, 0].to(q.device)
            if tok.numel() == 0:
                continue
            page = sel[:, 0].to(q.device)
            kk, vv = (x[page].transpose(1, 2).reshape(-1, hkv, d)[tok] for x in (kd, vb))
            sv = se[page][:, None, :].expand(-1, 16, -1).reshape(-1, hkv)[tok]
            s = torch.einsum("hgd,nhd->hgn", q[r].double().view(hkv, group, d), kk) * d ** -0.5
            ds = torch.einsum("h,nh->hn", qmax * 2.0 ** -17, kk.abs().sum(2)) * d ** -0.5
            p = torch.softmax(s, -1)
            w = p * sv.t()[:, None, :]
            ref, a = torch.einsum("hgn,nhd->hgd", w, vv), torch.einsum("hgn,nhd->hgd", w, vv.abs())
            moved = torch.einsum("hgn,hn,nhd->hgd", w, ds, vv.abs()) + a * torch.einsum("hgn,hn->hg", p, ds)[..., None]
            tol = (2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12) * a + 1.1 * moved
                   + 2.0 ** -19 * w.amax(-1)[..., None] * vv.abs().sum(0)[:, None, :] + 1e-30)
            yield r, ref.reshape(-1, d), tol.reshape(-1, d)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("group,hkv", [(1, 4), (4, 2), (11, 5), (33, 2), (64, 3)])
@pytest.mark.parametrize("spread", ["2^8", "all"])
def test_attention_peaked_scores_over_spread_scales(d, group, hkv, spread):
    """Scores of a dozen units, V's scales up to 2^16 apart, or anywhere a scale may be."""
    seed = group * 2 + d
    wl = _dag(seed, n_req=5, max_nodes=8, max_len=200, max_new=3, hq=hkv * group, hkv=hkv, d=d)
    k8, v8, sc = pools_of(wl.batch.num_pages, hkv, d, seed, spread=8)
    sc[..., 0] = 2.0 ** -4
    if spread == "all":
        sc[..., 1] = torch.exp2(torch.randint(-60, 41, sc[..., 1].shape, generator=torch.Generator().manual_seed(seed)).float()).cuda()
    out, step, _, q, _, _ = _attend(wl.batch, hkv * group, hkv, d, seed, pools=(k8, v8, sc), check=False)
    for r, ref, tol in bound64(q, k8, v8, sc, step.t, group):
        over = (out[r].double() - ref).abs() > tol
        assert not over.any(), (r, over.nonzero()[:4].tolist())


@pytest.mark.parametrize("d", [64, 128])
def test_attention_large_scores_and_one_heavy_token(d):
    """A token whose weight is far above a long tail that together weighs as much, and scores that grow along the history
    (the running reference moves again and again)."""
    n = 3000
    batch = _batch_of([[([], n, 1)]])
    step_q = torch.zeros(1, 4, d, device="cuda").bfloat16()
    step_q[..., 0] = 1.0
    k8, v8, sc = pools_of(batch.num_pages, 2, d, 41)
    sc[..., 0] = 1.0
    pages = torch.from_numpy(batch.page_idx[:(n + 16) // 16].astype(np.int64)).cuda()

    def keys(col0):
        k = torch.zeros(batch.num_pages, 2, 16, d, device="cuda")
        flat = torch.zeros(pages.numel() * 16, device="cuda")
        flat[:n + 1] = col0
        k[pages, :, :, 0] = flat.view(-1, 1, 16).expand(-1, 2, -1)
        return k.to(torch.float8_e4m3fn).view(torch.uint8).contiguous()

    sink = torch.zeros(n + 1, device="cuda")
    sink[7] = 8.0                                        # e^8 = 2981: as much as the other 3000 tokens together
    _attend(batch, 4, 2, d, 41, pools=(keys(sink), v8, sc), q=step_q, sm_scale=1.0)
    _attend(batch, 4, 2, d, 41, pools=(keys(sink.flip(0)), v8, sc), q=step_q, sm_scale=1.0)
    ramp = torch.linspace(-30, 60, n + 1, device="cuda")
    _attend(batch, 4, 2, d, 41, pools=(keys(ramp), v8, sc), q=step_q, sm_scale=2.0)
    _attend(batch, 4, 2, d, 41, pools=(keys(-ramp), v8, sc), q=step_q, sm_scale=2.0)


@pytest.mark.parametrize("d", [64, 128])
def test_attention_ignores_what_lies_behind_the_tokens(d):
    """Unused slots of a page hold NaN bytes, unused pages NaN scales."""
    batch = _batch_of([[([], 21, 0), ([0], 3, 1), ([0], 30, 2)], [([], 130, 1)]])
    k8, v8, sc = pools_of(batch.num_pages, 2, d, 51)
    used = torch.zeros(batch.num_pages, 16, dtype=torch.bool)
    for node in range(batch.n_nodes):
        n = int(batch.node_len[node] + batch.node_new[node])
        for p in range((n + 15) // 16):
            used[int(batch.page_idx[batch.page_off[node] + p]), :min(16, n - 16 * p)] = True
    hole = (~used).cuda()[:, None, :, None].expand_as(k8)
    clean, *_ = _attend(batch, 8, 2, d, 51, pools=(k8, v8, sc))
    k8[hole], v8[hole] = 0x7F, 0xFF
    sc[~used.any(1).cuda()] = float("nan")
    dirty, *_ = _attend(batch, 8, 2, d, 51, pools=(k8, v8, sc), check=False)
    assert torch.equal(clean, dirty)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("which", [0, 1])
def test_attention_lost_block_reaches_only_rows_that_see_it(d, which):
    batch = _batch_of([[([], 64, 0), ([0], 20, 1), ([0], 30, 1), ([0], 140, 1)], [([], 30, 1)]])
    clean, step, (k8, v8, sc), q, geom, ws = _attend(batch, 8, 2, d, 61)
    page = int(batch.page_idx[batch.page_off[2]])          # a page of the second branch
    sc[page, 1, which] = float("nan")
    B, _ = _mods()
    out = torch.empty_like(clean)
    B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, k8, v8, sc, out, ws)
    lost = torch.zeros_like(out, dtype=torch.bool)
    lost[1, 4:] = True                                     # its row, the query heads of KV head 1
    assert torch.isnan(out[lost]).all() and torch.equal(out[~lost], clean[~lost])


@pytest.mark.parametrize("d", [64, 128])
def test_attention_tables_of_the_callers_own(d):
    """A row that no entry names and a group without entries get zeros; a page may stand in several groups."""
    B, _ = _mods()
    i32 = lambda *x: torch.tensor(x, dtype=torch.int32, device="cuda")
    t = {"pos_id": i32(*[0] * 7), "slot": torch.full((7,), -1, dtype=torch.int64, device="cuda"), "counts": i32(6, 3, 3, 2, 0, 0, 0, 0),
         "group_row_off": i32(0, 3, 5, 6, 6), "group_ent_off": i32(0, 2, 2, 3, 3), "group_tile_off": i32(0, 1, 1, 2, 2),
         "entries": torch.tensor([[4, 16, 0b001, 0], [2, 5, 0b101, 0], [4, 9, 1, 0], [9, 9, 9, 9]], dtype=torch.int32, device="cuda")}
    tables = B.StepTables(**t, rows_per_group=16)
    k8, v8, sc = pools_of(6, 2, d, 71)
    q = torch.randn(7, 8, d, device="cuda").bfloat16()
    out = torch.full_like(q, 7.0)
    geom = B.make_geom(8, 2, d, 6, "bf16")
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    B.mv_dag_decode_attn_fp8_blk(tables, geom, q, k8, v8, sc, out, ws)
    assert B.mv_step_tables_read_status(tables) == 0
    assert (out[1] == 0).all() and (out[3:5] == 0).all() and (out[6] == 7.0).all()
    check_out(out, attend64(q, k8, v8, sc, t, 4))
    # a page id outside the pool is skipped and reported
    t["entries"][1, 0] = 6
    B.mv_dag_decode_attn_fp8_blk(tables, geom, q, k8, v8, sc, out, ws)
    assert B.mv_step_tables_read_status(tables) == 1


# ------------------------------------------------------------------------------------------------ a run of them together

def _same_as_definition(wl, state):
    B, _ = _mods()
    t = state.steps.t
    check_out(state.out, attend64(state.q_rot, state.k_pages, state.v_pages, state.kv_scale, t, wl.geom.group))


@pytest.mark.parametrize("hq,hkv,d", [(32, 8, 128), (8, 2, 64)])
def test_step_against_the_oracle(hq, hkv, d):
    """Build, write and attend on a workload whose history went in through the same calls: against the oracle on raw
    values, within what an 8-bit cache does (half a step, 2^-4, per element of K and V), and against the definition on the cache itself."""
    _, runtime = _mods()
    wl = synth.random_dag_workload(5, "decode", n_req=3, max_nodes=9, max_len=150, geom=synth.Geometry(hq, hkv, d, 16, "bf16", value_scale=0.5))
    st = runtime.DecodeStateFP8Blk(wl)
    got = st.step()
    assert st.steps.read_status() == 0
    check_tables(st.steps, wl.batch)
    _same_as_definition(wl, st)
    row = 0
    for r in range(wl.batch.n_req):
        vals = synth.request_values(wl, r)
        want = O.decode_request(batch_dict(wl.batch), r, vals["q"], vals["k"], vals["v"])
        g = got[row:row + want.shape[0]].double().cpu().numpy()
        row += want.shape[0]
        assert np.linalg.norm(g - want) <= 2.0 ** -4 * np.linalg.norm(want)


def test_generation_loop_with_the_scheduler():
    """The frontier scheduler drives the calls through forks and joins; after every step the output is the attention over the cache as
    it stands, and every token of the cache is the quantised rotation of what was given for it."""
    B, runtime = _mods()
    hq, hkv, d, pages = 8, 2, 128, 64
    sched = B.Scheduler(16, pages)
    sched.add_request([[], [0], [0], [1, 2]], [37, 5, 3, 4])
    sched.add_request([[], [0], [1]], [16, 18, 2])
    geom = B.make_geom(hq, hkv, d, pages, "bf16")
    k8, v8, sc = (torch.zeros(pages, hkv, 16, d, dtype=torch.uint8, device="cuda"), torch.zeros(pages, hkv, 16, d, dtype=torch.uint8, device="cuda"),
                  torch.zeros(pages, hkv, 2, device="cuda"))
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    g = torch.Generator(device="cuda").manual_seed(0)
    written = {}
    steps = 0
    while True:
        s = sched.step()
        if s is None:
            break
        batch = synth.DagBatch(s["n_req"], *(s[k] for k in ("node_off", "node_len", "node_new", "parent_off", "parent_idx", "page_off", "page_idx")),
                               16, pages)
        if steps == 0:   # the roots' tokens, once
            roots = np.asarray([1 if s["parent_off"][v + 1] == s["parent_off"][v] else 0 for v in range(batch.n_nodes)])
            hist = synth.DagBatch(batch.n_req, batch.node_off, np.zeros_like(batch.node_len), batch.node_len * roots, batch.parent_off, batch.parent_idx,
                                  batch.page_off, batch.page_idx, 16, pages)
            hs = runtime.StepOnDevice(hist, hq // hkv, blocks=False)
            n = hs.tables.max_rows
            k, v = (torch.randn(n, hkv, d, generator=g, device="cuda").bfloat16() for _ in range(2))
            B.mv_rope_write_kv_fp8_blk(hs.build(), geom, None, k, v, None, None, k8, v8, sc)
            for i, sl in enumerate(hs.t["slot"].tolist()):
                written[sl] = (int(hs.t["pos_id"][i]), k[i], v[i])
        step = runtime.StepOnDevice(batch, hq // hkv)
        t = step.build()
        n = t.max_rows
        q, k, v = (torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
        q_rot, out = torch.empty_like(q), torch.empty_like(q)
        B.mv_rope_write_kv_fp8_blk(t, geom, q, k, v, q_rot, None, k8, v8, sc)
        B.mv_dag_decode_attn_fp8_blk(t, geom, q_rot, k8, v8, sc, out, ws)
        assert step.read_status() == 0
        check_tables(step, batch)
        check_out(out, attend64(q_rot, k8, v8, sc, step.t, hq // hkv))
        for i, sl in enumerate(step.t["slot"].tolist()):
            if sl % 16 == 0:   # a page that a finished request gave back starts afresh
                written = {x: y for x, y in written.items() if x // 16 != sl // 16}
            written[sl] = (int(step.t["pos_id"][i]), k[i], v[i])
        sched.commit()
        steps += 1
    assert steps >= 9
    for sl, (pos, k, v) in written.items():
        want = O.rope_rotate(k[None].cpu().double().numpy(), [pos])[0]
        got = k8[sl // 16, :, sl % 16].view(torch.float8_e4m3fn).double().cpu().numpy() * sc[sl // 16, :, 0].double().cpu().numpy()[:, None]
        # once rounded, and among the subnormals of a scale that grew later once more
        assert (np.abs(got - want) <= np.abs(want) * 2.0 ** -4 + 2.0 ** -9 * sc[sl // 16, :, 0].double().cpu().numpy()[:, None] + 1e-6).all()


def test_captured_step_follows_lengths_on_the_device():
    """One graph holds the whole step; its replays, with node_len advanced on the device, equal eager steps on a second cache.
    New pages of a node are listed beforehand."""
    B, runtime = _mods()
    hq, hkv, d = 16, 4, 128
    lens, room = [90, 13, 16, 31], 40
    reqs = [[([], lens[0] + r, 0)] + [([0], n + r, 1) for n in lens[1:]] for r in range(3)]
    batch = _batch_of([[(p, n + (room if w else 0), w) for p, n, w in r] for r in reqs])     # pages for what is to come
    batch.node_len = np.asarray([n for r in reqs for _, n, _ in r], np.int32)
    geom = B.make_geom(hq, hkv, d, batch.num_pages, "bf16")
    rows = int(batch.node_new.sum())
    sides = []
    for _ in range(2):
        k8, v8, sc = pools_of(batch.num_pages, hkv, d, 81)
        step = runtime.StepOnDevice(batch, hq // hkv, max_rows=rows + 1, max_entries=600)
        ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
        q = torch.zeros(rows + 1, hq, d, device="cuda").bfloat16()
        k, v = (torch.zeros(rows + 1, hkv, d, device="cuda").bfloat16() for _ in range(2))
        sides.append(dict(pools=(k8, v8, sc), step=step, ws=ws, q=q, k=k, v=v, q_rot=torch.zeros_like(q), out=torch.zeros_like(q)))

    def one(s):
        t = s["step"].build()
        B.mv_rope_write_kv_fp8_blk(t, geom, s["q"], s["k"], s["v"], s["q_rot"], None, *s["pools"])
        B.mv_dag_decode_attn_fp8_blk(t, geom, s["q_rot"], *s["pools"], s["out"], s["ws"])
        s["step"].arrays["node_len"] += s["step"].arrays["node_new"]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    one(sides[0])                                   # a set-up call, undone below
    torch.cuda.synchronize()
    sides[0]["step"].arrays["node_len"] -= sides[0]["step"].arrays["node_new"]
    for x, y in zip(sides[0]["pools"], sides[1]["pools"]):
        x.copy_(y)
    with torch.cuda.graph(graph, stream=side):
        one(sides[0])
    g = torch.Generator(device="cuda").manual_seed(4)
    for i in range(room):
        for name in ("q", "k", "v"):
            x = torch.randn(sides[0][name].shape, generator=g, device="cuda").bfloat16()
            sides[0][name].copy_(x)
            sides[1][name].copy_(x)
        graph.replay()
        one(sides[1])
        assert sides[0]["step"].read_status() == 0
        for x, y in zip(sides[0]["pools"], sides[1]["pools"]):
            assert torch.equal(x, y), i
        assert torch.equal(sides[0]["out"], sides[1]["out"]), i
        if i % 13 == 0:
            s = sides[0]
            check_out(s["out"], attend64(s["q_rot"], *s["pools"], s["step"].t, hq // hkv))
    # one step further the pages end: the step reports it and is empty
    before = [x.clone() for x in sides[0]["pools"]]
    for _ in range(18):
        graph.replay()
    assert sides[0]["step"].read_status() == 3
    del graph


def test_streams_and_repeatability():
    """The same call on another stream and again: the same bits; two calls on two streams with their own workspaces."""
    B, _ = _mods()
    rng = np.random.default_rng(9)
    reqs = [[([], int(rng.integers(200, 3000)), 0)] + [([0], int(rng.integers(0, 60)), 1) for _ in range(4)] for _ in range(20)]
    batch = _batch_of(reqs)
    for d in (64, 128):
        out, step, pools, q, geom, ws = _attend(batch, 16, 2, d, 91)
        outs = [torch.zeros_like(q) for _ in range(6)]
        wss = [ws.clone() for _ in range(2)]
        streams = [torch.cuda.Stream() for _ in range(2)]
        torch.cuda.synchronize()
        for i, o in enumerate(outs):
            B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, *pools, o, wss[i % 2], streams[i % 2].cuda_stream)
        torch.cuda.synchronize()
        for o in outs:
            assert torch.equal(o, out)


def test_binding_refuses_what_the_kernels_would_misread():
    B, runtime = _mods()
    batch = _batch_of([[([], 9, 1)]])
    step = runtime.StepOnDevice(batch, 4)
    geom = B.make_geom(8, 2, 128, batch.num_pages, "bf16")
    k8, v8, sc = pools_of(batch.num_pages, 2, 128, 1)
    q = torch.zeros(1, 8, 128, device="cuda").bfloat16()
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    call = lambda **kw: B.mv_dag_decode_attn_fp8_blk(step.tables, geom, *({"q": q, "k": k8, "v": v8, "s": sc, "o": q.clone(), "w": ws} | kw).values())
    call()
    wide = torch.zeros(1, 16, 128, device="cuda").bfloat16()
    for kw in ({"q": q.float()}, {"q": wide[:, ::2]}, {"q": q.cpu()}, {"k": k8[:-1]}, {"s": sc.double()}, {"o": None}):
        with pytest.raises(ValueError):
            call(**kw)
    with pytest.raises(B.MvError) as e:
        call(w=ws[:-256])
    assert e.value.status == 5
