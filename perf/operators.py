"""Workloads of the device-planned, block-scaled 8-bit decode path: what each call gets, its plain form and its definition.

Three operators that follow one another in a decode step whose lengths live on the GPU:

``tables``   batch description on the device -> positions, slots and the block table of every group of rows
``write``    rotary embedding of q and k, K and V stored in 8 bits with a power-of-two scale per (page, KV head)
``attn``     attention of every row over the pages its block table names

A batch is a set of request DAGs: a shared prefix, layers of branches, sometimes a join; the last layer (or the join)
receives the step's new tokens.  ``run`` computes a pass with elementary torch operations, or with the library's calls
where ``own`` is true.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
E_MIN, E_MAX = -60, 40      # range of the scale exponents
K_TOP, V_TOP = 316.0, 448.0  # largest raw magnitude a block of scale 1 takes (316 * sqrt 2 < 448, the format's largest value)


# ---------------------------------------------------------------------------------------------------- cases

def _case(name, op, heads, n_req, prefix, branches, blen, layers=1, join=0.0, new=1, prefill=False, layout=1, vis=0, pos=0):
    c = {"op": op, "hq": heads[0], "hkv": heads[1], "d": heads[2], "n_req": n_req, "prefix_lo": prefix[0], "prefix_hi": prefix[1],
         "branches_lo": branches[0], "branches_hi": branches[1], "blen_lo": blen[0], "blen_hi": blen[1], "layers": layers, "join": join,
         "new": new, "prefill": prefill, "layout": layout, "vis": vis, "pos": pos}
    return c if name is None else {"name": name, **c}


def listed():
    small, large, half = (32, 8, 128), (64, 8, 128), (8, 2, 64)
    return [
        # the step's tables of a single short request (four branches behind a prompt): pure latency
        _case("tables of one request", "tables", small, 1, (384, 384), (4, 4), (70, 70)),
        # of a full serving batch: prompts of mixed lengths, 2 to 8 branches, a quarter of them at a join
        _case("tables of a serving batch", "tables", large, 128, (512, 16384), (2, 8), (64, 1024), join=0.25, layout=2),
        # of many long requests in layered DAGs, the longest list of pages
        _case("tables of 512 layered requests", "tables", small, 512, (512, 16384), (1, 6), (64, 512), layers=3, layout=3),
        # the cache write of one decode step of a small batch: one token per branch, pages already partly filled
        _case("write of a decode step", "write", small, 16, (512, 2048), (4, 4), (64, 512), layout=4),
        # a prompt with its whole reasoning DAG written at once, about 16 thousand tokens
        _case("write of a DAG prompt", "write", small, 1, (4096, 4096), (6, 6), (256, 768), layers=4, prefill=True, layout=5),
        # runs of five new tokens per branch (accepted drafts, text after a join) with 64-element heads
        _case("write of short runs, head 64", "write", half, 37, (1, 700), (1, 5), (1, 333), new=5, layout=6),
        # a short request alone: what a single user's step costs
        _case("attention of one request", "attn", small, 1, (384, 384), (4, 4), (70, 70), layout=7),
        # 16 requests with four branches each over a 2048-token prompt
        _case("attention of 16 requests", "attn", small, 16, (2048, 2048), (4, 4), (64, 512), layout=8),
        # 32 layered DAGs over 4096-token prompts
        _case("attention of 32 layered requests", "attn", small, 32, (4096, 4096), (1, 6), (64, 512), layers=3, layout=9),
        # the serving batch with groups of eight query heads: the largest
        _case("attention of a serving batch", "attn", large, 128, (512, 16384), (2, 8), (64, 1024), join=0.25, layout=10),
        # one very long history with two branches: the work has to be split along the keys
        _case("attention of a long request", "attn", small, 1, (65536, 65536), (2, 2), (129, 1000), layout=11),
        # 64-element heads, odd lengths, a few tokens at once per branch
        _case("attention of short runs, head 64", "attn", half, 37, (1, 700), (1, 5), (1, 333), new=3, layout=12),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["tables", "write", "attn", "attn"])
    heads = rng.choice([(32, 8, 128), (64, 8, 128), (40, 8, 128), (16, 16, 128), (24, 1, 128), (8, 2, 64), (32, 8, 64), (4, 1, 64)])
    lo = log(1, 16384)
    hi = log(lo, 16384) if lo < 16384 else lo
    blo = log(1, 1024)
    bhi = log(blo, 1024) if blo < 1024 else blo
    branches = rng.randint(1, 8)
    layers = rng.choice([1, 1, 2, 3, 4])
    most = {"tables": 512, "write": 128, "attn": 128}[op]
    tokens = hi + branches * bhi * layers
    n_req = max(1, min(log(1, most), int((600_000 if op != "tables" else 3_000_000) / tokens)))
    prefill = op == "write" and rng.random() < 0.4
    if prefill:
        n_req = max(1, min(n_req, 16_000 // tokens))
        hi, lo = min(hi, 8192), min(lo, 8192)
        bhi, blo = min(bhi, 256), min(blo, 256)
    return _case(None, op, heads, n_req, (lo, hi), (rng.randint(1, branches), branches), (blo, bhi), layers, rng.choice([0.0, 0.25, 1.0]),
                 rng.choice([1, 1, 1, 2, 5, 17]), prefill, rng.randint(1, 1 << 30), rng.choice([0, 0, 0, 1]), rng.choice([0, 0, 0, 1]))


def _requests(case):
    """The DAGs of a case: per request a list of (parents, tokens held, new tokens)."""
    r = np.random.default_rng(case["layout"])

    def log(lo, hi):
        return int(round(math.exp(r.uniform(math.log(lo), math.log(hi))))) if hi > lo else lo

    out = []
    for _ in range(case["n_req"]):
        nodes, prev = [([], log(case["prefix_lo"], case["prefix_hi"]))], [0]
        for layer in range(case["layers"]):
            cur = []
            for _ in range(int(r.integers(case["branches_lo"], case["branches_hi"] + 1))):
                parents = [0] if layer == 0 else sorted(int(prev[i]) for i in r.permutation(len(prev))[:int(r.integers(1, 3))])
                cur.append(len(nodes))
                nodes.append((parents, int(r.integers(case["blen_lo"], case["blen_hi"] + 1))))
            prev = cur
        if r.random() < case["join"]:
            nodes.append((list(prev), int(r.integers(0, case["blen_hi"] + 1))))
            prev = [len(nodes) - 1]
        if case["prefill"]:
            out.append([(p, 0, n) for p, n in nodes])
        else:
            out.append([(p, n, int(r.integers(1, case["new"] + 1)) if v in prev else 0) for v, (p, n) in enumerate(nodes)])
    return out


def _batch(case, seed):
    """Host arrays of the batch; the pages are dealt out from a shuffled pool."""
    node_off, length, new, parent_off, parent_idx, page_off = [0], [], [], [0], [], [0]
    for req in _requests(case):
        for parents, ln, nw in req:
            length.append(ln)
            new.append(nw)
            parent_idx.extend(parents)
            parent_off.append(len(parent_idx))
            page_off.append(page_off[-1] + (ln + nw + PAGE - 1) // PAGE)
        node_off.append(len(length))
    num_pages = page_off[-1] + page_off[-1] // 8 + 1
    page_idx = np.random.default_rng([seed, 77]).permutation(num_pages)[:page_off[-1]]
    b = {"node_off": node_off, "node_len": length, "node_new": new, "parent_off": parent_off, "parent_idx": parent_idx or [0],
         "page_off": page_off, "page_idx": page_idx}
    b = {k: np.asarray(v, np.int32) for k, v in b.items()}
    return b, num_pages


def _host_tables(case, b, blocks=True):
    """The step's tables by their definition, node by node.  Without ``blocks`` only positions and slots."""
    per = max(1, 64 // (case["hq"] // case["hkv"]))
    pos_id, slot, group_rows, group_ents, group_tiles, entries = [], [], [0], [0], [0], []
    for r in range(case["n_req"]):
        lo, hi = int(b["node_off"][r]), int(b["node_off"][r + 1])
        n = hi - lo
        ln, nw = b["node_len"][lo:hi].astype(np.int64), b["node_new"][lo:hi].astype(np.int64)
        parents = [[int(p) for p in b["parent_idx"][b["parent_off"][g]:b["parent_off"][g + 1]]] for g in range(lo, hi)]
        layer, sees = [], []
        for v in range(n):
            layer.append(1 + max(layer[p] for p in parents[v]) if parents[v] else 0)
            sees.append({v}.union(*[sees[p] for p in parents[v]]))
        if case["vis"] == 1:
            sees = [{v} | {u for u in range(n) if layer[u] < layer[v]} for v in range(n)]
        start, end = [0] * n, [0] * n
        if case["pos"] == 0:
            for v in range(n):
                start[v] = max([end[p] for p in parents[v]], default=0)
                end[v] = start[v] + int(ln[v] + nw[v])
        else:
            before = 0
            for k in range(max(layer) + 1):
                at = [v for v in range(n) if layer[v] == k]
                for v in at:
                    start[v], end[v] = before, before + int(ln[v] + nw[v])
                before = max(end[v] for v in at)
        rows = []
        for v in range(n):
            pages = b["page_idx"][b["page_off"][lo + v]:b["page_off"][lo + v + 1]].astype(np.int64)
            t = np.arange(ln[v], ln[v] + nw[v])
            pos_id.append(start[v] + t)
            slot.append(pages[t // PAGE] * PAGE + t % PAGE)
            rows += [(v, j) for j in range(int(nw[v]))]
        for r0 in range(0, len(rows) if blocks else 0, per):
            group = rows[r0:r0 + per]
            found = 0
            for u in range(n):
                tot = int(ln[u] + nw[u])
                bits = [(i, v, j) for i, (v, j) in enumerate(group) if u in sees[v]]
                if not bits or not tot:
                    continue
                p = np.arange((tot + PAGE - 1) // PAGE)
                full = np.minimum(PAGE, tot - PAGE * p)
                cnt = np.stack([np.clip(int(ln[u]) + j + 1 - PAGE * p, 0, PAGE) if v == u else full for _, v, j in bits], 1)
                bit = np.array([1 << i for i, _, _ in bits], np.uint64)
                mine = []
                for c in range(1, PAGE + 1):
                    mask = np.where(cnt == c, bit, np.uint64(0)).sum(1, dtype=np.uint64)
                    at = np.flatnonzero(mask)
                    low = (mask[at] & np.uint64(0xffffffff)).astype(np.uint32).view(np.int32)
                    high = (mask[at] >> np.uint64(32)).astype(np.uint32).view(np.int32)
                    mine.append(np.stack([at, np.full(len(at), c), low, high], 1).astype(np.int64))
                e = np.concatenate(mine)
                e = e[np.lexsort((e[:, 1], e[:, 0]))]
                e[:, 0] = b["page_idx"][b["page_off"][lo + u] + e[:, 0]]
                entries.append(e)
                found += len(e)
            group_rows.append(group_rows[-1] + len(group))
            group_ents.append(group_ents[-1] + found)
            group_tiles.append(group_tiles[-1] + (found + 7) // 8)
    pos_id, slot = np.concatenate(pos_id), np.concatenate(slot)
    return {"pos_id": pos_id, "slot": slot, "group_row_off": group_rows, "group_ent_off": group_ents, "group_tile_off": group_tiles,
            "entries": np.concatenate(entries) if entries else np.zeros((0, 4), np.int64)}


def _sizes(t):
    """Capacities a caller would set aside: a little more than this step needs."""
    return {"rows": len(t["pos_id"]) + 5, "groups": len(t["group_row_off"]) - 1 + 3, "entries": len(t["entries"]) + 9}


def _padded_tables(t):
    """The tables as the arrays of those capacities hold them: unused rows have slot -1, unused groups are empty."""
    z = _sizes(t)

    def fill(x, n, value, dtype):
        x = np.asarray(x, np.int64)
        return np.concatenate([x, np.full((n - len(x),) + x.shape[1:], value, np.int64)]).astype(dtype)

    out = {"pos_id": fill(t["pos_id"], z["rows"], 0, np.int32), "slot": fill(t["slot"], z["rows"], -1, np.int64)}
    for k in ("group_row_off", "group_ent_off", "group_tile_off"):
        out[k] = fill(t[k], z["groups"] + 1, t[k][-1], np.int32)
    out["entries"] = fill(t["entries"], z["entries"], 0, np.int32)
    out["counts"] = np.array([len(t["pos_id"]), len(t["group_row_off"]) - 1, len(t["entries"]), t["group_tile_off"][-1], 0, 0, 0, 0], np.int32)
    return out


# ---------------------------------------------------------------------------------------------------- inputs

def _normal(shape, seed, what, dtype=torch.bfloat16):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed * 1009 + what)
    return torch.randn(shape, generator=g, device="cuda", dtype=dtype)


def _scale_of(amax, top):
    """Smallest power of two, inside the range of the format's scales, at which ``amax`` is at most ``top``."""
    e = torch.ceil(torch.log2(amax.double() / top)).clamp(E_MIN, E_MAX)  # amax = 0: the lowest
    s = torch.exp2(e).float()
    return torch.where(torch.isfinite(amax), s, torch.full_like(s, math.nan))


def _pools(case, num_pages, seed):
    """A cache that earlier steps have filled: every block at the scale its values need."""
    k8, v8, sc = [], [], torch.empty(num_pages, case["hkv"], 2, device="cuda")
    step = max(1, (1 << 26) // (case["hkv"] * PAGE * case["d"]))
    for lo in range(0, num_pages, step):
        hi = min(num_pages, lo + step)
        for which, (pool, top) in enumerate(((k8, K_TOP), (v8, V_TOP))):
            x = _normal((hi - lo, case["hkv"], PAGE, case["d"]), seed, 100 + 2 * lo + which, torch.float32)
            s = _scale_of(x.abs().amax((2, 3)), top)
            sc[lo:hi, :, which] = s
            pool.append((x / s[:, :, None, None]).to(torch.float8_e4m3fn).view(torch.uint8))
    return torch.cat(k8), torch.cat(v8), sc


def prepare(case, seed):
    b, num_pages = _batch(case, seed)
    t = _host_tables(case, b, blocks=case["op"] != "write")
    z = _sizes(t)
    s = {"case": case, "num_pages": num_pages, "per": max(1, 64 // (case["hq"] // case["hkv"])), "z": z}
    if case["op"] == "tables":
        s["batch"] = {k: torch.from_numpy(v).cuda() for k, v in b.items()}
        s["most_nodes"] = int(np.diff(b["node_off"]).max())
        s["tables"] = {"pos_id": torch.zeros(z["rows"], dtype=torch.int32, device="cuda"),
                       "slot": torch.zeros(z["rows"], dtype=torch.int64, device="cuda"),
                       **{k: torch.zeros(z["groups"] + 1, dtype=torch.int32, device="cuda") for k in ("group_row_off", "group_ent_off", "group_tile_off")},
                       "entries": torch.zeros(z["entries"], 4, dtype=torch.int32, device="cuda"),
                       "counts": torch.zeros(8, dtype=torch.int32, device="cuda")}
    else:
        s["tables"] = {k: torch.from_numpy(v).cuda() for k, v in _padded_tables(t).items()}
        s["k_pages"], s["v_pages"], s["scale"] = _pools(case, num_pages, seed)
        rows = z["rows"]
        s["q"] = _normal((rows, case["hq"], case["d"]), seed, 1)
        if case["op"] == "write":
            s["k"], s["v"] = (_normal((rows, case["hkv"], case["d"]), seed, 2 + i) for i in range(2))
            s["q_rot"], s["k_rot"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        else:
            s["out"] = torch.zeros_like(s["q"])
    if own:  # the handles a program keeps beside its arrays, and its workspace
        from paper_2602_07529_b200 import binding as B
        s["B"] = B
        s["h_tables"] = B.StepTables(**s["tables"], rows_per_group=s["per"])
        if case["op"] == "tables":
            s["h_batch"] = B.DeviceBatch(case["n_req"], **s["batch"], num_pages=num_pages, max_req_nodes=s["most_nodes"], vis_mode=case["vis"],
                                         pos_mode=case["pos"])
            s["workspace"] = torch.empty(B.mv_step_tables_workspace_bytes(s["h_batch"]), dtype=torch.uint8, device="cuda")
        else:
            s["geom"] = B.make_geom(case["hq"], case["hkv"], case["d"], num_pages, "bf16")
            if case["op"] == "attn":
                s["workspace"] = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(s["geom"]), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------- the passes

def run(s):
    return {"tables": _tables, "write": _write, "attn": _attn}[s["case"]["op"]](s)


def _tables(s):
    if own:
        s["B"].mv_step_tables_build(s["h_batch"], s["h_tables"], s["workspace"])
        return s["tables"]
    case, b, per, z = s["case"], {k: v.long() for k, v in s["batch"].items()}, s["per"], s["z"]
    dev = b["node_off"].device
    off, n_req, n = b["node_off"], case["n_req"], s["most_nodes"]
    nodes = b["node_len"].numel()
    local = torch.arange(n, device=dev)
    have = off[:-1, None] + local < off[1:, None]
    at = (off[:-1, None] + local).clamp(max=nodes - 1)
    ln, nw = torch.where(have, b["node_len"][at], 0), torch.where(have, b["node_new"][at], 0)
    req = torch.bucketize(torch.arange(nodes, device=dev), off, right=True) - 1
    child = torch.bucketize(torch.arange(int(b["parent_off"][-1]), device=dev), b["parent_off"], right=True) - 1
    parent = torch.zeros(n_req, n, n, dtype=torch.bool, device=dev)
    parent[req[child], child - off[req[child]], b["parent_idx"][:child.numel()]] = True
    # layers, positions and who sees whom, node after node (parents come first)
    layer, start, end = (torch.zeros(n_req, n, dtype=torch.long, device=dev) for _ in range(3))
    sees = torch.zeros(n_req, n, n, dtype=torch.bool, device=dev)
    for v in range(n):
        par = parent[:, v]
        layer[:, v] = torch.where(par, layer + 1, 0).amax(1)
        start[:, v] = torch.where(par, end, 0).amax(1)
        end[:, v] = start[:, v] + ln[:, v] + nw[:, v]
        sees[:, v] = (par[:, :, None] & sees).any(1)
        sees[:, v, v] = True
    if case["vis"] == 1:
        sees = (layer[:, None, :] < layer[:, :, None]) | torch.eye(n, dtype=torch.bool, device=dev)
        sees &= have[:, None, :] & have[:, :, None]
    if case["pos"] == 1:
        before = torch.zeros(n_req, 1, dtype=torch.long, device=dev)
        for k in range(n):
            start = torch.where(layer == k, before, start)
            before = torch.maximum(before, torch.where((layer == k) & have, before + ln + nw, 0).amax(1, keepdim=True))
    # one row per new token
    new = b["node_new"]
    n_rows = int(new.sum())
    first = new.cumsum(0) - new
    node = torch.repeat_interleave(torch.arange(nodes, device=dev), new)
    j = torch.arange(n_rows, device=dev) - first[node]
    t = b["node_len"][node] + j
    r = req[node]
    pos_id = start[r, node - off[r]] + t
    slot = b["page_idx"][b["page_off"][node] + t // PAGE] * PAGE + t % PAGE
    # groups of at most `per` rows of one request
    rows_of = torch.where(have, nw, 0).sum(1)
    groups_of = (rows_of + per - 1) // per
    n_groups = int(groups_of.sum())
    g_first, r_first = groups_of.cumsum(0) - groups_of, rows_of.cumsum(0) - rows_of
    g_req = torch.repeat_interleave(torch.arange(n_req, device=dev), groups_of)
    g_idx = torch.arange(n_groups, device=dev) - g_first[g_req]
    g_row0 = r_first[g_req] + g_idx * per
    g_rows = torch.minimum(rows_of[g_req] - g_idx * per, torch.tensor(per, device=dev))
    # (group, node, page): how many tokens each row of the group sees of the page
    pair_g = torch.repeat_interleave(torch.arange(n_groups, device=dev), (off[1:] - off[:-1])[g_req])
    per_req = (off[1:] - off[:-1])[g_req]
    pair_u = torch.arange(pair_g.numel(), device=dev) - (per_req.cumsum(0) - per_req)[pair_g]
    tot = (ln + nw)[g_req[pair_g], pair_u]
    n_pages = (tot + PAGE - 1) // PAGE
    bits = torch.arange(per, device=dev)
    row = (g_row0[pair_g, None] + bits).clamp(max=n_rows - 1)
    visible = (bits < g_rows[pair_g, None]) & sees[g_req[pair_g, None], (node[row] - off[g_req[pair_g]][:, None]).clamp(0, n - 1), pair_u[:, None]]
    keep = visible.any(1)
    pair_g, pair_u, tot, n_pages, row, visible = (x[keep] for x in (pair_g, pair_u, tot, n_pages, row, visible))
    which = torch.repeat_interleave(torch.arange(pair_g.numel(), device=dev), n_pages)
    p = torch.arange(which.numel(), device=dev) - (n_pages.cumsum(0) - n_pages)[which]
    u = off[g_req[pair_g]][which] + pair_u[which]
    full = (tot[which] - PAGE * p).clamp(max=PAGE)
    mine = node[row][which] == u[:, None]
    cnt = torch.where(mine, (t[row][which] + 1 - PAGE * p[:, None]).clamp(0, PAGE), full[:, None])
    cnt = torch.where(visible[which], cnt, 0)
    exists = torch.zeros(which.numel(), PAGE + 1, dtype=torch.bool, device=dev).scatter_(1, cnt, True)[:, 1:]
    e, c = exists.nonzero(as_tuple=True)
    hit = cnt[e] == c[:, None] + 1
    word = hit * (1 << (bits % 32))
    masks = [torch.where(bits < 32, word, 0).sum(1), torch.where(bits >= 32, word, 0).sum(1)]
    masks = [torch.where(m >= 1 << 31, m - (1 << 32), m) for m in masks]
    found = torch.zeros(n_groups, dtype=torch.long, device=dev).index_add_(0, pair_g[which[e]], torch.ones_like(e))
    entries = torch.stack([b["page_idx"][b["page_off"][u[e]] + p[e]], c + 1, *masks], 1)

    def pad(x, m, value, dtype):
        out = torch.full((m,) + x.shape[1:], value, dtype=dtype, device=dev) if not torch.is_tensor(value) else value.to(dtype).expand(m).clone()
        out[:x.shape[0]] = x.to(dtype)
        return out

    def offsets(x):
        x = torch.cat([x.new_zeros(1), x.cumsum(0)])
        return pad(x, z["groups"] + 1, x[-1], torch.int32)

    tiles = (found + 7) // 8
    counts = torch.stack([new.sum(), groups_of.sum(), found.sum(), tiles.sum()] + [new.sum() * 0] * 4).to(torch.int32)
    return {"pos_id": pad(pos_id, z["rows"], 0, torch.int32), "slot": pad(slot, z["rows"], -1, torch.int64), "group_row_off": offsets(g_rows),
            "group_ent_off": offsets(found), "group_tile_off": offsets(tiles), "entries": pad(entries, z["entries"], 0, torch.int32), "counts": counts}


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _write(s):
    t = s["tables"]
    if own:
        s["B"].mv_rope_write_kv_fp8_blk(s["h_tables"], s["geom"], s["q"], s["k"], s["v"], s["q_rot"], s["k_rot"], s["k_pages"], s["v_pages"], s["scale"])
    else:
        d = s["case"]["d"]
        live = t["slot"] >= 0
        slot, pos = t["slot"][live], t["pos_id"][live]
        i = torch.arange(d // 2, device=pos.device, dtype=torch.float64)
        angle = pos.double()[:, None] * torch.pow(torch.tensor(10000.0, dtype=torch.float64, device=pos.device), -2.0 * i / d)
        cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]

        def rotate(x):
            lo, hi = x[live].float().split(d // 2, -1)
            return torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1)

        k_rot, v = rotate(s["k"]), s["v"][live].float()
        s["q_rot"][live], s["k_rot"][live] = rotate(s["q"]).bfloat16(), k_rot.bfloat16()
        page, off = slot // PAGE, slot % PAGE
        pages, at = page.unique(return_inverse=True)
        first = torch.full_like(pages, PAGE).scatter_reduce(0, at, off, "amin")
        for which, (pool, raw, x, top) in enumerate(((s["k_pages"], s["k"][live].float(), k_rot, K_TOP), (s["v_pages"], v, v, V_TOP))):
            amax = torch.zeros(pages.numel(), s["case"]["hkv"], device=pos.device).index_reduce_(0, at, raw.abs().amax(-1), "amax")
            need, old = _scale_of(amax, top), s["scale"][pages, :, which]
            scale = torch.where(first[:, None] > 0, torch.maximum(old, need), need)
            # what the block already holds moves to its new scale
            blocks = pool[pages].view(torch.float8_e4m3fn)
            moved = _e4m3(blocks.float() * (old / scale)[:, :, None, None])
            keep = (torch.arange(PAGE, device=pos.device) < first[:, None])[:, None, :, None]
            pool[pages] = torch.where(keep, moved.view(torch.uint8), pool[pages])
            pool[page, :, off] = _e4m3(x / scale[at][:, :, None]).view(torch.uint8)
            s["scale"][pages, :, which] = scale
    return {"q_rot": s["q_rot"], "k_rot": s["k_rot"], "k_pages": s["k_pages"].view(torch.float8_e4m3fn), "v_pages": s["v_pages"].view(torch.float8_e4m3fn),
            "scale": s["scale"]}


def _attn(s):
    t, case = s["tables"], s["case"]
    if own:
        s["B"].mv_dag_decode_attn_fp8_blk(s["h_tables"], s["geom"], s["q"], s["k_pages"], s["v_pages"], s["scale"], s["out"], s["workspace"])
        return s["out"]
    hkv, d, per = case["hkv"], case["d"], s["per"]
    g = case["hq"] // hkv
    dev = s["q"].device
    row_off, ent_off = t["group_row_off"].long(), t["group_ent_off"].long()
    n_groups = int(t["counts"][1])
    rows, ents = row_off[1:] - row_off[:-1], ent_off[1:] - ent_off[:-1]
    width = int(ents.max())
    # every group's pages side by side, padded to the longest list
    at = ent_off[:n_groups, None] + torch.arange(width, device=dev)
    there = torch.arange(width, device=dev) < ents[:n_groups, None]
    e = t["entries"].long()[torch.where(there, at, 0)]
    page, mask = e[..., 0], (e[..., 2] & 0xffffffff) | (e[..., 3] << 32)
    held = there[..., None] & (torch.arange(PAGE, device=dev) < e[..., 1:2])

    def load(pool, which):
        x = pool[page].view(torch.float8_e4m3fn).float()
        x *= s["scale"][page][..., which][..., None, None]
        x.masked_fill_(~held[:, :, None, :, None], 0.0)
        return x.permute(0, 2, 1, 3, 4).reshape(n_groups, hkv, width * PAGE, d)

    bit = torch.arange(per, device=dev)
    q_row = (row_off[:n_groups, None] + bit).clamp(max=s["q"].shape[0] - 1)
    q = s["q"][q_row].float().view(n_groups, per, hkv, g, d).permute(0, 2, 1, 3, 4).reshape(n_groups, hkv, per * g, d)
    score = torch.matmul(q, load(s["k_pages"], 0).transpose(2, 3)) / math.sqrt(d)
    see = (((mask[:, None] >> bit[:, None]) & 1) > 0)[..., None] & held[:, None]                       # group, row, page, token
    see = see.reshape(n_groups, 1, per, 1, width * PAGE)
    score = score.view(n_groups, hkv, per, g, width * PAGE).masked_fill_(~see, -math.inf)
    score -= score.amax(-1, keepdim=True).clamp(min=-3e38)
    score.exp_()
    total = score.sum(-1, keepdim=True)
    score /= total
    out = torch.matmul(score.view(n_groups, hkv, per * g, width * PAGE), load(s["v_pages"], 1))
    out = out.view(n_groups, hkv, per, g, d).permute(0, 2, 1, 3, 4).reshape(n_groups, per, hkv * g, d)
    live = bit < rows[:n_groups, None]
    s["out"][q_row[live]] = out[live].bfloat16()
    return s["out"]


# ---------------------------------------------------------------------------------------------------- by definition, in 64 bits

def exact(case, seed):
    b, num_pages = _batch(case, seed)
    if case["op"] == "tables":
        return None if case["n_req"] > 256 else {k: torch.from_numpy(v) for k, v in _padded_tables(_host_tables(case, b)).items()}
    s = prepare(case, seed)
    t = {k: v.cpu() for k, v in s["tables"].items()}
    d, hkv = case["d"], case["hkv"]
    if case["op"] == "attn":
        g = case["hq"] // hkv
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for i in range(int(t["counts"][1])):
            r0, r1 = int(t["group_row_off"][i]), int(t["group_row_off"][i + 1])
            e = t["entries"][int(t["group_ent_off"][i]):int(t["group_ent_off"][i + 1])].long()
            page = e[:, 0].cuda()
            k, v = (p[page].view(torch.float8_e4m3fn).double() * s["scale"][page, :, w].double()[:, :, None, None] for w, p in enumerate((s["k_pages"], s["v_pages"])))
            for r in range(r0, r1):
                word = e[:, 2] if r - r0 < 32 else e[:, 3]
                see = (((word >> ((r - r0) % 32)) & 1) > 0)[:, None] & (torch.arange(PAGE) < e[:, 1:2])
                see = see.reshape(-1).cuda().nonzero()[:, 0]
                for h in range(hkv):
                    kk, vv = (x[:, h].reshape(-1, d)[see] for x in (k, v))
                    w = torch.softmax(s["q"][r, h * g:(h + 1) * g].double() @ kk.T * d ** -0.5, -1)
                    out[r, h * g:(h + 1) * g] = w @ vv
        return out
    rows = int((t["slot"] >= 0).sum())
    slot = t["slot"][:rows].cuda()
    theta = 10000.0 ** (-2.0 * torch.arange(d // 2, dtype=torch.float64, device="cuda") / d)
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), t["pos_id"][:rows].cuda().double()[:, None] * theta)[:, None]

    def rotate(x):
        z = torch.complex(x[:rows, :, :d // 2].double(), x[:rows, :, d // 2:].double()) * turn
        y = torch.zeros(x.shape, dtype=torch.float64, device="cuda")
        y[:rows, :, :d // 2], y[:rows, :, d // 2:] = z.real, z.imag
        return y

    out = {"q_rot": rotate(s["q"]), "k_rot": rotate(s["k"])}
    scale = s["scale"].double()
    pools = [p.view(torch.float8_e4m3fn).double() for p in (s["k_pages"], s["v_pages"])]
    page, off = (slot // PAGE).tolist(), (slot % PAGE).tolist()
    r0 = 0
    while r0 < rows:  # runs of new tokens in one page
        r1 = r0 + 1
        while r1 < rows and page[r1] == page[r0] and off[r1] == off[r1 - 1] + 1:
            r1 += 1
        for w, (raw, x, top) in enumerate(((s["k"], out["k_rot"], K_TOP), (s["v"], s["v"].double(), V_TOP))):
            need = torch.exp2(torch.ceil(torch.log2(raw[r0:r1].double().abs().amax((0, 2)) / top)).clamp(E_MIN, E_MAX))
            if off[r0]:
                new = torch.maximum(scale[page[r0], :, w], need)
                pools[w][page[r0], :, :off[r0]] *= (scale[page[r0], :, w] / new)[:, None, None]
            else:
                new = need
            scale[page[r0], :, w] = new
            pools[w][page[r0], :, off[r0]:off[r1 - 1] + 1] = (x[r0:r1] / new[:, None]).transpose(0, 1)
        r0 = r1
    return {**out, "k_pages": pools[0], "v_pages": pools[1], "scale": scale}


# ---------------------------------------------------------------------------------------------------- what a pass cannot do without

def work(case):
    b, _ = _batch(case, 0)
    t = _host_tables(case, b, blocks=case["op"] != "write")
    rows, ents = len(t["pos_id"]), len(t["entries"])
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    if case["op"] == "tables":
        read = 4 * sum(len(x) for x in b.values())
        return {"bytes": read + 12 * rows + 12 * len(t["group_row_off"]) + 16 * ents, "flops": 0}
    if case["op"] == "write":
        blocks = len(np.unique(t["slot"] // PAGE))
        return {"bytes": rows * (12 + (2 * hq * 2 + 3 * hkv * 2 + 2 * hkv) * d) + blocks * hkv * 16, "flops": rows * (hq + hkv) * d * 3}
    pages = len(np.unique(t["entries"][:, 0]))
    seen = sum(bin(int(m) & 0xffffffff).count("1") * int(c) for _, c, lo, hi in t["entries"] for m in (lo, hi))
    return {"bytes": pages * hkv * (2 * PAGE * d + 8) + 16 * ents + 2 * 2 * rows * hq * d, "flops": 4 * seen * hq * d}
