"""Workloads of a prompt's chunk against the block-scaled 8-bit cache, and of what surrounds it: what each call gets, its plain
form and its definition.

``rotate``  rotary embedding of q and k in the backbones' forms (halves or pairs, part of the head, stretched for long contexts),
            and its backward pass
``write``   the same rotation fused with the write of K and V into the block-scaled cache
``pages``   pages of many pools copied at once (forks, compaction)
``tables``  batch description on the device -> query tiles and page lists of a step with any number of new tokens per node
``chunk``   attention of those new tokens over the cache, causal inside their node

A batch is a set of request DAGs: a shared prefix and layers of branches; the last layer receives the new tokens, or, where
``fresh``, every node's tokens are new.  ``run`` computes a pass with elementary torch operations, or with the library's calls
where ``own`` is true.
"""
import math

import numpy as np
import torch

own = False

PAGE = 16
KEYS = 8                    # pages of a key tile
E_MIN, E_MAX = -60, 40      # range of the scale exponents
K_TOP, V_TOP = 316.0, 448.0  # largest raw magnitude a block of scale 1 takes (316 * sqrt 2 < 448, the format's largest value)
PLAIN, LINEAR, BASE, RAMP = 0, 1, 2, 3  # how the angles are stretched


# ---------------------------------------------------------------------------------------------------- cases

def _form(layout, first, part, base=10000.0, scaling=PLAIN, factor=1.0, length=8192, slow=1.0, fast=32.0, amplitude=1.0):
    """A rotary form: ``part`` elements from ``first`` on, as two halves (0) or as pairs of neighbours (1)."""
    return {"layout": layout, "first": first, "part": part, "base": base, "scaling": scaling, "factor": factor, "length": length,
            "slow": slow, "fast": fast, "amplitude": amplitude}


def _rotate(name, heads, rows, pos, dtype, backward, packed, form, seed):
    return {"name": name, "op": "rotate", "hq": heads[0], "hkv": heads[1], "d": heads[2], "rows": rows, "pos": pos, "dtype": dtype,
            "backward": backward, "packed": packed, **form, "layout_seed": seed}


def _write(name, heads, n_req, held, new, pos, form, seed):
    return {"name": name, "op": "write", "hq": heads[0], "hkv": heads[1], "d": heads[2], "n_req": n_req, "held": held, "new": new,
            "pos": pos, **form, "layout_seed": seed}


def _pages(name, heads, pools, kind, num_pages, moves, seed):
    return {"name": name, "op": "pages", "hkv": heads[1], "d": heads[2], "layers": pools, "kind": kind, "num_pages": num_pages,
            "moves": moves, "layout_seed": seed}


def _dag(name, op, heads, n_req, prefix, branches, blen, new, seed, layers=1, fresh=False, vis=0):
    return {"name": name, "op": op, "hq": heads[0], "hkv": heads[1], "d": heads[2], "n_req": n_req, "prefix_lo": prefix[0],
            "prefix_hi": prefix[1], "branches_lo": branches[0], "branches_hi": branches[1], "blen_lo": blen[0], "blen_hi": blen[1],
            "new_lo": new[0], "new_hi": new[1], "layers": layers, "fresh": fresh, "vis": vis, "layout_seed": seed}


def listed():
    small, half = (32, 8, 128), (8, 2, 64)
    return [
        # q and k of one decode step of 16 requests with four branches, half of the head rotated in pairs, out of one packed projection
        _rotate("rotary of a decode step, pairs", small, 64, 20000, "bf16", False, True, _form(1, 0, 64), 1),
        # the gradients of q and k of a prompt of 17 thousand tokens on their way back through the rotation, stretched by turns
        _rotate("rotary backward of a prompt", small, 17021, 131072, "bf16", True, False,
                _form(0, 0, 128, 500000.0, RAMP, 8.0, 8192, 1.0, 4.0), 2),
        # the cache write of a decode step: one token for each of 64 branches, pairs, the last 64 elements of the head
        _write("write of a decode step, pairs", small, 64, 2048, 1, 20000, _form(1, 64, 64), 3),
        # a prompt's chunk written at once: 8 requests of about 2000 tokens, long context with an amplitude
        _write("write of a chunk, stretched", small, 8, 700, 2048, 131072, _form(0, 0, 128, 10000.0, RAMP, 16.0, 4096, 1.0, 32.0, 1.2772589), 4),
        # a fork: the partly filled last pages of sixteen branches, in the two 16-bit pools of one layer
        _pages("pages of a fork", small, 1, "bf16", 512, 16, 5),
        # a pool is compacted: 3000 of 8000 pages of four layers move, 8-bit pools and their scales
        _pages("pages of a compaction", small, 4, "fp8", 8000, 3000, 6),
        # tables of one prompt of 600 tokens behind a page or two: pure latency
        _dag("tables of one chunk", "tables", small, 1, (24, 24), (1, 1), (0, 0), (600, 600), 7),
        # of 128 requests of mixed lengths with runs of new tokens on every branch
        _dag("tables of 128 requests", "tables", small, 128, (512, 16384), (2, 8), (64, 512), (1, 300), 8),
        # a short prompt alone
        _dag("chunk of a short prompt", "chunk", small, 1, (0, 0), (1, 1), (0, 0), (50, 50), 9),
        # 24 requests with odd numbers of tokens on every branch, 64-element heads
        _dag("chunks on branches, head 64", "chunk", half, 24, (1, 2048), (1, 5), (1, 333), (1, 133), 10),
        # the next 2048 tokens of a document of 64 thousand
        _dag("chunk of a long document", "chunk", small, 1, (65536, 65536), (1, 1), (0, 0), (2048, 2048), 11),
        # a prompt with its whole reasoning DAG, about 17 thousand tokens, all of them new: the largest
        _dag("chunk of a DAG prompt", "chunk", (64, 8, 128), 1, (4096, 4096), (6, 6), (256, 768), (0, 0), 12, layers=4, fresh=True),
    ]


def draw(rng):
    def log(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    op = rng.choice(["rotate", "rotate", "write", "pages", "tables", "chunk", "chunk", "chunk"])
    heads = rng.choice([(32, 8, 128), (64, 8, 128), (40, 8, 128), (16, 16, 128), (24, 1, 128), (12, 2, 128), (8, 2, 64), (32, 8, 64), (4, 1, 64)])
    seed = rng.randint(1, 1 << 30)
    part = 16 * rng.randint(1, heads[2] // 16)
    form = _form(rng.randint(0, 1), 16 * rng.randint(0, (heads[2] - part) // 16), part, rng.choice([10000.0, 500000.0]),
                 rng.choice([PLAIN, LINEAR, BASE, RAMP]), rng.choice([2.0, 8.0, 32.5]), rng.choice([2048, 8192]), 1.0, rng.choice([4.0, 32.0]),
                 rng.choice([1.0, 1.0, 1.2079442, 0.75]))
    if op == "rotate":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 17000 * 40 * 128 // ((heads[0] + heads[1]) * heads[2]) // (2 if dtype == "f32" else 1)
        c = _rotate(None, heads, log(1, min(most, 40000)), log(1, 1 << 20), dtype, rng.random() < 0.5, rng.random() < 0.5, form, seed)
    elif op == "write":
        new = log(1, 3000)
        c = _write(None, heads, max(1, min(log(1, 128), 16000 // new)), log(1, 4096), new, log(1, 1 << 20), form, seed)
    elif op == "pages":
        n = log(4, 8000)
        c = _pages(None, heads, rng.randint(1, 4), rng.choice(["bf16", "fp8"]), n, log(1, max(1, 3 * n // 8)), seed)
    else:
        fresh = rng.random() < 0.3
        lo = log(1, 16384) if rng.random() < 0.8 else 0
        hi = log(lo, 16384) if 0 < lo < 16384 else lo
        layers = rng.choice([1, 1, 2, 3]) if op == "chunk" else rng.choice([1, 2, 4])
        branches = rng.randint(1, 8)
        blen, new = log(1, 1024), log(1, 2048)
        if fresh:
            hi, lo, new = min(hi, 4096), min(lo, 4096), 0
            blen = max(1, min(blen, 12000 // (branches * layers)))
        if op == "chunk":  # pairs of a new token and what it sees, times the query heads
            def cost():
                return (hi + branches * blen * layers if fresh else branches * new) * (hi + layers * blen + new) * heads[0]
            while cost() > 4.0e9:
                hi, lo, blen, new = (x - x // 4 for x in (hi, lo, blen, new))
        tokens = hi + branches * (blen * layers + new)
        rows = tokens if fresh else branches * new
        n_req = max(1, min(log(1, 128), 600_000 // tokens, 16_000 // rows, int(4.0e9 / cost()) if op == "chunk" else 128))
        c = _dag(None, op, heads, n_req, (lo, hi), (rng.randint(1, branches), branches), (rng.randint(0, blen) if not fresh else max(1, blen // 2), blen),
                 (max(1, new // 3) if not fresh else 0, new), seed, layers, fresh, rng.choice([0, 0, 0, 1]))
    del c["name"]
    return c


# ---------------------------------------------------------------------------------------------------- batches of DAGs

def _requests(case):
    """The DAGs of a case: per request a list of (parents, tokens held, new tokens)."""
    r = np.random.default_rng(case["layout_seed"])

    def log(lo, hi):
        return int(round(math.exp(r.uniform(math.log(lo), math.log(hi))))) if hi > lo > 0 else hi

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
        if case["fresh"]:
            out.append([(p, 0, n) for p, n in nodes])
        else:
            out.append([(p, n, int(r.integers(case["new_lo"], case["new_hi"] + 1)) if v in prev else 0) for v, (p, n) in enumerate(nodes)])
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
    return {k: np.asarray(v, np.int32) for k, v in b.items()}, num_pages


def _rows_per_tile(case):
    return 2 * (128 // (case["hq"] // case["hkv"]))


def _host_tables(case, b):
    """Query tiles and page lists by their definition, node by node."""
    per = _rows_per_tile(case)
    tiles, entries, nodes, rows, unit, n_ents = [], [], [], 0, 0, 0
    for r in range(case["n_req"]):
        lo, hi = int(b["node_off"][r]), int(b["node_off"][r + 1])
        n = hi - lo
        parents = [[int(p) for p in b["parent_idx"][b["parent_off"][g]:b["parent_off"][g + 1]]] for g in range(lo, hi)]
        layer, sees = [], []
        for v in range(n):
            layer.append(1 + max(layer[p] for p in parents[v]) if parents[v] else 0)
            sees.append(set().union(*[sees[p] | {p} for p in parents[v]]))
        if case["vis"] == 1:
            sees = [{u for u in range(n) if layer[u] < layer[v]} for v in range(n)]
        for v in range(n):
            ln, nw = int(b["node_len"][lo + v]), int(b["node_new"][lo + v])
            if nw == 0:
                continue
            mine = []
            for u in sorted(sees[v]) + [v]:
                tot = int(b["node_len"][lo + u]) + int(b["node_new"][lo + u])
                pages = b["page_idx"][b["page_off"][lo + u]:b["page_off"][lo + u] + (tot + PAGE - 1) // PAGE]
                mine.append(np.stack([pages, np.minimum(PAGE, tot - PAGE * np.arange(len(pages)))], 1))
            own_pages = len(mine[-1])
            mine = np.concatenate(mine)
            before = len(mine) - own_pages
            nodes.append((rows, nw, n_ents, len(mine), before, ln))
            for j in range(0, nw, per):
                m = min(per, nw - j)
                units = (before + (ln + j + m + PAGE - 1) // PAGE + KEYS - 1) // KEYS
                tiles.append((rows + j, m, n_ents, before, ln + j, unit, units, 0))
                unit += units
            entries.append(mine)
            n_ents += len(mine)
            rows += nw
    return {"tiles": np.asarray(tiles, np.int32).reshape(-1, 8), "entries": np.concatenate(entries).astype(np.int32) if entries else np.zeros((0, 2), np.int32),
            "counts": np.asarray([rows, len(tiles), n_ents, unit, 0, 0, 0, 0], np.int32), "nodes": nodes}


def _sizes(t):
    """Capacities a caller would set aside: a little more than this step needs."""
    return {"rows": int(t["counts"][0]) + 5, "tiles": len(t["tiles"]) + 3, "entries": len(t["entries"]) + 9}


def _padded(t):
    z = _sizes(t)
    out = {"tiles": np.zeros((z["tiles"], 8), np.int32), "entries": np.zeros((z["entries"], 2), np.int32), "counts": t["counts"]}
    for k in ("tiles", "entries"):
        out[k][:len(t[k])] = t[k]
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


def _theta(case):
    """Angle per position of every rotated pair, in 64 bits."""
    part, base, s = case["part"], case["base"], case["factor"]
    i = np.arange(part // 2, dtype=np.float64)
    if case["scaling"] == BASE:
        base = base * s ** (part / max(part - 2.0, 1.0))
    theta = base ** (-2.0 * i / part)
    if case["scaling"] == LINEAR:
        theta = theta / s
    if case["scaling"] == RAMP:  # by the turns a pair makes over the length it was trained on
        turns = case["length"] * theta / (2 * math.pi)
        keep = np.clip((turns - case["slow"]) / (case["fast"] - case["slow"]), 0.0, 1.0)
        theta = (1 - keep) * theta / s + keep * theta
    return theta


def _write_rows(case, seed):
    """Slots and positions of the new tokens: every request goes on in its last page; the pages come from a shuffled pool."""
    r = np.random.default_rng(case["layout_seed"])
    slots, pos, used = [], [], 0
    pages = []
    for _ in range(case["n_req"]):
        held, new = int(r.integers(0, case["held"] + 1)), int(r.integers(max(1, case["new"] - case["new"] // 8), case["new"] + 1))
        t = np.arange(held, held + new)
        pages.append((used, t))
        used += (held + new + PAGE - 1) // PAGE
        pos.append(t + int(r.integers(0, case["pos"])))
    num_pages = used + used // 8 + 1
    ids = np.random.default_rng([seed, 78]).permutation(num_pages).astype(np.int64)
    slots = [ids[first + t // PAGE] * PAGE + t % PAGE for first, t in pages]
    return np.concatenate(slots), np.concatenate(pos), num_pages


def _own_form(s, B):
    c = s["case"]
    return B.RopeForm(c["layout"], c["part"], first=c["first"], base=c["base"], scaling=("plain", "linear", "base", "ramp")[c["scaling"]], factor=c["factor"],
                      length=c["length"], slow=c["slow"], fast=c["fast"], amplitude=c["amplitude"])


def prepare(case, seed):
    s = {"case": case}
    if own:
        from paper_2602_07529_b200 import binding as B
        s["B"] = B
    if case["op"] == "rotate":
        hq, hkv, d, n = case["hq"], case["hkv"], case["d"], case["rows"]
        dt = torch.bfloat16 if case["dtype"] == "bf16" else torch.float32
        if case["packed"]:  # q, k and v of a token side by side, as one projection leaves them
            x = _normal((n, hq + 2 * hkv, d), seed, 1, dt)
            s["q"], s["k"] = x[:, :hq], x[:, hq:hq + hkv]
        else:
            s["q"], s["k"] = _normal((n, hq, d), seed, 1, dt), _normal((n, hkv, d), seed, 2, dt)
        g = np.random.default_rng([seed, 79])
        s["pos"] = torch.from_numpy(g.integers(0, case["pos"], n).astype(np.int32)).cuda()
        s["q_out"], s["k_out"] = (torch.zeros(x.shape, dtype=dt, device="cuda") for x in (s["q"], s["k"]))
        if own:
            s["form"], s["geom"] = _own_form(s, B), B.make_geom(hq, hkv, d, 0, case["dtype"])
        return s
    if case["op"] == "write":
        slot, pos, num_pages = _write_rows(case, seed)
        rows = len(slot) + 5
        s["tables"] = {"pos_id": torch.zeros(rows, dtype=torch.int32, device="cuda"), "slot": torch.full((rows,), -1, dtype=torch.int64, device="cuda"),
                       "counts": torch.zeros(8, dtype=torch.int32, device="cuda")}
        s["tables"]["pos_id"][:len(slot)] = torch.from_numpy(pos.astype(np.int32)).cuda()
        s["tables"]["slot"][:len(slot)] = torch.from_numpy(slot).cuda()
        s["k_pages"], s["v_pages"], s["scale"] = _pools(case, num_pages, seed)
        s["q"] = _normal((rows, case["hq"], case["d"]), seed, 1)
        s["k"], s["v"] = (_normal((rows, case["hkv"], case["d"]), seed, 2 + i) for i in range(2))
        s["q_rot"], s["k_rot"] = torch.zeros_like(s["q"]), torch.zeros_like(s["k"])
        if own:
            s["form"], s["geom"] = _own_form(s, B), B.make_geom(case["hq"], case["hkv"], case["d"], num_pages, "bf16")
            s["h_tables"] = B.StepTables(**s["tables"])
        return s
    if case["op"] == "pages":
        n, hkv, d = case["num_pages"], case["hkv"], case["d"]
        r = np.random.default_rng([seed, 80])
        ids = r.permutation(n)
        moves = min(case["moves"], n // 2)
        s["src"], s["dst"] = (torch.from_numpy(x.astype(np.int32)).cuda() for x in (ids[:moves], ids[moves:2 * moves]))
        s["pools"] = []
        for layer in range(case["layers"]):
            for which in range(2):
                x = _normal((n, hkv, d // 64, PAGE, 64), seed, 10 * layer + which)
                s["pools"].append(x if case["kind"] == "bf16" else x.to(torch.float8_e4m3fn).view(torch.uint8).view(n, hkv, PAGE, d))
            if case["kind"] == "fp8":
                s["pools"].append(torch.exp2(_normal((n, hkv, 2), seed, 10 * layer + 5, torch.float32).round()))
        if own:
            s["h_pools"] = B.PagePools(s["pools"])
        return s
    b, num_pages = _batch(case, seed)
    t = _host_tables(case, b)
    z, per = _sizes(t), _rows_per_tile(case)
    s["z"], s["per"], s["num_pages"] = z, per, num_pages
    if case["op"] == "tables":
        s["batch"] = {k: torch.from_numpy(v).cuda() for k, v in b.items()}
        s["most_nodes"] = int(np.diff(b["node_off"]).max())
        s["tables"] = {"tiles": torch.zeros(z["tiles"], 8, dtype=torch.int32, device="cuda"),
                       "entries": torch.zeros(z["entries"], 2, dtype=torch.int32, device="cuda"),
                       "counts": torch.zeros(8, dtype=torch.int32, device="cuda")}
    else:
        s["tables"] = {k: torch.from_numpy(v).cuda() for k, v in _padded(t).items()}
        s["nodes"] = t["nodes"]
        s["k_pages"], s["v_pages"], s["scale"] = _pools(case, num_pages, seed)
        s["q"] = _normal((z["rows"], case["hq"], case["d"]), seed, 1)
        s["out"] = torch.zeros_like(s["q"])
    if own:
        s["h_tables"] = B.ChunkTables(**s["tables"], max_rows=z["rows"], rows_per_tile=per)
        if case["op"] == "tables":
            s["h_batch"] = B.DeviceBatch(case["n_req"], **s["batch"], num_pages=num_pages, max_req_nodes=s["most_nodes"], vis_mode=case["vis"])
            s["workspace"] = torch.empty(B.mv_chunk_tables_workspace_bytes(s["h_batch"]), dtype=torch.uint8, device="cuda")
        else:
            s["geom"] = B.make_geom(case["hq"], case["hkv"], case["d"], num_pages, "bf16")
            s["workspace"] = torch.empty(B.mv_chunk_attn_workspace_bytes(s["geom"]), dtype=torch.uint8, device="cuda")
    return s


# ---------------------------------------------------------------------------------------------------- the passes

def run(s):
    return {"rotate": _run_rotate, "write": _run_write, "pages": _run_pages, "tables": _run_tables, "chunk": _run_chunk}[s["case"]["op"]](s)


def _turned(case, pos, x, backward=False):
    """x [n][heads][d] in 32 bits, rotated; angles in 64."""
    theta = torch.from_numpy(_theta(case)).to(pos.device)
    angle = pos.double()[:, None] * theta
    cos, sin = (f.float()[:, None] * case["amplitude"] for f in (angle.cos(), -angle.sin() if backward else angle.sin()))
    y = x.float().clone()
    part = y[..., case["first"]:case["first"] + case["part"]]
    if case["layout"] == 0:
        lo, hi = part.split(case["part"] // 2, -1)
        part.copy_(torch.cat([lo * cos - hi * sin, hi * cos + lo * sin], -1))
    else:
        lo, hi = part[..., 0::2], part[..., 1::2]
        part.copy_(torch.stack([lo * cos - hi * sin, hi * cos + lo * sin], -1).flatten(-2))
    return y


def _run_rotate(s):
    if own:
        s["B"].mv_rope_rotate(s["form"], s["geom"], s["pos"], s["q"], s["k"], s["q_out"], s["k_out"], backward=s["case"]["backward"])
    else:
        for x, y in ((s["q"], s["q_out"]), (s["k"], s["k_out"])):
            y.copy_(_turned(s["case"], s["pos"], x, s["case"]["backward"]))
    return {"q": s["q_out"], "k": s["k_out"]}


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _grown(case, amax):
    """What the rule of the K scale looks at: the largest raw magnitude, times the amplitude where that is above one."""
    return amax.float() * max(1.0, case["amplitude"])


def _run_write(s):
    t, case = s["tables"], s["case"]
    if own:
        s["B"].mv_rope_write_kv_fp8_blk_form(s["h_tables"], s["geom"], s["form"], s["q"], s["k"], s["v"], s["q_rot"], s["k_rot"], s["k_pages"],
                                             s["v_pages"], s["scale"])
    else:
        live = t["slot"] >= 0
        slot, pos = t["slot"][live], t["pos_id"][live]
        k_rot, v = _turned(case, pos, s["k"][live]), s["v"][live].float()
        s["q_rot"][live], s["k_rot"][live] = _turned(case, pos, s["q"][live]).bfloat16(), k_rot.bfloat16()
        page, off = slot // PAGE, slot % PAGE
        pages, at = page.unique(return_inverse=True)
        first = torch.full_like(pages, PAGE).scatter_reduce(0, at, off, "amin")
        for which, (pool, raw, x, top) in enumerate(((s["k_pages"], _grown(case, s["k"][live].abs()), k_rot, K_TOP), (s["v_pages"], v, v, V_TOP))):
            amax = torch.zeros(pages.numel(), case["hkv"], device=pos.device).index_reduce_(0, at, raw.abs().amax(-1), "amax")
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


def _run_pages(s):
    if own:
        s["B"].mv_pages_copy(s["h_pools"], s["src"], s["dst"])
    else:
        src, dst = s["src"].long(), s["dst"].long()
        for p in s["pools"]:
            p[dst] = p[src]
    return s["pools"]


def _run_tables(s):
    if own:
        s["B"].mv_chunk_tables_build(s["h_batch"], s["h_tables"], s["workspace"])
        return s["tables"]
    case, b, per = s["case"], {k: v.long() for k, v in s["batch"].items()}, s["per"]
    dev = b["node_off"].device
    off, n_req, n = b["node_off"], case["n_req"], s["most_nodes"]
    nodes = b["node_len"].numel()
    local = torch.arange(n, device=dev)
    have = off[:-1, None] + local < off[1:, None]
    at = (off[:-1, None] + local).clamp(max=nodes - 1)
    tot = torch.where(have, b["node_len"][at] + b["node_new"][at], 0)
    req = torch.bucketize(torch.arange(nodes, device=dev), off, right=True) - 1
    child = torch.bucketize(torch.arange(int(b["parent_off"][-1]), device=dev), b["parent_off"], right=True) - 1
    parent = torch.zeros(n_req, n, n, dtype=torch.bool, device=dev)
    parent[req[child], child - off[req[child]], b["parent_idx"][:child.numel()]] = True
    # layers and who sees whom, node after node (parents come first)
    layer = torch.zeros(n_req, n, dtype=torch.long, device=dev)
    sees = torch.zeros(n_req, n, n, dtype=torch.bool, device=dev)
    for v in range(n):
        par = parent[:, v]
        layer[:, v] = torch.where(par, layer + 1, 0).amax(1)
        sees[:, v] = (par[:, :, None] & sees).any(1) | par
    if case["vis"] == 1:
        sees = (layer[:, None, :] < layer[:, :, None]) & have[:, None, :] & have[:, :, None]
    # the receiving nodes, and their lists: other nodes' pages first, their own last
    v = (b["node_new"] > 0).nonzero()[:, 0]
    ln, nw = b["node_len"][v], b["node_new"][v]
    pages = (tot + PAGE - 1) // PAGE                                        # [request][node]
    rv, lv = req[v], v - off[req[v]]
    others = torch.where(sees[rv, lv], pages[rv], 0)                        # [receiving node][node]
    mine = torch.zeros_like(others).scatter_(1, lv[:, None], pages[rv, lv][:, None])
    before, found = others.sum(1), (others + mine).sum(1)
    first = found.cumsum(0) - found
    order = torch.cat([others, pages[rv, lv][:, None]], 1)                  # runs of pages, in the order of the list
    node = torch.cat([off[rv][:, None] + local, v[:, None]], 1)
    run = torch.repeat_interleave(torch.arange(order.numel(), device=dev), order.flatten())
    p = torch.arange(run.numel(), device=dev) - (order.flatten().cumsum(0) - order.flatten())[run]
    u = node.flatten()[run]
    entries = torch.stack([b["page_idx"][b["page_off"][u] + p], ((b["node_len"] + b["node_new"])[u] - PAGE * p).clamp(max=PAGE)], 1)
    # tiles of at most `per` rows
    count = (nw + per - 1) // per
    which = torch.repeat_interleave(torch.arange(v.numel(), device=dev), count)
    j = (torch.arange(which.numel(), device=dev) - (count.cumsum(0) - count)[which]) * per
    rows = torch.minimum(nw[which] - j, torch.tensor(per, device=dev))
    key0 = ln[which] + j
    units = (before[which] + (key0 + rows + PAGE - 1) // PAGE + KEYS - 1) // KEYS
    row0 = (nw.cumsum(0) - nw)[which] + j
    tiles = torch.stack([row0, rows, first[which], before[which], key0, units.cumsum(0) - units, units, torch.zeros_like(units)], 1)
    out = {"tiles": torch.zeros_like(s["tables"]["tiles"]), "entries": torch.zeros_like(s["tables"]["entries"])}
    out["tiles"][:tiles.shape[0]] = tiles.to(torch.int32)
    out["entries"][:entries.shape[0]] = entries.to(torch.int32)
    zero = nw.sum() * 0
    out["counts"] = torch.stack([nw.sum(), count.sum(), found.sum(), units.sum()] + [zero] * 4).to(torch.int32)
    return out


def _run_chunk(s):
    t, case = s["tables"], s["case"]
    if own:
        s["B"].mv_dag_chunk_attn_fp8_blk(s["h_tables"], s["geom"], s["q"], s["k_pages"], s["v_pages"], s["scale"], s["out"], s["workspace"])
        return s["out"]
    hkv, d = case["hkv"], case["d"]
    g = case["hq"] // hkv
    dev = s["q"].device
    for row0, rows, ent0, n_ent, before, held in s["nodes"]:
        e = t["entries"][ent0:ent0 + n_ent].long()
        there = (torch.arange(PAGE, device=dev) < e[:, 1:2]).flatten()

        def load(pool, which):
            x = pool[e[:, 0]].view(torch.float8_e4m3fn).float() * s["scale"][e[:, 0]][..., which][..., None, None]
            return x.permute(1, 0, 2, 3).reshape(hkv, n_ent * PAGE, d)[:, there]

        k, v = load(s["k_pages"], 0), load(s["v_pages"], 1)
        key = (torch.arange(n_ent * PAGE, device=dev) - before * PAGE)[there]    # index inside the node itself; negative: another node's
        step = max(1, (1 << 29) // (case["hq"] * key.numel()))
        for j0 in range(0, rows, step):
            j1 = min(rows, j0 + step)
            q = s["q"][row0 + j0:row0 + j1].float().view(j1 - j0, hkv, g, d).permute(1, 2, 0, 3).reshape(hkv, g * (j1 - j0), d)
            score = torch.matmul(q, k.transpose(1, 2)).mul_(d ** -0.5).view(hkv, g, j1 - j0, -1)
            score.masked_fill_(key > held + torch.arange(j0, j1, device=dev)[:, None], -math.inf)
            score -= score.amax(-1, keepdim=True)
            score.exp_()
            score /= score.sum(-1, keepdim=True)
            out = torch.matmul(score.view(hkv, g * (j1 - j0), -1), v)
            s["out"][row0 + j0:row0 + j1] = out.view(hkv, g, j1 - j0, d).permute(2, 0, 1, 3).reshape(j1 - j0, hkv * g, d).bfloat16()
    return s["out"]


# ---------------------------------------------------------------------------------------------------- by definition, in 64 bits

def _turned_exact(case, pos, x, backward=False):
    """Complex numbers times a unit one (and the amplitude), in 64 bits."""
    angle = pos.double()[:, None] * torch.from_numpy(_theta(case)).cuda()
    turn = torch.polar(torch.full_like(angle, case["amplitude"]), -angle if backward else angle)[:, None]
    y = x.double().clone()
    f, half = case["first"], case["part"] // 2
    re, im = (slice(f, f + half), slice(f + half, f + 2 * half)) if case["layout"] == 0 else (slice(f, f + 2 * half, 2), slice(f + 1, f + 2 * half, 2))
    z = torch.complex(y[..., re], y[..., im]) * turn
    y[..., re], y[..., im] = z.real, z.imag
    return y


def exact(case, seed):
    if case["op"] == "tables":
        b, _ = _batch(case, seed)
        return {k: torch.from_numpy(v) for k, v in _padded(_host_tables(case, b)).items()}
    s = prepare(case, seed)
    if case["op"] == "rotate":
        return {k: _turned_exact(case, s["pos"], s[k], case["backward"]) for k in ("q", "k")}
    if case["op"] == "pages":
        out = []
        for p in s["pools"]:
            x = p.cpu().clone()
            for a, c in zip(s["src"].tolist(), s["dst"].tolist()):  # no page is both
                x[c] = x[a]
            out.append(x if x.dtype == torch.uint8 else x.double())
        return out
    d, hkv = case["d"], case["hkv"]
    if case["op"] == "chunk":
        g = case["hq"] // hkv
        out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
        for row0, rows, ent0, n_ent, before, held in s["nodes"]:
            e = s["tables"]["entries"][ent0:ent0 + n_ent].long()
            page = e[:, 0]
            there = torch.arange(PAGE, device="cuda") < e[:, 1:2]
            for h in range(hkv):
                k, v = ((p[page, h].view(torch.float8_e4m3fn).double() * s["scale"][page, h, w].double()[:, None, None])[there]
                        for w, p in enumerate((s["k_pages"], s["v_pages"])))
                seen = int(there[:before].sum())  # tokens of other nodes; then the node's own, in order
                step = max(1, (1 << 27) // (g * k.shape[0]))
                for j0 in range(0, rows, step):
                    j = torch.arange(j0, min(rows, j0 + step), device="cuda")
                    q = s["q"][row0 + j, h * g:(h + 1) * g].double()
                    score = torch.einsum("jgd,kd->jgk", q, k) * d ** -0.5
                    limit = seen + held + j + 1
                    score = torch.where(torch.arange(k.shape[0], device="cuda") < limit[:, None, None], score, -math.inf)
                    out[row0 + j, h * g:(h + 1) * g] = torch.einsum("jgk,kd->jgd", torch.softmax(score, -1), v)
        return out
    rows = int((s["tables"]["slot"] >= 0).sum())
    slot, pos = s["tables"]["slot"][:rows], s["tables"]["pos_id"][:rows]
    out = {}
    for name in ("q", "k"):
        y = torch.zeros(s[name].shape, dtype=torch.float64, device="cuda")
        y[:rows] = _turned_exact(case, pos, s[name][:rows])
        out[name + "_rot"] = y
    scale = s["scale"].double()
    pools = [p.view(torch.float8_e4m3fn).double() for p in (s["k_pages"], s["v_pages"])]
    page, off = (slot // PAGE).tolist(), (slot % PAGE).tolist()
    r0 = 0
    while r0 < rows:  # runs of new tokens in one page
        r1 = r0 + 1
        while r1 < rows and page[r1] == page[r0] and off[r1] == off[r1 - 1] + 1:
            r1 += 1
        for w, (raw, x, top) in enumerate(((s["k"], out["k_rot"], K_TOP), (s["v"], s["v"].double(), V_TOP))):
            amax = raw[r0:r1].abs().amax((0, 2))
            if w == 0:
                amax = _grown(case, amax)
            need = torch.exp2(torch.ceil(torch.log2(amax.double() / top)).clamp(E_MIN, E_MAX))
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
    hkv, d = case["hkv"], case["d"]
    if case["op"] == "pages":
        page = hkv * PAGE * d * 2 * 2 if case["kind"] == "bf16" else hkv * (PAGE * d * 2 + 8)
        moves = min(case["moves"], case["num_pages"] // 2)
        return {"bytes": moves * (2 * case["layers"] * page + 8), "flops": 0}
    hq = case["hq"]
    if case["op"] == "rotate":
        size = 2 if case["dtype"] == "bf16" else 4
        return {"bytes": case["rows"] * (4 + 2 * size * (hq + hkv) * d), "flops": case["rows"] * (hq + hkv) * case["part"] * 3}
    if case["op"] == "write":
        slot, _, _ = _write_rows(case, 0)
        rows, blocks = len(slot), len(np.unique(slot // PAGE))
        return {"bytes": rows * (12 + (2 * hq * 2 + 3 * hkv * 2 + 2 * hkv) * d) + blocks * hkv * 16, "flops": rows * (hq + hkv) * case["part"] * 3}
    b, _ = _batch(case, 0)
    t = _host_tables(case, b)
    rows, n_tiles, ents = (int(x) for x in t["counts"][:3])
    if case["op"] == "tables":
        return {"bytes": 4 * sum(len(x) for x in b.values()) + 32 * n_tiles + 8 * ents, "flops": 0}
    pages = len(np.unique(t["entries"][:, 0]))
    pairs = 0
    for _, n, ent0, _, before, held in t["nodes"]:
        pairs += n * (int(t["entries"][ent0:ent0 + before, 1].sum()) + held) + n * (n + 1) // 2
    return {"bytes": pages * hkv * (2 * PAGE * d + 8) + 8 * ents + 32 * n_tiles + 2 * 2 * rows * hq * d, "flops": 4 * pairs * hq * d}
