"""Chunks of new tokens over the block-scaled 8-bit cache: tables by their definition, attention against 64 bits.

Tolerances, fixed before the first run:
  tables  whole numbers: equal.
  out     bf16 rounds by at most 2^-8 of the value.  Every weight is rounded to bf16, off by at most 2^-8 of itself, which moves an output by
          at most 2^-8 A, A = sum_j p_j |V_j| / sum_j p_j.  Keys and values are exact; a score is a sum of at most 128 exact products in 32
          bits, off by at most 128 * 2^-24 S, S = sum |q_i k_i| (times the softmax scale): another 2^-17 S' A with S' the largest such sum over
          the row's keys, doubled for the reference that is subtracted; the power, the sums and the division: under 2^-12 A together (sums in
          32 bits over at most 2^12 terms in a chain of 2^5 per tile)."""
import dataclasses

import numpy as np
import pytest
import torch

from paper_2602_07529_b200 import synth
from test_gpu_fp8_blk import visible_counts

pytestmark = pytest.mark.gpu


def _mods():
    from paper_2602_07529_b200 import binding as B, runtime
    return B, runtime


def batch_of(reqs, seed=0, slack=1.3, vis=0):
    """reqs: per request a list of (parents, tokens held, new tokens)."""
    b = synth.build_batch(reqs, rng=np.random.default_rng(seed), slack=slack)
    return dataclasses.replace(b, vis_mode=vis)


def random_reqs(seed, n_req=5, most_new=90):
    rng = np.random.default_rng(seed)
    out = []
    for _ in range(n_req):
        n = int(rng.integers(1, 9))
        nodes = []
        for v in range(n):
            k = int(rng.integers(0, min(v, 3) + 1)) if v else 0
            parents = sorted(int(x) for x in rng.permutation(v)[:k])
            nodes.append((parents, int(rng.choice([0, 0, 1, 15, 16, 17, 40, 133])), int(rng.choice([0, 0, 1, 2, 16, 31, most_new]))))
        out.append(nodes)
    return out


# ------------------------------------------------------------------------------------------------ tables

def want_tables(b, per):
    tiles, entries, rows, unit, ents = [], [], 0, 0, 0
    for r in range(b.n_req):
        lo, hi = int(b.node_off[r]), int(b.node_off[r + 1])
        layer, anc = [], []
        par = [[int(p) for p in b.parent_idx[b.parent_off[g]:b.parent_off[g + 1]]] for g in range(lo, hi)]
        for v in range(hi - lo):
            layer.append(1 + max(layer[p] for p in par[v]) if par[v] else 0)
            anc.append(set().union(*[anc[p] | {p} for p in par[v]]))
        for v in range(hi - lo):
            ln, nw = int(b.node_len[lo + v]), int(b.node_new[lo + v])
            if not nw:
                continue
            sees = sorted(anc[v]) if b.vis_mode == 0 else [u for u in range(hi - lo) if layer[u] < layer[v]]
            mine = []
            for u in sees + [v]:
                if u == v:
                    before = len(mine)
                tot = int(b.node_len[lo + u] + b.node_new[lo + u])
                mine += [(int(b.page_idx[b.page_off[lo + u] + p]), min(16, tot - 16 * p)) for p in range((tot + 15) // 16)]
            for j in range(0, nw, per):
                m = min(per, nw - j)
                units = (before + (ln + j + m + 15) // 16 + 7) // 8
                tiles.append((rows + j, m, ents, before, ln + j, unit, units, 0))
                unit += units
            entries += mine
            ents += len(mine)
            rows += nw
    return np.asarray(tiles, np.int64).reshape(-1, 8), np.asarray(entries, np.int64).reshape(-1, 2), [rows, len(tiles), ents, unit, 0, 0, 0, 0]


def check_tables(chunk, b):
    t = {k: v.cpu().numpy() for k, v in chunk.t.items()}
    tiles, entries, counts = want_tables(b, chunk.tables.c_tables.rows_per_tile)
    assert list(t["counts"]) == counts
    assert np.array_equal(t["tiles"][:len(tiles)], tiles) and np.array_equal(t["entries"][:len(entries)], entries)
    assert not t["tiles"][len(tiles):].any() and not t["entries"][len(entries):].any()


@pytest.mark.parametrize("vis", [0, 1])
@pytest.mark.parametrize("group", [1, 4, 5, 24, 128])
@pytest.mark.parametrize("seed", range(4))
def test_tables(seed, group, vis):
    _, rt = _mods()
    b = batch_of(random_reqs(seed, n_req=[1, 5, 40, 3][seed], most_new=[700, 90, 33, 257][seed]), seed, vis=vis)
    chunk = rt.ChunkOnDevice(b, group)
    chunk.build()
    assert chunk.read_status() == 0
    check_tables(chunk, b)


def test_tables_many_receiving_nodes_and_empty_requests():
    """More than 64 receiving nodes in a request (several sweeps), requests without nodes or without new tokens."""
    _, rt = _mods()
    rng = np.random.default_rng(3)
    wide = [([], 5, 1)] + [(sorted({0, int(rng.integers(0, v))}), int(rng.integers(0, 40)), int(rng.integers(0, 3))) for v in range(1, 300)]
    for reqs in ([wide], [[], wide, [], [([], 30, 0)], wide[:70], []], [[([], 3, 0)]], [[]]):
        for vis in (0, 1):
            b = batch_of(reqs, 1, vis=vis)
            chunk = rt.ChunkOnDevice(b, 8)
            chunk.build()
            assert chunk.read_status() == 0
            check_tables(chunk, b)


def test_tables_capacities():
    """Exactly enough fits, one less of anything leaves an empty step and MV_ERR_WORKSPACE; more tables than the step needs keep the rest."""
    B, rt = _mods()
    b = batch_of(random_reqs(7), 7)
    tiles, entries, counts = want_tables(b, 64)
    for kw, ok in (({}, True), ({"max_tiles": len(tiles) - 1}, False), ({"max_entries": len(entries) - 1}, False), ({"max_rows": counts[0] - 1}, False)):
        full = {"max_rows": counts[0], "max_tiles": len(tiles), "max_entries": len(entries), **kw}
        chunk = rt.ChunkOnDevice(b, 4, **full)
        B.mv_chunk_tables_build(chunk.batch, chunk.tables, chunk.workspace)
        assert B.mv_chunk_tables_read_status(chunk.tables) == (0 if ok else 5)
        if ok:
            check_tables(chunk, b)
        else:
            assert not chunk.t["counts"].cpu().numpy()[[0, 1, 2, 3, 5, 6, 7]].any() and not chunk.t["tiles"].any() and not chunk.t["entries"].any()


def test_tables_bad_arrays():
    """What the arrays hold wrongly is found on the device; the step is then empty, and the attention touches nothing."""
    B, rt = _mods()
    b = batch_of([[([], 20, 3), ([0], 4, 2), ([0, 1], 0, 5)], [([], 9, 9)]], 2)
    for name, at, value, want in (("parent_idx", 1, 2, 2), ("parent_idx", 0, -1, 2), ("node_len", 1, 30, 3), ("node_new", 0, -1, 1), ("page_idx", 0, b.num_pages, 1),
                                  ("page_idx", 2, -1, 1), ("page_off", 1, 100, 1), ("page_off", 2, 0, 1), ("parent_off", 2, 9, 1), ("node_off", 1, 7, 1), ("node_off", 0, 1, 1)):
        chunk = rt.ChunkOnDevice(b, 4)
        chunk.arrays[name][at] = value
        B.mv_chunk_tables_build(chunk.batch, chunk.tables, chunk.workspace)
        assert B.mv_chunk_tables_read_status(chunk.tables) == want, (name, at, value)
        assert not chunk.t["counts"].cpu().numpy()[[0, 1, 2, 3]].any()
        q = torch.ones(chunk.tables.max_rows, 8, 128, dtype=torch.bfloat16, device="cuda")
        out = torch.full_like(q, 5.0)
        geom = B.make_geom(8, 2, 128, b.num_pages, "bf16")
        pools = [torch.zeros(b.num_pages, 2, 16, 128, dtype=torch.uint8, device="cuda") for _ in range(2)]
        B.mv_dag_chunk_attn_fp8_blk(chunk.tables, geom, q, *pools, torch.ones(b.num_pages, 2, 2, device="cuda"), out,
                                    torch.empty(B.mv_chunk_attn_workspace_bytes(geom), dtype=torch.uint8, device="cuda"))
        assert (out == 5).all()


# ------------------------------------------------------------------------------------------------ attention

class Case:
    """A step with a cache of random bytes: N(0, 1) values under scales of about 1, stale bytes behind every node's tokens."""

    def __init__(self, reqs, heads, seed=0, vis=0, scales=(0, 0), k_size=1.0, q_size=1.0, sm_scale=0.0, max_rows=None):
        self.B, rt = _mods()
        self.hq, self.hkv, self.d = heads
        self.b = batch_of(reqs, seed, vis=vis)
        self.chunk = rt.ChunkOnDevice(self.b, self.hq // self.hkv, max_rows=max_rows)
        g = torch.Generator(device="cuda").manual_seed(seed)
        n = self.b.num_pages
        rnd = lambda *s: torch.randn(*s, generator=g, device="cuda")
        self.geom = self.B.make_geom(self.hq, self.hkv, self.d, n, "bf16", sm_scale=sm_scale)
        e = torch.randint(scales[0], scales[1] + 1, (n, self.hkv, 2), generator=g, device="cuda")
        self.scale = torch.exp2(e.double()).float()
        self.k8, self.v8 = ((rnd(n, self.hkv, 16, self.d) * s).to(torch.float8_e4m3fn).view(torch.uint8) for s in (k_size, 1.0))
        self.q = (rnd(self.chunk.tables.max_rows, self.hq, self.d) * q_size).bfloat16()
        self.out = torch.full_like(self.q, 7.0)
        self.ws = torch.full((self.B.mv_chunk_attn_workspace_bytes(self.geom),), 0xff, dtype=torch.uint8, device="cuda")
        self.seen = visible_counts(self.b)
        self.chunk.build()
        assert self.chunk.read_status() == 0
        held = {}
        for _, s in self.seen:
            for p, c in s.items():
                held[p] = max(held.get(p, 0), c)
        for p in range(n):     # stale bytes, the format's NaN among them
            for pool, byte in ((self.k8, 0x7f), (self.v8, 0xff)):
                pool[p, :, held.get(p, 0):] = byte

    def run(self, stream=None):
        self.B.mv_dag_chunk_attn_fp8_blk(self.chunk.tables, self.geom, self.q, self.k8, self.v8, self.scale, self.out, self.ws, stream)
        assert self.chunk.read_status(stream) == 0
        return self.out

    def check(self, rows=None):
        g = self.hq // self.hkv
        c = self.geom.sm_scale or self.d ** -0.5
        rows = range(len(self.seen)) if rows is None else rows
        for r in rows:
            page = torch.tensor(list(self.seen[r][1]), device="cuda")
            count = torch.tensor(list(self.seen[r][1].values()), device="cuda")
            there = (torch.arange(16, device="cuda") < count[:, None]).flatten()
            k, v = ((p[page].view(torch.float8_e4m3fn).double() * self.scale[page][..., w].double()[..., None, None]).permute(1, 0, 2, 3).reshape(self.hkv, -1, self.d)[:, there]
                    for w, p in enumerate((self.k8, self.v8)))
            q = self.q[r].double().view(self.hkv, g, self.d)
            score = torch.einsum("hgd,hkd->hgk", q, k) * c
            p = torch.softmax(score, -1)
            ref = torch.einsum("hgk,hkd->hgd", p, v)
            A = torch.einsum("hgk,hkd->hgd", p, v.abs())
            S = torch.einsum("hgd,hkd->hgk", q.abs(), k.abs()).amax(-1, keepdim=True) * c
            tol = 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -12 + 2.0 ** -16 * S) * A
            err = (self.out[r].double().view(self.hkv, g, self.d) - ref).abs()
            assert (err <= tol).all(), (r, float((err / tol).max()), int(there.sum()))
        n = len(self.seen)
        assert (self.out[n:] == 7).all()      # rows behind the step are left as they were


HEADS = [(32, 8, 128), (8, 2, 64), (16, 16, 128), (24, 1, 128), (12, 2, 64), (40, 8, 128), (128, 1, 64), (64, 1, 128), (3, 3, 64), (9, 3, 128)]


@pytest.mark.parametrize("heads", HEADS)
@pytest.mark.parametrize("seed", [0, 1, 2])
def test_random_dags(seed, heads):
    case = Case(random_reqs(seed + 10, n_req=4, most_new=70), heads, seed, vis=seed % 2, scales=(-2, 2), max_rows=700)
    case.run()
    case.check()


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64)])
@pytest.mark.parametrize("held", [0, 1, 15, 16, 127, 128, 129, 1000])
@pytest.mark.parametrize("new", [1, 2, 16, 17, 63, 64, 65, 200])
def test_one_node(new, held, heads):
    """One node alone: every length around pages, key tiles and query tiles."""
    case = Case([[([], held, new)]], heads, new + held, max_rows=new + 3)
    case.run()
    case.check()


def test_one_token_of_one_head():
    case = Case([[([], 0, 1)]], (1, 1, 64), 5)
    case.run()
    case.check()
    v = case.v8[case.b.page_idx[0], 0, 0].view(torch.float8_e4m3fn).float() * case.scale[case.b.page_idx[0], 0, 1]
    assert torch.equal(case.out[0, 0].float(), v)     # a single key: its value


@pytest.mark.parametrize("heads", [(32, 8, 128), (64, 8, 128), (8, 1, 64)])
def test_long_history_is_split(heads):
    """Few rows over a long history: the work is cut over all SMs and joined."""
    case = Case([[([], 20001, 0), ([0], 5, 37)]], heads, 3)
    case.run()
    case.check(rows=[0, 1, 17, 36])


def test_many_short_nodes():
    """Lists of many partly filled pages: masks inside every key tile."""
    reqs = [[([], 3, 0)] + [([0] if v == 1 else [v - 1], 1 + v % 18, 0) for v in range(1, 60)] + [([59], 2, 75)]]
    for heads in ((8, 2, 128), (8, 8, 64)):
        case = Case(reqs, heads, 4)
        case.run()
        case.check()


def test_layers_that_all_receive():
    """A DAG prompt written at once: receiving nodes see each other in full."""
    case = Case([[([], 0, 100), ([0], 0, 70), ([0], 0, 33), ([1, 2], 0, 41), ([3], 0, 1), ([3], 0, 129)]], (16, 4, 128), 6)
    case.run()
    case.check()


def test_every_byte_at_every_scale():
    """All values of the format, subnormals and zeros of both signs among them, at scales 2^-60 .. 2^40: a node of one token gives them back."""
    B, rt = _mods()
    codes = torch.tensor([c for c in range(256) if c & 0x7f != 0x7f], dtype=torch.uint8, device="cuda")
    exps = list(range(-60, 41)) + [-80]
    reqs = [[([], 0, 1)] for _ in exps]
    for d in (64, 128):
        case = Case(reqs, (4, 2, d), 8)
        for x, e in enumerate(exps):
            page = int(case.b.page_idx[x])
            fill = codes.repeat(2)[: 2 * 254]
            for h in range(2):
                at = (x * 97 + h * 127) % 254
                case.v8[page, h, 0] = fill[at:at + d] if at + d <= len(fill) else fill[:d]
            case.scale[page] = 2.0 ** e
        case.run()
        for x, e in enumerate(exps):
            page = int(case.b.page_idx[x])
            v = case.v8[page, :, 0].view(torch.float8_e4m3fn).double() * 2.0 ** e
            assert torch.equal(case.out[x].double(), v.repeat_interleave(2, 0)), e
    # a scale of zero counts as 2^-80
    case.scale.zero_()
    case.run()
    assert (case.out.float().abs() <= 448.0 * 2.0 ** -80).all()


@pytest.mark.parametrize("scales", [(-60, -50), (-8, 8), (36, 40)])
def test_scales_of_values(scales):
    """V far up and down (K held near one by its own): scales enter exactly."""
    case = Case([[([], 70, 0), ([0], 30, 50)]], (8, 2, 128), 9, scales=scales)
    case.scale[..., 0] = 1.0
    case.run()
    case.check()


def test_scales_of_keys():
    """K far up: scores beyond any weight but the largest; K far down: all alike."""
    for e, sm in ((40, 2.0 ** -41), (30, 0.0), (-60, 0.0), (8, 2.0 ** -9), (7, 2.0 ** -10)):
        case = Case([[([], 100, 0), ([0], 3, 40)]], (4, 2, 64), 10, sm_scale=sm)
        case.scale[..., 0] = 2.0 ** e
        case.run()
        if e != 30:
            case.check()
        else:     # one key takes all of a row: its value comes back (keys of equal scores aside, which do not happen here)
            assert torch.isfinite(case.out[:40].float()).all()
            r = 39
            page, count = list(case.seen[r][1]), list(case.seen[r][1].values())
            k = torch.cat([case.k8[p, 0, :c] for p, c in zip(page, count)]).view(torch.float8_e4m3fn).double()
            v = torch.cat([case.v8[p, 0, :c].view(torch.float8_e4m3fn).double() * float(case.scale[p, 0, 1]) for p, c in zip(page, count)])
            best = int((k @ case.q[r, 0].double()).argmax())
            assert torch.equal(case.out[r, 0].double(), v[best])


@pytest.mark.parametrize("q_size", [30.0, 0.0])
def test_peaked_and_flat_rows(q_size):
    """References that leap from tile to tile; weights that are all one."""
    case = Case([[([], 900, 0), ([0], 60, 70)]], (8, 2, 128), 11, q_size=q_size)
    case.run()
    case.check()


@pytest.mark.parametrize("which", [0, 1])
def test_nan_scale_reaches_those_who_see_it(which):
    """A page of another branch, of an ancestor, and one in the middle of the chunk itself."""
    reqs = [[([], 40, 0), ([0], 200, 100), ([0], 30, 0), ([2], 10, 40)]]
    clean = Case(reqs, (8, 2, 128), 12)
    clean.run()
    ref = clean.out.clone()
    po, pi = clean.b.page_off, clean.b.page_idx
    for page in (int(pi[po[2] + 1]), int(pi[po[1] + 15]), int(pi[po[0]]), int(pi[po[3] + 2])):
        case = Case(reqs, (8, 2, 128), 12)
        case.scale[page, 1, which] = float("nan")
        case.run()
        for r, (_, seen) in enumerate(case.seen):
            lost = page in seen
            got = case.out[r].view(2, 4, 128)
            assert torch.equal(got[0], ref[r].view(2, 4, 128)[0])
            assert bool(torch.isnan(got[1]).all()) == lost and (lost or torch.equal(got[1], ref[r].view(2, 4, 128)[1])), r


def test_rows_that_are_not_finite_spoil_themselves_only():
    reqs = [[([], 300, 0), ([0], 3, 90)]]
    clean = Case(reqs, (8, 2, 128), 13)
    clean.run()
    case = Case(reqs, (8, 2, 128), 13)
    case.q[5, 3, 7], case.q[80, 0, 0] = float("nan"), float("inf")
    case.run()
    same = (case.out == clean.out).all(-1)
    assert sorted(map(tuple, (~same[:90]).nonzero().tolist())) == [(5, 3), (80, 0)]


def test_same_bits_on_every_call():
    case = Case(random_reqs(21), (32, 8, 128), 14)
    first = case.run().clone()
    for _ in range(3):
        case.out.fill_(7.0)
        case.ws.fill_(0)
        assert torch.equal(case.run(), first)


def test_smaller_tiles_of_the_callers_own():
    """rows_per_tile below the most: other tiles, the same rows."""
    B, rt = _mods()
    case = Case([[([], 33, 0), ([0], 7, 150)]], (16, 4, 128), 15)
    ref = case.run().clone()
    for per in (1, 7, 31, 32, 33):
        t = {"tiles": torch.zeros(400, 8, dtype=torch.int32, device="cuda"), "entries": torch.zeros(400, 2, dtype=torch.int32, device="cuda"),
             "counts": torch.zeros(8, dtype=torch.int32, device="cuda")}
        tables = B.ChunkTables(**t, max_rows=case.q.shape[0], rows_per_tile=per)
        B.mv_chunk_tables_build(case.chunk.batch, tables, case.chunk.workspace)
        case.out.fill_(7.0)
        B.mv_dag_chunk_attn_fp8_blk(tables, case.geom, case.q, case.k8, case.v8, case.scale, case.out, case.ws)
        assert B.mv_chunk_tables_read_status(tables) == 0
        case.check(rows=range(0, 150, 7))
        # sums are taken over the same key tiles, but may be cut elsewhere
        assert (case.out.float() - ref.float()).abs().max() <= 2.0 ** -5


@pytest.mark.parametrize("word,value", [(0, -1), (0, 1000), (1, 0), (1, 65), (2, -5), (2, 100000), (3, -1), (3, 90000), (4, -1), (4, 1 << 30), (5, -3), (6, 0), (6, 4), (6, 1 << 20)])
def test_records_that_do_not_fit_are_skipped(word, value):
    """A tile's record that would lead outside the arrays: the status says so, the rows of the other tile stand."""
    B, rt = _mods()
    case = Case([[([], 40, 64)], [([], 40, 64)]], (16, 4, 128), 16)
    good = case.run().clone()
    case.chunk.t["tiles"][1, word] = value
    case.out.fill_(7.0)
    B.mv_dag_chunk_attn_fp8_blk(case.chunk.tables, case.geom, case.q, case.k8, case.v8, case.scale, case.out, case.ws)
    assert B.mv_chunk_tables_read_status(case.chunk.tables) == 1
    if word != 5:      # (the key tiles before a tile say which CTA takes what: with a wrong count neighbours may be left out too)
        assert (case.out[64:] == 7).all() and torch.equal(case.out[:64], good[:64])


def test_pages_outside_the_pool_are_skipped():
    B, rt = _mods()
    for column, value in ((0, -1), (0, 10 ** 6), (1, 0), (1, 17)):
        case = Case([[([], 40, 64)], [([], 40, 64)]], (16, 4, 128), 17)
        good = case.run().clone()
        first = int(case.chunk.t["tiles"][1, 2])
        case.chunk.t["entries"][first + 1, column] = value
        case.out.fill_(7.0)
        B.mv_dag_chunk_attn_fp8_blk(case.chunk.tables, case.geom, case.q, case.k8, case.v8, case.scale, case.out, case.ws)
        assert B.mv_chunk_tables_read_status(case.chunk.tables) == 1
        assert torch.equal(case.out[:64], good[:64]) and torch.isfinite(case.out.float()).all()


def test_captured_step_grows():
    """Tables and attention captured once; the lengths on the device advance from replay to replay."""
    B, rt = _mods()
    reqs = [[([], 50, 0), ([0], 10, 40)], [([], 7, 33)]]
    grown = [[([], 50, 0), ([0], 50, 21)], [([], 40, 40)]]
    b0, b1 = batch_of(reqs, 18), None
    room = [[([], 50, 0), ([0], 60, 40)], [([], 50, 40)]]     # the same pages for both steps
    br = batch_of(room, 18)
    mk = lambda r: dataclasses.replace(br, node_len=np.asarray([n[1] for q in r for n in q], np.int32), node_new=np.asarray([n[2] for q in r for n in q], np.int32))
    steps = [mk(reqs), mk(grown)]
    case = Case(room, (8, 2, 128), 18, max_rows=90)
    case.chunk = rt.ChunkOnDevice(steps[0], 4, max_rows=90, max_tiles=8, max_entries=64)
    case.out = torch.full_like(case.q, 7.0)
    run = lambda: (case.chunk.build(), B.mv_dag_chunk_attn_fp8_blk(case.chunk.tables, case.geom, case.q, case.k8, case.v8, case.scale, case.out, case.ws))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        run()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        run()
    for b in (steps[1], steps[0], steps[1]):
        for name in ("node_len", "node_new"):
            case.chunk.arrays[name].copy_(torch.from_numpy(getattr(b, name)))
        case.out.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert case.chunk.read_status() == 0
        case.b, case.seen = b, visible_counts(b)
        case.check(rows=range(0, len(case.seen), 5))


def test_tensors_aligned_to_16_bytes_only():
    """q_rot and out at addresses that are multiples of 16 bytes and not of 32."""
    case = Case([[([], 40, 0), ([0], 3, 90)]], (8, 2, 128), 19, max_rows=95)
    ref = case.run().clone()
    room = [torch.full((case.q.numel() + 8,), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    shifted = [x[8:].view(case.q.shape) for x in room]
    assert all(x.data_ptr() % 32 == 16 for x in shifted)
    shifted[0].copy_(case.q)
    case.q, case.out = shifted
    assert torch.equal(case.run(), ref) and (room[1][:8] == 7).all()


def test_two_streams_with_workspaces_of_their_own():
    cases = [Case(random_reqs(30 + i), (32, 8, 128), 30 + i) for i in range(2)]
    refs = [c.run().clone() for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for _ in range(5):
        for c, s in zip(cases, streams):
            c.B.mv_dag_chunk_attn_fp8_blk(c.chunk.tables, c.geom, c.q, c.k8, c.v8, c.scale, c.out, c.ws, s)
    torch.cuda.synchronize()
    assert all(torch.equal(c.out, r) for c, r in zip(cases, refs))


def test_chunk_by_chunk_is_the_prompt_at_once():
    """A prompt written and attended in pieces against the same prompt in one step, and single tokens against the decode call."""
    B, rt = _mods()
    n, hq, hkv, d = 157, 8, 2, 128
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    pages = (n + 15) // 16 + 2
    geom = B.make_geom(hq, hkv, d, pages, "bf16")
    ids = np.random.default_rng(5).permutation(pages).astype(np.int32)[:(n + 15) // 16]

    def run(cuts, last_by_decode=False):
        k8, v8 = (torch.zeros(pages, hkv, 16, d, dtype=torch.uint8, device="cuda") for _ in range(2))
        sc = torch.zeros(pages, hkv, 2, device="cuda")
        out = torch.zeros(n, hq, d, dtype=torch.bfloat16, device="cuda")
        ws = torch.empty(B.mv_chunk_attn_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
        for a, z in zip(cuts[:-1], cuts[1:]):
            one = lambda x: np.asarray([x], np.int32)
            b = synth.DagBatch(1, np.asarray([0, 1], np.int32), one(a), one(z - a), np.asarray([0, 0], np.int32), np.zeros(0, np.int32), np.asarray([0, len(ids)], np.int32),
                               ids, 16, pages)
            c = rt.ChunkOnDevice(b, hq // hkv)
            t = c.build()
            part = [x[a:z].contiguous() for x in (q, k, v)]
            qr, o = torch.empty_like(part[0]), torch.empty_like(part[0])
            B.mv_rope_write_kv_fp8_blk(c.steps.tables, geom, *part, qr, None, k8, v8, sc)
            B.mv_dag_chunk_attn_fp8_blk(t, geom, qr, k8, v8, sc, o, ws)
            assert c.read_status() == 0
            if last_by_decode and z == n:
                s = rt.StepOnDevice(b, hq // hkv)
                dws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
                o2 = torch.empty_like(o)
                B.mv_dag_decode_attn_fp8_blk(s.build(), geom, qr, k8, v8, sc, o2, dws)
                assert (o2.float() - o.float()).abs().max() <= 2.0 ** -6 * 3      # both within 2^-8 (|out| + 2 A), A below 3 here
            out[a:z] = o
        return out, k8, v8, sc

    # the pages' scales grow with what is written, and what a page held moves to a larger scale without loss but among the subnormals:
    # with every page's scale fixed beforehand by its largest element there is nothing to move
    k[:, :, 0], v[:, :, 0] = 6.0, 6.0
    whole, *cache = run([0, n])
    for cuts in ([0, 16, 157], [0, 1, 2, 3, 100, 156, 157], [0, 64, 128, 157]):
        got, *c2 = run(cuts, cuts[-2] == 156)
        assert all(torch.equal(x, y) for x, y in zip(cache, c2))
        assert (got.float() - whole.float()).abs().max() <= 2.0 ** -6 * 7         # |out|, A below 7


def test_runtime_state_against_the_definition():
    """History, write and attention through the runtime's state, with the geometry's own rotation and with a form."""
    B, rt = _mods()
    wl = synth.config2(n_req=3, prefix=100, branches=3, branch_len=40, new_tokens=21)
    for form in (None, B.RopeForm(B.ROPE_PAIRS, 64, first=32, base=5e5)):
        st = rt.ChunkStateFP8Blk(wl, form=form)
        out = st.step()
        assert st.chunk.read_status() == 0
        seen = visible_counts(wl.batch)
        g = wl.geom
        case = Case.__new__(Case)
        case.b, case.seen, case.hq, case.hkv, case.d = wl.batch, seen, g.n_q_heads, g.n_kv_heads, g.head_dim
        case.geom, case.q, case.k8, case.v8, case.scale, case.out = st.geom, st.q_rot, st.k_pages, st.v_pages, st.kv_scale, out
        case.check(rows=range(0, len(seen), 11))


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (5, 5, 128), (148, 148, 64)])
@pytest.mark.parametrize("held", [(0,), (400, 3), (600, 20, 1), (9000,), (20, 5000, 700, 130, 1, 1)])
def test_few_tiles_of_unlike_lengths(heads, held):
    """Steps of few query tiles, whose lists stay whole, are cut into equal pieces, or lie on the line where they are too unlike."""
    case = Case([[([], n, 0 if n else 3), ([0], 0, 1 + i)] for i, n in enumerate(held)], heads, 41, max_rows=40)
    case.run()
    case.check(rows=range(0, len(case.seen), 3))
