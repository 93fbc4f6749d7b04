"""Host-side refusals of the chunk tables and the chunk attention (nothing is launched: the addresses are never followed)."""
import ctypes as C
import math

import pytest

from paper_2602_07529_b200 import binding as B
from test_step_refusals import INVALID, OK, P, UNSUPPORTED, WORKSPACE, batch, shape


def tables(**kw):
    t = B._ChunkTables(64, 4, 64, 32, P, P, P)
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def build(b=None, s=None, t=None, ws=P, ws_bytes=1 << 20):
    ref = lambda x: None if x is None else C.byref(x)
    return B.lib.mv_chunk_tables_build(ref(b), ref(s), ref(t), ws, ws_bytes, None)


@pytest.mark.parametrize("b,s,t,want", [
    (None, {}, {}, INVALID), ({}, None, {}, INVALID), ({}, {}, None, INVALID),
    ({"n_req": -1}, {}, {}, INVALID), ({"page_size": 32}, {}, {}, INVALID), ({"vis_mode": 2}, {}, {}, INVALID),
    ({"node_off": None}, {}, {}, INVALID), ({"node_new": None}, {}, {}, INVALID), ({"parent_idx": None}, {}, {}, INVALID),
    ({"page_idx": None}, {}, {}, INVALID), ({}, {"n_pages": -1}, {}, INVALID), ({}, {"num_pages": -5}, {}, INVALID),
    ({}, {"max_req_nodes": 0}, {}, UNSUPPORTED), ({}, {"max_req_nodes": 2049}, {}, UNSUPPORTED),
    ({}, {}, {"max_rows": -1}, INVALID), ({}, {}, {"max_tiles": -1}, INVALID), ({}, {}, {"max_entries": -1}, INVALID),
    ({}, {}, {"tiles": None}, INVALID), ({}, {}, {"entries": None}, INVALID), ({}, {}, {"counts": None}, INVALID),
    ({}, {}, {"tiles": P + 8}, INVALID), ({}, {}, {"entries": P + 4}, INVALID), ({}, {}, {"counts": P + 2}, INVALID),
    ({}, {}, {"rows_per_tile": 0}, UNSUPPORTED), ({}, {}, {"rows_per_tile": 257}, UNSUPPORTED),
])
def test_build_refuses(b, s, t, want):
    assert build(None if b is None else batch(**b), None if s is None else shape(**s), None if t is None else tables(**t)) == want


def test_build_refuses_workspaces():
    need = B.lib.mv_chunk_tables_workspace_bytes(2)
    assert need > 0 and need % 256 == 0 and B.lib.mv_chunk_tables_workspace_bytes(5000) >= 5000 * 20
    for ws, n in ((None, need), (P, need - 1), (P + 128, need)):
        assert build(batch(), shape(), tables(), ws, n) == WORKSPACE
    assert B.lib.mv_chunk_tables_read_status(None, None, C.byref(C.c_int32())) == INVALID


def attend(t, g, p=(P, P, P, P, P + 4096), ws=P, ws_bytes=1 << 30):
    q, k, v, s, o = p
    return B.lib.mv_dag_chunk_attn_fp8_blk(C.byref(t) if t else None, C.byref(g) if g else None, q, k, v, s, o, ws, ws_bytes, None)


def test_attention_refuses():
    g = B.make_geom(32, 8, 128, 100, "bf16")   # G = 4: 64 rows per tile
    assert attend(None, g) == INVALID and attend(tables(), None) == INVALID
    for kw in ({"max_rows": -1}, {"max_tiles": -1}, {"max_entries": -1}, {"counts": None}, {"tiles": None}, {"entries": None}, {"tiles": P + 8},
               {"entries": P + 8}, {"counts": P + 1}):
        assert attend(tables(**kw), g) == INVALID, kw
    for kw in ({"rows_per_tile": 0}, {"rows_per_tile": 65}):
        assert attend(tables(**kw), g) == UNSUPPORTED
    for i in range(5):
        for bad in (None, P + 8):
            p = [P, P, P, P, P + 4096]
            p[i] = bad
            assert attend(tables(), g, p) == INVALID
    assert attend(tables(), g, [P] * 5) == INVALID                       # out is q_rot
    assert attend(tables(max_rows=0), g) == OK
    assert attend(tables(max_tiles=0), g) == INVALID                     # rows that no tile could name, and an output that waits for them
    assert attend(tables(max_tiles=0), g, [None, P, P, P, None]) == OK
    need = B.lib.mv_chunk_attn_workspace_bytes(C.byref(g))
    assert need > 0 and B.lib.mv_chunk_attn_workspace_bytes(C.byref(B.make_geom(8, 3, 128, 1, "bf16"))) == 0
    for ws, n in ((None, need), (P, need - 1), (P + 128, need)):
        assert attend(tables(), g, ws=ws, ws_bytes=n) == WORKSPACE
    for bad in (math.nan, math.inf, -1.0):
        assert attend(tables(), B.make_geom(32, 8, 128, 100, "bf16", sm_scale=bad)) == INVALID
    for geom in (B.make_geom(32, 8, 128, 100, "f32"), B.make_geom(32, 8, 96, 100, "bf16"), B.make_geom(32, 7, 128, 100, "bf16"),
                 B.make_geom(129, 1, 128, 100, "bf16"), B.make_geom(32, 8, 128, 1 << 24, "bf16"), B.make_geom(32, 8, 128, 100, "bf16", page_size=32)):
        assert attend(tables(rows_per_tile=1), geom) == UNSUPPORTED
    assert attend(tables(max_tiles=1 << 30), g) == UNSUPPORTED


def test_attention_refuses_outputs_that_overlap_its_input():
    """q_rot and out have max_rows rows of 32 heads of 128: one may end where the other begins, no closer."""
    g, t = B.make_geom(32, 8, 128, 100, "bf16"), tables(max_rows=16)
    size, at = 16 * 32 * 128 * 2, 1 << 30
    for shift in (16, size - 16, -16, 16 - size):
        assert attend(t, g, (at, P, P, P, at + shift)) == INVALID, shift


def test_attention_refuses_a_scale_that_is_infinite_in_binary_logarithms():
    assert attend(tables(), B.make_geom(32, 8, 128, 100, "bf16", sm_scale=3.3e38), (1 << 30, P, P, P, 1 << 40)) == INVALID
