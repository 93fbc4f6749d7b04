"""Host-side refusals of the device-planned decode path: every one is found before anything is launched, so the C entry
points are called here with addresses that are never followed."""
import ctypes as C

import pytest

from paper_2602_07529_b200 import binding as B

OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 4, 5
P = 0x100000  # an aligned address nobody reads


def tables(**kw):
    t = B._StepTables(16, 4, 64, 4, *([P] * 7))
    for k, v in kw.items():
        setattr(t, k, v)
    return t


def batch(**kw):
    b = B._DagBatch(2, *([P] * 7), 16, 0, 0)
    for k, v in kw.items():
        setattr(b, k, v)
    return b


def shape(**kw):
    s = B._StepShape(6, 8, 40, 6, 100)
    for k, v in kw.items():
        setattr(s, k, v)
    return s


def build(b=None, s=None, t=None, ws=P, ws_bytes=1 << 20):
    ref = lambda x: None if x is None else C.byref(x)
    return B.lib.mv_step_tables_build(ref(b), ref(s), ref(t), ws, ws_bytes, None)


@pytest.mark.parametrize("b,s,t,want", [
    (None, {}, {}, INVALID), ({}, None, {}, INVALID), ({}, {}, None, INVALID),
    ({"n_req": -1}, {}, {}, INVALID), ({"page_size": 32}, {}, {}, INVALID), ({"vis_mode": 2}, {}, {}, INVALID),
    ({"pos_mode": -1}, {}, {}, INVALID), ({"node_off": None}, {}, {}, INVALID), ({"node_len": None}, {}, {}, INVALID),
    ({"parent_idx": None}, {}, {}, INVALID), ({"page_idx": None}, {}, {}, INVALID), ({}, {"n_nodes": -1}, {}, INVALID),
    ({}, {"num_pages": -5}, {}, INVALID), ({}, {"max_req_nodes": 0}, {}, UNSUPPORTED), ({}, {"max_req_nodes": 2049}, {}, UNSUPPORTED),
    ({}, {}, {"max_rows": -1}, INVALID), ({}, {}, {"pos_id": None}, INVALID), ({}, {}, {"counts": None}, INVALID),
    ({}, {}, {"rows_per_group": 0}, UNSUPPORTED), ({}, {}, {"rows_per_group": 65}, UNSUPPORTED),
    ({}, {}, {"group_tile_off": None}, INVALID), ({}, {}, {"entries": None}, INVALID), ({}, {}, {"entries": P + 4}, INVALID),
])
def test_build_refuses(b, s, t, want):
    assert build(None if b is None else batch(**b), None if s is None else shape(**s), None if t is None else tables(**t)) == want


def test_build_refuses_workspaces():
    need = B.lib.mv_step_tables_workspace_bytes(2)
    assert need > 0 and need % 256 == 0 and B.lib.mv_step_tables_workspace_bytes(5000) >= 5000 * 20
    for ws, n in ((None, need), (P, need - 1), (P + 128, need)):
        assert build(batch(), shape(), tables(), ws, n) == WORKSPACE
    assert B.lib.mv_step_tables_read_status(None, None, C.byref(C.c_int32())) == INVALID


def write(t, g, ptrs):
    return B.lib.mv_rope_write_kv_fp8_blk(None if t is None else C.byref(t), C.byref(g), *ptrs, None)


def test_write_refuses():
    g = B.make_geom(8, 2, 128, 100, "bf16")
    good = [P] * 8  # q, k, v, q_rot, k_rot, k_pages, v_pages, scale
    assert write(None, g, good) == INVALID
    assert write(tables(counts=None), g, good) == INVALID
    assert write(tables(slot=None), g, good) == INVALID
    assert write(tables(), B.make_geom(8, 2, 128, 100, "f32"), good) == UNSUPPORTED
    assert write(tables(), B.make_geom(8, 2, 96, 100, "bf16"), good) == UNSUPPORTED
    assert write(tables(), B.make_geom(8, 3, 128, 100, "bf16"), good) == UNSUPPORTED
    assert write(tables(), B.make_geom(8, 2, 128, 100, "bf16", rope_base=-1.0), good) == INVALID
    for i in range(8):
        if i != 4:  # k_rot is optional
            assert write(tables(), g, good[:i] + [None] + good[i + 1:]) == INVALID, i
        assert write(tables(), g, good[:i] + [P + 8] + good[i + 1:]) == INVALID, i
    assert write(tables(max_rows=0), g, [None] * 8) == OK  # nothing to write, nothing launched


def attend(t, g, ptrs, ws=P, n=None):
    n = B.lib.mv_decode_fp8_blk_workspace_bytes(C.byref(g)) if n is None else n
    return B.lib.mv_dag_decode_attn_fp8_blk(None if t is None else C.byref(t), C.byref(g), *ptrs, ws, n, None)


def test_attention_refuses():
    g = B.make_geom(8, 2, 128, 100, "bf16")
    need = B.lib.mv_decode_fp8_blk_workspace_bytes(C.byref(g))
    good = [P] * 5  # q, k_pages, v_pages, scale, out
    assert attend(None, g, good) == INVALID
    assert attend(tables(counts=None), g, good) == INVALID
    assert attend(tables(max_entries=-1), g, good) == INVALID
    assert attend(tables(group_ent_off=None), g, good) == INVALID
    assert attend(tables(entries=None), g, good) == INVALID
    assert attend(tables(), B.make_geom(8, 2, 128, 100, "f32"), good) == UNSUPPORTED
    assert attend(tables(), B.make_geom(130, 1, 128, 100, "bf16"), good) == UNSUPPORTED     # 130 query heads of one KV head
    assert attend(tables(rows_per_group=17), g, good) == UNSUPPORTED                        # 17 * 4 > 64
    assert attend(tables(rows_per_group=0), g, good) == UNSUPPORTED
    for i in range(5):
        assert attend(tables(), g, good[:i] + [None] + good[i + 1:]) == INVALID, i
        assert attend(tables(), g, good[:i] + [P + 8] + good[i + 1:]) == INVALID, i
    for ws, n in ((None, need), (P, need - 1), (P + 64, need)):
        assert attend(tables(), g, good, ws, n) == WORKSPACE
    assert attend(tables(), B.make_geom(8, 2, 128, 2 ** 31 // 32, "bf16"), good) == UNSUPPORTED  # rows of the pool beyond 31 bits
    assert attend(tables(max_entries=2 ** 31 - 1), B.make_geom(8, 8, 128, 100, "bf16"), good) == UNSUPPORTED
    assert attend(tables(max_rows=0), g, [None] * 5) == OK
    assert attend(tables(max_groups=0), g, [None] * 5) == OK
    assert B.lib.mv_decode_fp8_blk_workspace_bytes(C.byref(B.make_geom(8, 2, 96, 100, "bf16"))) == 0


def test_binding_checks_tensors():
    """The Python wrappers look at what the C calls cannot see: dtype, layout, size and device."""
    import torch
    i32 = lambda n: torch.zeros(n, dtype=torch.int32)
    with pytest.raises(ValueError, match="node_off"):
        B.DeviceBatch(1, i32(2), i32(1), i32(1), i32(2), i32(1), i32(2), i32(1), num_pages=4, max_req_nodes=1)
    with pytest.raises(ValueError, match="pos_id"):
        B.StepTables(i32(4), torch.zeros(4, dtype=torch.int64), i32(8))
