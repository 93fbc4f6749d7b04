"""The captured decode step where it has to stop, and q-vectors that are not numbers."""
import numpy as np
import pytest
import torch

from test_gpu_fp8_blk import _batch_of, _mods, pools_of

pytestmark = pytest.mark.gpu


def test_captured_step_that_finds_no_room_touches_nothing():
    """Replays go on after a node's pages are full: the step reports it and leaves cache, scales and outputs as they were."""
    B, runtime = _mods()
    hq, hkv, d, room = 16, 4, 128, 3
    batch = _batch_of([[([], 40, 0), ([0], 13, 1), ([0], 16, 1)], [([], 20, 0), ([0], 13, 1)]])   # nodes of 13 tokens: room for three more
    geom = B.make_geom(hq, hkv, d, batch.num_pages, "bf16")
    step = runtime.StepOnDevice(batch, hq // hkv, max_entries=600)
    n = step.tables.max_rows
    k8, v8, sc = pools_of(batch.num_pages, hkv, d, 81)
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    q, k, v = (torch.randn(n, h, d, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    q_rot, k_rot, out = torch.zeros_like(q), torch.zeros_like(k), torch.zeros_like(q)

    def one():
        t = step.build()
        B.mv_rope_write_kv_fp8_blk(t, geom, q, k, v, q_rot, k_rot, k8, v8, sc)
        B.mv_dag_decode_attn_fp8_blk(t, geom, q_rot, k8, v8, sc, out, ws)
        step.arrays["node_len"] += step.arrays["node_new"]

    one()
    torch.cuda.synchronize()
    step.arrays["node_len"] -= step.arrays["node_new"]
    graph = torch.cuda.CUDAGraph()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        one()
    for _ in range(room):
        graph.replay()
        assert step.read_status() == 0
    state = [x.clone() for x in (k8, v8, sc, q_rot, k_rot, out)]
    for x in (q, k, v):
        x.mul_(2.0)
    for _ in range(3):
        graph.replay()
        assert step.read_status() == 3
        assert step.t["counts"].tolist() == [0, 0, 0, 0, 3, 0, 0, 0]
        for x, y in zip(state, (k8, v8, sc, q_rot, k_rot, out)):
            assert torch.equal(x, y)
    del graph


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_a_q_vector_that_is_not_finite_spoils_itself_only(d, bad):
    B, runtime = _mods()
    batch = _batch_of([[([], 1500 + 40 * r, 0)] + [([0], 9 * b, 1) for b in range(8)] for r in range(30)])
    step = runtime.StepOnDevice(batch, 4)
    step.build()
    geom = B.make_geom(16, 4, d, batch.num_pages, "bf16")
    pools = pools_of(batch.num_pages, 4, d, 5)
    ws = torch.empty(B.mv_decode_fp8_blk_workspace_bytes(geom), dtype=torch.uint8, device="cuda")
    q = torch.randn(step.tables.max_rows, 16, d, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda").bfloat16()
    clean, dirty = torch.empty_like(q), torch.empty_like(q)
    B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, *pools, clean, ws)
    lost = torch.zeros(q.shape[:2], dtype=torch.bool, device="cuda")
    lost[3, 2] = lost[100, 15] = lost[170] = True
    q[lost, d - 3] = bad
    B.mv_dag_decode_attn_fp8_blk(step.tables, geom, q, *pools, dirty, ws)
    assert step.read_status() == 0
    assert torch.isnan(dirty[lost]).all() and torch.equal(dirty[~lost], clean[~lost])
