"""mv_pages_copy on the GPU: exact copies and nothing else changed."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def pools_of(n, sizes, seed):
    g = torch.Generator(device="cuda").manual_seed(seed)
    return [torch.randint(0, 256, (n, b), generator=g, dtype=torch.uint8, device="cuda") for b in sizes]


def check(n, sizes, src, dst, count=None, seed=0):
    from paper_2602_07529_b200 import binding as B
    pools = pools_of(n, sizes, seed)
    want = [p.clone() for p in pools]
    up = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    c = None if count is None else up([count])
    status = up([0])
    B.mv_pages_copy(B.PagePools(pools), up(src), up(dst), c, status)
    k = len(src) if count is None else max(0, min(count, len(src)))
    good = [(a, b) for a, b in zip(src[:k], dst[:k]) if 0 <= a < n and 0 <= b < n]
    for w in want:
        if good:
            w[[b for _, b in good]] = w[[a for a, _ in good]]
    assert all(torch.equal(p, w) for p, w in zip(pools, want))
    assert int(status) == (0 if len(good) == k else 1)


@pytest.mark.parametrize("sizes", [[32768], [16384, 16384, 64], [8, 4096, 12], [16400], [4], [65536 + 16, 48], [16384 + 4, 1020]])
def test_sizes(sizes):
    rng = np.random.default_rng(1)
    for n, moves in ((2, 1), (40, 17), (700, 333)):
        ids = rng.permutation(n).tolist()
        check(n, sizes, ids[:moves], ids[moves:2 * moves], seed=n)


def test_one_source_many_destinations_and_itself():
    check(50, [4096, 8], [3, 3, 3, 7, 9], [10, 11, 12, 7, 13])


def test_none():
    check(5, [64], [], [])


@pytest.mark.parametrize("count", [0, 1, 4, 5, 6, 1000, -3])
def test_count_on_the_device(count):
    check(30, [1024, 64, 8], [0, 1, 2, 3, 4], [10, 11, 12, 13, 14], count)


@pytest.mark.parametrize("bad", [-1, 30, 1 << 30, -(1 << 31)])
def test_pages_outside_are_skipped(bad):
    check(30, [4096, 8], [0, bad, 2, 3], [10, 11, 12, bad])


def test_many_pools():
    from paper_2602_07529_b200 import binding as B
    check(20, [256, 64, 8, 4] * 64, [1, 2], [3, 4])
    with pytest.raises(B.MvError, match="UNSUPPORTED"):
        check(4, [16] * 257, [1], [2])


def test_offsets_past_32_bits():
    """A pool of 5 GB: pages whose byte offsets need more than 32 bits."""
    from paper_2602_07529_b200 import binding as B
    n, b = 320, 16 << 20
    pool = torch.empty(n, b, dtype=torch.uint8, device="cuda")
    for p in (0, 300, 310, 5):
        pool[p] = p % 251
    up = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    B.mv_pages_copy(B.PagePools([pool]), up([300, 0]), up([5, 319]))
    assert (pool[5] == 300 % 251).all() and (pool[319] == 0).all() and (pool[310] == 310 % 251).all() and (pool[300] == 300 % 251).all()


def test_captured_and_on_another_stream():
    from paper_2602_07529_b200 import binding as B
    pools = pools_of(64, [4096, 64], 3)
    src, dst, count = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([1, 2, 3], [11, 12, 13], [2]))
    pp = B.PagePools(pools)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.mv_pages_copy(pp, src, dst, count)
    want = [p.clone() for p in pools]
    graph.replay()
    for w in want:
        w[[11, 12]] = w[[1, 2]]
    torch.cuda.synchronize()
    assert all(torch.equal(p, w) for p, w in zip(pools, want))
    src.copy_(torch.tensor([20, 21, 22]))
    count.fill_(3)
    graph.replay()
    for w in want:
        w[[11, 12, 13]] = w[[20, 21, 22]]
    torch.cuda.synchronize()
    assert all(torch.equal(p, w) for p, w in zip(pools, want))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.mv_pages_copy(pp, dst, src, stream=side)
    side.synchronize()
    assert all(torch.equal(p[20], p[11]) for p in pools)


def test_lists_from_the_host_outlive_the_call():
    """copy_pages on a stream that is still busy: the lists' memory is not handed out again before that stream has read it."""
    from paper_2602_07529_b200 import runtime
    pools = pools_of(64, [4096, 64], 4)
    want = [p.clone() for p in pools]
    for w in want:
        w[40:48] = w[8:16]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        torch.cuda._sleep(50_000_000)      # some tens of milliseconds
    runtime.copy_pages(pools, range(8, 16), range(40, 48), stream=side)
    runtime.copy_pages(pools, [], [], stream=side)
    later = [torch.full((8,), 63, dtype=torch.int32, device="cuda") for _ in range(8)]
    torch.cuda.synchronize()
    assert len(later) == 8 and all(torch.equal(p, w) for p, w in zip(pools, want))


def test_binding_refuses():
    from paper_2602_07529_b200 import binding as B
    pools = pools_of(8, [64, 16], 1)
    up = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    for bad in ([], [pools[0], pools[1][:4]], [pools[0].cpu()], [pools[0][:, :32]]):
        with pytest.raises(ValueError):
            B.PagePools(bad)
    pp = B.PagePools(pools)
    for a, b in ((up([1]), up([1, 2])), (up([1]).long(), up([2]).long()), (up([1]).cpu(), up([2]).cpu())):
        with pytest.raises(ValueError):
            B.mv_pages_copy(pp, a, b)


def test_cloned_request_decodes_like_its_own():
    """A request is cloned in mid-page and the pool compacted; its rows' attention is the same as the request's own."""
    from paper_2602_07529_b200 import binding as B, runtime, synth
    n, hq, hkv, d = 40, 8, 2, 128
    geom = synth.Geometry(hq, hkv, d)
    g = torch.Generator(device="cuda").manual_seed(2)
    rnd = lambda *s: torch.randn(*s, generator=g, device="cuda").bfloat16()
    c_geom = B.make_geom(hq, hkv, d, n, "bf16")
    kp, vp = rnd(*runtime.pool_shape(n, geom)), rnd(*runtime.pool_shape(n, geom))
    s = B.Scheduler(16, n)
    s.add_request([[], [0]], [20, 9])      # three pages, of which the clone's copies take the lower two
    a = s.add_request([[], [0], [0]], [37, 40, 40])

    def step(kp, vp, q, k, v):
        b = s.step()
        batch = synth.DagBatch(b["n_req"], b["node_off"], b["node_len"], b["node_new"], b["parent_off"], b["parent_idx"], b["page_off"], b["page_idx"], 16, n, 0, 0)
        pod = runtime.PlanOnDevice(batch, geom=geom)
        rows = len(b["row_req"])
        ws = torch.empty(pod.plan.workspace_bytes(c_geom, B.OP_DECODE_ATTN), dtype=torch.uint8, device="cuda")
        qr, out = torch.empty_like(q[:rows]), torch.empty_like(q[:rows])
        B.mv_rope_write_kv(pod.plan, c_geom, q[:rows].contiguous(), k[:rows].contiguous(), v[:rows].contiguous(), qr, None, kp, vp)
        B.mv_dag_decode_attn(pod.plan, c_geom, qr, kp, vp, out, ws)
        s.commit()
        return b, out

    for _ in range(11):      # the first request ends: its pages below are free again
        step(kp, vp, rnd(3, hq, d), rnd(3, hkv, d), rnd(3, hkv, d))
    b_id, src, dst = s.clone_request(a)
    assert len(src) == 2
    runtime.copy_pages([kp, vp], src, dst)
    src, dst, top = s.compact(100)
    assert len(src) > 0
    runtime.copy_pages([kp, vp], src, dst)
    # the same new tokens for the request and its clone give the same rows
    q, k, v = rnd(2, hq, d).repeat(2, 1, 1), rnd(2, hkv, d).repeat(2, 1, 1), rnd(2, hkv, d).repeat(2, 1, 1)
    for _ in range(7):
        b, out = step(kp, vp, q, k, v)
        assert list(b["row_req"]) == [a, a, b_id, b_id] and b["page_idx"].max() < top + 8
        x, y = out[:2].float(), out[2:].float()
        # the streams may be split differently: weights are rounded to bf16 (2^-9 of each, so of |V|) on either side, and both results (2^-8)
        assert torch.isfinite(x).all() and (x - y).abs().max() <= 2.0 ** -8 * float(vp.abs().max()) + 2.0 ** -7 * x.abs().max()
