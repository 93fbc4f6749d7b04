"""Page copies on the host side: refusals of the call, and the lists the scheduler makes (clones of a request, compaction)."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_07529_b200 import binding as B
from test_step_refusals import INVALID, OK, P, UNSUPPORTED


def copy(pools=((P, 64),), num_pages=10, src=P, dst=P, n=4, count=None, status=None):
    arr = (B._PagePool * max(1, len(pools)))(*[B._PagePool(*p) for p in pools])
    return B.lib.mv_pages_copy(arr, len(pools), num_pages, src, dst, n, count, status, None)


def test_copy_refuses():
    assert copy(n=0) == OK and copy(num_pages=0) == OK and copy(n=0, src=None, dst=None) == OK
    assert B.lib.mv_pages_copy(None, 1, 10, P, P, 4, None, None, None) == INVALID
    for kw in ({"pools": ()}, {"pools": ((None, 64),)}, {"pools": ((P, 0),)}, {"pools": ((P, -16),)}, {"pools": ((P, 66),)}, {"pools": ((P + 2, 64),)},
               {"num_pages": -1}, {"n": -1}, {"src": None}, {"dst": None}, {"src": P + 1}, {"dst": P + 2}, {"count": P + 3}, {"status": P + 1}):
        assert copy(**kw) == INVALID, kw
    for kw in ({"pools": ((P, 64),) * 257}, {"num_pages": 1 << 31}, {"pools": ((P, (1 << 31) + 16),)}, {"pools": ((P, 1 << 31),), "n": (1 << 31) - 1}):
        assert copy(**kw) == UNSUPPORTED, kw


class Model:
    """The content of a pool under the scheduler's rules: every page holds (request lineage, node, index) marks of its 16 tokens."""

    def __init__(self, n):
        self.page = np.zeros((n, 16), np.int64)

    def copy(self, src, dst):
        assert not set(src.tolist()) & set(dst.tolist()) and len(set(dst.tolist())) == len(dst)
        self.page[dst] = self.page[src]

    def step(self, s, tok):
        """Writes a mark for each row's token; returns what every row sees: {(request, node): marks of the nodes it reads}."""
        b = s.step()
        if b is None:
            return None
        seen, row = {}, 0
        for r in range(b["n_req"]):
            lo, hi = b["node_off"][r], b["node_off"][r + 1]
            pages = [b["page_idx"][b["page_off"][v]:b["page_off"][v + 1]] for v in range(lo, hi)]
            parents = [b["parent_idx"][b["parent_off"][v]:b["parent_off"][v + 1]] for v in range(lo, hi)]
            vis = []
            for v in range(hi - lo):
                vis.append({v}.union(*[vis[p] for p in parents[v]]))
            here = []
            for v in range(hi - lo):
                if b["node_new"][lo + v]:
                    t = b["node_len"][lo + v]
                    key = (int(b["row_req"][row]), int(b["row_node"][row]))
                    self.page[pages[v][t // 16], t % 16] = tok(key, int(t))
                    here.append((key, v))
                    row += 1
            for key, v in here:
                seen[key] = [[int(self.page[pages[u][i // 16], i % 16]) for i in range(b["node_len"][lo + u] + b["node_new"][lo + u])] for u in sorted(vis[v])]
        return seen


NET = ([[], [0], [0], [1, 2], [3]], [21, 30, 19, 18, 5])


@pytest.mark.parametrize("at", [0, 1, 15, 16, 17, 20, 31, 40])
def test_clone_shares_what_is_complete(at):
    s, m = B.Scheduler(16, 64), Model(64)
    a = s.add_request(*NET)
    # the prompt's marks
    first = s.step()
    for i in range(21):
        m.page[first["page_idx"][i // 16], i % 16] = 1000 + i
    tok = lambda key, t: (key[0] + 1) * 100000 + key[1] * 1000 + t
    for _ in range(at):
        m.step(s, tok)
        s.commit()
    if at == 0:
        s.commit(np.zeros(2, np.uint8))
    before = s.stats()["pages_in_use"]
    b, src, dst = s.clone_request(a)
    done = at if at else 1
    running = [n for n, k in ((30, 1), (19, 2)) if done < n] if done < 30 else [18]
    left = done if done < 30 else done - 30
    want = len(running) if left % 16 else 0
    assert len(src) == len(dst) == want and s.stats()["pages_in_use"] == before + want and b == a + 1
    m.copy(src, dst)
    # from here on both write their own tokens; each sees the common past and its own future only
    history = {}
    while True:
        seen = m.step(s, tok)
        if seen is None:
            break
        for (req, node), marks in seen.items():
            other = 2 - req      # marks begin with the request's number + 1
            for x in sum(marks, []):
                assert x < 100000 or x // 100000 == 1 or req == b
                if req == a:
                    assert x // 100000 != 2
            mine = marks[-1]
            written = [t for t, x in enumerate(mine) if x // 100000 == req + 1]
            history.setdefault((req, node), []).append(len(mine))
        s.commit()
    for node in (3, 4):
        assert history[(a, node)] == history[(b, node)]
    assert s.stats()["pages_in_use"] == 0 and s.stats()["requests_live"] == 0
    assert (s.page_refs(range(64)) == 0).all()


def test_clone_refuses():
    s = B.Scheduler(16, 4)
    a = s.add_request([[], [0]], [16, 20])
    for bad in (-1, 1, 7):
        with pytest.raises(B.MvError, match="INVALID"):
            s.clone_request(bad)
    s.step()
    with pytest.raises(B.MvError, match="INVALID"):
        s.clone_request(a)                      # between a step and its commit
    with pytest.raises(B.MvError, match="INVALID"):
        s.compact(4)
    s.commit()
    clones = [s.clone_request(a)[0] for _ in range(2)]
    with pytest.raises(B.MvError, match="PAGE_CAPACITY"):
        s.clone_request(a)                      # the pool is used up; nothing has changed
    assert s.stats()["requests_live"] == 3 and s.stats()["pages_in_use"] == 4 and clones == [1, 2]
    assert list(s.page_refs(range(4))) == [6, 1, 1, 1]     # the prompt's page: three owners, three readers
    n = C.c_int32(0)
    rid = C.c_int32(0)
    assert B.lib.mv_sched_clone_request(s._h, a, C.byref(rid), 0, None, None, C.byref(n)) == 5 and n.value == 1
    assert B.lib.mv_sched_compact(s._h, -1, None, None, C.byref(n), None) == INVALID
    assert B.lib.mv_sched_compact(s._h, 2, None, None, C.byref(n), None) == INVALID
    assert B.lib.mv_sched_compact(None, 0, None, None, C.byref(n), None) == INVALID


@pytest.mark.parametrize("seed", range(6))
@pytest.mark.parametrize("most", [0, 1, 3, 1000])
def test_compaction_changes_nothing_that_is_seen(seed, most):
    """Random requests come, are cloned and end; the pool is compacted now and then.  What rows see is what they see without it."""
    def play(compact):
        rng = np.random.default_rng(seed)
        s, m = B.Scheduler(16, 200), Model(200)
        out = []
        tok = lambda key, t: (key[0] + 1) * 100000 + key[1] * 1000 + t
        for step in range(120):
            if rng.random() < 0.15 and s.stats()["pages_in_use"] < 100:
                s.add_request([[], [0], [0], [1, 2]], [int(x) for x in rng.integers(1, 40, 4)])
            if rng.random() < 0.1:
                try:
                    _, src, dst = s.clone_request(int(rng.integers(0, 5)))
                    m.copy(src, dst)
                except B.MvError:
                    pass
            go = rng.random() < 0.3
            if compact and go:
                used = (s.page_refs(range(200)) > 0)
                src, dst, top = s.compact(most)
                m.copy(src, dst)
                now = (s.page_refs(range(200)) > 0)
                assert now.sum() == used.sum() and len(src) <= most and used[src].all() and not used[dst].any() and (src > dst).all()
                assert top == (int(np.flatnonzero(now)[-1]) + 1 if now.any() else 0)
                if most == 1000:
                    assert now[:now.sum()].all()
            seen = m.step(s, tok)
            if seen is not None:
                out.append({k: [[x for x in n if x] for n in v] for k, v in seen.items()})
                s.commit()
        return out
    a, b = play(False), play(True)
    # prompts are never written here, so pages hold zeros or left-overs there: compare the marks of steps (rows' own lineage)
    keep = lambda run: [{k: [[x for x in n if x // 100000] for n in v[1:]] for k, v in step.items()} for step in run]
    assert keep(a) == keep(b)
