"""What a cloned request and its original read afterwards, token by token: the common past, then each its own tokens only."""
import numpy as np
import pytest

from paper_2602_07529_b200 import binding as B
from test_pages_host import NET, Model

SEES = {1: (0, 1), 2: (0, 2), 3: (0, 1, 2, 3), 4: (0, 1, 2, 3, 4)}
LENGTH = NET[1]                       # 21 30 19 18 5: nodes 1 and 2 run together, then 3, then 4
STARTS = {1: 0, 2: 0, 3: 30, 4: 48}   # the step that writes a node's first token


def mark(req, node, t):
    return (req + 1) * 100000 + node * 1000 + t


def written(node, steps):
    """Tokens of the node after so many steps."""
    return LENGTH[0] if node == 0 else max(0, min(LENGTH[node], steps - STARTS[node]))


def play(at, copies=True):
    """Clones after `at` steps and plays to the end.  Rows (step, request, node) that read anything but what they should."""
    s, m = B.Scheduler(16, 64), Model(64)
    a = s.add_request(*NET)
    wrong, clone, pages = [], None, 0
    for step in range(sum(LENGTH)):
        if step == at:
            clone, src, dst = s.clone_request(a)
            pages = len(src)
            if copies:
                m.copy(src, dst)
        if step == 0:     # the prompt's marks, once its pages are known
            first = s.step()
            if first is not None:
                for i in range(LENGTH[0]):
                    m.page[first["page_idx"][i // 16], i % 16] = 1000 + i
        seen = m.step(s, lambda key, t: mark(*key, t))
        if seen is None:
            break
        both = [a] if clone is None else [a, clone]
        nodes = [v for v in SEES if STARTS[v] <= step < STARTS[v] + LENGTH[v]]
        assert sorted(seen) == sorted((r, v) for r in both for v in nodes)
        for (req, node), lists in seen.items():
            want = []
            for u in SEES[node]:
                past = written(u, at) if req != a else written(u, step + 1)    # by the original; the rest by the request itself
                want.append([1000 + t if u == 0 else mark(a if t < past else req, u, t) for t in range(written(u, step + 1))])
            if lists != want:
                wrong.append((step, req, node))
        s.commit()
    assert step == 53 and s.stats()["pages_in_use"] == 0 and s.stats()["requests_live"] == 0 and (s.page_refs(range(64)) == 0).all()
    return wrong, pages


CLONED_AT = [0, 1, 15, 16, 17, 18, 19, 20, 29, 30, 31, 40, 46, 47, 48, 49, 52]


@pytest.mark.parametrize("at", CLONED_AT)
def test_each_reads_the_common_past_and_its_own(at):
    wrong, pages = play(at)
    assert wrong == []
    assert pages == sum(0 < written(v, at) < LENGTH[v] and written(v, at) % 16 != 0 for v in SEES)


@pytest.mark.parametrize("at", CLONED_AT)
def test_a_copy_that_is_left_out_is_seen(at):
    """The clone then reads what its new pages held before, from the step after the clone on; the original reads what it should."""
    wrong, pages = play(at, copies=False)
    assert bool(wrong) == (pages > 0) and all(req != 0 for _, req, _ in wrong)
    if pages:
        assert wrong[0][0] == at
