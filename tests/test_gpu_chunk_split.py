"""Chunk attention with its lists cut, left whole and joined: no page of a list is lost or taken twice.

V counts: element e of a token's value is one where its page's place in the list is e modulo head_dim, and zero elsewhere, so an output element is
the share of the weight that falls on those pages, ref = sum of p_j over them.  Tolerance, fixed before the first run, relative to ref itself
(everything is positive): weights rounded to bf16, 2^-8; the result, 2^-8; scores off by at most 2^-16 S, S = sum |q_i k_i| times the softmax scale
(here at most 12, checked), which is below 2^-12 of a weight; powers, sums and the division 2^-12: together 2^-7 + 2^-11.
That every page counts is checked on the reference: each one's share of its element is at least four times that for rows that see it in full."""
import numpy as np
import pytest
import torch

from test_gpu_chunk import Case

pytestmark = pytest.mark.gpu

TOL = 2.0 ** -7 + 2.0 ** -11


def counting(reqs, heads, seed, max_entries=None, max_tiles=None):
    case = Case(reqs, heads, seed, k_size=0.25, max_rows=sum(n[2] for r in reqs for n in r) + 2)
    held, place = {}, {}
    for _, seen in case.seen:
        for at, (p, c) in enumerate(seen.items()):
            held[p] = max(held.get(p, 0), c)
            place.setdefault(p, at)
    for p, c in held.items():
        case.v8[p, :, :c] = 0
        case.v8[p, :, :c, place[p] % case.d] = 0x38     # one
    case.place = place
    if max_entries or max_tiles:
        from paper_2602_07529_b200 import runtime
        t = case.chunk.tables
        case.chunk = runtime.ChunkOnDevice(case.b, heads[0] // heads[1], max_rows=t.max_rows, max_entries=max_entries, max_tiles=max_tiles)
        case.chunk.build()
        assert case.chunk.read_status() == 0
    return case


def check(case):
    g, hkv, d = case.hq // case.hkv, case.hkv, case.d
    least = 1.0
    for r, (_, seen) in enumerate(case.seen):
        page = torch.tensor(list(seen), device="cuda")
        count = torch.tensor(list(seen.values()), device="cuda")
        there = torch.arange(16, device="cuda") < count[:, None]
        k = case.k8[page].view(torch.float8_e4m3fn).double() * case.scale[page][..., 0].double()[..., None, None]      # [page][head][16][d]
        q = case.q[r].double().view(hkv, g, d)
        S = torch.einsum("hgd,phtd->hgpt", q.abs(), k.nan_to_num().abs())[:, :, there].amax() * d ** -0.5
        assert float(S) <= 12
        score = torch.einsum("hgd,phtd->hgpt", q, k.nan_to_num()) * d ** -0.5
        score = score.masked_fill(~there, -torch.inf)
        w = torch.softmax(score.flatten(2), -1).view(score.shape).sum(-1)                   # a page's weight
        cls = torch.tensor([case.place[p] % d for p in seen], device="cuda")
        ref = torch.zeros(hkv, g, d, dtype=torch.float64, device="cuda").index_add_(2, cls, w)
        got = case.out[r].double().view(hkv, g, d)
        assert ((got - ref).abs() <= TOL * ref).all(), (r, float(((got - ref).abs() / ref.clamp(min=1e-30)).max()))
        full = count == 16
        if full.any():
            least = min(least, float((w / ref[:, :, cls])[:, :, full].min()))
    assert least >= 4 * TOL, least
    assert (case.out[len(case.seen):] == 7).all()


@pytest.mark.parametrize("heads", [(32, 8, 128), (64, 8, 128), (8, 2, 64), (8, 1, 64), (5, 5, 128)])
@pytest.mark.parametrize("held,new", [(2000, 3), (6001, 37), (1030, 300)])
def test_cut_lists(held, new, heads):
    """Few rows over a history: cut over the SMs and joined."""
    case = counting([[([], held, 0), ([0], 5, new)]], heads, held + new)
    case.run()
    check(case)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (64, 8, 64)])
@pytest.mark.parametrize("room", [None, 4000])
@pytest.mark.parametrize("tiles", [1, 2, 3, 4, 5, 6, 9, 17])
def test_short_lists_whole_and_cut(tiles, room, heads):
    """Lists around the lengths up to which they stay whole, in tables just large enough (there the joining launch may be left out) and in roomy ones."""
    case = counting([[([], 128 * tiles - 40, 40)]], heads, tiles, max_entries=room)
    case.run()
    check(case)


@pytest.mark.parametrize("heads", [(32, 8, 128), (8, 2, 64), (16, 16, 64)])
@pytest.mark.parametrize("n_req,held,new", [(16, 350, 10), (5, 900, 120), (16, 90, 40), (3, 130, 500)])
def test_many_lists(n_req, held, new, heads):
    """More lists than stay with one share each: lengths that differ, some cut, some whole."""
    case = counting([[([], held + 37 * i, 0), ([0], 3, new + i % 3)] for i in range(n_req)], heads, n_req + held)
    case.run()
    check(case)


def test_more_query_tiles_than_are_dealt():
    """40 query tiles of one request and of several: the shares of the line of cost end inside lists."""
    for reqs in ([[([], 700, 0), ([0], 0, 2500)]], [[([], 500 + 100 * i, 0)] + [([0], 4, 9 + j) for j in range(9)] for i in range(5)]):
        case = counting(reqs, (8, 2, 64), 77)
        case.run()
        check(case)
