"""Refusals of the block-scaled decode path that say what a call would silently leave undone (host side, nothing is launched)."""
from paper_2602_07529_b200 import binding as B
from test_step_refusals import INVALID, OK, P, attend, tables


def test_attention_refuses_tables_without_groups():
    """Tables of positions and slots only: the call has no group to answer for, so tensors that wait for an answer are refused."""
    g = B.make_geom(8, 2, 128, 100, "bf16")
    assert attend(tables(max_groups=0, max_entries=0), g, [P] * 5) == INVALID
    assert attend(tables(max_groups=0), g, [P, P, P, P, None]) == INVALID
    assert attend(tables(max_groups=0), g, [None, P, P, P, P]) == INVALID
    assert attend(tables(max_rows=0, max_groups=0), g, [P] * 5) == OK
