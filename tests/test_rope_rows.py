"""How many tokens mv_rope_rotate turns, and where it takes them from (nothing is launched: the tensors are on the host)."""
import pytest
import torch

from paper_2602_07529_b200 import binding as B


def heads(n, h, d=64):
    return torch.zeros(n, h, d, dtype=torch.bfloat16)


@pytest.mark.parametrize("q_rows,k_rows", [(4, 5), (5, 4), (0, 1), (1, 0)])
def test_q_and_k_have_the_same_tokens(q_rows, k_rows):
    """A k of more tokens than q would keep the rest of k_out as it was, without a word; one of fewer never fitted."""
    form, geom = B.RopeForm(B.ROPE_HALVES, 64), B.make_geom(4, 2, 64, 0, "bf16")
    q, k = heads(q_rows, 4), heads(k_rows, 2)
    pos = torch.zeros(8, dtype=torch.int32)
    with pytest.raises(ValueError, match=f"q has {q_rows} tokens, k {k_rows}"):
        B.mv_rope_rotate(form, geom, pos, q, k, torch.empty_like(q), torch.empty_like(k))


def test_a_single_token_has_no_stride():
    """The distance to a second token that is not there is not looked at; with two it is."""
    room = torch.zeros(2 * 1001, dtype=torch.bfloat16)
    one, two = (torch.as_strided(room, (n, 4, 64), (1001, 64, 1)) for n in (1, 2))
    assert B._heads_at(one, "q", 1, 4, 64, torch.bfloat16, -1) == (room.data_ptr(), 256)
    assert B._heads_at(two, "q", 1, 4, 64, torch.bfloat16, -1) == (room.data_ptr(), 256)
    assert B._heads_at(two, "q", 2, 4, 64, torch.bfloat16, -1) == (room.data_ptr(), 1001)


def test_a_plan_on_another_gpu_is_refused():
    """The plan's positions are memory of the GPU it was uploaded to: a launch on another one must not read them."""
    from paper_2602_07529_b200 import synth
    wl = synth.config1()
    plan = B.Plan(wl.batch)
    assert plan.index is None       # not uploaded
    plan.index = 3                  # as if on a GPU that the tensors are not on
    form, geom = B.RopeForm(B.ROPE_HALVES, 64), B.make_geom(4, 2, 64, 0, "bf16")
    q = heads(4, 4)
    with pytest.raises(ValueError, match="plan is on cuda:3"):
        B.mv_rope_rotate(form, geom, plan, q, None, q, None)


class Uploads:
    """A device buffer as far as Plan.upload looks at one."""

    def __init__(self, index):
        self.index = index

    numel = element_size = data_ptr = lambda self: 0

    def get_device(self):
        return self.index


def test_an_upload_says_where_the_plan_is(monkeypatch):
    from paper_2602_07529_b200 import synth
    plan = B.Plan(synth.config1().batch)
    with pytest.raises(B.MvError):
        plan.upload(Uploads(2), stream=0)      # too small: nothing is uploaded
    assert plan.index is None
    monkeypatch.setattr(B.lib, "mv_plan_upload", lambda *a: 0, raising=False)
    plan.upload(Uploads(2), stream=0)
    assert plan.index == 2
