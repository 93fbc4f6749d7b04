"""mv_rope_rotate refuses outputs that lie over another tensor of the call, row by row.

Nothing is launched and no address is followed: a call that is not refused for its rows is refused for its 8192 query heads."""
import ctypes as C

import numpy as np
import pytest

from paper_2602_07529_b200 import binding as B
from test_rope_form_refusals import form
from test_step_refusals import INVALID, P, UNSUPPORTED

HQ, D = 8192, 64
Q = HQ * D * 2            # bytes of a token's query heads
FAR = 1 << 40


def rotate(hkv, q, k, qo, ko, n, pos=P + (1 << 50)):
    """Each tensor as (address, stride in bytes) or None."""
    el = lambda t: (None, 0) if t is None else (t[0], t[1] // 2)
    return B.lib.mv_rope_rotate(C.byref(form(rotary_dim=D)[1]), C.byref(B.make_geom(HQ, hkv, D, 0, "bf16")), pos, n, 0, *el(q), *el(k), *el(qo), *el(ko), None)


def test_outputs_over_other_tensors():
    q, k, qo, ko = (P, Q), (P + FAR, 256), (P + 2 * FAR, Q), (P + 3 * FAR, 256)
    ok = lambda *a, n=8: rotate(2, *a, n) == UNSUPPORTED
    refused = lambda *a, n=8: rotate(2, *a, n) == INVALID
    assert ok(q, k, qo, ko) and ok(q, k, q, k) and ok(q, None, qo, None) and ok(None, k, None, k)
    for at in (16, Q - 16, 8 * Q - 16, 16 - 8 * Q, -16):      # q_out shifted over q
        assert refused(q, None, (q[0] + at, Q), None), at
    for at in (8 * Q, -8 * Q):
        assert ok(q, None, (q[0] + at, Q), None), at
    assert refused(q, k, k, ko) and refused(q, k, qo, q[:1] + (256,)) and refused(q, k, qo, (qo[0] + 5 * Q, 256)) and refused(q, k, (k[0] - Q + 16, Q), k)
    # q and k side by side in the rows of one projection, in place, to another such one, and with an output over its neighbour
    s = Q + 512
    a, b = (P, s), (P + Q, s)
    assert ok(a, b, a, b) and ok(a, b, (P + FAR, s), (P + FAR + Q, s)) and ok(a, None, a, None)
    assert refused(a, b, a, (P + Q - 16, s)) and refused(a, b, b, a) and ok(a, b, a, (P + Q + 256, s)) and refused(a, b, a, (P + Q + 240, s))
    # rows of another stride: the first fits a gap, the second does not
    assert refused((P, 2 * Q), None, (P + Q, Q), None, n=2) and ok((P, 2 * Q), None, (P + Q, 3 * Q), None, n=2) and ok((P, 2 * Q), None, (P + Q, Q), None, n=1)
    # positions are an input too
    assert rotate(2, q, None, qo, None, 8, pos=qo[0] + 3 * Q + 4) == INVALID and rotate(2, q, None, qo, None, 8, pos=qo[0] + 8 * Q) == UNSUPPORTED
    assert rotate(2, q, k, q, ko, 8, pos=ko[0]) == INVALID and rotate(2, q, k, q, k, 8, pos=q[0]) == INVALID
    assert rotate(2, q, None, q, None, 8, pos=q[0] - 32) == UNSUPPORTED and rotate(2, q, None, q, None, 8, pos=q[0] - 28) == INVALID


def test_many_tokens_and_large_addresses():
    n = (1 << 31) - 1
    one = lambda a, b, n: rotate(1, None, a, None, b, n)
    s, row = 4096, 2 * D
    assert one((P, s), (P + row, s), n) == UNSUPPORTED and one((P, s), (P + row - 16, s), n) == INVALID          # interleaved
    assert one((P, s), (P + s * (n - 1) + row - 16, s), n) == INVALID and one((P, s), (P + s * n, s), n) == UNSUPPORTED
    assert one((1 << 61, 1 << 31), (1 << 40, 1 << 31), 1 << 20) == UNSUPPORTED
    assert one(((1 << 61) + 16, 1 << 31), (1 << 61, 1 << 31), 1 << 20) == INVALID
    assert one((P, row), (P + 16, row), 0) == 0


@pytest.mark.parametrize("seed", range(20))
def test_against_every_pair_of_rows(seed):
    rng = np.random.default_rng(seed)
    met = set()
    for _ in range(300):
        n = int(rng.integers(1, 6))
        if rng.random() < 0.5:      # k and k_out: rows of 128 bytes
            la = lb = 2 * D
            sa = la + 16 * int(rng.integers(0, 20))
            sb = sa if rng.random() < 0.5 else lb + 16 * int(rng.integers(0, 20))
            a, b = P, P + 16 * int(rng.integers(-80, 80))
            got = rotate(1, None, (a, sa), None, (b, sb), n)
        else:                       # q, and k_out of longer rows with gaps
            hkv = int(2 ** rng.integers(0, 13))
            la, lb = Q, hkv * D * 2
            sa = la + 16 * int(rng.integers(0, 2 * lb // 16 + 2))
            sb = sa if rng.random() < 0.5 and sa >= lb else lb + 16 * int(rng.integers(0, 2 * la // 16))
            a, b = P, P + 16 * int(rng.integers(-n * sb // 16, n * sa // 16))
            got = rotate(hkv, (a, sa), (P + FAR, lb), (P + 2 * FAR, la), (b, sb), n)
        if a == b:
            continue                # in place, or refused for its stride
        want = any(a + i * sa < b + j * sb + lb and b + j * sb < a + i * sa + la for i in range(n) for j in range(n))
        assert got == (INVALID if want else UNSUPPORTED), (a, sa, la, b - a, sb, lb, n)
        met.add(want)
    assert met == {False, True}
