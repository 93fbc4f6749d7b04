"""Rotary embedding at positions up to 2^30, the most that tables built on the device hold, against extended precision.

Bound: bf16 rounds by 2^-8 of the value; the angle pos * theta is a rounded double below 2^30 (off by 2^-24), theta is within an ulp of its
value or two (2^-52 of it, so 2^-22 in the angle), cosine and sine are floats (2^-23): 2^-21 of the pair's length in all."""
import numpy as np
import pytest
import torch

pytestmark = pytest.mark.gpu


def rotate_extended(x, pos, base):
    """[T, H, d] rotated in 80-bit arithmetic."""
    d = x.shape[-1]
    theta = np.longdouble(base) ** (-2.0 * np.arange(d // 2, dtype=np.longdouble) / d)
    a = np.asarray(pos, np.longdouble)[:, None] * theta
    c, s = np.cos(a)[:, None], np.sin(a)[:, None]
    lo, hi = x[..., :d // 2].astype(np.longdouble), x[..., d // 2:].astype(np.longdouble)
    return np.concatenate([lo * c - hi * s, hi * c + lo * s], -1).astype(np.float64)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("base", [10000.0, 500000.0, 1.0])
def test_positions_up_to_2_30(d, base):
    from paper_2602_07529_b200 import binding as B
    rng = np.random.default_rng(3)
    pos = np.concatenate([[0, 1, 2 ** 20 + 3, 2 ** 24 + 1, 2 ** 25 - 1, 2 ** 27 + 5, 2 ** 29 + 1, 2 ** 30 - 1, 2 ** 30],
                          rng.integers(2 ** 25, 2 ** 30, 1200), np.exp(rng.uniform(0, np.log(2 ** 30), 1200)).astype(np.int64)])
    n, hq, hkv = len(pos), 4, 2
    tables = B.StepTables(torch.from_numpy(pos.astype(np.int32)).cuda(), torch.full((n,), 0, dtype=torch.int64, device="cuda") + torch.arange(n, device="cuda") * 16,
                          torch.zeros(8, dtype=torch.int32, device="cuda"))
    geom = B.make_geom(hq, hkv, d, n, "bf16", rope_base=base)
    g = torch.Generator(device="cuda").manual_seed(5)
    q, k, v = (torch.randn(n, h, d, generator=g, device="cuda").bfloat16() for h in (hq, hkv, hkv))
    q_rot, k_rot = torch.empty_like(q), torch.empty_like(k)
    pools = [torch.zeros(n, hkv, 16, d, dtype=torch.uint8, device="cuda") for _ in range(2)]
    sc = torch.zeros(n, hkv, 2, device="cuda")
    B.mv_rope_write_kv_fp8_blk(tables, geom, q, k, v, q_rot, k_rot, *pools, sc)
    assert B.mv_step_tables_read_status(tables) == 0
    for got, x in ((q_rot, q), (k_rot, k)):
        x = x.cpu().double().numpy()
        ref = rotate_extended(x, pos, base)
        pair = np.sqrt(x[..., :d // 2] ** 2 + x[..., d // 2:] ** 2)
        tol = 2.0 ** -8 * np.abs(ref) + 2.0 ** -21 * np.concatenate([pair, pair], -1)
        assert (np.abs(got.cpu().double().numpy() - ref) <= tol).all()
