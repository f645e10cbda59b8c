"""What sa_cache_attend_plan says and refuses (no GPU needed)."""
import ctypes as C

import pytest

import paper_2412_06198_amd as sa


def _context(hq, hkv, block=64):
    c = sa.SaConfig()
    c.n_q_heads, c.n_kv_heads, c.head_dim = hq, hkv, 128
    c.seq_len, c.block, c.last_q = 512, block, 32
    return sa.sa_create(sa.sa_default_budgets(c, 0.5))


@pytest.mark.parametrize("heads", [(1, 1), (8, 2), (32, 8), (32, 32), (128, 1), (128, 128)])
def test_plans_stay_inside_the_scratch(heads):
    ctx = _context(*heads)
    slots = sa.sa_cache_attend_scratch_bytes(ctx) // (128 * 4 + 8)
    for n in (1, 2, 5, 31, 33, 100, 257, 1000, 2048, 20000):
        for pos in (0, 1, 31, 32, 500, 5000, 131072, 2 ** 30 - n):
            rows, splits = sa.sa_cache_attend_plan(ctx, n, pos)
            assert rows in (32, 128) and 1 <= splits <= 256
            assert splits == 1 or heads[0] * n * splits <= slots, (n, pos, splits)
            assert splits <= -(-(pos + n) // 32)
            if heads[0] // heads[1] * n <= 32:
                assert rows == 32
    sa.sa_destroy(ctx)


def test_refusals():
    ctx = _context(8, 2)
    sa.sa_cache_attend_plan(ctx, 1, 2 ** 30 - 1)
    for n, pos in ((0, 0), (-1, 5), (1, -1), (2 ** 27, 0), (1, 2 ** 30), (2 ** 62, 0), (1, 2 ** 62)):
        with pytest.raises(sa.SaError) as e:
            sa.sa_cache_attend_plan(ctx, n, pos)
        assert e.value.status == 1
    out = C.c_int32()
    lib = sa.library()
    assert lib.sa_cache_attend_plan(None, 1, 0, C.byref(out), C.byref(out)) == 1
    assert lib.sa_cache_attend_plan(ctx, 1, 0, None, C.byref(out)) == 1
    assert lib.sa_cache_attend_plan(ctx, 1, 0, C.byref(out), None) == 1
    sa.sa_destroy(ctx)
