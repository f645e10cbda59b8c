"""Causal attention over the 4-bit cache where the sums of a row's waves or splits are near the ends of what each of them may hold: scores 20 to 60 above or below
0 and values of one sign or very large, so that a part that holds by itself is joined with others like it, or with parts that were done once more.

Tolerance: that of test_gpu_cache4_attend.py, and fp32 scores as large as they are here: 16 roundings of 2^-24 of sum |q k| in exponents of 2, from the products and
from subtracting or adding to a reference of that size.  An exponent off by x changes an output by x ln 2 (sum p |v| + |o|) at most."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from oracle import cache4 as oc

pytestmark = pytest.mark.gpu

SCALE = 128.0 ** -0.5
UNIT = 32 * 1.5 * SCALE  # score of a query of ones on a group of keys of 1.5


def _made(hq, hkv, n, before, sizes, peaks=(), low=()):
    """A session, a cache and what it stands for: keys 1.5 in their first group (6 for those in `low`), 0 or, for `peaks`, 1.5 in the second one, N(0,1)
    behind; values 1 to 1.25 times the size of their group, those of the peaks negative."""
    gen = torch.Generator(device="cuda").manual_seed(31)
    tokens = before + n
    K = torch.randn((hkv, tokens, 128), generator=gen, device="cuda")
    V = 1 + torch.rand((hkv, tokens, 128), generator=gen, device="cuda") / 4
    K[..., :32], K[..., 32:64] = 1.5, 0.0
    V *= torch.tensor(sizes, device="cuda").repeat_interleave(32)
    for t in low:
        K[:, t, :32] = 6.0
    for t in peaks:
        K[:, t, 32:64] = 1.5
        V[:, t] *= -1
    ses = sa.Session(hq, hkv, 256, 64, 32, keep=0.5)
    c = ses.cache4(tokens)
    K, V = K.bfloat16(), V.bfloat16()
    ses.append(c, K, V, 0)
    ses.read(c, K, V)
    return ses, c, K.double(), V.double()


def _check(made, n, before, offset, above=0.0, at=()):
    """offset: natural logarithms that the scores are moved by, a number or one for each of the n rows; above: that much more for the peaks; at: the rows that are
    compared."""
    ses, c, keys, vals = made
    hq, g = ses.cfg.n_q_heads, ses.cfg.n_q_heads // ses.cfg.n_kv_heads
    gen = torch.Generator(device="cuda").manual_seed(32)
    Q = torch.randn((hq, n, 128), generator=gen, device="cuda")
    Q[..., :32] = torch.as_tensor(offset, device="cuda", dtype=torch.float32).expand(n)[None, :, None] / UNIT
    Q[..., 32:64] = above / UNIT
    Q = Q.bfloat16()
    O = torch.full_like(Q, 7.0)
    ses.attend(c, Q, before, O)
    torch.cuda.synchronize()
    rows, _ = sa.sa_cache4_attend_plan(ses.ctx, n, before)
    of_p = 2.0 ** -15 if rows == 16 or (rows == 32 and g * n <= 64) else 2.0 ** -8
    at = torch.tensor(at, device="cuda")
    q = Q[:, at].double()
    left = torch.from_numpy(oc.query_left_out(q.cpu().numpy(), np.float32(SCALE) * np.float32(1.4426950408889634))).cuda()
    later = (torch.arange(before + n, device="cuda")[None] > before + at[:, None]).repeat(g, 1)
    for h in range(0, hq, g):
        k, v, rows_of = keys[h // g], vals[h // g], slice(h, h + g)
        kt, x = k.T.contiguous(), q[rows_of].reshape(-1, 128)
        p = torch.softmax((x @ kt * SCALE).masked_fill_(later, -torch.inf), -1)
        o = p @ v
        spread = p @ v.abs() + o.abs()
        off = (left[rows_of].reshape(-1, 128) @ kt).abs_().masked_fill_(later, 0).amax(-1, keepdim=True)
        off += 2.0 ** -20 * SCALE * np.log2(np.e) * (x.abs() @ kt.abs_()).amax(-1, keepdim=True)
        tol = 2.0 ** -8 * o.abs() + (of_p + 2.0 ** -12 + np.log(2) * off) * spread
        got = O[rows_of, at].reshape(-1, 128).double()
        ok = (got - o).abs() <= tol
        assert ok.all(), (h, offset, above, got[~ok][:3].tolist(), o[~ok][:3].tolist())


# heads, tokens, before, (rows of a workgroup, whether in splits): waves joined, few splits, many splits
FORMS = [((32, 8), 500, 0, (32, False)), ((64, 8), 191, 640, (32, False)), ((32, 8), 50, 5000, (32, True)), ((32, 1), 4, 100000, (32, True)), ((8, 1), 8, 131000, (32, True)),
         ((128, 2), 130, 5, (128, False)), ((32, 8), 200, 8009, (128, True)), ((64, 1), 47, 90000, (128, True)), ((8, 1), 30, 130000, (128, True)), ((4, 4), 3, 0, (16, False)),
         ((8, 2), 5, 10003, (16, True))]


def _form(heads, n, before, form, sizes, **more):
    print(f"case attend4 join {heads} {n} {before} {form} {sizes}", flush=True)
    made = _made(*heads, n, before, sizes, **more)
    rows, splits = sa.sa_cache4_attend_plan(made[0].ctx, n, before)
    assert (rows, splits > 1) == form, (rows, splits)
    return made, sorted({i * (n - 1) // 12 for i in range(13)} | {min(1, n - 1)})


@pytest.mark.parametrize("sizes", [(0.1, 0.1, 0.1, 0.1), (0.01, 1.0, 60.0, 1000.0)])
@pytest.mark.parametrize("heads,n,before,form", FORMS)
def test_all_scores_near_the_upper_end(heads, n, before, form, sizes):
    made, at = _form(heads, n, before, form, sizes)
    for offset in (40.0, 43.0, 45.0, 46.0, 47.0, 48.0, 48.5, 49.0, 49.5, 50.0, 51.0, 52.0, 53.0, 54.0, 55.0, 57.0):
        _check(made, n, before, float(offset), at=at)


@pytest.mark.parametrize("heads,n,before,form", FORMS)
def test_all_scores_near_the_lower_end(heads, n, before, form):
    made, at = _form(heads, n, before, form, (0.01, 1.0, 60.0, 1000.0))
    for offset in (-36.0, -31.0, -29.5, -28.0, -27.0, -26.0, -24.0):
        _check(made, n, before, float(offset), at=at)


@pytest.mark.parametrize("exponent", [60, 72, 76, 80, 88])
@pytest.mark.parametrize("heads,n,before,form", FORMS)
def test_values_near_the_upper_end(heads, n, before, form, exponent):
    made, at = _form(heads, n, before, form, (2.0 ** exponent, 1.0, 2.0 ** (exponent - 3), 2.0 ** (exponent - 20)))
    for offset in (0.0, 8.0):
        _check(made, n, before, offset, at=at)


@pytest.mark.parametrize("heads,n,before,form", FORMS)
def test_parts_that_hold_beside_parts_that_do_not(heads, n, before, form):
    # a key above the many: its wave or split is done once more, and the others together weigh as much
    tokens = before + n
    peak = [max(0, before - 3) if before else 0]
    made, at = _form(heads, n, before, form, (1.0, 0.1, 0.02, 0.5), peaks=peak)
    for offset in np.arange(42.5, 55.0, 1.0):
        for above in (5.0, 9.5, np.log(tokens), np.log(tokens) + 2):
            _check(made, n, before, float(offset), float(above), at=at)


@pytest.mark.parametrize("heads,n,before,form", FORMS)
def test_rows_of_many_offsets(heads, n, before, form):
    made, at = _form(heads, n, before, form, (0.1, 1.0, 60.0, 1000.0), peaks=[before // 2])
    for above in (0.0, 9.0):
        _check(made, n, before, np.resize(np.arange(44.0, 60.0, 0.77)[::-1].copy(), n), above, at=at)
        _check(made, n, before, np.resize(np.arange(-70.0, 90.0, 11.3), n), above, at=at)


def test_splits_of_long_walks():
    """Splits of more than 256 tiles of 64 keys: each looks at its first tile ahead, whose scores are 45 below the others, or 36 above."""
    heads, n, before = (32, 8), 300, 130700
    ses = sa.Session(*heads, 256, 64, 32, keep=0.5)
    rows, splits = sa.sa_cache4_attend_plan(ses.ctx, n, before)
    assert rows == 128 and splits > 1 and (before + n) // 64 // splits >= 256, (rows, splits)
    low = set()
    for tiles in range(before // 64, (before + n) // 64 + 2):
        per = -(-tiles // splits)
        low |= {64 * per * sp + i for sp in range(splits) for i in range(64) if 64 * per * sp + i < before}
    for exponent in (0, 48, 49, 50):
        print(f"case attend4 join long walk 2^{exponent}", flush=True)
        made = _made(*heads, n, before, (2.0 ** exponent,) * 4, low=[sorted(low)])
        for offset in (-15.0, 12.0):
            _check(made, n, before, offset, at=[0, 1, 150, 298, 299])
