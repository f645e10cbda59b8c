"""Causal attention over the 8-bit cache where many rows read many keys (600 thousand and more over all sets of 32 rows), which
workgroups of 128 rows take, but at the edge: K multiplied as codes, Q cut into two.  Against fp64 on the values that the cache stands for; the reference runs
on the GPU, one plain product per head.

Tolerance: as in test_gpu_cache_attend.py.  Q = hi + lo is exact, but for elements below 2^-14 of their row's largest, which are
off by 2^-23 of it: 2^-16 sum |k| scale at most in a score, inside the 2^-12."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa

pytestmark = pytest.mark.gpu


def _fill(ses, b, tokens, kind, seed, change=None):
    """A cache of `tokens` random tokens, filled by append, and what it stands for."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    hkv = ses.cfg.n_kv_heads
    K, V = (torch.randn((hkv, tokens, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    K[..., 5::32] *= 4
    if change:
        change(K, V)
    c = ses.cache(-(-tokens // b) * b + b, kind)
    for t in c.tensors:  # what stands behind the tokens is never read: NaN there
        t.view(torch.uint8).fill_(0x7F)
    ses.append(c, K, V, 0)
    full = tokens // b * b
    kinds = (torch.float8_e4m3fn, torch.float8_e5m2)[kind]

    def read(codes, scale, rows):
        x = codes[:, :full].view(kinds).double() * scale[:, :full // b].double().repeat_interleave(b, 1)[..., None]
        return torch.cat([x, rows[:, :tokens - full].double()], 1)

    return c, read(c.k, c.k_scale, c.k_open), read(c.v, c.v_scale, c.v_open), gen


def _reference(q, keys, vals, pos, scale=128 ** -0.5):
    hq, n, g = q.shape[0], q.shape[1], q.shape[0] // keys.shape[0]
    o, tol = torch.empty(q.shape, dtype=torch.float64, device="cuda"), torch.empty(q.shape, dtype=torch.float64, device="cuda")
    later = torch.arange(pos + n, device="cuda") > pos + torch.arange(n, device="cuda")[:, None]
    for h in range(hq):
        s = (q[h].double() @ keys[h // g].T.contiguous()) * scale
        s.masked_fill_(later, -torch.inf)
        p = torch.softmax(s, -1)
        o[h] = p @ vals[h // g]
        tol[h] = 2.0 ** -8 * o[h].abs() + (2.0 ** -8 + 2.0 ** -12) * (p @ vals[h // g].abs() + o[h].abs())
    return o, tol


def _many(hq, hkv, n, tokens):
    return -(-(hq // hkv * n) // 32) * hkv * tokens > 600000 and hq // hkv * n > 32


def _check(hq, hkv, b, n, pos, kind=sa.SA_CACHE_E4M3, seed=1, scale=0.0, many=True):
    print(f"case rows hq={hq} hkv={hkv} b={b} n={n} pos={pos} kind={kind}", flush=True)
    assert not many or _many(hq, hkv, n, pos + n)
    ses = sa.Session(hq, hkv, 4 * b, b, 32, keep=0.5, softmax_scale=scale)
    c, keys, vals, gen = _fill(ses, b, pos + n, kind, seed)
    q = torch.randn((hq, n, 128), generator=gen, device="cuda").bfloat16()
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    want, tol = _reference(q, keys, vals, pos, scale or 128 ** -0.5)
    err = (o.double() - want).abs()
    assert (err <= tol).all(), float((err / tol).max())
    return ses, c, q, o


@pytest.mark.parametrize("kind", [sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("rest", [0, 1, 63, 64, 100])
def test_ends_of_the_open_block(b, kind, rest):
    # splits; the last tokens in no, a short, a full and two tiles of the open block
    _check(8, 8, b, 200, 11008 - 200 + rest, kind)


@pytest.mark.parametrize("heads", [(4, 1), (6, 2), (24, 3), (32, 8), (128, 1), (5, 5)])
@pytest.mark.parametrize("n", [33, 130, 257])
def test_heads_and_rows(heads, n):
    hq, hkv = heads
    sets = -(-(hq // hkv * n) // 32) * hkv
    _check(hq, hkv, 64, n, max(700, 600000 // sets + 100), seed=2)


@pytest.mark.parametrize("pos", [0, 1, 63, 100, 900])
def test_a_workgroup_per_row_tile(pos):
    # 288 workgroups without splits, the second ones of a compute unit in the opposite order; tiles that some rows see
    _check(32, 32, 64, 1100, pos, seed=3)
    _check(24, 24, 128, 1500, pos, sa.SA_CACHE_E5M2, seed=3)


def test_many_row_tiles():
    _check(16, 2, 64, 5000, 700, seed=4)     # 626 workgroups


@pytest.mark.parametrize("heads,n,pos", [((32, 8), 700, 0), ((32, 8), 700, 700), ((64, 8), 350, 0), ((24, 3), 1000, 500), ((24, 3), 700, 0),
                                         ((32, 8), 500, 1500), ((8, 1), 4000, 0), ((5, 5), 1111, 3), ((128, 8), 200, 1)])
def test_sets_of_32_rows_over_a_full_card(heads, n, pos):
    # one to four workgroups of 32 rows a compute unit, from the longest row tile down or from the shortest up
    _check(*heads, 64, n, pos, seed=13, many=False)


def test_scale_of_the_softmax():
    _check(8, 8, 64, 200, 11000, seed=5, scale=0.3)


def test_queries_of_uneven_elements():
    # rows of large and tiny elements, zeros, and a row of zeros: what the two codes of an element hold
    print("case rows queries", flush=True)
    ses = sa.Session(8, 8, 256, 64, 32, keep=0.5)
    n, pos = 200, 11000
    c, keys, vals, gen = _fill(ses, 64, pos + n, 0, 6)
    q = torch.randn((8, n, 128), generator=gen, device="cuda")
    q *= 2.0 ** torch.randint(-9, 3, (8, n, 128), generator=gen, device="cuda")
    q[:, ::7] *= 2.0 ** -60
    q[:, 3::7] = 0
    q[:, 5::7, ::2] = 0
    q = q.bfloat16()
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    want, tol = _reference(q, keys, vals, pos)
    assert ((o.double() - want).abs() <= tol).all()


def test_non_finite_queries():
    print("case rows NaN in queries", flush=True)
    ses = sa.Session(8, 8, 256, 64, 32, keep=0.5)
    n, pos = 200, 11000
    c, keys, vals, gen = _fill(ses, 64, pos + n, 0, 7)
    q = torch.randn((8, n, 128), generator=gen, device="cuda").bfloat16()
    q[2, 17, 9], q[5, 199, 64] = float("nan"), float("inf")
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    bad = torch.zeros((8, n, 128), dtype=torch.bool, device="cuda")
    bad[2, 17] = bad[5, 199] = True
    assert torch.equal(torch.isnan(o), bad)


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("back", [0, 3, 90, 199, 5000])
def test_non_finite_values(value, back):
    print(f"case rows non-finite V {value} {back}", flush=True)
    hq, n, pos = 8, 200, 11000
    at = pos + n - 1 - back

    def change(K, V):
        V[:, at, 9] = value
        V[:, at, 64] = value

    ses = sa.Session(hq, hq, 256, 64, 32, keep=0.5)
    c, keys, vals, gen = _fill(ses, 64, pos + n, sa.SA_CACHE_E5M2, 8, change)
    q = torch.randn((hq, n, 128), generator=gen, device="cuda").bfloat16()
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    bad = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
    bad[:, max(0, at - pos):, 9] = bad[:, max(0, at - pos):, 64] = True
    got = o.double()
    assert (torch.isnan(got[bad]) if value != value else got[bad] == value).all()
    vals[:, at, 9] = vals[:, at, 64] = 0
    want, tol = _reference(q, keys, vals, pos)
    assert ((got - want).abs() <= tol)[~bad].all()


def test_nan_keys_of_later_tokens():
    print("case rows NaN in K", flush=True)
    hq, n, pos = 8, 200, 11000

    def change(K, V):
        K[:, pos + 150, 3] = float("nan")

    ses = sa.Session(hq, hq, 256, 128, 32, keep=0.5)
    c, keys, vals, gen = _fill(ses, 128, pos + n, 0, 9, change)
    q = torch.randn((hq, n, 128), generator=gen, device="cuda").bfloat16()
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    bad = torch.isnan(o).any(-1)
    assert bad[:, 150:].all() and not bad[:, :150].any()


def test_strides_and_in_place():
    print("case rows strides", flush=True)
    ses, c, q, want = _check(8, 8, 64, 200, 11000, seed=10)
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)
    room = torch.full((200, 8, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    ses.attend(c, turned, 11000, room[..., :128].transpose(0, 1))
    assert torch.equal(room[..., :128].transpose(0, 1), want) and (room[..., 128:] == 7.0).all()
    ses.attend(c, q, 11000, q)
    assert torch.equal(q, want)


def test_replays():
    print("case rows graph", flush=True)
    ses, c, q, _ = _check(8, 8, 64, 200, 11000, seed=11)
    o = torch.empty_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.attend(c, q, 11000, o)
    for rep in range(3):
        q.copy_(torch.randn_like(q))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(o)
        ses.attend(c, q, 11000, want)
        torch.cuda.synchronize()
        assert torch.equal(o, want), rep


def test_large_scores():
    # logits of hundreds: the running maximum moves often.  Queries 12 times as large: scores off by 12 x 2^-12 at most, which
    # moves a weight by that part of itself, and an output by that part of the largest |v - o|, below 8 where it counts
    print("case rows large scores", flush=True)
    ses = sa.Session(8, 8, 256, 64, 32, keep=0.5)
    n, pos = 200, 11000
    c, keys, vals, gen = _fill(ses, 64, pos + n, 0, 12)
    q = (torch.randn((8, n, 128), generator=gen, device="cuda") * 12).bfloat16()
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    want, tol = _reference(q, keys, vals, pos)
    assert ((o.double() - want).abs() <= tol + 12 * 2.0 ** -12 * 8).all()
