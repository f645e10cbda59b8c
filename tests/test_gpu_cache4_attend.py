"""Causal attention of the newest tokens over the 4-bit cache, against fp64 on the values that the cache stands for.

Tolerance: half a step of bf16 of the output, 2^-8 |o|; a probability as multiplied, 2^-8 of itself in bf16 or 2^-15 in two parts, normalised
by the sum of what is multiplied, and fp32 scores as in the decode step, 2^-12: of sum p |v| + |o|; an exponent (of 2) off by x, x ln 2 of
that too: what the three codes of a query leave out, as the oracle cuts it, times the key."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from gpu_util import dev_bf16, host_f64
from oracle import cache4 as oc
from test_gpu_cache_decode import _f64

pytestmark = pytest.mark.gpu


def _setup(Hq, Hkv, tokens, seed=1, change=None, **options):
    ses = sa.Session(Hq, Hkv, 256, 64, 32, keep=0.5, **options)
    Q, K, V = gen.random_qkv(Hq, Hkv, tokens, 128, seed=seed)
    if change:
        change(Q, K, V)
    c = ses.cache4(tokens + 37)
    for t in c.tensors:  # what stands behind the tokens is never read: NaN there
        t.fill_(0xFF)
    ses.append(c, dev_bf16(K), dev_bf16(V), 0)
    return ses, c, Q, oc.read(_f64(K)), oc.read(_f64(V))


def _reference(q, keys, vals, pos, rows, scale=128.0 ** -0.5):
    """q [Hq, n, 128]; o and the tolerance.  rows: query rows of a KV head that a workgroup takes."""
    hq, n, g = q.shape[0], q.shape[1], q.shape[0] // keys.shape[0]
    o, tol = np.empty(q.shape), np.empty(q.shape)
    later = np.arange(pos + n)[None] > pos + np.arange(n)[:, None]
    of_p = 2.0 ** -15 if rows == 16 or (rows == 32 and g * n <= 64) else 2.0 ** -8
    for h in range(hq):
        s = q[h] @ keys[h // g].T * scale
        s[later] = -np.inf
        off = np.log(2) * np.abs(oc.query_left_out(q[h], np.float32(scale) * np.float32(1.4426950408889634)) @ keys[h // g].T)
        off[later] = 0
        p = np.exp(s - s.max(-1, keepdims=True))
        p /= p.sum(-1, keepdims=True)
        o[h] = p @ vals[h // g]
        spread = p @ np.abs(vals[h // g]) + np.abs(o[h])
        tol[h] = 2.0 ** -8 * np.abs(o[h]) + (of_p + 2.0 ** -12 + off.max(-1, keepdims=True)) * spread
    return o, tol


def _check(ses, c, Q, keys, vals, n, scale=128.0 ** -0.5):
    tokens = keys.shape[1]
    pos = tokens - n
    Qd = dev_bf16(Q[:, pos:])
    O = torch.full_like(Qd, 7.0)
    ses.attend(c, Qd, pos, O)
    torch.cuda.synchronize()
    want, tol = _reference(_f64(Q[:, pos:]), keys, vals, pos, sa.sa_cache4_attend_plan(ses.ctx, n, pos)[0], scale)
    err = np.abs(host_f64(O) - want)
    assert (err <= tol).all(), (n, tokens, float((err / tol).max()))
    return O


@pytest.mark.parametrize("heads", [(4, 4), (8, 2), (6, 2), (8, 1), (24, 3), (32, 1), (40, 1)])
def test_one_token(heads):
    for L in (1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 500, 1024, 1087):
        print(f"case attend4 one heads={heads} L={L}", flush=True)
        _check(*_setup(*heads, L), 1)


@pytest.mark.parametrize("heads", [(4, 4), (6, 2), (8, 1)])
@pytest.mark.parametrize("n", [2, 4, 5, 8, 9, 17, 33, 64, 65, 127, 200, 513])
def test_drafts_and_chunks(heads, n):
    print(f"case attend4 chunk heads={heads} n={n}", flush=True)
    for before in (0, 1, 70, 640, 1500):
        _check(*_setup(*heads, before + n, seed=2), n)


def test_whole_prompt():
    print("case attend4 prompt", flush=True)
    _check(*_setup(4, 1, 1000, seed=3), 1000)
    _check(*_setup(32, 8, 200, seed=4), 200)


@pytest.mark.parametrize("n", [1, 3, 40, 300])
def test_long_cache_in_splits(n):
    print(f"case attend4 long n={n}", flush=True)
    _check(*_setup(4, 2, 20000 + 77, seed=5), n)


@pytest.mark.parametrize("n", [1, 7, 150])
def test_uneven_queries_and_softmax_scale(n):
    # a few elements far above the others of their group, rows of tiny and of large queries
    print(f"case attend4 uneven n={n}", flush=True)

    def change(Q, K, V):
        q = gen.bf16_bits_to_f32(Q)
        q[..., 3::32] *= 32
        q[:, ::3] *= 2.0 ** -20
        q[:, 1::5, 40:70] = 0
        Q[:] = gen.f32_to_bf16_bits(q)
    _check(*_setup(4, 2, 400, seed=6, change=change, softmax_scale=0.02), n, scale=float(np.float32(0.02)))


def test_strides():
    print("case attend4 strides", flush=True)
    ses, c, Q, keys, vals = _setup(6, 2, 333, seed=7)
    for n in (3, 100):
        pos = 333 - n
        want = _check(ses, c, Q, keys, vals, n)
        Qd = dev_bf16(Q[:, pos:]).transpose(0, 1).contiguous().transpose(0, 1)   # tokens outermost
        room = torch.full((n, 6, 136), 7.0, dtype=torch.bfloat16, device="cuda")
        ses.attend(c, Qd, pos, room[..., :128].transpose(0, 1))
        torch.cuda.synchronize()
        assert torch.equal(room[..., :128].transpose(0, 1), want) and (room[..., 128:] == 7.0).all()
        Qi = Qd.clone()
        ses.attend(c, Qi, pos, Qi)   # in place
        torch.cuda.synchronize()
        assert torch.equal(Qi, want)


@pytest.mark.parametrize("n,heads", [(1, (4, 1)), (5, (4, 1)), (100, (4, 1)), (300, (2, 2))])
def test_nan_groups_reach_only_rows_that_see_them(n, heads):
    # a value of V that is no number, among the new tokens and before: its group of 32, of the rows that see it
    print(f"case attend4 non-finite V n={n} heads={heads}", flush=True)
    tokens = 260 + n
    for at in (tokens - n // 2 - 1, tokens - 1, tokens - n + 1 if n > 1 else 5, 100):
        def change(Q, K, V):
            V[:, at, 9] = 0x7F80
            V[:, at, 64] = 0x7FC0
        ses, c, Q, keys, vals = _setup(*heads, tokens, 8, change)
        pos = tokens - n
        Qd = dev_bf16(Q[:, pos:])
        O = torch.full_like(Qd, 7.0)
        ses.attend(c, Qd, pos, O)
        torch.cuda.synchronize()
        got = host_f64(O)
        bad = np.zeros(got.shape, bool)
        bad[:, max(0, at - pos):, 0:32] = bad[:, max(0, at - pos):, 64:96] = True
        assert np.isnan(got[bad]).all()
        clean = vals.copy()
        clean[:, at, 0:32] = clean[:, at, 64:96] = 0
        ref, tol = _reference(_f64(Q[:, pos:]), keys, clean, pos, sa.sa_cache4_attend_plan(ses.ctx, n, pos)[0])
        assert (np.abs(got - ref) <= tol)[~bad].all()


@pytest.mark.parametrize("n", [1, 4, 150])
def test_nan_keys_and_queries(n):
    print(f"case attend4 non-finite K, Q n={n}", flush=True)
    tokens = 200 + n
    at = tokens - min(2, n)

    def change(Q, K, V):
        K[:2, at, 3] = 0x7FC0
        Q[3, tokens - 1, 77] = 0xFF80
    ses, c, Q, keys, vals = _setup(4, 4, tokens, change=change)
    Qd = dev_bf16(Q[:, tokens - n:])
    O = torch.empty_like(Qd)
    ses.attend(c, Qd, tokens - n, O)
    torch.cuda.synchronize()
    bad = np.zeros((4, n), bool)
    bad[:2, at - (tokens - n):] = True
    bad[3, -1] = True
    assert np.array_equal(np.isnan(host_f64(O)), np.broadcast_to(bad[..., None], O.shape))


def test_scores_that_are_all_nan():
    print("case attend4 NaN rows", flush=True)

    def change(Q, K, V):
        K[0, :, 5] = 0x7F80
    for n, tokens in ((1, 700), (3, 40), (200, 300)):
        ses, c, Q, keys, vals = _setup(4, 2, tokens, change=change)
        Qd = dev_bf16(Q[:, tokens - n:])
        O = torch.empty_like(Qd)
        ses.attend(c, Qd, tokens - n, O)
        torch.cuda.synchronize()
        assert torch.isnan(O[:2]).all() and torch.isfinite(O[2:]).all()


@pytest.mark.parametrize("n,before", [(1, 3000), (6, 3000), (200, 900)])
def test_same_bytes_in_a_replayed_graph_and_on_another_stream(n, before):
    print(f"case attend4 graph n={n}", flush=True)
    ses, c, Q, keys, vals = _setup(8, 2, before + n, seed=9)
    want = _check(ses, c, Q, keys, vals, n)
    Qd = dev_bf16(Q[:, before:])
    O = torch.empty_like(Qd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.attend(c, Qd, before, O)
    for rep in range(4):
        O.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(O, want), rep
        other = torch.empty_like(Qd)
        ses.attend(c, torch.randn_like(Qd), before, other)      # eager calls between the replays
        torch.cuda.synchronize()
    with torch.cuda.stream(side):
        O.fill_(7.0)
        ses.attend(c, Qd, before, O)
    side.synchronize()
    assert torch.equal(O, want)
