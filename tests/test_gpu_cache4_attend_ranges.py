"""Causal attention over the 4-bit cache where scores lie far from 0, or values are very large or small: a kernel may sum 2^exponent as it is, and has to
notice where that leaves fp32.

Tolerance: that of test_gpu_cache4_attend.py, and fp32 scores as large as they are here: 16 roundings of 2^-24 of sum |q k| in exponents of 2,
from the products and from subtracting a reference of that size."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from gpu_util import dev_bf16, host_f64
from oracle import cache4 as oc
from test_gpu_cache4_attend import _reference, _setup
from test_gpu_cache_decode import _f64

pytestmark = pytest.mark.gpu

SHAPES = [(1, 2, 2, 300), (4, 4, 1, 700), (40, 8, 2, 500), (150, 4, 1, 90), (150, 4, 4, 4000), (200, 32, 8, 3000), (61, 128, 2, 0), (130, 128, 2, 5), (47, 64, 1, 9000)]  # n, heads, before


def _write(bits, values):
    bits[:] = gen.f32_to_bf16_bits(values.astype(np.float32))


def _run(n, hq, hkv, before, change, seed=11):
    ses, c, Q, keys, vals = _setup(hq, hkv, before + n, seed, change)
    q = Q[:, before:]
    O = torch.full(q.shape, 7.0, dtype=torch.bfloat16, device="cuda")
    ses.attend(c, dev_bf16(q), before, O)
    torch.cuda.synchronize()
    want, tol = _reference(_f64(q), keys, vals, before, sa.sa_cache4_attend_plan(ses.ctx, n, before)[0])
    size = np.abs(_f64(q)) @ np.repeat(np.abs(keys), hq // hkv, 0).transpose(0, 2, 1) * 128.0 ** -0.5 * np.log2(np.e)
    spread = np.abs(vals).max() if vals.size else 0.0
    got = host_f64(O)
    assert np.isfinite(got).all()
    err, tol = np.abs(got - want), tol + 2.0 ** -20 * np.log(2) * size.max(-1, keepdims=True) * 2 * spread
    assert (err <= tol).all(), (float((err / tol).max()), np.argwhere(err > tol)[:3])


def _shift(Q, K, offsets):
    """Scores of row t of every head moved by offsets[t] (natural logarithms): the first group of K a constant."""
    k, q = gen.bf16_bits_to_f32(K), gen.bf16_bits_to_f32(Q)
    k[..., :32] = 1.5
    q[..., :32] = (np.asarray(offsets, np.float32) / np.float32(32 * 1.5 * 128.0 ** -0.5))[None, :, None]
    _write(K, k)
    _write(Q, q)


@pytest.mark.parametrize("n,hq,hkv,before", SHAPES)
@pytest.mark.parametrize("offset", [-300.0, -60.0, -12.0, 30.0, 68.0, 75.0, 250.0])
def test_scores_far_from_zero(n, hq, hkv, before, offset):
    print(f"case attend4 far scores {n} {hq} {hkv} {before} {offset}", flush=True)
    _run(n, hq, hkv, before, lambda Q, K, V: _shift(Q, K, np.full(Q.shape[1], offset)))


@pytest.mark.parametrize("n,hq,hkv,before", SHAPES)
def test_rows_far_from_each_other(n, hq, hkv, before):
    print(f"case attend4 far rows {n} {hq} {hkv} {before}", flush=True)
    _run(n, hq, hkv, before, lambda Q, K, V: _shift(Q, K, np.resize([0.0, 200.0, -200.0, 5.0, 90.0, -15.0, 0.0], Q.shape[1])))


@pytest.mark.parametrize("n,hq,hkv,before", SHAPES)
def test_one_key_far_above_the_others(n, hq, hkv, before):
    # late in the walk, so that what was summed before it has to shrink: in the last tile that all see, and among the new ones
    print(f"case attend4 late peak {n} {hq} {hkv} {before}", flush=True)

    def change(Q, K, V):
        k, q = gen.bf16_bits_to_f32(K), gen.bf16_bits_to_f32(Q)
        q[..., :32] = 4.0
        k[..., :32] = 0.0
        k[:, before - 3, :32] = 4.0
        k[:, before // 2, :32] = 3.0
        _write(K, k)
        _write(Q, q)
    _run(n, hq, hkv, before, change)


@pytest.mark.parametrize("n,hq,hkv,before", SHAPES)
@pytest.mark.parametrize("exponent,offset", [(110, 0.0), (110, 25.0), (-98, 0.0), (-98, -13.0)])
def test_values_large_and_small(n, hq, hkv, before, exponent, offset):
    print(f"case attend4 values 2^{exponent} {offset} {n} {hq} {hkv} {before}", flush=True)

    def change(Q, K, V):
        _write(V, gen.bf16_bits_to_f32(V) * np.float32(2.0 ** exponent))
        _shift(Q, K, np.full(Q.shape[1], offset))
    _run(n, hq, hkv, before, change)


@pytest.mark.parametrize("first,later", [(0.0, 0.0), (-60.0, -60.0), (75.0, 75.0), (0.0, 120.0), (-60.0, 75.0), (-60.0, -250.0)])
def test_long_walks(first, later):
    """64 heads, 1024 tokens behind 16500: every workgroup walks over 256 tiles of 64 keys and more.  Scores of the first tile, and of the others, far from 0."""
    print(f"case attend4 long walk {first} {later}", flush=True)
    hq, hkv, n, before = 64, 8, 1024, 16500

    def change(Q, K, V):
        q, k = gen.bf16_bits_to_f32(Q), gen.bf16_bits_to_f32(K)
        q[..., :32] = 1.5
        k[..., :32] = later / (32 * 1.5 * 128.0 ** -0.5)  # before it becomes codes: about that far
        k[:, :64, :32] = first / (32 * 1.5 * 128.0 ** -0.5)
        _write(Q, q)
        _write(K, k)
    ses, c, Q, keys, vals = _setup(hq, hkv, before + n, 5, change)
    rows, splits = sa.sa_cache4_attend_plan(ses.ctx, n, before)
    assert (rows, splits) == (128, 1)
    O = torch.full((hq, n, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ses.attend(c, dev_bf16(Q[:, before:]), before, O)
    torch.cuda.synchronize()
    got = host_f64(O)
    assert np.isfinite(got).all()
    for t in (0, 1, 15, 100, 511, 512, 777, 1023):
        q, k, v = _f64(Q[:, before + t:before + t + 1]), keys[:, :before + t + 1], vals[:, :before + t + 1]
        want, tol = _reference(q, k, v, before + t, rows)
        size = np.abs(q) @ np.repeat(np.abs(k), hq // hkv, 0).transpose(0, 2, 1) * 128.0 ** -0.5 * np.log2(np.e)
        err, tol = np.abs(got[:, t:t + 1] - want), tol + 2.0 ** -20 * np.log(2) * size.max(-1, keepdims=True) * 2 * np.abs(v).max()
        assert (err <= tol).all(), (t, float((err / tol).max()))


@pytest.mark.parametrize("rows,n,hq,hkv,before,far", [(32, 130, 64, 1, 0, 10), (32, 130, 64, 1, 0, 31), (32, 191, 64, 8, 642, 30), (32, 150, 6, 2, 3007, 2950),
                                                      (128, 160, 128, 2, 0, 10), (128, 130, 128, 2, 5, 63), (128, 333, 128, 2, 1000, 1020),
                                                      (128, 90, 32, 8, 8000, 7990), (16, 61, 8, 2, 337, 250), (16, 12, 16, 2, 3001, 2999)])
def test_a_far_key_of_a_wave_that_ends_inside_a_tile(rows, n, hq, hkv, before, far):
    """The wave that ends with the last, partial tile takes its whole tiles with all their keys when it starts anew."""
    print(f"case attend4 far key {n} {hq} {hkv} {before} {far}", flush=True)

    def change(Q, K, V):
        q, k = gen.bf16_bits_to_f32(Q), gen.bf16_bits_to_f32(K)
        q[..., :32], k[..., :32] = 1.5, 0.0
        k[:, far, :32] = 200.0 / (32 * 1.5 * 128.0 ** -0.5)
        _write(Q, q)
        _write(K, k)
    ses = sa.Session(hq, hkv, 256, 64, 32, keep=0.5)
    assert sa.sa_cache4_attend_plan(ses.ctx, n, before)[0] == rows
    _run(n, hq, hkv, before, change)
