"""The decode step over the prefill index with K and V out of the 4-bit cache, against the fp64 oracle of the step on the
values that the cache stands for.

Tolerance: half a step of bf16 of the output, 2^-8 |o|, and fp32 arithmetic: scores off by 128 roundings of 2^-24 of
sum |q k| scale (under 10 here, after scale and log2 e: 2^-13 in all), probabilities in fp32; together under
2^-12 (sum p |v| + |o|)."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from oracle import cache4 as oc
from oracle import decode as dec
from oracle import oracle as orc
from gpu_util import dev_bf16, download_index, host_f64, random_index, upload_index
from test_gpu_cache_decode import _f64, _reference

pytestmark = pytest.mark.gpu


def _case(Hq, Hkv, N, b, extra, override, positions, seed, index=None, keep=0.2, **options):
    print(f"case 4-bit decode Hq={Hq} Hkv={Hkv} N={N} b={b} {options}", flush=True)
    Q, K, V = gen.random_qkv(Hq, Hkv, N + extra, 128, seed=seed)
    ses = sa.Session(Hq, Hkv, N, b, min(64, N), keep=keep, **options)
    Qd, Kd, Vd = dev_bf16(Q), dev_bf16(K), dev_bf16(V)
    if index is None:
        ses.estimate(Qd[:, :N].contiguous(), Kd[:, :N].contiguous())
        ses.build_index(override)
        torch.cuda.synchronize()
        index = download_index(ses)
    else:
        index = index(ses)
        upload_index(ses, index)
    c = ses.cache4(N + extra + 3)
    for t in c.tensors:  # what stands behind the tokens is never read: NaN there
        t.fill_(0xFF)
    at = 0
    for pos in positions:
        ses.append(c, Kd[:, at:pos + 1], Vd[:, at:pos + 1], at)
        at = pos + 1
        q = Qd[:, pos].contiguous()
        o = torch.full_like(q, 7.0)
        ses.decode_cached(c, q, pos, o)
        torch.cuda.synchronize()
        want, tol = _reference(_f64(Q[:, pos]), oc.read(_f64(K[:, :at])), oc.read(_f64(V[:, :at])), b, index, N, pos)
        err = np.abs(host_f64(o) - want)
        assert (err <= tol).all(), (pos, float((err / tol).max()))
    return ses, c


def test_patterns_and_positions():
    _case(6, 2, 1024, 64, 150, [h % 3 for h in range(6)], [1024, 1025, 1030, 1087, 1088, 1151, 1170], 401)
    _case(4, 4, 640, 128, 260, [1, 1, 2, 0], [640, 641, 766, 767, 768, 895, 896], 402)


@pytest.mark.parametrize("options", [dict(diagonal_select=1), dict(block_select=1), dict(block_select=2)])
def test_over_the_selection_options(options):
    _case(4, 2, 1024, 64, 20, [1, 2, 1, 2], [1024, 1043], 403, **options)


@pytest.mark.parametrize("heads", [(1, 1), (24, 3), (128, 2), (8, 1)])
def test_heads(heads):
    _case(*heads, 512, 64, 80, [h % 3 for h in range(heads[0])], [512, 575, 590], 404)


def test_short_prompts():
    _case(2, 1, 64, 64, 70, [1, 2], [64, 127, 133], 405)
    _case(2, 1, 128, 128, 130, [1, 0], [128, 255, 257], 406)


def test_many_generated_tokens():
    _case(4, 2, 512, 64, 3000, [0, 1, 2, 1], [512, 2000, 3511], 407)


@pytest.mark.parametrize("seed", range(6))
def test_hand_made_indexes(seed):
    # arbitrary blocks, columns, diagonals (some heads keep nothing of the prompt), duplicates between the parts
    N, b = 640, 64

    def make(ses):
        return random_index(np.random.default_rng(seed), 6, N, b, ses.cfg.k_vertical, ses.cfg.k_slash, ses.cap_b)

    _case(6, 3, N, b, 100, None, [N, N + 63, N + 64, N + 99], 410 + seed, index=make, k_blocks=120, k_vertical=100, k_slash=40)


def test_nothing_kept_of_the_prompt():
    def make(ses):
        z = np.zeros(2, np.int32)
        return orc.Index(z, z, np.full((2, ses.cfg.k_vertical), -1, np.int32), z, np.full((2, ses.cfg.k_slash), -1, np.int32),
                         np.zeros((2, 11), np.int32), np.full((2, ses.cap_b), -1, np.int32))

    _case(2, 1, 640, 64, 70, None, [640, 702, 703, 704], 420, index=make)


def test_same_bytes_every_time_and_in_a_replayed_graph():
    ses, c = _case(8, 2, 2048, 64, 40, [h % 3 for h in range(8)], [2048, 2087], 430)
    q = torch.randn(8, 128, device="cuda").bfloat16()
    want, o = torch.empty_like(q), torch.empty_like(q)
    ses.decode_cached(c, q, 2087, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.decode_cached(c, q, 2087, o)
    for rep in range(4):
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), rep
        q2, o2, w2 = torch.randn_like(q), torch.empty_like(q), torch.empty_like(q)
        ses.decode_cached(c, q2, 2087, w2)          # eager steps between the replays
        ses.decode_cached(c, q2, 2087, o2)
        torch.cuda.synchronize()
        assert torch.equal(o2, w2)


def test_nan_of_kept_and_other_keys():
    # a NaN in K or V of a key reaches the heads that keep it and no other; in V its whole group
    print("case 4-bit decode NaN", flush=True)
    N, b, pos = 640, 64, 660
    Q, K, V = gen.random_qkv(2, 1, N + 40, 128, seed=431)
    ses = sa.Session(2, 1, N, b, 64, keep=0.5)
    ix = orc.Index(np.ones(2, np.int32), np.array([1, 0], np.int32), np.full((2, ses.cfg.k_vertical), -1, np.int32),
                   np.zeros(2, np.int32), np.full((2, ses.cfg.k_slash), -1, np.int32),
                   np.tile(np.array([0] * 10 + [1], np.int32), (2, 1)), np.full((2, ses.cap_b), -1, np.int32))
    ix.cols[0, 0] = 70
    ix.blkcols[:, 0] = 9
    upload_index(ses, ix)
    V[0, 70, 37] = 0x7F80
    K[0, 80, 3] = 0x7FC0   # kept by nobody
    c = ses.cache4(704)
    ses.append(c, dev_bf16(K)[:, :pos + 1], dev_bf16(V)[:, :pos + 1], 0)
    o = torch.empty((2, 128), dtype=torch.bfloat16, device="cuda")
    ses.decode_cached(c, dev_bf16(Q)[:, pos].contiguous(), pos, o)
    bad = np.zeros((2, 128), bool)
    bad[0, 32:64] = True
    assert (np.isnan(host_f64(o)) == bad).all()


@pytest.mark.parametrize("many", [False, True])
def test_nan_scores_of_whole_heads(many):
    # NaN in every score of a head, of a workgroup or of a wave: the head's output is NaN, the others' are not
    print(f"case 4-bit decode NaN scores {many}", flush=True)
    N, b = (8192, 64) if many else (64, 64)
    pos = N + 40
    Q, K, V = gen.random_qkv(4, 2, pos + 1, 128, seed=432)
    ses = sa.Session(4, 2, N, b, 64, keep=0.9)
    ses.estimate(dev_bf16(Q)[:, :N].contiguous(), dev_bf16(K)[:, :N].contiguous())
    ses.build_index([1, 1, 1, 1])
    K[1, :512 if many else 64, 7] = 0x7FC0
    c = ses.cache4(N + 64)
    ses.append(c, dev_bf16(K), dev_bf16(V), 0)
    q = dev_bf16(Q)[:, pos].contiguous()
    q[1, 9] = float("nan")
    o = torch.empty_like(q)
    ses.decode_cached(c, q, pos, o)
    torch.cuda.synchronize()
    index = download_index(ses)
    bad = [False, True] + [bool((np.asarray(dec.kept_keys(index, h, N, b, pos)) < (512 if many else 64)).any()) for h in (2, 3)]
    assert bad[2] and bad[3]
    assert (np.isnan(host_f64(o)) == np.array(bad)[:, None]).all()
