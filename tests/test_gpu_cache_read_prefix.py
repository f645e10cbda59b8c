"""Session.read without a number of tokens: a cache that was filled through append() knows how many it holds, so that any part of it is read as it is, a prefix that
ends inside a block among them."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from oracle import cache as oc8
from oracle import cache4 as oc4
from gpu_util import dev_bf16, host_f64
from helpers import f64
from test_gpu_cache4_append import _values

pytestmark = pytest.mark.gpu

KINDS = ["e2m1", sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2]


def _setup(kind, block, tokens):
    ses = sa.Session(3, 3, 4 * block, block, 32, keep=0.5)
    K, V = _values(3, tokens, 1), _values(3, tokens, 2)
    c = ses.cache4(tokens + 70) if kind == "e2m1" else ses.cache(-(-tokens // block) * block + block, kind)
    return ses, c, K, V


def _held(kind, block, bits):
    return oc4.read(f64(bits).numpy()) if kind == "e2m1" else oc8.read(f64(bits).numpy(), block, kind)


def _read(ses, c, lo, hi):
    k, v = (torch.full((3, hi - lo, 128), 7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ses.read(c, k, v, lo)
    torch.cuda.synchronize()
    return host_f64(k), host_f64(v)


def _check(ses, c, kind, block, K, V, tokens):
    keys, vals = _held(kind, block, K[:, :tokens]), _held(kind, block, V[:, :tokens])
    for lo, hi in {(0, 1), (0, tokens), (tokens - 1, tokens), (tokens // 3, tokens - tokens // 4), (0, tokens - block // 2), (tokens // 2, tokens - 1), (0, block)}:
        if 0 <= lo < hi <= tokens:
            k, v = _read(ses, c, lo, hi)
            assert np.array_equal(k, keys[:, lo:hi]) and np.array_equal(v, vals[:, lo:hi]), (tokens, lo, hi)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [64, 128])
def test_prefixes(kind, block):
    for tokens in (2, block - 1, block, block + 1, 2 * block + 40, 457):
        print(f"case read prefix kind={kind} block={block} tokens={tokens}", flush=True)
        ses, c, K, V = _setup(kind, block, tokens)
        ses.append(c, dev_bf16(K), dev_bf16(V), 0)
        assert c.tokens == tokens
        _check(ses, c, kind, block, K, V, tokens)


@pytest.mark.parametrize("kind", KINDS)
def test_in_several_calls(kind):
    print(f"case read prefix calls kind={kind}", flush=True)
    block, tokens = 64, 300
    ses, c, K, V = _setup(kind, block, tokens)
    assert c.tokens == 0
    Kd, Vd, at = dev_bf16(K), dev_bf16(V), 0
    for n in (100, 0, 27, 1, 1, 62, 64, 45):
        ses.append(c, Kd[:, at:at + n], Vd[:, at:at + n], at)
        at += n
        assert c.tokens == at
        _check(ses, c, kind, block, K, V, at)
    append = sa.sa_cache4_append if kind == "e2m1" else sa.sa_cache_append
    append(ses.ctx, c, sa.SaRows(), sa.SaRows(), 0, 200, ses.stream())
    assert c.tokens == 200
    with pytest.raises(sa.SaError):
        ses.append(c, Kd, Vd, 2 ** 20)   # no room: the cache holds what it held
    assert c.tokens == 200


@pytest.mark.parametrize("kind", KINDS[1:])
def test_taken_back(kind):
    print(f"case read prefix taken back kind={kind}", flush=True)
    block, tokens = 64, 200
    ses, c, K, V = _setup(kind, block, tokens)
    Kd, Vd = dev_bf16(K), dev_bf16(V)
    ses.append(c, Kd[:, :190], Vd[:, :190], 0)
    kept = c.k_open.clone(), c.v_open.clone()
    ses.append(c, Kd[:, 190:195], Vd[:, 190:195], 190)   # fills a block
    _check(ses, c, kind, block, K, V, 195)
    for x, y in zip((c.k_open, c.v_open), kept):
        x.copy_(y)
    ses.append(c, Kd[:, :0], Vd[:, :0], 190)             # none of them stays
    _check(ses, c, kind, block, K, V, 190)
    ses.append(c, Kd[:, 150:170], Vd[:, 150:170], 150)   # back inside the open block
    _check(ses, c, kind, block, K, V, 170)


@pytest.mark.parametrize("kind", KINDS[1:])
def test_buffers_from_elsewhere(kind):
    # nothing says how many tokens they hold: the number given, or as many as the call reads up to
    print(f"case read prefix buffers kind={kind}", flush=True)
    block, tokens = 64, 200
    ses, c, K, V = _setup(kind, block, tokens)
    ses.append(c, dev_bf16(K), dev_bf16(V), 0)
    own = sa.Cache(*c.tensors, kind)
    assert own.tokens is None
    keys = _held(kind, block, K)
    out = torch.empty((3, 170, 128), dtype=torch.bfloat16, device="cuda")
    ses.read(own, out, None, 30)
    torch.cuda.synchronize()
    assert np.array_equal(host_f64(out), keys[:, 30:])
    ses.read(own, out, None, 0, tokens)
    torch.cuda.synchronize()
    assert np.array_equal(host_f64(out), keys[:, :170])
    own.tokens = tokens
    out.fill_(7.0)
    ses.read(own, out, None, 0)
    torch.cuda.synchronize()
    assert np.array_equal(host_f64(out), keys[:, :170])
