"""Reading the 8-bit and the 4-bit cache back into bf16, against the fp64 oracles: the values are equal."""
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


def _setup(kind, heads, block, tokens, seed=1, bits=None):
    """A session, a cache of `tokens` tokens with NaN behind them, and the values that it stands for."""
    ses = sa.Session(heads, heads, 4 * block, block, 32, keep=0.5)
    K, V = bits or (_values(heads, tokens, seed), _values(heads, tokens, seed + 1))
    c = ses.cache4(tokens + 70) if kind == "e2m1" else ses.cache(-(-tokens // block) * block + block, kind)
    for t in c.tensors:
        t.view(torch.uint8).fill_(0xFF)
    ses.append(c, dev_bf16(K), dev_bf16(V), 0)
    read = oc4.read if kind == "e2m1" else lambda x: oc8.read(x, block, kind)
    with np.errstate(invalid="ignore"):
        return ses, c, read(f64(K).numpy()), read(f64(V).numpy())


def _out(heads, n):
    return torch.full((heads, n, 128), 7.0, dtype=torch.bfloat16, device="cuda")


def _same(got, want):
    return np.array_equal(host_f64(got), want, equal_nan=True)


@pytest.mark.parametrize("kind", KINDS)
@pytest.mark.parametrize("block", [64, 128])
def test_ranges(kind, block):
    for tokens in (1, 63, 64, 65, 128, 200, 457):
        print(f"case read kind={kind} block={block} tokens={tokens}", flush=True)
        ses, c, keys, vals = _setup(kind, 3, block, tokens)
        for lo, hi in {(0, tokens), (tokens - 1, tokens), (tokens // 2, tokens), (0, 1), (tokens // 3, max(tokens // 3 + 1, tokens - 3))}:
            k, v = _out(3, hi - lo), _out(3, hi - lo)
            ses.read(c, k, v, lo, tokens)
            torch.cuda.synchronize()
            assert _same(k, keys[:, lo:hi]) and _same(v, vals[:, lo:hi]), (lo, hi)


@pytest.mark.parametrize("kind", KINDS)
def test_sides_strides_and_what_is_left_alone(kind):
    print(f"case read strides kind={kind}", flush=True)
    tokens, lo, n = 333, 50, 270
    ses, c, keys, vals = _setup(kind, 4, 64, tokens)
    room = torch.full((n + 2, 4, 2, 136), 7.0, dtype=torch.bfloat16, device="cuda")   # tokens outermost, K and V side by side
    ses.read(c, room[1:n + 1, :, 0, :128].transpose(0, 1), room[1:n + 1, :, 1, :128].transpose(0, 1), lo, tokens)
    torch.cuda.synchronize()
    assert _same(room[1:n + 1, :, 0, :128].transpose(0, 1), keys[:, lo:lo + n]) and _same(room[1:n + 1, :, 1, :128].transpose(0, 1), vals[:, lo:lo + n])
    assert (room[..., 128:] == 7.0).all() and (room[0] == 7.0).all() and (room[-1] == 7.0).all()
    k, v = _out(4, 5), _out(4, 5)
    ses.read(c, k, None, tokens - 5)
    ses.read(c, None, v, tokens - 5)
    torch.cuda.synchronize()
    assert _same(k, keys[:, -5:]) and _same(v, vals[:, -5:])
    before = [t.view(torch.uint8).clone() for t in c.tensors]   # NaN is no value to compare
    ses.read(c, k[:, :0], v[:, :0], 3, tokens)
    torch.cuda.synchronize()
    assert _same(k, keys[:, -5:]) and all(torch.equal(a, b.view(torch.uint8)) for a, b in zip(before, c.tensors))


@pytest.mark.parametrize("kind", KINDS)
def test_values_that_are_no_numbers(kind):
    print(f"case read non-finite kind={kind}", flush=True)
    x = _values(2, 130, 9)
    x[0, 3, 7], x[1, 90, 100], x[1, 129, 5], x[0, 128, 127], x[0, 60] = 0x7F80, 0xFFC1, 0xFF80, 0x7FC0, 0
    ses, c, keys, vals = _setup(kind, 2, 64, 130, bits=(x, np.ascontiguousarray(x[:, ::-1])))
    k, v = _out(2, 130), _out(2, 130)
    ses.read(c, k, v)
    torch.cuda.synchronize()
    assert _same(k, keys) and _same(v, vals)


@pytest.mark.parametrize("kind", KINDS)
def test_every_code(kind):
    # all bytes as codes under several scales, the least and the largest among them
    print(f"case read codes kind={kind}", flush=True)
    ses = sa.Session(1, 1, 256, 64, 32, keep=0.5)
    codes = np.arange(256, dtype=np.uint8)
    if kind == "e2m1":
        c = ses.cache4(256)
        raw, sc = np.resize(np.random.default_rng(3).permutation(codes), (1, 256, 64)), np.zeros((1, 256, 4), np.uint8)
        raw[0, :, :] = (np.arange(256)[:, None] + 5 * np.arange(64)) & 255
        sc[0] = np.array([27, 100, 127, 252])[(np.arange(256)[:, None] + np.arange(4)) % 4]
        sc[0, ::17, 1] = 255
        want = oc4.values(raw, sc)
        k = _out(1, 256)
        c.k.copy_(torch.from_numpy(raw)); c.k_scale.copy_(torch.from_numpy(sc))
        ses.read(c, k, None)
    else:
        c = ses.cache(256, kind)
        raw = np.resize(codes, (1, 256, 128))
        sc = np.array([[2.0 ** -100, 2.0 ** -3, 1.0, 2.0 ** 100]], np.float32)
        want = oc8.values(kind)[raw] * np.repeat(sc.astype(np.float64), 64, 1)[..., None]
        k = _out(1, 256)
        c.k.copy_(torch.from_numpy(raw)); c.k_scale.copy_(torch.from_numpy(sc))
        ses.read(c, k, None)
    torch.cuda.synchronize()
    assert _same(k, want)


def test_session_refusals():
    print("case read refusals", flush=True)
    ses, c, keys, _ = _setup("e2m1", 2, 64, 100)
    for k, v, pos, tokens in ((None, None, 0, None), (_out(3, 5), None, 0, None), (_out(2, 5).float(), None, 0, None), (_out(2, 5), _out(2, 6), 0, None),
                              (_out(2, 5), None, 0, 4), (_out(2, 5), None, -1, None), (_out(2, 5), None, 166, None), (_out(2, 5).cpu(), None, 0, None),
                              (_out(1, 5).expand(2, 5, 128), None, 0, None)):
        with pytest.raises(sa.SaError):
            ses.read(c, k, v, pos, tokens)
    other = sa.Session(4, 4, 256, 64, 32, keep=0.5)
    with pytest.raises(sa.SaError):
        other.read(c, _out(4, 5), None)
    with pytest.raises(sa.SaError):
        other.append(c, _out(4, 5), _out(4, 5), 0)
    wide = sa.Session(2, 2, 256, 128, 32, keep=0.5)   # a 4-bit cache has no blocks: any session of its heads
    k = _out(2, 100)
    wide.read(c, k, None)
    torch.cuda.synchronize()
    assert _same(k, keys)
