"""The 8-bit cache on the GPU against its fp64 oracle: codes, scales and open rows are equal, to the bit."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from oracle import cache as oc
from gpu_util import dev_bf16, host_f64
from helpers import f64

pytestmark = pytest.mark.gpu

FILL = 0x5A


def _session(hkv, block):
    return sa.Session(hkv, hkv, 4 * block, block, 32, keep=0.5)


def _values(heads, n, seed):
    """N(0,1) with spread dimensions, rows of tiny and of large values, zeros."""
    rng = np.random.default_rng(seed)
    x = rng.standard_normal((heads, n, 128), dtype=np.float32)
    x[..., 5::32] *= 8
    x *= np.float32(2.0) ** rng.integers(-12, 3, (heads, n, 1)).astype(np.float32)
    x[:, ::7, 3] = 0
    return gen.f32_to_bf16_bits(x)


def _empty(ses, capacity, kind):
    c = ses.cache(capacity, kind)
    for t in c.tensors:
        t.view(torch.uint8).fill_(FILL)
    return c


def _check(c, side, bits, block, kind, what=""):
    x = f64(bits).numpy()
    codes, scales, rest = oc.contents(x, block, kind)
    full = codes.shape[1]
    raw, sc, op = ((c.k, c.k_scale, c.k_open), (c.v, c.v_scale, c.v_open))[side]
    got = oc.values(kind)[raw.cpu().numpy()]
    assert np.array_equal(got[:, :full], codes, equal_nan=True), what
    assert (sc.cpu().numpy()[:, :full // block] == scales).all(), what
    assert np.array_equal(op.cpu().view(torch.int16).numpy().view(np.uint16)[:, :rest.shape[1]], bits[:, full:]), what
    # what no token belongs to keeps what it held
    assert (raw.cpu().numpy()[:, full:] == FILL).all() and (sc.cpu().view(torch.uint8).numpy().reshape(sc.shape[0], -1)[:, 4 * (full // block):] == FILL).all(), what


@pytest.mark.parametrize("kind", [sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2])
@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("n", [1, 63, 64, 65, 127, 128, 129, 300, 512])
def test_one_call(kind, block, n):
    print(f"case append kind={kind} block={block} n={n}", flush=True)
    ses = _session(3, block)
    c = _empty(ses, 640, kind)
    K, V = _values(3, n, 1), _values(3, n, 2)
    ses.append(c, dev_bf16(K), dev_bf16(V), 0)
    torch.cuda.synchronize()
    _check(c, 0, K, block, kind, "K")
    _check(c, 1, V, block, kind, "V")


@pytest.mark.parametrize("block", [64, 128])
@pytest.mark.parametrize("parts", [[1] * 131, [30, 60, 1, 37, 200, 5], [64, 64, 64, 64, 64], [127, 2, 127, 2], [130, 0, 190, 64, 63]])
def test_bytes_do_not_depend_on_the_calls(block, parts):
    print(f"case append block={block} parts={parts[:6]}", flush=True)
    ses, n = _session(2, block), sum(parts)
    K, V = _values(2, n, 3), _values(2, n, 4)
    Kd, Vd = dev_bf16(K), dev_bf16(V)
    c = _empty(ses, 512, sa.SA_CACHE_E4M3)
    at = 0
    for p in parts:
        ses.append(c, Kd[:, at:at + p], Vd[:, at:at + p], at)
        at += p
    torch.cuda.synchronize()
    _check(c, 0, K, block, sa.SA_CACHE_E4M3, "K")
    _check(c, 1, V, block, sa.SA_CACHE_E4M3, "V")


def test_taken_back_inside_the_open_block():
    print("case append taken back", flush=True)
    ses = _session(2, 64)
    K, V = _values(2, 140, 5), _values(2, 140, 6)
    c = _empty(ses, 256, sa.SA_CACHE_E4M3)
    ses.append(c, dev_bf16(_values(2, 120, 7))[:, :120], dev_bf16(V)[:, :120], 0)   # drafts, 100 of them kept
    ses.append(c, dev_bf16(K)[:, :64], dev_bf16(V)[:, :64], 0)
    ses.append(c, dev_bf16(K)[:, 64:], dev_bf16(V)[:, 64:], 64)
    torch.cuda.synchronize()
    _check(c, 0, K, 64, sa.SA_CACHE_E4M3)
    _check(c, 1, V, 64, sa.SA_CACHE_E4M3)


@pytest.mark.parametrize("kind", [sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2])
def test_every_bf16_value(kind):
    # all 65536 bit patterns: each in a block whose largest magnitude is its own exponent's, and beside the largest finite one
    print(f"case append every value kind={kind}", flush=True)
    ses = _session(1, 64)
    order = np.argsort((np.arange(65536) & 0x7FFF) * 2 + (np.arange(65536) >> 15), kind="stable").astype(np.uint16)
    ascending = order.reshape(1, 512, 128)
    mixed = np.random.default_rng(8).permutation(order).reshape(1, 512, 128)
    c = _empty(ses, 512, kind)
    ses.append(c, dev_bf16(ascending), dev_bf16(mixed), 0)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        _check(c, 0, ascending, 64, kind, "ascending")
        _check(c, 1, mixed, 64, kind, "mixed")


@pytest.mark.parametrize("kind", [sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2])
def test_blocks_of_zeros_tiny_and_non_finite_values(kind):
    print(f"case append edges kind={kind}", flush=True)
    ses = _session(1, 64)
    x = _values(1, 6 * 64, 9)
    x[0, :64] = 0
    x[0, 1, 1] = 0x8000
    x[0, 64:128] = 0x0001                # the least subnormal: below the least scale
    x[0, 128:192, :] = 0x7F7F            # the largest finite value
    x[0, 200, 7] = 0x7F80
    x[0, 201, 8] = 0xFFC1
    x[0, 256:320] = 0xFF80               # nothing finite
    c = _empty(ses, 384, kind)
    ses.append(c, dev_bf16(x), dev_bf16(x[:, ::-1]), 0)
    torch.cuda.synchronize()
    _check(c, 0, x, 64, kind)
    _check(c, 1, np.ascontiguousarray(x[:, ::-1]), 64, kind)


def test_strides():
    print("case append strides", flush=True)
    ses, n = _session(4, 64), 200
    K, V = _values(4, n, 10), _values(4, n, 11)
    packed = torch.cat([dev_bf16(K).transpose(0, 1), dev_bf16(V).transpose(0, 1)], 1).contiguous()   # [n, 8, 128]
    c = _empty(ses, 256, sa.SA_CACHE_E4M3)
    ses.append(c, packed[:, :4].transpose(0, 1), packed[:, 4:].transpose(0, 1), 0)
    torch.cuda.synchronize()
    _check(c, 0, K, 64, sa.SA_CACHE_E4M3)
    _check(c, 1, V, 64, sa.SA_CACHE_E4M3)


def test_far_into_a_long_cache():
    # offsets of the last heads pass 2^31 bytes
    print("case append far", flush=True)
    ses, cap = _session(8, 128), 3 * 2 ** 20
    assert 8 * cap * 128 > 2 ** 31
    c = ses.cache(cap)
    K, V = _values(8, 300, 12), _values(8, 300, 13)
    pos = cap - 384
    for t in c.tensors:
        t.view(torch.uint8).fill_(FILL)
    ses.append(c, dev_bf16(K), dev_bf16(V), pos)
    torch.cuda.synchronize()
    tail = sa.Cache(c.k[:, pos:].contiguous(), c.v[:, pos:].contiguous(), c.k_scale[:, pos // 128:].contiguous(),
                    c.v_scale[:, pos // 128:].contiguous(), c.k_open, c.v_open)
    _check(tail, 0, K, 128, sa.SA_CACHE_E4M3)
    _check(tail, 1, V, 128, sa.SA_CACHE_E4M3)
    assert (c.k[:, :pos] == FILL).all() and (c.v[:, :pos] == FILL).all()
