"""The 4-bit cache at addresses past 2^32 bytes: long caches, many heads of them, and rows with wide strides.

A cache of zero keys is given one key with a score above 60; all others, 70 million at most, have score 0 and weigh under
2^27 e^-60 = 2^-59 of it, so the output is that key's value, to bf16's rounding of the weight's sum (none) and of the value (none): equal."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from oracle import cache4 as oc
from oracle import oracle as orc
from gpu_util import host_f64, upload_index
from test_gpu_cache4_attend import _reference

pytestmark = pytest.mark.gpu

ONES = 0x22  # two codes of 1


def _cache(ses, cap):
    c = ses.cache4(cap)
    c.k.zero_()
    c.v.random_(0, 256)
    c.k_scale.fill_(127)
    c.v_scale.random_(120, 135)
    return c


def _value(c, head, at):
    return oc.values(c.v[head, at].cpu().numpy(), c.v_scale[head, at].cpu().numpy())


@pytest.mark.parametrize("n", [1, 40, 200])
@pytest.mark.parametrize("hq", [1, 4])
def test_a_far_key_of_one_head(n, hq):
    print(f"case far attend4 n={n} hq={hq}", flush=True)
    cap = 2 ** 26 + 2 ** 20 + 1
    ses = sa.Session(hq, 1, 512, 128, 64, keep=0.5)
    c = _cache(ses, cap)
    tokens = cap - 300
    assert tokens * 64 > 2 ** 32
    q = torch.full((hq, n, 128), 8.0, dtype=torch.bfloat16, device="cuda")  # score of a key of ones: 8 * 128 / sqrt(128) = 90
    o = torch.empty_like(q)
    for far in (tokens - 1000, 2 ** 26 + 77, 2 ** 25 - 1, 3):
        c.k[0, far] = ONES
        ses.attend(c, q, tokens - n, o)
        assert (host_f64(o) == _value(c, 0, far)).all(), far
        c.k[0, far] = 0


@pytest.mark.parametrize("n", [1, 20, 130])
def test_heads_past_32_bits(n):
    print(f"case far attend4 heads n={n}", flush=True)
    ses = sa.Session(72, 72, 512, 64, 64, keep=0.5)
    cap = 2 ** 20
    assert 64 * cap * 64 >= 2 ** 32
    c = _cache(ses, cap)
    heads = torch.arange(72, device="cuda")
    at = heads * 7000 + 5
    c.k[heads, at] = ONES
    q = torch.full((72, n, 128), 8.0, dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    ses.attend(c, q, cap - 30 - n, o)
    assert (host_f64(o) == _value(c, heads, at)[:, None]).all()


def test_a_step_over_heads_past_32_bits():
    print("case far decode4 heads", flush=True)
    H, N, b = 72, 640, 64
    ses = sa.Session(H, H, N, b, 64, keep=0.5)
    cap = 2 ** 20
    c = _cache(ses, cap)
    z = np.zeros(H, np.int32)
    ix = orc.Index(z, z, np.full((H, ses.cfg.k_vertical), -1, np.int32), z, np.full((H, ses.cfg.k_slash), -1, np.int32),
                   np.zeros((H, N // b + 1), np.int32), np.full((H, ses.cap_b), -1, np.int32))
    upload_index(ses, ix)
    heads = torch.arange(H, device="cuda")
    at = heads * 7000 + 700
    c.k[heads, at] = ONES
    q = torch.full((H, 128), 8.0, dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    ses.decode_cached(c, q, cap - 30, o)
    assert (host_f64(o) == _value(c, heads, at)).all()


def test_wide_strides():
    print("case far append4, read", flush=True)
    n, wide = 300, 2 ** 31 + 1024
    room = torch.zeros(3 * wide + n * 128, dtype=torch.bfloat16, device="cuda")
    rows = room.as_strided((4, n, 128), (wide, 128, 1))
    near = torch.randn(4, n, 128, device="cuda").bfloat16()
    rows.copy_(near)
    ses = sa.Session(4, 4, 512, 64, 64, keep=0.5)
    a, c = ses.cache4(512), ses.cache4(512)
    ses.append(a, rows, rows, 0)
    ses.append(c, near, near, 0)
    for x, y in zip(a.tensors, c.tensors):
        assert torch.equal(x[:, :n], y[:, :n])
    ses.read(a, rows, None)
    ses.read(a, near, None)
    assert torch.equal(rows, near)
    e = ses.cache(512)
    ses.append(e, near, near, 0)
    ses.read(e, None, rows)
    ses.read(e, None, near)
    assert torch.equal(rows, near)


def test_read_of_8_bits_past_32_bits():
    print("case far read", flush=True)
    cap = 2 ** 25 + 128
    ses = sa.Session(2, 2, 512, 64, 64, keep=0.5)
    c = ses.cache(cap)
    K = torch.randn(2, 300, 128, device="cuda").bfloat16()
    ses.append(c, K, K, cap - 320)
    near = ses.cache(512)
    ses.append(near, K, K, 0)
    x, y = torch.empty_like(K), torch.empty_like(K)
    ses.read(c, x, None, cap - 320)
    ses.read(near, y, None, 0)
    assert torch.equal(x, y)


def test_more_row_tiles_than_a_grid_is_deep():
    """128 heads on 2 KV heads, 66000 tokens at once: 33000 tiles of 128 query rows a KV head, over the 32768 that stand one behind the other."""
    print("case attend4 33000 row tiles", flush=True)
    hq, hkv, n = 128, 2, 66000
    ses = sa.Session(hq, hkv, 256, 64, 32, keep=0.5)
    c = ses.cache4(n)
    made = torch.Generator(device="cuda").manual_seed(3)
    K, V = (torch.randn((hkv, n, 128), generator=made, device="cuda").bfloat16() for _ in range(2))
    ses.append(c, K, V, 0)
    ses.read(c, K, V)
    Q = torch.randn((hq, n, 128), generator=made, device="cuda", dtype=torch.bfloat16)
    assert sa.sa_cache4_attend_plan(ses.ctx, n, 0) == (128, 1)
    O = torch.full_like(Q, 7.0)
    ses.attend(c, Q, 0, O)
    torch.cuda.synchronize()
    assert not bool((O == 7.0).all(-1).any())
    for t in (0, 1, 2, 447, 448, 449, 33000, 65535, 65536, 65999):  # 2 tokens a tile: the first 232 tiles stand beside the KV heads
        want, tol = _reference(host_f64(Q[:, t:t + 1]), host_f64(K[:, :t + 1]), host_f64(V[:, :t + 1]), t, 128)
        err = np.abs(host_f64(O[:, t:t + 1]) - want)
        assert (err <= tol).all(), (t, float((err / tol).max()))
