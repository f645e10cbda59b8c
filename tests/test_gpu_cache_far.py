"""Addresses past 2^32 bytes: long caches, many heads of them, and rows with wide strides.

A cache of zero keys is given one key with a score above 60; all others, 34 million at most, have score 0 and weigh under
2^25 e^-60 = 2^-61 of it, so the output is that key's value, to bf16's rounding of the weight's sum (none) and of the value (none): equal."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from oracle import oracle as orc
from gpu_util import upload_index

pytestmark = pytest.mark.gpu

ONE = 0x38  # 1 in e4m3


def _cache(ses, cap):
    c = ses.cache(cap)
    c.k.zero_()
    c.v.random_(0, 120)
    c.k_scale.fill_(1.0)
    c.v_scale.fill_(1.0)
    c.k_open.zero_()
    c.v_open.normal_()
    return c


@pytest.mark.parametrize("n", [1, 200])
@pytest.mark.parametrize("hq", [1, 4])
def test_a_far_key_of_one_head(n, hq):
    print(f"case far attend n={n} hq={hq}", flush=True)
    cap = 2 ** 25 + 2 ** 20
    ses = sa.Session(hq, 1, 512, 128, 64, keep=0.5)
    c = _cache(ses, cap)
    tokens = cap - 300
    assert tokens * 128 > 2 ** 32
    q = torch.full((hq, n, 128), 8.0, dtype=torch.bfloat16, device="cuda")  # score of a key of ones: 8 * 128 / sqrt(128) = 90
    o = torch.empty_like(q)
    for far in (tokens - 1000, 2 ** 25 + 77, 2 ** 24 - 1, 3):
        c.k[0, far] = ONE
        ses.attend(c, q, tokens - n, o)
        want = c.v[0, far].view(torch.float8_e4m3fn).to(torch.bfloat16)
        assert torch.equal(o, want.expand(hq, n, 128)), far
        c.k[0, far] = 0


@pytest.mark.parametrize("n", [1, 130])
def test_heads_past_32_bits(n):
    print(f"case far attend heads n={n}", flush=True)
    ses = sa.Session(72, 72, 512, 64, 64, keep=0.5)
    cap = 2 ** 19
    assert 64 * cap * 128 >= 2 ** 32
    c = _cache(ses, cap)
    tokens = cap - 30
    at = torch.arange(72, device="cuda") * 7000 + 5
    c.k[torch.arange(72, device="cuda"), at] = ONE
    q = torch.full((72, n, 128), 8.0, dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    ses.attend(c, q, tokens - n, o)
    want = c.v[torch.arange(72, device="cuda"), at].view(torch.float8_e4m3fn).to(torch.bfloat16)
    assert torch.equal(o, want[:, None].expand(72, n, 128))


def test_a_step_over_heads_past_32_bits():
    print("case far decode heads", flush=True)
    H, N, b = 72, 640, 64
    ses = sa.Session(H, H, N, b, 64, keep=0.5)
    cap = 2 ** 19
    c = _cache(ses, cap)
    z = np.zeros(H, np.int32)
    ix = orc.Index(z, z, np.full((H, ses.cfg.k_vertical), -1, np.int32), z, np.full((H, ses.cfg.k_slash), -1, np.int32),
                   np.zeros((H, N // b + 1), np.int32), np.full((H, ses.cap_b), -1, np.int32))
    upload_index(ses, ix)
    at = torch.arange(H, device="cuda") * 7000 + 700
    c.k[torch.arange(H, device="cuda"), at] = ONE
    q = torch.full((H, 128), 8.0, dtype=torch.bfloat16, device="cuda")
    o = torch.empty_like(q)
    ses.decode_cached(c, q, cap - 30, o)
    assert torch.equal(o, c.v[torch.arange(H, device="cuda"), at].view(torch.float8_e4m3fn).to(torch.bfloat16))


def test_appends_and_wide_strides():
    print("case far append", flush=True)
    n, wide = 300, 2 ** 31 + 1024
    room = torch.empty(3 * wide + n * 128, dtype=torch.bfloat16, device="cuda")
    rows = room.as_strided((4, n, 128), (wide, 128, 1))
    near = torch.randn(4, n, 128, device="cuda").bfloat16()
    rows.copy_(near)
    ses = sa.Session(4, 4, 512, 64, 64, keep=0.5)
    a, c = ses.cache(512), ses.cache(512)
    ses.append(a, rows, rows, 0)
    ses.append(c, near, near, 0)
    for x, y in zip(a.tensors[:4], c.tensors[:4]):
        assert torch.equal(x[:, :256 if x.dtype == torch.uint8 else 4], y[:, :256 if x.dtype == torch.uint8 else 4])
    assert torch.equal(a.k_open[:, :44], c.k_open[:, :44])
    rot = sa.Rotary()
    ses.rotate(rot, rows, None, rows, None, 5)
    ses.rotate(rot, near, None, near, None, 5)
    assert torch.equal(rows, near)


def test_append_past_32_bits():
    print("case far append cache", flush=True)
    cap = 2 ** 25 + 128
    ses = sa.Session(2, 2, 512, 64, 64, keep=0.5)
    K = torch.randn(2, 100, 128, device="cuda").bfloat16()
    c, near = ses.cache(cap), ses.cache(128)
    c.k.fill_(0x7F)
    ses.append(c, K, K, cap - 128)
    ses.append(near, K, K, 0)
    assert torch.equal(c.k[:, cap - 128:cap - 64], near.k[:, :64]) and torch.equal(c.k_open[:, :36], near.k_open[:, :36])
    assert torch.equal(c.k_scale[:, -2], near.k_scale[:, 0]) and (c.k[:, cap - 64:] == 0x7F).all() and (c.k[:, :cap - 128] == 0x7F).all()
