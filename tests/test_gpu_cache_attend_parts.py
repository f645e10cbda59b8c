"""Attention over the 8-bit cache for at most 64 query rows a KV head (steps, drafted tokens): probabilities in two parts, so that an
output is off by little more than its own rounding.

Tolerance: 2^-8 |o| (half a step of bf16), and d (sum p |v| + |o|) with d = 2^-15 of the rest of a probability in bf16, 2^-22 of
the exponential, keys 2^-24 of the sums, and a score's error, 140 roundings of 2^-24 of sum |q k| scale."""
import pytest
import torch

import paper_2412_06198_amd as sa

pytestmark = pytest.mark.gpu


def _contents(codes, scales, rows, kind, b, tokens):
    full = tokens // b * b
    f8 = (torch.float8_e4m3fn, torch.float8_e5m2)[kind]
    x = codes[:, :full].view(f8).double() * scales[:, :full // b].double().repeat_interleave(b, 1)[..., None]
    return torch.cat([x, rows[:, :tokens - full].double()], 1)


def _setup(hq, hkv, b, n, tokens, kind, seed, change=None):
    print(f"case parts hq={hq} hkv={hkv} b={b} n={n} tokens={tokens} kind={kind}", flush=True)
    ses = sa.Session(hq, hkv, 4 * b, b, 32, keep=0.5)
    assert sa.sa_cache_attend_plan(ses.ctx, n, tokens - n)[0] == 32
    gen = torch.Generator(device="cuda").manual_seed(seed)
    K, V = (torch.randn((hkv, tokens, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    V[..., 5::32] *= 4
    if change:
        change(K, V)
    c = ses.cache(tokens // b * b + b, kind)
    ses.append(c, K, V, 0)
    q = torch.randn((hq, n, 128), generator=gen, device="cuda").bfloat16()
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, tokens - n, o)
    return q, o, _contents(c.k, c.k_scale, c.k_open, kind, b, tokens), _contents(c.v, c.v_scale, c.v_open, kind, b, tokens)


def _reference(q, keys, vals):
    hq, n, g, tokens = q.shape[0], q.shape[1], q.shape[0] // keys.shape[0], keys.shape[1]
    pos = tokens - n
    o, tol = (torch.empty(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    later = torch.arange(tokens, device="cuda") > pos + torch.arange(n, device="cuda")[:, None]
    for h in range(hq):
        x, kt, v = q[h].double(), keys[h // g].T.contiguous(), vals[h // g]
        p = torch.softmax((x @ kt * 128 ** -0.5).masked_fill(later, -torch.inf), -1)
        o[h] = p @ v
        d = torch.expm1(140 * 2.0 ** -24 * 128 ** -0.5 * (x.abs() @ kt.abs()).amax(-1)) + 2.0 ** -15 + 2.0 ** -22 + tokens * 2.0 ** -24
        tol[h] = 2.0 ** -8 * o[h].abs() + d[:, None] * (p @ v.abs() + o[h].abs())
    return o, tol


@pytest.mark.parametrize("kind", [sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("heads,n", [((32, 8), 1), ((8, 1), 1), ((8, 1), 4), ((8, 1), 5), ((8, 1), 8), ((4, 4), 33), ((128, 2), 1), ((6, 2), 21)])
def test_little_more_than_the_rounding(heads, n, b, kind):
    for tokens in (n, n + 90, 1000, 4133, 20003):
        q, o, keys, vals = _setup(*heads, b, n, tokens, kind, tokens)
        want, tol = _reference(q, keys, vals)
        err = (o.double() - want).abs() / tol
        assert (err <= 1).all(), float(err.max())


@pytest.mark.parametrize("value", [float("inf"), float("-inf")])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("n", [1, 8])
def test_infinite_values_of_small_weights(n, b, value):
    # keys with scores down to some 70 below the row's largest: weights of 2^-100 and less, whose rest is small or nearly 0
    tokens = 3000

    def change(K, V):
        K[:, ::50] *= torch.linspace(-1, 1, 60, device="cuda")[:, None].bfloat16() * 4
        V[:, 150::300, 9] = value    # seen by all rows, in full blocks
        V[:, -1, 70] = value         # in the open block, by the last row

    q, o, keys, vals = _setup(8, 1, b, n, tokens, sa.SA_CACHE_E5M2, 3, change)
    bad = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
    bad[..., 9] = bad[:, -1, 70] = True
    assert (o[bad] == value).all()
    vals[:, 150::300, 9] = vals[:, -1, 70] = 0
    want, tol = _reference(q, keys, vals)
    assert ((o.double() - want).abs() <= tol)[~bad].all()
