"""Causal attention over the 8-bit cache in each of its forms: 32 and 128 query rows a workgroup, with and without splits of the
keys, as sa_cache_attend_plan says of the shapes below (asserted in every case); both types of codes, both sizes of block.
Against fp64 on the values that the cache stands for, on the GPU, one plain product per head.

Tolerance, per element: half a step of bf16 of the output, 2^-8 |o|; and what moves a weight by a part d of itself moves the
output by d (sum p |v| + |o|) at most: probabilities rounded to bf16 2^-8, fp32 sums over the keys (keys 2^-24), the exponential
2^-22, and a score's error: 140 roundings (128 products, their sums, scale, exponent) of 2^-24 of sum |q k| scale, and Q cut into
two codes, each element off by 2^-14 / 224 of the row's largest at most."""
import pytest
import torch

import paper_2412_06198_amd as sa

pytestmark = pytest.mark.gpu

E4M3, E5M2 = sa.SA_CACHE_E4M3, sa.SA_CACHE_E5M2
# query heads, KV heads, new tokens, tokens before them (about), rows of a workgroup, whether the keys are split
SHAPES = {"32 rows": (32, 8, 64, 300, 32, False), "32 rows, splits": (8, 8, 40, 2900, 32, True),
          "128 rows": (32, 8, 1500, 100, 128, False), "128 rows of a head": (32, 32, 1500, 40, 128, False),
          "128 rows, splits": (32, 8, 257, 5100, 128, True)}
FORMS = [name for name in SHAPES if name != "128 rows of a head"]
MANY = [name for name in SHAPES if name.startswith("128")]


def _case(shape, b, rest, kind, seed, scale=0.0, change=None):
    """A session, a cache whose last block holds `rest` tokens, K and V as the cache stands for them, the queries, pos."""
    hq, hkv, n, before, rows, split = SHAPES[shape]
    tokens = (before + n) // b * b + rest
    pos = tokens - n
    print(f"case kernels {shape} b={b} rest={rest} kind={kind} seed={seed}", flush=True)
    ses = sa.Session(hq, hkv, 4 * b, b, 32, keep=0.5, softmax_scale=scale)
    taken, parts = sa.sa_cache_attend_plan(ses.ctx, n, pos)
    assert taken == rows and (parts > 1) == split, (taken, parts)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    K, V = (torch.randn((hkv, tokens, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    K[..., 5::32] *= 4
    q = torch.randn((hq, n, 128), generator=gen, device="cuda").bfloat16()
    if change:
        change(q, K, V, pos)
    c = ses.cache(tokens // b * b + b, kind)
    for t in c.tensors:  # what stands behind the tokens is never read: NaN there
        t.view(torch.uint8).fill_(0x7F)
    ses.append(c, K, V, 0)
    full = tokens // b * b
    f8 = (torch.float8_e4m3fn, torch.float8_e5m2)[kind]

    def read(codes, scales, rows):
        x = codes[:, :full].view(f8).double() * scales[:, :full // b].double().repeat_interleave(b, 1)[..., None]
        return torch.cat([x, rows[:, :rest].double()], 1)

    return ses, c, read(c.k, c.k_scale, c.k_open), read(c.v, c.v_scale, c.v_open), q, pos


def _reference(q, keys, vals, pos, scale=128 ** -0.5):
    hq, n, g, tokens = q.shape[0], q.shape[1], q.shape[0] // keys.shape[0], keys.shape[1]
    o, tol = (torch.empty(q.shape, dtype=torch.float64, device="cuda") for _ in range(2))
    later = torch.arange(tokens, device="cuda") > pos + torch.arange(n, device="cuda")[:, None]
    for h in range(hq):
        x, k, v = q[h].double(), keys[h // g], vals[h // g]
        kt, size = k.T.contiguous(), k.abs().nan_to_num(0, 0, 0)
        p = torch.softmax((x @ kt * scale).masked_fill(later, -torch.inf), -1)
        o[h] = p @ v
        d = (140 * 2.0 ** -24 * (x.abs() @ size.T.contiguous()).masked_fill(later, 0).amax(-1)
             + 2.0 ** -14 / 224 * x.abs().amax(-1) * size.sum(-1).max()) * scale
        d = torch.expm1(d) + 2.0 ** -8 + 2.0 ** -22 + tokens * 2.0 ** -24
        tol[h] = 2.0 ** -8 * o[h].abs() + d[:, None] * (p @ v.abs() + o[h].abs())
    return o, tol


def _attend(ses, c, q, pos):
    o = torch.full_like(q, 7.0)
    ses.attend(c, q, pos, o)
    return o


def _near(o, want, tol, where=None):
    err = (o.double() - want).abs() / tol
    if where is not None:
        err = err[where]
    assert (err <= 1).all(), float(err.max())


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("shape", SHAPES)
def test_ends_of_the_open_block(shape, b, kind):
    # the last tokens in no tile, a short one, a full one but a row, two
    for rest in (0, 1, 63) if b == 64 else (0, 1, 64, 100):
        ses, c, keys, vals, q, pos = _case(shape, b, rest, kind, rest)
        _near(_attend(ses, c, q, pos), *_reference(q, keys, vals, pos))


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("shape", FORMS)
def test_scale_and_large_scores(shape, kind):
    def change(q, K, V, pos):
        q *= 8

    ses, c, keys, vals, q, pos = _case(shape, 64, 17, kind, 1, scale=0.05)
    _near(_attend(ses, c, q, pos), *_reference(q, keys, vals, pos, 0.05))
    ses, c, keys, vals, q, pos = _case(shape, 128, 70, kind, 2, change=change)  # scores of some tens: the running maximum moves often
    _near(_attend(ses, c, q, pos), *_reference(q, keys, vals, pos))


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("shape", FORMS)
def test_queries_of_uneven_elements(shape, kind):
    # rows of large and tiny elements, tiny rows, zeros, and rows of zeros: what the two codes of an element hold
    def change(q, K, V, pos):
        gen = torch.Generator(device="cuda").manual_seed(9)
        q *= 2.0 ** torch.randint(-20, 3, q.shape, generator=gen, device="cuda")
        q[:, ::7] *= 2.0 ** -60
        q[:, 3::7] = 0
        q[:, 5::7, ::2] = 0

    ses, c, keys, vals, q, pos = _case(shape, 64, 30, kind, 3, change=change)
    _near(_attend(ses, c, q, pos), *_reference(q, keys, vals, pos))


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("shape", FORMS)
def test_non_finite_queries(shape, kind):
    def change(q, K, V, pos):
        q[2, 17, 9], q[5, 39, 64], q[5, 20, 100] = float("nan"), float("inf"), float("-inf")

    ses, c, keys, vals, q, pos = _case(shape, 128, 90, kind, 4, change=change)
    o = _attend(ses, c, q, pos)
    bad = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
    bad[2, 17] = bad[5, 39] = bad[5, 20] = True  # an infinite query has scores of both infinities
    assert torch.equal(torch.isnan(o), bad)
    _near(o, *_reference(q.nan_to_num(0, 0, 0), keys, vals, pos), where=~bad)


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("shape", FORMS)
def test_nan_keys_of_later_tokens(shape, b, kind):
    n = SHAPES[shape][2]
    for late in (n // 2, n - 1, 1):
        def change(q, K, V, pos):
            K[:, pos + late, 3] = float("nan")

        ses, c, keys, vals, q, pos = _case(shape, b, 25, kind, 5, change=change)
        o = _attend(ses, c, q, pos)
        assert torch.isnan(o[:, late:]).all()
        keys[:, pos + late] = 0  # no row that is compared sees it
        _near(o[:, :late], *_reference(q[:, :late].contiguous(), keys[:, :pos + late], vals[:, :pos + late], pos))


@pytest.mark.parametrize("value", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("b", [64, 128])
@pytest.mark.parametrize("shape", FORMS)
def test_non_finite_values(shape, b, value):
    # V of a token that all rows see, that some see, in full blocks and in the open one; codes that have infinities, and
    # those that have NaN alone
    n = SHAPES[shape][2]
    for kind, back in ((E5M2, 0), (E5M2, 3), (E4M3, n // 2), (E5M2, n // 2), (E5M2, n - 2), (E5M2, n + 40)):
        def change(q, K, V, pos):
            V[:, pos + n - 1 - back, 9] = value
            V[:, pos + n - 1 - back, 64] = value

        ses, c, keys, vals, q, pos = _case(shape, b, 45, kind, 6, change=change)
        at = pos + n - 1 - back
        stands = vals[0, at, 9].item()  # NaN for an infinity in a full block of e4m3
        o = _attend(ses, c, q, pos)
        bad = torch.zeros(o.shape, dtype=torch.bool, device="cuda")
        bad[:, max(0, at - pos):, 9] = bad[:, max(0, at - pos):, 64] = True
        got = o.double()
        assert (torch.isnan(got[bad]) if stands != stands else got[bad] == stands).all()
        vals[:, at, 9] = vals[:, at, 64] = 0
        _near(o, *_reference(q, keys, vals, pos), where=~bad)


@pytest.mark.parametrize("kind", [E4M3, E5M2])
@pytest.mark.parametrize("shape", FORMS)
def test_strides_in_place_and_replays(shape, kind):
    ses, c, keys, vals, q, pos = _case(shape, 64, 33, kind, 7)
    hq, n, _ = q.shape
    want = _attend(ses, c, q, pos)
    _near(want, *_reference(q, keys, vals, pos))
    turned = q.transpose(0, 1).contiguous().transpose(0, 1)  # tokens outermost
    room = torch.full((n, hq, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    ses.attend(c, turned, pos, room[..., :128].transpose(0, 1))
    assert torch.equal(room[..., :128].transpose(0, 1), want) and (room[..., 128:] == 7.0).all()
    x = q.clone()
    ses.attend(c, x, pos, x)
    assert torch.equal(x, want)
    o = torch.empty_like(q)
    ses.attend_scratch()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.attend(c, q, pos, o)
    for rep in range(3):
        q.copy_(torch.randn_like(q))
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, _attend(ses, c, q, pos)), rep
