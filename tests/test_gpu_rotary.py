"""Rotary positions on the GPU against the fp64 oracle.

Tolerance: one rounding to bf16, half a step = 2^-8 of the value, and the fp32 arithmetic before it: sine and cosine to
2^-22 (an angle exact to 2^-32 of a turn, as fp32 2^-25 of half a turn, and a few ulp of the function), two products
and a sum, together under 2^-20 (|x| + |y|) amplitude."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from oracle import rotary as orot
from gpu_util import dev_bf16, host_f64
from helpers import f64

pytestmark = pytest.mark.gpu


def _session(hq=4, hkv=2):
    return sa.Session(hq, hkv, 512, 64, 64, keep=0.3)


def _bits(heads, n, seed):
    return gen.f32_to_bf16_bits(np.random.default_rng(seed).standard_normal((heads, n, 128), dtype=np.float32))


def _check(got, bits, positions, config, what):
    dim = config.get("rotary_dim", 128) or 128
    w = orot.frequencies(dim, config.get("theta", 10000.0) or 10000.0, config.get("scaling", 0), config.get("factor", 1.0),
                         config.get("low", 1.0), config.get("high", 4.0), config.get("original_len", 8192.0))
    amp = orot.amplitude(config.get("scaling", 0), config.get("factor", 1.0), config.get("amplitude", 0.0))
    x = f64(bits).numpy()
    want = orot.rotate(x, positions, w, config.get("layout", 0) == sa.SA_ROTARY_INTERLEAVED, bool(config.get("transposed", 0)), amp)
    part = np.sqrt(np.maximum(want ** 2, 0))
    half = dim // 2
    both = np.zeros_like(x)
    a, b = (np.arange(0, dim, 2), np.arange(1, dim, 2)) if config.get("layout", 0) else (np.arange(half), np.arange(half, dim))
    both[..., a] = both[..., b] = np.abs(x[..., a]) + np.abs(x[..., b])
    tol = 2.0 ** -8 * part + 2.0 ** -20 * amp * both
    err = np.abs(host_f64(got) - want)
    assert (err <= tol).all(), (what, float((err - tol).max()))
    assert (host_f64(got)[..., dim:] == x[..., dim:]).all(), what


CONFIGS = [dict(), dict(layout=1), dict(rotary_dim=64), dict(rotary_dim=64, layout=1), dict(rotary_dim=96), dict(rotary_dim=40),
           dict(rotary_dim=36, layout=1), dict(rotary_dim=36), dict(rotary_dim=20), dict(rotary_dim=2), dict(rotary_dim=2, layout=1), dict(rotary_dim=126),
           dict(transposed=1), dict(layout=1, transposed=1, amplitude=0.7), dict(scaling=sa.SA_SCALING_LINEAR, factor=4.0),
           dict(scaling=sa.SA_SCALING_BASE, factor=8.0), dict(rotary_dim=2, scaling=sa.SA_SCALING_BASE, factor=8.0),
           dict(scaling=sa.SA_SCALING_WAVELENGTH, theta=500000.0, factor=8.0, low=1.0, high=4.0, original_len=8192),
           dict(scaling=sa.SA_SCALING_RAMP, theta=1e6, factor=4.0, low=1.0, high=32.0, original_len=32768),
           dict(scaling=sa.SA_SCALING_RAMP, rotary_dim=64, layout=1, factor=16.0, low=1.0, high=32.0, original_len=4096, transposed=1)]


@pytest.mark.parametrize("config", CONFIGS, ids=lambda c: "-".join(f"{k}{v}" for k, v in c.items()) or "default")
def test_layouts_dims_and_scalings(config):
    print(f"case rotary {config}", flush=True)
    ses, n, pos = _session(), 37, 131000
    rot = sa.Rotary(**config)
    Q, K = _bits(4, n, 1), _bits(2, n, 2)
    Qd, Kd = dev_bf16(Q), dev_bf16(K)
    Qo, Ko = torch.full_like(Qd, 7.0), torch.full_like(Kd, 7.0)
    ses.rotate(rot, Qd, Kd, Qo, Ko, pos=pos)
    at = np.arange(pos, pos + n)
    _check(Qo, Q, at, config, "Q")
    _check(Ko, K, at, config, "K")
    ses.rotate(rot, Qd, Kd, Qd, Kd, pos=pos)      # in place
    assert torch.equal(Qd, Qo) and torch.equal(Kd, Ko)


@pytest.mark.parametrize("heads", [(1, 1), (6, 2), (24, 3), (128, 1)])
@pytest.mark.parametrize("n", [1, 2, 33, 700])
def test_heads_and_lengths(heads, n):
    print(f"case rotary heads={heads} n={n}", flush=True)
    ses = _session(*heads)
    rot = sa.Rotary()
    Q, K = _bits(heads[0], n, 3), _bits(heads[1], n, 4)
    Qd, Kd = dev_bf16(Q), dev_bf16(K)
    Qo, Ko = torch.full_like(Qd, 7.0), torch.full_like(Kd, 7.0)
    ses.rotate(rot, Qd, Kd, Qo, Ko, pos=5)
    _check(Qo, Q, np.arange(5, 5 + n), {}, "Q")
    _check(Ko, K, np.arange(5, 5 + n), {}, "K")


def test_positions_far_negative_repeated():
    print("case rotary positions", flush=True)
    ses, rot = _session(), sa.Rotary()
    at = np.array([0, 2 ** 31 - 1, -(2 ** 31), -1, 131072, 131072, 16777217, 3, 3], np.int32)
    Q, K = _bits(4, len(at), 5), _bits(2, len(at), 6)
    Qd, Kd = dev_bf16(Q), dev_bf16(K)
    Qo, Ko = torch.full_like(Qd, 7.0), torch.full_like(Kd, 7.0)
    ses.rotate(rot, Qd, Kd, Qo, Ko, positions=torch.from_numpy(at).cuda())
    _check(Qo, Q, at, {}, "Q")
    _check(Ko, K, at, {}, "K")
    ses.rotate(rot, Qd, None, Qo, None, pos=2 ** 31 - len(at))
    _check(Qo, Q, np.arange(2 ** 31 - len(at), 2 ** 31), {}, "last positions")


def test_strides_and_one_side():
    # tokens outermost, heads inside, as projections give them; outputs in another order, what lies between untouched
    print("case rotary strides", flush=True)
    ses, rot, n = _session(), sa.Rotary(layout=1, rotary_dim=64), 19
    Q, K = _bits(4, n, 7), _bits(2, n, 8)
    packed = torch.cat([dev_bf16(Q).transpose(0, 1), dev_bf16(K).transpose(0, 1)], 1).contiguous()   # [n, 6, 128]
    Qd, Kd = packed[:, :4].transpose(0, 1), packed[:, 4:].transpose(0, 1)
    room = torch.full((4, n, 136), 7.0, dtype=torch.bfloat16, device="cuda")
    Qo, Ko = room[..., :128], torch.full((2, n, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    ses.rotate(rot, Qd, Kd, Qo, Ko, pos=9)
    at = np.arange(9, 9 + n)
    _check(Qo, Q, at, dict(layout=1, rotary_dim=64), "Q")
    _check(Ko, K, at, dict(layout=1, rotary_dim=64), "K")
    assert (room[..., 128:] == 7.0).all()
    before = packed.clone()
    ses.rotate(rot, None, Kd, None, Kd, pos=9)     # one side in place inside the packed tensor
    assert torch.equal(packed[:, :4], before[:, :4]) and torch.equal(packed[:, 4:].transpose(0, 1), Ko)
    ses.rotate(rot, Qd[:, :0], Kd[:, :0], Qd[:, :0], Kd[:, :0])  # no rows


@pytest.mark.parametrize("layout", [0, 1])
def test_transposed_is_the_gradient(layout):
    # <g, R x> = <R^T g, x> for the map as computed, and against differences: R is linear, so R(x + d) - R(x) = R d.
    # bf16 outputs: each side is off by at most 2^-8 of its terms' magnitudes.
    print(f"case rotary gradient layout={layout}", flush=True)
    ses, n = _session(1, 1), 16
    config = dict(layout=layout, rotary_dim=96, amplitude=1.3)
    fwd, back = sa.Rotary(**config), sa.Rotary(transposed=1, **config)
    X, G = _bits(1, n, 9), _bits(1, n, 10)
    Xd, Gd = dev_bf16(X), dev_bf16(G)
    Y, D = torch.empty_like(Xd), torch.empty_like(Gd)
    ses.rotate(fwd, Xd, None, Y, None, pos=77)
    ses.rotate(back, Gd, None, D, None, pos=77)
    x, g, y, d = (host_f64(t) for t in (Xd, Gd, Y, D))
    room = 2.0 ** -8 * (np.abs(g * y) + np.abs(d * x)).sum()
    assert abs((g * y).sum() - (d * x).sum()) <= room
    step = dev_bf16(gen.f32_to_bf16_bits(np.random.default_rng(11).standard_normal((1, n, 128), dtype=np.float32)))
    moved, Ym = Xd.float() + step.float(), torch.empty_like(Xd)
    ses.rotate(fwd, moved.bfloat16(), None, Ym, None, pos=77)
    delta = host_f64(moved.bfloat16()) - x
    change = (g * (host_f64(Ym) - y)).sum()
    assert abs(change - (d * delta).sum()) <= 2.0 ** -8 * (np.abs(g) * (np.abs(host_f64(Ym)) + np.abs(y)) + np.abs(d * delta)).sum()


def test_nan_stays_in_its_pair():
    print("case rotary NaN", flush=True)
    ses, n = _session(1, 1), 4
    Q = _bits(1, n, 12)
    Q[0, 2, 5] = 0x7FC0
    Qd = dev_bf16(Q)
    Qo = torch.empty_like(Qd)
    ses.rotate(sa.Rotary(), Qd, None, Qo, None, pos=3)
    bad = np.zeros((1, n, 128), bool)
    bad[0, 2, [5, 69]] = True
    assert (np.isnan(host_f64(Qo)) == bad).all()


def test_replays_on_another_stream():
    print("case rotary graph", flush=True)
    ses, rot, n = _session(), sa.Rotary(), 65
    Qd, Kd = dev_bf16(_bits(4, n, 13)), dev_bf16(_bits(2, n, 14))
    at = torch.arange(n, dtype=torch.int32, device="cuda")
    Qo, Ko = torch.empty_like(Qd), torch.empty_like(Kd)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.rotate(rot, Qd, Kd, Qo, Ko, positions=at)
    for rep in range(3):
        at += 100
        Qo.fill_(7.0)
        Ko.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        Qe, Ke = torch.empty_like(Qd), torch.empty_like(Kd)
        ses.rotate(rot, Qd, Kd, Qe, Ke, positions=at)
        torch.cuda.synchronize()
        assert torch.equal(Qo, Qe) and torch.equal(Ko, Ke), rep
