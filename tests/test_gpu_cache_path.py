"""The operators together, as a serving program runs a layer: rotated prompt, index and sparse prefill, the cache filled, sparse
decode steps with each token rotated and appended, then a further turn attended densely; and the session's refusals."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from oracle import cache as oc
from oracle import decode as dec
from oracle import rotary as orot
from gpu_util import dev_bf16, download_index, host_f64

pytestmark = pytest.mark.gpu


def _layer(seed, Hq=8, Hkv=2, N=2048, b=64, extra=200):
    Q, K, V = gen.random_qkv(Hq, Hkv, N + extra, 128, seed=seed)
    ses = sa.Session(Hq, Hkv, N, b, 64, keep=0.2)
    return ses, sa.Rotary(theta=500000.0), (dev_bf16(Q), dev_bf16(K), dev_bf16(V))


def _run(ses, rot, tensors, steps, turn, step):
    """What a program does; returns the outputs of the prefill, of `steps` decode steps and of a turn of `turn` tokens."""
    Q, K, V = tensors
    N = ses.cfg.seq_len
    q, k, v = (x[:, :N].contiguous() for x in (Q, K, V))
    ses.rotate(rot, q, k, q, k)
    O = torch.empty_like(q)
    ses.estimate_and_index(q, k)
    ses.prefill(q, k, v, O)
    cache = ses.cache(N + 256)
    ses.append(cache, k, v, 0)
    outs = []
    for pos in range(N, N + steps):
        outs.append(step(ses, rot, cache, Q[:, pos:pos + 1], K[:, pos:pos + 1], V[:, pos:pos + 1], pos))
    at = N + steps
    qt, kt = torch.empty_like(Q[:, at:at + turn]), torch.empty_like(K[:, at:at + turn])
    ses.rotate(rot, Q[:, at:at + turn], K[:, at:at + turn], qt, kt, pos=at)
    ses.append(cache, kt, V[:, at:at + turn], at)
    T = torch.empty_like(qt)
    ses.attend(cache, qt, at, T)
    return O, outs, T, cache


def _eager_step(ses, rot, cache, q, k, v, pos):
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    ses.rotate(rot, q, k, qr, kr, pos=pos)
    ses.append(cache, kr, v, pos)
    o = torch.empty((q.shape[0], 128), dtype=torch.bfloat16, device="cuda")
    ses.decode_cached(cache, qr.view(-1, 128), pos, o)
    return o


def test_prompt_steps_and_a_further_turn():
    print("case path", flush=True)
    ses, rot, tensors = _layer(21)
    N, b, steps, turn = 2048, 64, 70, 90
    O, outs, T, cache = _run(ses, rot, tensors, steps, turn, _eager_step)
    torch.cuda.synchronize()
    ix = download_index(ses)
    # in fp64, every value rounded to bf16 where the path does
    w = orot.frequencies(128, 500000.0)
    tokens = N + steps + turn
    at = np.arange(tokens)

    def turned(x):
        y = orot.rotate(host_f64(x[:, :tokens]), at, w)
        return torch.from_numpy(y).bfloat16().double().numpy()

    q, k, v = turned(tensors[0]), turned(tensors[1]), host_f64(tensors[2][:, :tokens])

    def near(got, want, what):
        # keys that the kernel rotated one bf16 step apart from fp64's change the scores by up to 2^-7 of a few terms, and a
        # code of e4m3 beside them by 2^-3 of its value
        d = np.abs(got - want)
        assert np.isfinite(got).all() and d.max() <= 2e-2 and d.mean() <= 2e-3, (what, d.max(), d.mean())

    for i, o in enumerate(outs):
        pos = N + i
        kc, vc = oc.read(k[:, :pos + 1], b, 0), oc.read(v[:, :pos + 1], b, 0)
        for h in (0, 3, 7) if i % 10 else range(8):
            keys = dec.kept_keys(ix, h, N, b, pos)
            s = kc[h // 4, keys] @ q[h, pos] / np.sqrt(128.0)
            p = np.exp(s - s.max())
            near(host_f64(o)[h], (p / p.sum()) @ vc[h // 4, keys], (pos, h))
        if i == 12:
            break
    kc, vc = oc.read(k, b, 0), oc.read(v, b, 0)
    for h in range(8):
        s = q[h, N + steps:] @ kc[h // 4].T / np.sqrt(128.0)
        s[np.arange(tokens)[None] > np.arange(N + steps, tokens)[:, None]] = -np.inf
        p = np.exp(s - s.max(-1, keepdims=True))
        near(host_f64(T)[h], (p / p.sum(-1, keepdims=True)) @ vc[h // 4], ("turn", h))


def test_recorded_steps_of_two_layers():
    # two layers, each with its session and cache, a step of both recorded once and replayed on new tokens of the same
    # position, with eager steps between: every replay gives the eager bytes
    print("case path graph", flush=True)
    layers = [_layer(22), _layer(23, Hq=6, Hkv=3)]
    N, pos = 2048, 2048 + 63                       # the token that fills its block
    state = []
    for ses, rot, (Q, K, V) in layers:
        q, k = Q[:, :N].contiguous(), K[:, :N].contiguous()
        ses.rotate(rot, q, k, q, k)
        ses.estimate_and_index(q, k)
        cache = ses.cache(N + 64)
        ses.append(cache, k, V[:, :N], 0)
        ses.append(cache, K[:, N:pos], V[:, N:pos], N)
        x = [t[:, pos:pos + 1].clone() for t in (Q, K, V)]
        out = [torch.empty_like(x[0]), torch.empty_like(x[1]), torch.empty((Q.shape[0], 128), dtype=torch.bfloat16, device="cuda")]
        state.append((ses, rot, cache, x, out))

    def step():
        for ses, rot, cache, (q, k, v), (qr, kr, o) in state:
            ses.rotate(rot, q, k, qr, kr, pos=pos)
            ses.append(cache, kr, v, pos)
            ses.decode_cached(cache, qr.view(-1, 128), pos, o)

    def snapshot():
        torch.cuda.synchronize()
        return [t.clone() for s in state for t in (s[4][2],) + s[2].tensors]

    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        step()
    for rep in range(4):
        for s in state:
            for t in s[3]:
                t.copy_(torch.randn_like(t))
        step()
        want = snapshot()
        for s in state:
            s[4][2].fill_(7.0)
            s[2].k[:, N:].fill_(9)
        graph.replay()
        for x, y in zip(snapshot(), want):
            assert torch.equal(x, y), rep


def test_two_streams_with_sessions_of_their_own():
    print("case path streams", flush=True)
    a, b = _layer(24), _layer(25)
    want = [_run(*l, 5, 40, _eager_step) for l in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, l in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append(_run(*l, 5, 40, _eager_step))
    torch.cuda.synchronize()
    for (O, outs, T, _), (O2, outs2, T2, _) in zip(want, got):
        assert torch.equal(O, O2) and torch.equal(T, T2) and all(torch.equal(x, y) for x, y in zip(outs, outs2))


def test_refusals_of_the_session():
    print("case path refusals", flush=True)
    ses = sa.Session(4, 2, 512, 64, 64, keep=0.3)
    rot, c = sa.Rotary(), ses.cache(640)
    q, k = torch.zeros(4, 3, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 3, 128, dtype=torch.bfloat16, device="cuda")
    other = sa.Session(4, 4, 512, 64, 64, keep=0.3)
    wide = sa.Session(4, 2, 512, 128, 64, keep=0.3)
    for call in (lambda: ses.rotate(rot, None, None, None, None), lambda: ses.rotate(rot, q, None, None, None),
                 lambda: ses.rotate(rot, q, None, q, k), lambda: ses.rotate(rot, q, k, q, k[:, :2]), lambda: ses.rotate(rot, q, q, q, q), lambda: ses.rotate(rot, q.float(), k, q, k),
                 lambda: ses.rotate(rot, q.cpu(), k, q, k), lambda: ses.rotate(rot, q.transpose(1, 2), k, q, k),
                 lambda: ses.rotate(rot, q, k, q, k, positions=torch.zeros(3, dtype=torch.int64, device="cuda")),
                 lambda: ses.rotate(rot, q, k, q, k, positions=torch.zeros(2, dtype=torch.int32, device="cuda")),
                 lambda: ses.rotate(rot, q, k, q, k, positions=torch.zeros(3, dtype=torch.int32)),
                 lambda: ses.rotate(rot, q[:1, :1].expand(4, 3, 128), k, q, k), lambda: ses.append(c, k, k[:, :2], 0),
                 lambda: ses.append(c, k, k, 638), lambda: ses.append(c, k.cpu(), k, 0), lambda: other.append(c, q, q, 0),
                 lambda: wide.append(c, k, k, 0), lambda: ses.attend(c, q, 0, q[:, :2]), lambda: ses.attend(c, q, 638, q),
                 lambda: ses.attend(c, q, 0, torch.empty(4, 1, 128, dtype=torch.bfloat16, device="cuda").expand(4, 3, 128)),
                 lambda: ses.decode_cached(c, q[:, 0], 511, q[:, 0]), lambda: ses.decode_cached(c, q[:, 0], 512, q[:, 0]),
                 lambda: ses.cache(100), lambda: ses.cache(640, 7) and ses.append(ses.cache(640, 7), k, k, 0),
                 lambda: sa.Cache(c.k, c.v[:, :64], c.k_scale, c.v_scale, c.k_open, c.v_open)):
        with pytest.raises(sa.SaError):
            call()
    ses.append(c, k, k, 0)
    torch.cuda.synchronize()


def test_first_attend_inside_a_capture():
    # the session's scratch is then allocated while recording, and serves eager calls after the graph is gone
    print("case path first attend recorded", flush=True)
    ses, other = (sa.Session(8, 2, 512, 64, 64, keep=0.3) for _ in range(2))
    gen = torch.Generator(device="cuda").manual_seed(5)
    K, V = (torch.randn((2, 5000, 128), generator=gen, device="cuda").bfloat16() for _ in range(2))
    c = ses.cache(5056)
    ses.append(c, K, V, 0)
    q = torch.randn((8, 1, 128), generator=gen, device="cuda").bfloat16()
    o, want = torch.empty_like(q), torch.empty_like(q)
    other.attend(c, q, 4999, want)
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.attend(c, q, 4999, o)
    for rep in range(3):
        o.fill_(7.0)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(o, want), rep
    del graph
    torch.cuda.empty_cache()
    filler = [torch.full((1 << 20,), 1e30, device="cuda") for _ in range(8)]
    o.fill_(7.0)
    ses.attend(c, q, 4999, o)
    torch.cuda.synchronize()
    assert torch.equal(o, want) and all((f == 1e30).all() for f in filler)
