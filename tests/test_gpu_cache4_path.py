"""The 4-bit cache as a serving program runs a layer: rotated prompt quantised as it is written, index and sparse prefill over what is read back,
decode steps with each token rotated and appended, a further turn attended densely, drafts taken back; eagerly, recorded, on two streams."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from harness import gen
from oracle import cache4 as oc
from oracle import decode as dec
from oracle import oracle as orc
from gpu_util import check_attention, dev_bf16, download_index, host_f64

pytestmark = pytest.mark.gpu


def _layer(seed, Hq=8, Hkv=2, N=1024, b=64, extra=200):
    Q, K, V = gen.random_qkv(Hq, Hkv, N + extra, 128, seed=seed)
    ses = sa.Session(Hq, Hkv, N, b, 64, keep=0.3)
    return ses, sa.Rotary(theta=500000.0), (dev_bf16(Q), dev_bf16(K), dev_bf16(V))


def _step(ses, rot, cache, q, k, v, pos):
    qr, kr = torch.empty_like(q), torch.empty_like(k)
    ses.rotate(rot, q, k, qr, kr, pos=pos)
    ses.append(cache, kr, v, pos)
    o = torch.empty((q.shape[0], 128), dtype=torch.bfloat16, device="cuda")
    ses.decode_cached(cache, qr.view(-1, 128), pos, o)
    return o, qr


def _run(ses, rot, tensors, steps, turn):
    Q, K, V = tensors
    N = ses.cfg.seq_len
    q, k = Q[:, :N].contiguous(), K[:, :N].contiguous()
    ses.rotate(rot, q, k, q, k)
    cache = ses.cache4(N + 190)
    ses.append(cache, k, V[:, :N], 0)
    kq, vq = torch.empty_like(k), torch.empty_like(k)
    ses.read(cache, kq, vq)
    O = torch.empty_like(q)
    ses.estimate_and_index(q, kq)
    ses.prefill(q, kq, vq, O)
    ses.append(cache, K[:, N:N + 9], V[:, N:N + 9], N)   # drafts, none of them kept
    outs = [_step(ses, rot, cache, Q[:, p:p + 1], K[:, p:p + 1], V[:, p:p + 1], p) for p in range(N, N + steps)]
    at = N + steps
    qt, kt = torch.empty_like(Q[:, at:at + turn]), torch.empty_like(K[:, at:at + turn])
    ses.rotate(rot, Q[:, at:at + turn], K[:, at:at + turn], qt, kt, pos=at)
    ses.append(cache, kt, V[:, at:at + turn], at)
    T = torch.empty_like(qt)
    ses.attend(cache, qt, at, T)
    return q, O, outs, qt, T, cache


def test_prompt_steps_and_a_further_turn():
    print("case path4", flush=True)
    ses, rot, tensors = _layer(41)
    N, b, steps, turn = 1024, 64, 30, 90
    q, O, outs, qt, T, cache = _run(ses, rot, tensors, steps, turn)
    tokens = N + steps + turn
    k, v = (torch.empty((2, tokens, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ses.read(cache, k, v)
    torch.cuda.synchronize()
    ix = download_index(ses)
    keys, vals = host_f64(k), host_f64(v)
    assert np.array_equal(vals, oc.read(host_f64(tensors[2][:, :tokens])))

    def bits(t):
        return t.cpu().view(torch.int16).numpy().view(np.uint16)

    check_attention(host_f64(O), orc.masked_rows(bits(q), bits(k[:, :N].contiguous()), bits(v[:, :N].contiguous()), b, ix)[0], "prefill")

    def near(got, query, at, kept, h):
        s = keys[h // 4, kept] @ query / np.sqrt(128.0)
        p = np.exp(s - s.max())
        p /= p.sum()
        w = vals[h // 4, kept]
        spread = p @ np.abs(w) + np.abs(p @ w)
        # probabilities in bf16 at most (2^-8), fp32 scores and what a query's codes leave out, 2^-9 together, the output's rounding
        assert (np.abs(got - p @ w) <= (2.0 ** -8 + 2.0 ** -9) * spread + 2.0 ** -8 * np.abs(p @ w)).all(), (at, h)

    for i, (o, qr) in enumerate(outs):
        for h in range(8):
            near(host_f64(o)[h], host_f64(qr)[h, 0], N + i, dec.kept_keys(ix, h, N, b, N + i), h)
    for h in range(8):
        for t in range(0, turn, 7):
            near(host_f64(T)[h, t], host_f64(qt)[h, t], ("turn", t), np.arange(N + steps + t + 1), h)


def test_recorded_steps_of_two_layers():
    # two layers, each with its session and cache, a step and drafted tokens of both recorded once and replayed on new tokens of the same
    # position, with eager ones between: every replay gives the eager bytes
    print("case path4 graph", flush=True)
    state = []
    for ses, rot, (Q, K, V) in (_layer(42), _layer(43, Hq=6, Hkv=3)):
        N = ses.cfg.seq_len
        q, k = Q[:, :N].contiguous(), K[:, :N].contiguous()
        ses.rotate(rot, q, k, q, k)
        ses.estimate_and_index(q, k)
        cache = ses.cache4(N + 64)
        ses.append(cache, k, V[:, :N], 0)
        x = [t[:, N:N + 5].clone() for t in (Q, K, V)]
        out = [torch.empty_like(x[0]), torch.empty_like(x[1]), torch.empty_like(x[0]), torch.empty((Q.shape[0], 128), dtype=torch.bfloat16, device="cuda"),
               torch.empty_like(x[1]), torch.empty_like(x[1])]
        ses.attend_scratch()
        state.append((ses, rot, cache, x, out))

    def step():
        for ses, rot, cache, (q, k, v), (qr, kr, o, one, kb, vb) in state:
            N = ses.cfg.seq_len
            ses.rotate(rot, q, k, qr, kr, pos=N)
            ses.append(cache, kr, v, N)
            ses.attend(cache, qr, N, o)
            ses.decode_cached(cache, qr[:, 4].contiguous(), N + 4, one)
            ses.read(cache, kb, vb, N)

    def snapshot():
        torch.cuda.synchronize()
        return [t.clone() for s in state for t in s[4][2:] + list(s[2].tensors)]

    step()
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
            for t in s[4][2:]:
                t.fill_(7.0)
            s[2].k[:, s[0].cfg.seq_len:s[0].cfg.seq_len + 5].fill_(9)
        graph.replay()
        for x, y in zip(snapshot(), want):
            assert torch.equal(x, y), rep


def test_two_streams_with_sessions_of_their_own():
    print("case path4 streams", flush=True)
    a, b = _layer(44), _layer(45)
    want = [_run(*l, 5, 40) for l in (a, b)]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for s, l in zip(streams, (a, b)):
        with torch.cuda.stream(s):
            got.append(_run(*l, 5, 40))
    torch.cuda.synchronize()
    for x, y in zip(want, got):
        assert torch.equal(x[1], y[1]) and torch.equal(x[4], y[4]) and all(torch.equal(m[0], n[0]) for m, n in zip(x[2], y[2]))


def test_refusals_of_the_session():
    print("case path4 refusals", flush=True)
    ses = sa.Session(4, 2, 512, 64, 64, keep=0.3)
    c = ses.cache4(640)
    q, k = torch.zeros(4, 3, 128, dtype=torch.bfloat16, device="cuda"), torch.zeros(2, 3, 128, dtype=torch.bfloat16, device="cuda")
    other = sa.Session(4, 4, 512, 64, 64, keep=0.3)
    for call in (lambda: ses.append(c, k, k[:, :2], 0), lambda: ses.append(c, k, k, 638), lambda: ses.append(c, k.cpu(), k, 0), lambda: ses.append(c, k.float(), k, 0),
                 lambda: other.append(c, q, q, 0), lambda: other.attend(c, q, 0, q), lambda: other.decode_cached(c, q[:, 0].contiguous(), 512, q[:, 0].contiguous()),
                 lambda: ses.attend(c, q, 0, q[:, :2]), lambda: ses.attend(c, q, 638, q), lambda: ses.attend(c, q, -1, q),
                 lambda: ses.attend(c, q, 0, torch.empty(4, 1, 128, dtype=torch.bfloat16, device="cuda").expand(4, 3, 128)),
                 lambda: ses.decode_cached(c, q[:, 0], 512, q[:, 0]), lambda: ses.decode_cached(c, q[:, 0].contiguous(), 511, q[:, 0].contiguous()),
                 lambda: ses.decode_cached(c, q[:, 0].contiguous(), 640, q[:, 0].contiguous()), lambda: ses.cache4(0), lambda: ses.cache4(2 ** 30 + 1),
                 lambda: sa.Cache4(c.k, c.v[:, :64], c.k_scale, c.v_scale), lambda: sa.Cache4(c.k, c.v, c.k_scale, c.v_scale.float())):
        with pytest.raises(sa.SaError):
            call()
    ses.append(c, k, k, 0)
    torch.cuda.synchronize()
