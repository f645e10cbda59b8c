"""Every form of the causal attention over the 4-bit cache, as sa_cache4_attend_plan names them: 16, 32 or 128 query rows a workgroup, with and without splits of
the keys; ragged lengths, masked tiles, uneven rows, strides, values that are no numbers. Tolerance: test_gpu_cache4_attend.py."""
import numpy as np
import pytest
import torch

import paper_2412_06198_amd as sa
from gpu_util import dev_bf16, host_f64
from test_gpu_cache4_attend import _check, _reference, _setup
from test_gpu_cache_decode import _f64

pytestmark = pytest.mark.gpu

# heads, tokens, before, (rows of a workgroup, whether in splits)
FORMS = [((4, 4), 3, 0, (16, False)), ((8, 2), 61, 333, (16, False)), ((4, 4), 700, 5, (16, False)), ((16, 2), 12, 3001, (16, True)), ((128, 2), 5, 3001, (16, True)),
         ((64, 1), 130, 0, (32, False)), ((64, 8), 191, 640, (32, False)), ((8, 1), 191, 2000, (32, True)), ((6, 2), 150, 3001, (32, True)),
         ((8, 8), 50, 9000, (32, True)), ((32, 8), 13, 9000, (32, True)), ((40, 1), 47, 4000, (32, True)),
         ((128, 2), 160, 0, (128, False)), ((128, 2), 130, 5, (128, False)), ((128, 2), 100, 70, (128, False)), ((64, 1), 400, 640, (128, False)),
         ((128, 2), 333, 1000, (128, False)), ((8, 1), 700, 6000, (128, True)), ((64, 1), 47, 9000, (128, True)), ((4, 4), 400, 20000, (128, True)),
         ((32, 8), 90, 8000, (128, True))]


def _made(heads, n, before, form, seed, change=None):
    made = _setup(*heads, before + n, seed, change)
    rows, splits = sa.sa_cache4_attend_plan(made[0].ctx, n, before)
    assert (rows, splits > 1) == form, (rows, splits)
    return made


@pytest.mark.parametrize("heads,n,before,form", FORMS)
def test_forms(heads, n, before, form):
    print(f"case attend4 form {heads} {n} {before} {form}", flush=True)
    _check(*_made(heads, n, before, form, 21), n)


@pytest.mark.parametrize("heads,n,before,form", [f for f in FORMS if f[0][0] * f[1] * (f[1] + f[2]) < 8e6])
def test_groups_that_are_nan(heads, n, before, form):
    # in a key that all rows see, in one that some do, in the last; several keys of a tile, several groups of a key
    print(f"case attend4 form NaN {heads} {n} {before} {form}", flush=True)
    tokens = before + n
    at = sorted({before // 2, max(before, tokens - n // 2 - 1), max(before, tokens - n // 2 - 2), tokens - 1})
    groups = [[0], [1, 3], [2], [3]][:len(at)]

    def change(Q, K, V):
        for j, gs in zip(at, groups):
            for g in gs:
                V[:, j, 32 * g + 5] = 0xFF80
    ses, c, Q, keys, vals = _made(heads, n, before, form, 22, change)
    Qd = dev_bf16(Q[:, before:])
    O = torch.full_like(Qd, 7.0)
    ses.attend(c, Qd, before, O)
    torch.cuda.synchronize()
    got, bad, clean = host_f64(O), np.zeros((heads[0], n, 128), bool), vals.copy()
    for j, gs in zip(at, groups):
        for g in gs:
            bad[:, max(0, j - before):, 32 * g:32 * g + 32] = True
            clean[:, j, 32 * g:32 * g + 32] = 0
    assert np.isnan(got[bad]).all()
    ref, tol = _reference(_f64(Q[:, before:]), keys, clean, before, form[0])
    assert (np.abs(got - ref) <= tol)[~bad].all()


@pytest.mark.parametrize("heads,n,before,form", [f for f in FORMS if f[0][0] * f[1] * (f[1] + f[2]) < 8e6])
def test_nan_keys_and_queries(heads, n, before, form):
    print(f"case attend4 form NaN keys {heads} {n} {before} {form}", flush=True)
    at = before + n // 2

    def change(Q, K, V):
        K[0, at, 100] = 0x7FC0
        Q[-1, before + n - 1, 3] = 0x7F80
    ses, c, Q, keys, vals = _made(heads, n, before, form, 23, change)
    Qd = dev_bf16(Q[:, before:])
    O = torch.empty_like(Qd)
    ses.attend(c, Qd, before, O)
    torch.cuda.synchronize()
    got, bad = host_f64(O), np.zeros((heads[0], n), bool)
    bad[:heads[0] // heads[1], n // 2:] = True
    bad[-1, -1] = True
    assert np.array_equal(np.isnan(got), np.broadcast_to(bad[..., None], got.shape))
    keys = np.nan_to_num(keys, nan=0.0)
    ref, tol = _reference(np.nan_to_num(_f64(Q[:, before:]), posinf=0.0), keys, vals, before, form[0])
    assert (np.abs(got - ref) <= tol)[~bad].all()


@pytest.mark.parametrize("heads,n,before,form", [FORMS[i] for i in (1, 3, 6, 7, 13, 18)])
def test_strides_in_place_and_replays(heads, n, before, form):
    print(f"case attend4 form strides {heads} {n} {before} {form}", flush=True)
    ses, c, Q, keys, vals = _made(heads, n, before, form, 24)
    want = _check(ses, c, Q, keys, vals, n)
    Qd = dev_bf16(Q[:, before:]).transpose(0, 1).contiguous().transpose(0, 1)   # tokens outermost
    room = torch.full((n, heads[0], 136), 7.0, dtype=torch.bfloat16, device="cuda")
    ses.attend(c, Qd, before, room[..., :128].transpose(0, 1))
    torch.cuda.synchronize()
    assert torch.equal(room[..., :128].transpose(0, 1), want) and (room[..., 128:] == 7.0).all()
    Qi = Qd.clone()
    ses.attend(c, Qi, before, Qi)   # in place
    torch.cuda.synchronize()
    assert torch.equal(Qi, want)
    O, side = torch.empty_like(want), torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        ses.attend(c, Qd, before, O)
    for rep in range(3):
        O.fill_(7.0)
        graph.replay()
        ses.attend(c, Qd, before, room[..., :128].transpose(0, 1))   # behind it, on the same scratch
        torch.cuda.synchronize()
        assert torch.equal(O, want) and torch.equal(room[..., :128].transpose(0, 1), want), rep


def test_a_cache_of_exactly_its_tokens():
    # no byte of room behind the last token: rows of the last tile that are not there are not read (the buffers end a larger one whose rest is NaN scales)
    print("case attend4 form exact capacity", flush=True)
    for heads, n, before in (((8, 2), 61, 333), ((8, 1), 191, 1000), ((128, 2), 130, 5)):
        ses, c, Q, keys, vals = _setup(*heads, before + n, seed=25)
        tight = sa.Cache4(*[t[:, :before + n].contiguous() for t in c.tensors])
        _check(ses, tight, Q, keys, vals, n)
