"""Refusals of the rotary and cache entry points: every call below is turned away before its first launch (no GPU needed)."""
import ctypes as C
import math

import pytest

import paper_2412_06198_amd as sa

A = 4096  # an address that is never read: every call that gets one is refused, or does nothing


def _cfg(**kw):
    c = sa.SaConfig()
    c.n_q_heads, c.n_kv_heads, c.head_dim = 8, 2, 128
    c.seq_len, c.block, c.last_q = 4096, 64, 64
    sa.sa_default_budgets(c, 0.1)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


@pytest.fixture
def ctx():
    c = sa.sa_create(_cfg())
    yield c
    sa.sa_destroy(c)


def _rows(data=A, head_stride=0, row_stride=0):
    return sa.SaRows(data, head_stride, row_stride)


def _cache(**kw):
    c = sa.SaCache(A, A, A, A, A, A, 8192, 0)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _refused(status, text, call, *args):
    with pytest.raises(sa.SaError) as e:
        call(*args)
    assert e.value.status == status and text in str(e.value), str(e.value)


@pytest.mark.parametrize("bad,status", [
    (dict(rotary_dim=130), 2), (dict(rotary_dim=7), 2), (dict(rotary_dim=-2), 2), (dict(layout=2), 1), (dict(layout=-1), 1),
    (dict(scaling=5), 1), (dict(scaling=-1), 1), (dict(transposed=2), 1), (dict(theta=1.0), 1), (dict(theta=-3.0), 1),
    (dict(theta=math.nan), 1), (dict(theta=math.inf), 1), (dict(scaling=1, factor=0.5), 1), (dict(scaling=1), 1),
    (dict(scaling=2, factor=math.inf), 1), (dict(scaling=3, factor=2.0), 1), (dict(scaling=3, factor=2.0, low=4.0, high=1.0, original_len=10), 1),
    (dict(scaling=4, factor=2.0, low=1.0, high=32.0), 1), (dict(scaling=4, factor=2.0, low=1.0, high=math.nan, original_len=10), 1),
    (dict(amplitude=-1.0), 1), (dict(amplitude=math.inf), 1), (dict(amplitude=1e300), 1), (dict(nonsense=1), 1)])
def test_rotary_configs(bad, status):
    with pytest.raises(sa.SaError) as e:
        sa.Rotary(**bad)
    assert e.value.status == status


def test_rotary_calls(ctx):
    rot = sa.Rotary()
    call = sa.sa_rotary_embed
    ok = _rows()
    call(ctx, rot, ok, ok, 0, 0, None, ok, ok)                       # no rows: nothing to do
    call(ctx, rot, _rows(0), _rows(0), 0, 0, None, _rows(0), _rows(0))
    _refused(1, "null", call, ctx, None, ok, ok, 4, 0, None, ok, ok)
    _refused(1, "null", call, ctx, rot, _rows(0), _rows(0), 4, 0, None, ok, ok)
    _refused(1, "null", call, ctx, rot, ok, ok, 4, 0, None, _rows(0), ok)
    _refused(1, "pos", call, ctx, rot, ok, ok, -1, 0, None, ok, ok)
    _refused(1, "pos", call, ctx, rot, ok, ok, 4, -1, None, ok, ok)
    _refused(1, "pos", call, ctx, rot, ok, ok, 4, 2 ** 31 - 3, None, ok, ok)
    _refused(1, "pos", call, ctx, rot, ok, ok, 2 ** 25 + 1, 0, A, ok, ok)
    _refused(1, "positions", call, ctx, rot, ok, ok, 4, 0, A + 2, ok, ok)
    _refused(1, "aligned", call, ctx, rot, _rows(A + 8), ok, 4, 0, None, ok, ok)
    _refused(1, "strides", call, ctx, rot, ok, _rows(A, 1024, 100), 4, 0, None, ok, ok)
    _refused(1, "strides", call, ctx, rot, ok, _rows(A, 0, 128), 4, 0, None, ok, ok)
    _refused(1, "strides", call, ctx, rot, ok, _rows(A, -512, 128), 4, 0, None, ok, ok)
    _refused(1, "strides", call, ctx, rot, ok, _rows(A, 516, 128), 4, 0, None, ok, ok)
    _refused(1, "strides", call, ctx, rot, ok, _rows(A, 512, 64), 4, 0, None, ok, ok)
    _refused(1, "overlap", call, ctx, rot, ok, ok, 4, 0, None, _rows(2 * A, 384, 128), ok)
    _refused(1, "overlap", call, ctx, rot, ok, ok, 4, 0, None, _rows(2 * A, 128, 896), ok)
    _refused(1, "in place", call, ctx, rot, ok, ok, 4, 0, None, _rows(A, 1024, 128), ok)


def test_cache_sizes(ctx):
    assert sa.sa_cache_bytes(ctx, 8192) == [2 * 8192 * 128] * 2 + [2 * 128 * 4] * 2 + [2 * 64 * 128 * 2] * 2
    for capacity in (0, -64, 100, 2 ** 30 + 64):
        _refused(1, "", sa.sa_cache_bytes, ctx, capacity)
    assert sa.sa_cache_bytes(ctx, 2 ** 30)[0] == 2 * 2 ** 30 * 128


CACHES = [(dict(k=0), 1, "null"), (dict(v_open=0), 1, "null"), (dict(v_scale=0), 1, "null"), (dict(v=A + 4), 1, "aligned"), (dict(k_open=A + 8), 1, "aligned"),
          (dict(k_scale=A + 2), 1, "aligned"), (dict(type=2), 1, "type"), (dict(type=-1), 1, "type"), (dict(capacity=100), 1, "capacity"),
          (dict(capacity=-64), 1, "capacity"), (dict(capacity=2 ** 30 + 64), 1, "capacity"), (dict(capacity=4096), 3, "room")]


@pytest.mark.parametrize("bad,status,text", CACHES, ids=lambda x: str(x) if isinstance(x, dict) else "")
def test_caches(ctx, bad, status, text):
    c, ok = _cache(**bad), _rows()
    ix = sa.SaIndex(*([A] * 7))
    scratch = sa.sa_cache_attend_scratch_bytes(ctx)
    _refused(status, text, sa.sa_cache_append, ctx, c, ok, ok, 1, 4096)
    _refused(status, text, sa.sa_cache_decode, ctx, c, A, ix, 4096, A)
    _refused(status, text, sa.sa_cache_attend, ctx, c, ok, 1, 4096, ok, A, scratch)


def test_cache_calls(ctx):
    c, ok = _cache(), _rows()
    sa.sa_cache_append(ctx, c, ok, ok, 0, 8192)
    sa.sa_cache_append(ctx, c, _rows(0), _rows(0), 0, 5)
    _refused(3, "room", sa.sa_cache_append, ctx, c, ok, ok, 1, 8192)
    _refused(3, "room", sa.sa_cache_append, ctx, c, ok, ok, 8193, 0)
    for n, pos in ((-1, 0), (1, -1), (2 ** 25 + 1, 0), (2 ** 62, 2 ** 62), (2 ** 63 - 1, 1)):
        _refused(1, "pos", sa.sa_cache_append, ctx, c, ok, ok, n, pos)
    _refused(1, "null", sa.sa_cache_append, ctx, None or c, _rows(0), ok, 1, 0)
    _refused(1, "aligned", sa.sa_cache_append, ctx, c, ok, _rows(A + 2), 1, 0)
    _refused(1, "strides", sa.sa_cache_append, ctx, c, ok, _rows(A, 128 * 9, 132), 9, 0)
    ix = sa.SaIndex(*([A] * 7))
    _refused(1, "null", sa.sa_cache_decode, ctx, c, 0, ix, 4096, A)
    _refused(1, "null", sa.sa_cache_decode, ctx, c, A, sa.SaIndex(A, A, A, A, A, A, 0), 4096, A)
    _refused(1, "aligned", sa.sa_cache_decode, ctx, c, A + 4, ix, 4096, A)
    _refused(1, "pos", sa.sa_cache_decode, ctx, c, A, ix, 4095, A)
    _refused(1, "pos", sa.sa_cache_decode, ctx, c, A, ix, 4096 + 2 ** 20, A)
    _refused(3, "room", sa.sa_cache_decode, ctx, c, A, ix, 8192, A)
    _refused(1, "workspace", sa.sa_cache_decode, ctx, c, A, ix, 4096, A)


def test_attend_calls(ctx):
    c, ok, size = _cache(), _rows(), sa.sa_cache_attend_scratch_bytes(ctx)
    call = sa.sa_cache_attend
    call(ctx, c, ok, 0, 0, ok, A, size)
    _refused(1, "scratch", call, ctx, c, ok, 1, 0, ok, 0, size)
    _refused(1, "scratch", call, ctx, c, ok, 1, 0, ok, A + 128, size)
    _refused(3, "scratch", call, ctx, c, ok, 1, 0, ok, A, size - 1)
    _refused(1, "pos", call, ctx, c, ok, -1, 0, ok, A, size)
    _refused(1, "pos", call, ctx, c, ok, 1, -1, ok, A, size)
    _refused(1, "pos", call, ctx, c, ok, 2 ** 27, 0, ok, A, size)
    _refused(3, "room", call, ctx, c, ok, 2, 8191, ok, A, size)
    _refused(1, "null", call, ctx, c, _rows(0), 1, 0, ok, A, size)
    _refused(1, "overlap", call, ctx, c, ok, 4, 0, _rows(2 * A, 384, 128), A, size)
    _refused(1, "in place", call, ctx, c, ok, 4, 0, _rows(A, 1024, 128), A, size)


@pytest.mark.parametrize("bad", [dict(k=(8192, 128)), dict(k_open=(256,)), dict(k_open=(2, 0, 128)), dict(v=(2, 8192, 64)), dict(k_scale=(2, 127))])
def test_buffers_of_a_cache(bad):
    torch = pytest.importorskip("torch")
    shapes = dict(k=(2, 8192, 128), v=(2, 8192, 128), k_scale=(2, 128), v_scale=(2, 128), k_open=(2, 64, 128), v_open=(2, 64, 128))
    kinds = dict(k=torch.uint8, v=torch.uint8, k_scale=torch.float32, v_scale=torch.float32, k_open=torch.bfloat16, v_open=torch.bfloat16)
    sa.Cache(**{name: torch.empty(shapes[name], dtype=kinds[name]) for name in shapes})
    shapes.update(bad)
    with pytest.raises(sa.SaError):
        sa.Cache(**{name: torch.empty(shapes[name], dtype=kinds[name]) for name in shapes})


def test_null_context_and_handles():
    lib = sa.library()
    assert lib.sa_cache_attend_scratch_bytes(None, C.byref(C.c_size_t())) == 1
    assert lib.sa_cache_bytes(None, 64, (C.c_size_t * 6)()) == 1
    assert lib.sa_rotary_create(None, C.byref(C.c_void_p())) == 1
    assert lib.sa_cache_append(None, None, _rows(), _rows(), 1, 0, None) == 1
    sa.sa_rotary_destroy(None)
