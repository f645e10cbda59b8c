"""Refusals of the 4-bit cache's entry points and of reading caches back: every call below is turned away before its first launch (no GPU needed)."""
import ctypes as C

import pytest

import paper_2412_06198_amd as sa

A = 4096  # an address that is never read: every call that gets one is refused, or does nothing


@pytest.fixture
def ctx():
    c = sa.SaConfig()
    c.n_q_heads, c.n_kv_heads, c.head_dim = 8, 2, 128
    c.seq_len, c.block, c.last_q = 4096, 64, 64
    sa.sa_default_budgets(c, 0.1)
    c = sa.sa_create(c)
    yield c
    sa.sa_destroy(c)


def _rows(data=A, head_stride=0, row_stride=0):
    return sa.SaRows(data, head_stride, row_stride)


def _cache(**kw):
    c = sa.SaCache4(A, A, A, A, 8192)
    for k, v in kw.items():
        setattr(c, k, v)
    return c


def _refused(status, text, call, *args):
    with pytest.raises(sa.SaError) as e:
        call(*args)
    assert e.value.status == status and text in str(e.value), str(e.value)


def test_sizes(ctx):
    assert sa.sa_cache4_bytes(ctx, 8191) == [2 * 8191 * 64] * 2 + [2 * 8191 * 4] * 2
    assert sa.sa_cache4_bytes(ctx, 2 ** 30)[0] == 2 * 2 ** 30 * 64
    for capacity in (0, -1, 2 ** 30 + 1):
        _refused(1, "", sa.sa_cache4_bytes, ctx, capacity)


CACHES = [(dict(k=0), 1, "null"), (dict(v=0), 1, "null"), (dict(k_scale=0), 1, "null"), (dict(v_scale=0), 1, "null"), (dict(k=A + 8), 1, "aligned"),
          (dict(v=A + 4), 1, "aligned"), (dict(k_scale=A + 2), 1, "aligned"), (dict(v_scale=A + 1), 1, "aligned"),
          (dict(capacity=0), 1, "capacity"), (dict(capacity=-64), 1, "capacity"), (dict(capacity=2 ** 30 + 1), 1, "capacity"), (dict(capacity=4096), 3, "room")]


@pytest.mark.parametrize("bad,status,text", CACHES, ids=lambda x: str(x) if isinstance(x, dict) else "")
def test_caches(ctx, bad, status, text):
    c, ok = _cache(**bad), _rows()
    ix = sa.SaIndex(*([A] * 7))
    scratch = sa.sa_cache_attend_scratch_bytes(ctx)
    _refused(status, text, sa.sa_cache4_append, ctx, c, ok, ok, 1, 4096)
    _refused(status, text, sa.sa_cache4_read, ctx, c, ok, ok, 1, 4096)
    _refused(status, text, sa.sa_cache4_decode, ctx, c, A, ix, 4096, A)
    _refused(status, text, sa.sa_cache4_attend, ctx, c, ok, 1, 4096, ok, A, scratch)


def test_append_and_read_calls(ctx):
    c, ok = _cache(), _rows()
    for call in (sa.sa_cache4_append, sa.sa_cache4_read):
        call(ctx, c, ok, ok, 0, 8192)
        call(ctx, c, _rows(0), _rows(0), 0, 5)
        _refused(3, "room", call, ctx, c, ok, ok, 1, 8192)
        _refused(3, "room", call, ctx, c, ok, ok, 8193, 0)
        for n, pos in ((-1, 0), (1, -1), (2 ** 25 + 1, 0), (2 ** 62, 2 ** 62), (2 ** 63 - 1, 1)):
            _refused(1, "pos", call, ctx, c, ok, ok, n, pos)
        _refused(1, "null", call, ctx, c, _rows(0), _rows(0), 1, 0)
        _refused(1, "aligned", call, ctx, c, ok, _rows(A + 2), 1, 0)
        _refused(1, "strides", call, ctx, c, ok, _rows(A, 128 * 9, 132), 9, 0)
    _refused(1, "null", sa.sa_cache4_append, ctx, c, ok, _rows(0), 1, 0)
    _refused(1, "overlap", sa.sa_cache4_read, ctx, c, ok, _rows(2 * A, 384, 128), 4, 0)
    _refused(1, "overlap", sa.sa_cache4_read, ctx, c, _rows(2 * A, 128, 136), _rows(0), 4, 0)


def test_reads_of_the_8_bit_cache(ctx):
    c, ok = sa.SaCache(A, A, A, A, A, A, 8192, 0), _rows()
    call = sa.sa_cache_read
    call(ctx, c, 8192, ok, ok, 0, 8192)
    call(ctx, c, 0, _rows(0), _rows(0), 0, 0)
    _refused(1, "tokens", call, ctx, c, 4000, ok, ok, 1, 4000)
    _refused(1, "tokens", call, ctx, c, -1, ok, ok, 0, 0)
    _refused(3, "room", call, ctx, c, 8193, ok, ok, 1, 0)
    for n, pos in ((-1, 0), (1, -1), (2 ** 25 + 1, 0), (2 ** 62, 2 ** 62), (2 ** 63 - 1, 1)):
        _refused(1, "pos", call, ctx, c, 2 ** 30, ok, ok, n, pos)
    _refused(1, "null", call, ctx, c, 10, _rows(0), _rows(0), 1, 0)
    _refused(1, "overlap", call, ctx, c, 10, _rows(2 * A, 384, 128), ok, 4, 0)
    _refused(1, "type", call, ctx, sa.SaCache(A, A, A, A, A, A, 8192, 2), 10, ok, ok, 4, 0)


def test_decode_calls(ctx):
    c, ix, call = _cache(), sa.SaIndex(*([A] * 7)), sa.sa_cache4_decode
    _refused(1, "null", call, ctx, c, 0, ix, 4096, A)
    _refused(1, "null", call, ctx, c, A, sa.SaIndex(A, A, A, A, A, A, 0), 4096, A)
    _refused(1, "aligned", call, ctx, c, A + 4, ix, 4096, A)
    _refused(1, "pos", call, ctx, c, A, ix, 4095, A)
    _refused(1, "pos", call, ctx, c, A, ix, 4096 + 2 ** 20, A)
    _refused(3, "room", call, ctx, c, A, ix, 8192, A)
    _refused(1, "workspace", call, ctx, c, A, ix, 4096, A)


def test_attend_calls(ctx):
    c, ok, size = _cache(), _rows(), sa.sa_cache_attend_scratch_bytes(ctx)
    call = sa.sa_cache4_attend
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
    for n, pos in ((0, 0), (-1, 5), (1, 2 ** 30), (2 ** 28, 0)):
        _refused(1, "", sa.sa_cache4_attend_plan, ctx, n, pos)
    rows, splits = sa.sa_cache4_attend_plan(ctx, 1, 100000)
    assert rows >= 1 and splits >= 1


@pytest.mark.parametrize("bad", [dict(k=(8192, 64)), dict(k=(2, 8192, 128)), dict(v=(2, 8192, 32)), dict(v=(2, 8191, 64)), dict(k_scale=(2, 8192)), dict(v_scale=(2, 8192, 1))])
def test_buffers_of_a_cache(bad):
    torch = pytest.importorskip("torch")
    shapes = dict(k=(2, 8192, 64), v=(2, 8192, 64), k_scale=(2, 8192, 4), v_scale=(2, 8192, 4))
    sa.Cache4(**{name: torch.empty(shapes[name], dtype=torch.uint8) for name in shapes})
    shapes.update(bad)
    with pytest.raises(sa.SaError):
        sa.Cache4(**{name: torch.empty(shapes[name], dtype=torch.uint8) for name in shapes})


def test_null_context():
    lib = sa.library()
    assert lib.sa_cache4_bytes(None, 64, (C.c_size_t * 4)()) == 1
    assert lib.sa_cache4_append(None, None, _rows(), _rows(), 1, 0, None) == 1
    assert lib.sa_cache4_read(None, None, _rows(), _rows(), 1, 0, None) == 1
    assert lib.sa_cache_read(None, None, 1, _rows(), _rows(), 1, 0, None) == 1
    assert lib.sa_cache4_attend(None, None, _rows(), 1, 0, _rows(), None, 0, None) == 1
