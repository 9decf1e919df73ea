"""Host side of the cache in pages, without a GPU: calls that are refused before any launch, the handle's checks."""
import ctypes as C

import pytest
import torch

from paper_2608_26140_b200 import binding as ab
from paper_2608_26140_b200 import build as abuild


@pytest.fixture(scope="module")
def lib():
    abuild.build()
    return ab.load_library()


@pytest.fixture
def handle(lib):
    h = C.c_void_p()
    assert lib.acache_create(C.byref(ab.ModelDesc(256, 4, 2, 64, 1024, 1e-5, 0, 2, 256, 128, 64, 32, 0, 0)), C.byref(h)) == ab.OK
    yield h
    assert lib.acache_launch_count(h) == 0
    lib.acache_destroy(h)


def cache(**kw):
    c = dict(k=4096, v=8192, page_stride=2 * 16 * 64, n_pages=8, page=16, table=256, table_stride=4)
    c.update(kw)
    return ab.PagedKV(**c)


def append(lib, h, kv, batch=1, ctx_len=64, k=None, v=None, q=None, q_out=None, n=2, lens=256, pos=None, counts=None, cos=None, sin=None):
    rows = ab.Rows(256, 2 * 128, 128)
    return lib.acache_paged_append(h, C.byref(kv), batch, ctx_len, C.byref(k or rows), C.byref(v or rows), C.byref(q) if q else None, q_out, n, lens, pos,
                                   counts, cos, sin, None)


def attend(lib, h, kv, batch=1, n=1, ctx_len=64, q=256, o=256):
    return lib.acache_paged_attention(h, C.byref(kv), batch, n, ctx_len, q, None, None, o, None, None)


def test_calls_without_workspace_are_rejected(lib, handle):
    assert append(lib, handle, cache()) == ab.ERR_WORKSPACE
    assert attend(lib, handle, cache()) == ab.ERR_WORKSPACE
    assert append(lib, None, cache()) == ab.ERR_INVALID_ARG
    assert attend(lib, None, cache()) == ab.ERR_INVALID_ARG


@pytest.fixture
def with_workspace(lib, handle):
    """A handle whose workspace is an address that no refused call touches: it is taken before the call fails for want of a GPU."""
    if torch.cuda.is_available():
        pytest.skip("the workspace of this test is no memory")
    assert lib.acache_set_workspace(handle, 1 << 20, lib.acache_workspace_bytes(handle), None) == ab.ERR_CUDA
    return handle


def test_bad_caches(lib, with_workspace):
    h = with_workspace
    for bad, code in [(dict(k=None), ab.ERR_INVALID_ARG), (dict(v=None), ab.ERR_INVALID_ARG), (dict(k=4104), ab.ERR_INVALID_ARG), (dict(table=None), ab.ERR_INVALID_ARG),
                      (dict(page=0), ab.ERR_UNSUPPORTED_SHAPE), (dict(page=24), ab.ERR_UNSUPPORTED_SHAPE), (dict(page=-16), ab.ERR_UNSUPPORTED_SHAPE),
                      (dict(page=2048, page_stride=1 << 20), ab.ERR_UNSUPPORTED_SHAPE), (dict(n_pages=0), ab.ERR_INVALID_ARG), (dict(n_pages=-1), ab.ERR_INVALID_ARG),
                      (dict(page_stride=2 * 16 * 64 - 8), ab.ERR_INVALID_ARG), (dict(page_stride=2 * 16 * 64 + 4), ab.ERR_INVALID_ARG),
                      (dict(table_stride=-1), ab.ERR_INVALID_ARG), (dict(table_stride=3), ab.ERR_INVALID_ARG)]:
        assert append(lib, h, cache(**bad)) == code, bad
        assert attend(lib, h, cache(**bad)) == code, bad


def test_bad_arguments(lib, with_workspace):
    h, rows = with_workspace, ab.Rows
    for bad in (dict(batch=-1), dict(batch=3), dict(ctx_len=-1), dict(ctx_len=65), dict(n=-1), dict(lens=None), dict(pos=256), dict(q=rows(256, 512, 256)), dict(q_out=256),
                dict(q=rows(256, 512, 248), q_out=256), dict(q=rows(264, 512, 256), q_out=256), dict(q=rows(256, 512, 256), q_out=264), dict(k=rows(None, 256, 128)),
                dict(k=rows(264, 256, 128)), dict(k=rows(256, 256, 120)), dict(v=rows(256, 256, 132)), dict(v=rows(256, 260, 128), batch=2), dict(v=rows(256, -256, 128), batch=2),
                dict(cos=256), dict(sin=256), dict(cos=256, sin=260)):
        assert append(lib, h, cache(), **bad) == ab.ERR_INVALID_ARG, bad
    for bad in (dict(batch=-1), dict(batch=3), dict(ctx_len=-1), dict(ctx_len=65), dict(n=-1), dict(n=1 << 30), dict(q=None), dict(o=None), dict(q=264), dict(o=264)):
        assert attend(lib, h, cache(), **bad) == ab.ERR_INVALID_ARG, bad
    # nothing to do
    assert append(lib, h, cache(), n=0) == ab.OK and append(lib, h, cache(), batch=0) == ab.OK
    assert attend(lib, h, cache(), n=0) == ab.OK and attend(lib, h, cache(), batch=0) == ab.OK
    # a very long table: the length is bounded by itself
    assert attend(lib, h, cache(page=1024, page_stride=1 << 17, table_stride=1 << 21), ctx_len=(1 << 30) + 1) == ab.ERR_INVALID_ARG


def test_the_handle_wants_pools_that_go_together():
    ctx = ab.Context.__new__(ab.Context)
    ctx.heads = (4, 2, 64)
    pool, table = torch.zeros((5, 2, 16, 64), dtype=torch.bfloat16), torch.zeros((3, 4), dtype=torch.int32)
    c = ctx.paged_kv(pool, pool.clone(), table)
    assert (c.page_stride, c.n_pages, c.page, c.table_stride) == (2 * 16 * 64, 5, 16, 4) and c.made_of == (3, 2, 64, False, -1)
    apart = torch.zeros((5, 3, 16, 64), dtype=torch.bfloat16)[:, :2]
    assert ctx.paged_kv(apart, torch.zeros((5, 3, 16, 64), dtype=torch.bfloat16)[:, 1:], table).page_stride == 3 * 16 * 64
    for bad in ((pool, pool[:3], table), (pool, apart, table), (pool.float(), pool, table), (pool, pool, table.long()), (pool, pool, table.t()), (pool, pool, table[0]),
                (pool.transpose(2, 3), pool.transpose(2, 3), table), (pool[:, :1], pool[:, :1], table)):
        with pytest.raises(ValueError):
            ctx.paged_kv(*bad)


def test_calls_want_one_device(monkeypatch):
    """The context's, the pages' and every tensor's: the current one, where the call runs."""
    ctx = ab.Context.__new__(ab.Context)
    ctx.heads, ctx.dtypes, ctx.gpu = (4, 2, 64), (torch.bfloat16, torch.float32, torch.int32), 0
    ctx._row_args = [(ab.Rows(), None) for _ in range(3)]
    cache = ab.PagedKV()
    cache.made_of = (3, 2, 64, True, 1)
    q, k, lens = torch.zeros((3, 1, 4, 64), dtype=torch.bfloat16), torch.zeros((3, 1, 2, 64), dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int32)
    logits, u, token = torch.zeros((2, 10)), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    calls = (lambda: ctx.paged_attention(cache, 16, q, q.clone()), lambda: ctx.paged_append(cache, 16, k, k.clone(), lens=lens))
    samples = (lambda: ctx.sample_tokens(logits, u, token), lambda: ctx.predict_sample(None, 1, None, 2, 1, None, None, 10, logits, u, 0.9, None, None, None))
    monkeypatch.setattr(ab, "_current_device", lambda: 1)
    for call in calls + samples:
        with pytest.raises(ValueError, match="a context on GPU 0 while GPU 1 is"):
            call()
    ctx.gpu = 1
    for call in calls + samples:                                 # tensors on the CPU
        with pytest.raises(ValueError, match="on cpu"):
            call()
    monkeypatch.setattr(ab, "_current_device", lambda: 0)
    ctx.gpu = 0
    for call in calls:
        with pytest.raises(ValueError, match="on GPU 1"):
            call()
