"""Host side of the sampling, without a GPU: calls that are refused before any launch."""
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
    assert lib.acache_create(C.byref(ab.ModelDesc(256, 4, 2, 64, 1024, 1e-5, 0, 2, 256, 128, 64, 32, 1280, 8)), C.byref(h)) == ab.OK
    yield h
    assert lib.acache_launch_count(h) == 0
    lib.acache_destroy(h)


def sample(lib, h, logits=256, kind=1, rows=2, vocab=100, stride=100, how=ab.Sampling(None, None, None, None, 1), u=256, token=256):
    return lib.acache_sample_tokens(h, logits, kind, rows, vocab, stride, C.byref(how) if how else None, u, token, None, None, None)


def predict(lib, h, vocab=1280, logits=256, how=ab.Sampling(None, None, None, None, 1), u=256, token=256, n=3):
    return lib.acache_predict_sample(h, 256, 4, 256, 1, n, 256, 256, vocab, logits, C.byref(how) if how else None, u, 0.5, token, 256, 256, None)


def test_refusals(lib, handle):
    if torch.cuda.is_available():
        pytest.skip("the workspace of this test is no memory")
    h = handle
    assert sample(lib, h) == ab.ERR_WORKSPACE and predict(lib, h) == ab.ERR_WORKSPACE
    assert sample(lib, None) == ab.ERR_INVALID_ARG and predict(lib, None) == ab.ERR_INVALID_ARG
    # the address is taken before the call fails for want of a GPU; no refused call touches it
    assert lib.acache_set_workspace(h, 1 << 20, lib.acache_workspace_bytes(h), None) == ab.ERR_CUDA
    bad = ab.ERR_INVALID_ARG
    for kw, code in ((dict(logits=None), bad), (dict(logits=258), bad), (dict(logits=257, kind=0), bad), (dict(kind=2), bad), (dict(kind=-1), bad), (dict(rows=-1), bad),
                     (dict(vocab=0), bad), (dict(vocab=-5), bad), (dict(stride=99), bad), (dict(how=None), bad), (dict(how=ab.Sampling(None, None, None, None, 0)), bad),
                     (dict(how=ab.Sampling(None, None, None, None, -2)), bad), (dict(u=None), bad), (dict(token=None), bad),
                     (dict(vocab=262145, stride=262145), ab.ERR_UNSUPPORTED_SHAPE), (dict(rows=(1 << 24) + 1), ab.ERR_UNSUPPORTED_SHAPE)):
        assert sample(lib, h, **kw) == code, kw
    assert sample(lib, h, rows=0) == ab.OK
    for kw, code in ((dict(how=None), bad), (dict(logits=None), bad), (dict(logits=260), bad), (dict(u=None), bad), (dict(token=None), bad), (dict(vocab=0), bad),
                     (dict(vocab=1408), bad), (dict(vocab=100), ab.ERR_UNSUPPORTED_SHAPE), (dict(n=-1), bad), (dict(n=17), bad),
                     (dict(how=ab.Sampling(None, None, None, None, 0)), bad)):
        assert predict(lib, h, **kw) == code, kw
    assert predict(lib, h, n=0) == ab.OK
