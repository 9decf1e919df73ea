"""The binding lets no cache through whose tensors a call would read or write past: tensors of the host, fewer requests than the
call has, other heads than the context's.  On the host, over a library that only notes that it was called."""
import pytest
import torch

from paper_2608_26140_b200 import binding as ab

H, HKV, D, CAP, BLOCK = 8, 2, 64, 128, 32


class Library:
    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append(name) or ab.OK


class OnGpu(torch.Tensor):
    """A tensor of the host that says it is on a GPU."""
    is_cuda = True


@pytest.fixture
def ctx(monkeypatch):
    monkeypatch.setattr(ab, "_stream", lambda: 0)
    c = ab.Context.__new__(ab.Context)
    c.lib, c.h, c.heads = Library(), None, (H, HKV, D)
    return c


def on_gpu(t):
    return t.as_subclass(OnGpu)


def tensors(batch, hkv=HKV, d=D, gpu=True):
    t = [torch.zeros((batch, hkv, CAP, d), dtype=torch.uint8) for _ in range(2)]
    t += [torch.zeros((batch, hkv, CAP // BLOCK), dtype=torch.uint8) for _ in range(2)]
    return [on_gpu(x) for x in t] if gpu else t


def calls(ctx, batch):
    rows = on_gpu(torch.zeros((batch, 3, HKV, D), dtype=torch.bfloat16))
    q = on_gpu(torch.zeros((batch, 3, H, D), dtype=torch.bfloat16))
    req = ab.Request()
    req.batch = batch
    return [lambda c: ctx.kv8_write(c, batch, CAP, rows, rows), lambda c: ctx.kv8_read(c, batch, CAP, rows, rows),
            lambda c: ctx.kv8_attention(c, batch, CAP, q, q), lambda c: ctx.layer_step_kv8(ab.LayerWeights(), req, c, q, 0, 0.0, 0, None, None, q)]


def test_caches_that_fit_go_through(ctx):
    for shared, batch, made in ((False, 2, 2), (False, 1, 2), (True, 5, 1)):
        c = ab.Context.kv8(*tensors(made), BLOCK, 0, shared=shared)
        for call in calls(ctx, batch):
            call(c)
    assert len(ctx.lib.calls) == 12


@pytest.mark.parametrize("made", [dict(batch=1), dict(batch=2, hkv=1), dict(batch=2, hkv=4), dict(batch=2, d=128), dict(batch=2, gpu=False)])
def test_caches_that_do_not_fit_are_refused(ctx, made):
    c = ab.Context.kv8(*tensors(**made), BLOCK, 0)
    for call in calls(ctx, 2):
        with pytest.raises(ValueError, match="cache"):
            call(c)
    assert not ctx.lib.calls


def test_a_tensor_of_the_host_among_those_of_a_cache_is_found(ctx):
    for i in range(4):
        t = tensors(2)
        t[i] = torch.zeros_like(t[i]).as_subclass(torch.Tensor)
        c = ab.Context.kv8(*t, BLOCK, 0)
        for call in calls(ctx, 2):
            with pytest.raises(ValueError, match="cache"):
                call(c)
    assert not ctx.lib.calls


def test_requests_in_the_same_place_are_no_cache_of_their_own():
    """Expanded codes would have been taken for a cache that is shared, with the exponents of its first request."""
    t = tensors(3)
    with pytest.raises(ValueError):
        ab.Context.kv8(t[0][:1].expand(3, HKV, CAP, D), t[1][:1].expand(3, HKV, CAP, D), t[2], t[3], BLOCK, 0)
    one = [x[:1] for x in t]
    alone = ab.Context.kv8(one[0].as_strided(one[0].shape, (0, CAP * D, D, 1)), one[1], *one[2:], BLOCK, 0)
    assert alone.batch_stride == HKV * CAP * D
