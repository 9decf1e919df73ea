"""What the binding refuses before acache_recompute_paged is called, without a GPU: the current device is made the CPU's number, so that tensors here are where
they should be, and the library is one that notes its calls."""
import ctypes as C
import types

import pytest
import torch

from paper_2608_26140_b200 import binding as ab

B, T, L, E, K, D, F, V = 2, 40, 16, 3, 4, 256, 384, 50
H, HKV, d = 4, 2, 64
BF16, F32, I32 = torch.bfloat16, torch.float32, torch.int32


class Elsewhere(torch.Tensor):
    def get_device(self):
        return 5


@pytest.fixture
def ctx(monkeypatch):
    monkeypatch.setattr(ab, "_current_device", lambda: -1)
    monkeypatch.setattr(ab, "_stream", lambda: 0)
    c = ab.Context.__new__(ab.Context)
    c.h, c.gpu, c.heads, c.desc, c.dtypes = None, -1, (H, HKV, d), ab.ModelDesc(hidden=D, ffn=F, qkv_bias=1), (BF16, F32, I32)
    c.calls = []
    c.lib = types.SimpleNamespace(acache_recompute_paged=lambda *a: c.calls.append(a) or ab.OK)
    return c


def tensors():
    bf = lambda *s: torch.zeros(s, dtype=BF16)  # noqa: E731
    w = dict(attn_norm_g=bf(D), wq=bf(H * d, D), wk=bf(HKV * d, D), wv=bf(HKV * d, D), bq=bf(H * d), bk=bf(HKV * d), bv=bf(HKV * d), wo=bf(D, H * d), mlp_norm_g=bf(D),
             w_gate=bf(F, D), w_up=bf(F, D), w_down=bf(D, F))
    r = dict(extra_rows=torch.zeros((B, E), dtype=I32), rope_cos=torch.zeros((T, d // 2)), rope_sin=torch.zeros((T, d // 2)), token_ids=torch.zeros((B, T), dtype=I32))
    a = dict(x=bf(V, D), anchor_idx=torch.zeros((B, K), dtype=I32), y=bf(B, K + E, D), lens=torch.zeros(B, dtype=I32))
    return w, r, a


def call(ctx, w, r, a, compact=0, k=K):
    weights = w if isinstance(w, ab.LayerWeights) else ab.Context.weights(w)
    req = r if isinstance(r, ab.Request) else ab.Context.request(B, T, 0, L, None, r["extra_rows"], r["rope_cos"], r["rope_sin"], token_ids=r["token_ids"], n_embed=V)
    cache = ab.PagedKV()
    cache.made_of = (B, HKV, d, True, -1)
    ctx.recompute_paged(weights, req, cache, a["x"], compact, a["anchor_idx"], k, a["y"], lens=a["lens"])


def test_tensors_that_fit_come_through(ctx):
    w, r, a = tensors()
    call(ctx, w, r, a)                                           # looked up
    call(ctx, w, r, {**a, "x": torch.zeros((B, K + E, D), dtype=BF16)}, compact=1)
    call(ctx, w, {**r, "token_ids": None}, {**a, "x": torch.zeros((B, T, D), dtype=BF16)})
    call(ctx, w, r, {**a, "anchor_idx": None, "y": torch.zeros((B, E, D), dtype=BF16), "lens": None}, k=0)
    call(ctx, w, r, {**a, "y": torch.zeros((B + 1, K + E, D), dtype=BF16), "x": torch.zeros((V + 9, D), dtype=BF16)})      # more than is wanted
    # what the library refuses itself
    call(ctx, w, r, {**a, "x": None})
    call(ctx, w, r, {**a, "anchor_idx": None, "y": torch.zeros((B, E, D), dtype=BF16)})
    call(ctx, ab.LayerWeights(), r, a)
    assert len(ctx.calls) == 8
    got = ctx.calls[0]
    assert (got[4], got[5], got[6], got[7], got[8], got[9]) == (a["x"].data_ptr(), 0, a["anchor_idx"].data_ptr(), K, a["lens"].data_ptr(), a["y"].data_ptr())


def worse(t):
    kinds = {BF16: torch.float16, F32: torch.float64, I32: torch.int64}
    return t.to(kinds[t.dtype]), t[:-1], t[:0], torch.zeros((*t.shape, 2), dtype=t.dtype)[..., 0], t.clone().as_subclass(Elsewhere)


@pytest.mark.parametrize("name", ["x", "anchor_idx", "y", "lens"])
def test_arguments_that_do_not_fit_are_refused(ctx, name):
    w, r, a = tensors()
    for bad in worse(a[name]):
        with pytest.raises(ValueError):
            call(ctx, w, r, {**a, name: bad})
    for compact, x in ((1, torch.zeros((B, K + E - 1, D), dtype=BF16)), (0, torch.zeros((V - 1, D), dtype=BF16))):
        with pytest.raises(ValueError):
            call(ctx, w, r, {**a, "x": x}, compact=compact)
    with pytest.raises(ValueError):
        call(ctx, w, {**r, "token_ids": None}, a)                # a table without indexes into it
    assert not ctx.calls


@pytest.mark.parametrize("name", ["attn_norm_g", "wq", "wk", "wv", "bq", "bk", "bv", "wo", "mlp_norm_g", "w_gate", "w_up", "w_down"])
def test_weights_that_do_not_fit_are_refused(ctx, name):
    w, r, a = tensors()
    for bad in worse(w[name]):
        if bad.numel() == 0:                                     # a NULL, which the library refuses
            continue
        with pytest.raises(ValueError, match=name + ":"):
            call(ctx, {**w, name: bad}, r, a)
    assert not ctx.calls
    one = ab.Context.weights(w)
    call(ctx, one, r, a)
    ctx.desc = ab.ModelDesc(hidden=2 * D, ffn=2 * F, qkv_bias=1)                # the same weights for another layer
    with pytest.raises(ValueError):
        call(ctx, one, r, {**a, "x": torch.zeros((V, 2 * D), dtype=BF16), "y": torch.zeros((B, K + E, 2 * D), dtype=BF16)})
    # an address put in by hand is the caller's affair
    one = ab.Context.weights({**w, name: w[name].double()})
    ctx.desc = ab.ModelDesc(hidden=D, ffn=F, qkv_bias=1)
    setattr(one, name, C.c_void_p(4096))
    call(ctx, one, r, a)


@pytest.mark.parametrize("name", ["extra_rows", "rope_cos", "rope_sin", "token_ids"])
def test_requests_that_do_not_fit_are_refused(ctx, name):
    w, r, a = tensors()
    for bad in worse(r[name]):
        if bad.numel() == 0:                                     # none, or a NULL, which the library refuses
            continue
        with pytest.raises(ValueError, match=name + ":"):
            call(ctx, w, {**r, name: bad}, a)
    assert not ctx.calls
    compact = {**a, "x": torch.zeros((B, K + E, D), dtype=BF16)}
    call(ctx, w, {**r, "token_ids": r["token_ids"].long()}, compact, compact=1)  # not looked at
