"""Thin ctypes binding of the C-ABI library (``include/acache.h``).

Argument marshalling only: every step of the path runs in the library's CUDA
kernels.  Tensors are ``torch`` CUDA tensors (used for device memory and the
current stream); there is no CPU fallback -- loading fails loudly if the
library has not been built (``python -m paper_2608_26140_b200.build``).
"""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, Optional

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libacache.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED_SHAPE, ERR_WORKSPACE, ERR_CUDA, ERR_TIMEOUT = range(6)
FLAG_BAD_INDEX, FLAG_WAIT_EXPIRED, FLAG_NONFINITE = 0x1, 0x2, 0x4
KV8_FORMATS = {"e4m3": 0, "int8": 1}
F_SCORE, F_SELECT, F_ACCUMULATE, F_SCORE_NORM_FULL, F_NO_RECOMPUTE, F_DROP_NON_ANCHOR = 0x1, 0x2, 0x4, 0x8, 0x10, 0x20

EXPORTS = ["acache_create", "acache_workspace_bytes", "acache_set_workspace", "acache_destroy",
           "acache_last_error", "acache_poll_status", "acache_launch_count", "acache_score_anchors",
           "acache_k_from_ratio", "acache_select_topk", "acache_recompute_anchors", "acache_scatter_kv",
           "acache_layer_step", "acache_layer_step_host", "acache_stage_timing", "acache_read_stage_times",
           "acache_score_anchors_static", "acache_predict_commit", "acache_denoise_step", "acache_probe_select",
           "acache_commit_update", "acache_generate_block", "acache_denoise_step_shared", "acache_recompute_rows_shared",
           "acache_decode_step_shared", "acache_generate_block_shared", "acache_layer_step_shared",
           "acache_host_x_in_place", "acache_score_kv_deviation", "acache_debug_expire_next_wait",
           "acache_kv8_write", "acache_kv8_read", "acache_kv8_attention", "acache_layer_step_kv8"]

STAGES = ["mask_q", "score", "topk", "gather_norm", "qkv", "attention", "oproj", "mlp_norm", "gate_up", "down"]


class ModelDesc(C.Structure):
    _fields_ = [("hidden", C.c_int32), ("n_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("ffn", C.c_int32), ("rms_eps", C.c_float),
                ("qkv_bias", C.c_int32), ("max_batch", C.c_int32), ("max_ctx", C.c_int32),
                ("max_affix", C.c_int32), ("max_rows", C.c_int32), ("max_masked", C.c_int32),
                ("max_vocab", C.c_int32), ("max_block", C.c_int32)]


class LayerWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("attn_norm_g", "wq", "wk", "wv", "bq", "bk", "bv", "wo",
                                          "mlp_norm_g", "w_gate", "w_up", "w_down")]


class KV(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("batch_stride", C.c_int64), ("ctx_capacity", C.c_int32)]


class KV8(C.Structure):
    _fields_ = [("k", C.c_void_p), ("v", C.c_void_p), ("k_exp", C.c_void_p), ("v_exp", C.c_void_p), ("batch_stride", C.c_int64),
                ("ctx_capacity", C.c_int32), ("block", C.c_int32), ("format", C.c_int32)]
    made_of = None      # of the tensors that Context.kv8 made it over: requests (shared: any number), KV heads, head dimension, all on a GPU


class Request(C.Structure):
    _fields_ = [("batch", C.c_int32), ("ctx_len", C.c_int32), ("affix_start", C.c_int32),
                ("affix_len", C.c_int32), ("masked_pos", C.c_void_p), ("n_masked", C.c_int32),
                ("extra_rows", C.c_void_p), ("n_extra", C.c_int32), ("rope_cos", C.c_void_p),
                ("rope_sin", C.c_void_p), ("token_ids", C.c_void_p), ("n_embed", C.c_int32)]


class AcacheError(RuntimeError):
    def __init__(self, status: int, msg: str):
        super().__init__(f"acache status {status}: {msg}")
        self.status = status


_lib = None


def load_library(path: Optional[str] = None) -> C.CDLL:
    """Loads libacache.so (once) and declares the prototypes."""
    global _lib
    if _lib is not None and path is None:
        return _lib
    p = path or LIB_PATH
    if not os.path.exists(p):
        raise RuntimeError(f"{p} is missing: build it with `python -m paper_2608_26140_b200.build` "
                           "(there is no CPU fallback)")
    lib = C.CDLL(p)
    vp, i32, u32, i64 = C.c_void_p, C.c_int32, C.c_uint32, C.c_int64
    lib.acache_create.argtypes = [C.POINTER(ModelDesc), C.POINTER(vp)]
    lib.acache_create.restype = C.c_int
    lib.acache_workspace_bytes.argtypes = [vp]
    lib.acache_workspace_bytes.restype = C.c_size_t
    lib.acache_set_workspace.argtypes = [vp, vp, C.c_size_t, vp]
    lib.acache_set_workspace.restype = C.c_int
    lib.acache_destroy.argtypes = [vp]
    lib.acache_destroy.restype = None
    lib.acache_last_error.argtypes = [vp]
    lib.acache_last_error.restype = C.c_char_p
    lib.acache_poll_status.argtypes = [vp, vp, C.POINTER(u32)]
    lib.acache_poll_status.restype = C.c_int
    lib.acache_debug_expire_next_wait.argtypes = [vp]
    lib.acache_debug_expire_next_wait.restype = C.c_int
    lib.acache_launch_count.argtypes = [vp]
    lib.acache_launch_count.restype = C.c_uint64
    lib.acache_score_anchors.argtypes = [vp, C.POINTER(Request), vp, C.POINTER(KV), vp, C.c_int, C.c_int, vp]
    lib.acache_score_anchors.restype = C.c_int
    lib.acache_score_kv_deviation.argtypes = [vp, C.POINTER(Request), C.POINTER(KV), C.POINTER(KV), vp, C.c_int, vp]
    lib.acache_score_kv_deviation.restype = C.c_int
    lib.acache_k_from_ratio.argtypes = [i32, C.c_double]
    lib.acache_k_from_ratio.restype = i32
    lib.acache_select_topk.argtypes = [vp, vp, i32, i32, i32, vp, vp]
    lib.acache_select_topk.restype = C.c_int
    lib.acache_recompute_anchors.argtypes = [vp, C.POINTER(LayerWeights), C.POINTER(Request), C.POINTER(KV),
                                             vp, C.c_int, vp, i32, vp, vp, vp, vp]
    lib.acache_recompute_anchors.restype = C.c_int
    lib.acache_scatter_kv.argtypes = [vp, C.POINTER(Request), C.POINTER(KV), vp, i32, vp, vp, vp]
    lib.acache_scatter_kv.restype = C.c_int
    lib.acache_layer_step.argtypes = [vp, C.POINTER(LayerWeights), C.POINTER(Request), C.POINTER(KV), vp, C.c_int,
                                      C.c_double, u32, vp, vp, vp, vp]
    lib.acache_layer_step.restype = C.c_int
    lib.acache_layer_step_host.argtypes = [vp, C.POINTER(LayerWeights), C.POINTER(Request), C.POINTER(KV), vp,
                                           C.c_double, u32, vp, vp, vp, vp]
    lib.acache_layer_step_host.restype = C.c_int
    lib.acache_host_x_in_place.argtypes = [vp]
    lib.acache_host_x_in_place.restype = C.c_int32
    lib.acache_score_anchors_static.argtypes = [C.POINTER(ModelDesc), C.POINTER(Request), vp, C.POINTER(KV), vp,
                                                C.c_int, C.c_int, vp]
    lib.acache_score_anchors_static.restype = C.c_int
    lib.acache_predict_commit.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp, i32, C.c_float, vp, vp, vp, vp]
    lib.acache_predict_commit.restype = C.c_int
    lib.acache_denoise_step.argtypes = [vp, i32, C.POINTER(LayerWeights), C.POINTER(KV), C.POINTER(Request), vp, vp, i32,
                                        vp, vp, C.POINTER(vp), vp, i32, vp, vp, i32, C.c_float, vp, vp, vp, vp]
    lib.acache_denoise_step.restype = C.c_int
    lib.acache_denoise_step_shared.argtypes = [vp, i32, C.POINTER(LayerWeights), C.POINTER(KV), C.POINTER(Request), vp, vp, i32,
                                               C.POINTER(vp), C.POINTER(vp), vp, vp, C.POINTER(vp), vp, i32, vp, vp, i32,
                                               C.c_float, vp, vp, vp, vp]
    lib.acache_denoise_step_shared.restype = C.c_int
    lib.acache_probe_select.argtypes = [vp, i32, C.POINTER(LayerWeights), C.POINTER(KV), C.POINTER(Request), vp,
                                        C.c_double, u32, vp, vp, vp, vp, vp]
    lib.acache_probe_select.restype = C.c_int
    lib.acache_commit_update.argtypes = [vp, vp, i32, vp, i32, i32, vp, vp, i32, C.c_float, vp, vp]
    lib.acache_commit_update.restype = C.c_int
    lib.acache_generate_block.argtypes = [vp, i32, C.POINTER(LayerWeights), C.POINTER(KV), C.POINTER(Request),
                                          C.POINTER(Request), vp, vp, i32, vp, vp, vp, vp, i32, vp, vp, i32, C.c_float,
                                          i32, i32, vp, vp, vp, vp, C.POINTER(i32), vp]
    lib.acache_generate_block.restype = C.c_int
    lib.acache_layer_step_shared.argtypes = [vp, C.POINTER(LayerWeights), C.POINTER(Request), C.POINTER(KV), vp, C.c_int,
                                             C.c_double, u32, vp, vp, vp, vp, vp, vp]
    lib.acache_layer_step_shared.restype = C.c_int
    lib.acache_recompute_rows_shared.argtypes = [vp, C.POINTER(LayerWeights), C.POINTER(Request), C.POINTER(Request),
                                                 C.POINTER(KV), vp, C.c_int, vp, i32, vp, vp, vp, vp, vp]
    lib.acache_recompute_rows_shared.restype = C.c_int
    lib.acache_decode_step_shared.argtypes = [vp, i32, C.POINTER(LayerWeights), C.POINTER(KV), C.POINTER(Request),
                                              C.POINTER(Request), vp, vp, i32, vp, C.POINTER(vp), C.POINTER(vp), vp, vp,
                                              C.POINTER(vp), vp, i32, vp, vp, i32, C.c_float, vp, vp, vp, vp]
    lib.acache_decode_step_shared.restype = C.c_int
    lib.acache_generate_block_shared.argtypes = [vp, i32, C.POINTER(LayerWeights), C.POINTER(KV), C.POINTER(Request),
                                                 C.POINTER(Request), vp, vp, i32, C.POINTER(vp), C.POINTER(vp), vp, vp, vp, vp,
                                                 i32, vp, vp, i32, C.c_float, i32, i32, vp, vp, vp, vp, C.POINTER(i32), vp]
    lib.acache_generate_block_shared.restype = C.c_int
    lib.acache_kv8_write.argtypes = [vp, C.POINTER(KV8), i32, i32, vp, vp, i64, i32, vp, i32, vp]
    lib.acache_kv8_write.restype = C.c_int
    lib.acache_kv8_read.argtypes = [vp, C.POINTER(KV8), i32, i32, vp, vp, i32, vp, i32, vp]
    lib.acache_kv8_read.restype = C.c_int
    lib.acache_kv8_attention.argtypes = [vp, C.POINTER(KV8), i32, i32, i32, vp, vp, vp, vp, vp, vp]
    lib.acache_kv8_attention.restype = C.c_int
    lib.acache_layer_step_kv8.argtypes = [vp, C.POINTER(LayerWeights), C.POINTER(Request), C.POINTER(KV8), vp, C.c_int,
                                          C.c_double, u32, vp, vp, vp, vp]
    lib.acache_layer_step_kv8.restype = C.c_int
    lib.acache_stage_timing.argtypes = [vp, C.c_int]
    lib.acache_stage_timing.restype = C.c_int
    lib.acache_read_stage_times.argtypes = [vp, C.POINTER(C.c_float)]
    lib.acache_read_stage_times.restype = C.c_int
    if path is None:
        _lib = lib
    return lib


def k_from_ratio(affix_len: int, ratio: float) -> int:
    return int(load_library().acache_k_from_ratio(int(affix_len), float(ratio)))


def score_anchors_static(desc: ModelDesc, req: Request, q_mask, kv: KV, scores, accumulate=False,
                         norm_full=False) -> int:
    """Scoring through the entry point that allocates nothing and needs no context or workspace
    (its scratch is a fixed array inside the library).  Returns the status code."""
    return int(load_library().acache_score_anchors_static(C.byref(desc), C.byref(req), _ptr(q_mask), C.byref(kv),
                                                          _ptr(scores), int(accumulate), int(norm_full), _stream()))


def _ptr(t) -> Optional[int]:
    """Device (or host) address of a tensor, an int, or None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _check_tensor(t, dtype, shape):
    if t.shape != shape or t.dtype is not dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"a tensor {tuple(t.shape)} of {t.dtype} on {t.device} where contiguous {tuple(shape)} of {dtype} on a GPU is wanted")


def _dense(t, strides):
    """All dimensions but the first as in a contiguous tensor; the stride of a dimension of one element says nothing."""
    return t.numel() == 0 or all(n == 1 or have == want for n, have, want in zip(t.shape[1:], t.stride()[1:], strides))


def _stream() -> int:
    """The current stream of the current device (torch.cuda.current_stream() builds an object around it: 3.3 us a call, this 0.2)."""
    import torch
    return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())


class Context:
    """One layer shape + workspace.  Mirrors the C entry points one to one."""

    def __init__(self, hidden, n_heads, n_kv_heads, head_dim, ffn, rms_eps, qkv_bias,
                 max_batch, max_ctx, max_affix, max_rows, max_masked, device="cuda:0", max_vocab=0, max_block=0):
        import torch
        self.lib = load_library()
        self.desc = ModelDesc(hidden, n_heads, n_kv_heads, head_dim, ffn, rms_eps, int(bool(qkv_bias)),
                              max_batch, max_ctx, max_affix, max_rows, max_masked, max_vocab, max_block)
        self.heads = (n_heads, n_kv_heads, head_dim)
        h = C.c_void_p()
        st = self.lib.acache_create(C.byref(self.desc), C.byref(h))
        if st != OK:
            raise AcacheError(st, "acache_create rejected the descriptor")
        self.h = h
        self.device = torch.device(device)
        nbytes = self.lib.acache_workspace_bytes(self.h)
        with torch.cuda.device(self.device):
            self.workspace = torch.empty(nbytes + 256, dtype=torch.uint8, device=self.device)
            base = self.workspace.data_ptr()
            self._ws_ptr = (base + 255) & ~255
            self._check(self.lib.acache_set_workspace(self.h, self._ws_ptr, nbytes, _stream()))
        self.workspace_bytes = nbytes

    @classmethod
    def for_shape(cls, shape, max_batch, max_ctx, max_affix, max_rows, max_masked, device="cuda:0", max_vocab=0,
                  max_block=0):
        return cls(shape.hidden, shape.n_heads, shape.n_kv_heads, shape.head_dim, shape.ffn, shape.rms_eps,
                   shape.qkv_bias, max_batch, max_ctx, max_affix, max_rows, max_masked, device, max_vocab, max_block)

    def close(self):
        if getattr(self, "h", None):
            self.lib.acache_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _check(self, st: int):
        if st != OK:
            raise AcacheError(st, self.lib.acache_last_error(self.h).decode())

    # ---- marshalling helpers ----
    @staticmethod
    def weights(w: Dict[str, object]) -> LayerWeights:
        lw = LayerWeights()
        for name, _ in LayerWeights._fields_:
            setattr(lw, name, _ptr(w.get(name)))
        return lw

    @staticmethod
    def kv(cache_k, cache_v) -> KV:
        B, cap, hkv, d = cache_k.shape
        return KV(cache_k.data_ptr(), cache_v.data_ptr(), cap * hkv * d, cap)

    @staticmethod
    def kv8(codes_k, codes_v, exp_k, exp_v, block, fmt, shared=False) -> KV8:
        """8-bit cache over one-byte codes [B, Hkv, capacity, d] and exponent bytes [B, Hkv, capacity / block]; fmt: a value of
        KV8_FORMATS.  Requests may lie further apart than their codes take.  shared: one request's cache for every request."""
        requests, hkv, cap, d = codes_k.shape
        for c, e in ((codes_k, exp_k), (codes_v, exp_v)):
            if c.element_size() != 1 or e.element_size() != 1:
                raise ValueError("codes and exponents are bytes")
            if c.shape != codes_k.shape or tuple(e.shape) != (c.shape[0], hkv, cap // block):
                raise ValueError(f"codes {tuple(c.shape)} and exponents {tuple(e.shape)} do not go together with blocks of {block}")
            if not _dense(c, (cap * d, d, 1)) or not e.is_contiguous() or (requests > 1 and c.stride(0) != codes_k.stride(0)):
                raise ValueError("the codes of a request and all exponents are contiguous")
        stride = codes_k.stride(0) if requests > 1 else hkv * cap * d
        if stride == 0 and not shared:
            raise ValueError("the codes of all requests lie in one place: shared=True is for that")
        c = KV8(_ptr(codes_k), _ptr(codes_v), _ptr(exp_k), _ptr(exp_v), 0 if shared else stride, cap, block, fmt)
        c.made_of = (float("inf") if shared else requests, hkv, d, all(t.is_cuda for t in (codes_k, codes_v, exp_k, exp_v)))
        return c

    def new_kv8(self, batch, ctx_capacity, block=64, fmt="e4m3"):
        """An empty 8-bit cache for this context's shape: (tensors to keep alive: codes k, v, exponents k, v; the KV8)."""
        import torch
        hkv, d = self.desc.n_kv_heads, self.desc.head_dim
        cap = -(-ctx_capacity // block) * block
        t = [torch.zeros((batch, hkv, cap, d), dtype=torch.uint8, device=self.device) for _ in range(2)]
        t += [torch.zeros((batch, hkv, cap // block), dtype=torch.uint8, device=self.device) for _ in range(2)]
        return t, self.kv8(*t, block, KV8_FORMATS[fmt])

    @staticmethod
    def pack_key_drop(drop):
        """Boolean [B, T] (True: the position does not exist as a key) as the bit mask of kv8_attention, int32 [B, ceil(T / 32)]."""
        import torch
        import torch.nn.functional as F
        B, T = drop.shape
        bits = F.pad(drop.to(torch.int64), (0, -T % 32)).view(B, -1, 32) << torch.arange(32, device=drop.device)
        return bits.sum(-1).to(torch.uint32).view(torch.int32)

    @staticmethod
    def request(batch, ctx_len, affix_start, affix_len, masked_pos, extra_rows, rope_cos, rope_sin,
                token_ids=None, n_embed=0) -> Request:
        nm = 0 if masked_pos is None else int(masked_pos.shape[1])
        ne = 0 if extra_rows is None else int(extra_rows.shape[1])
        return Request(batch, ctx_len, affix_start, affix_len, _ptr(masked_pos) if nm else None, nm,
                       _ptr(extra_rows) if ne else None, ne, _ptr(rope_cos), _ptr(rope_sin), _ptr(token_ids), n_embed)

    # ---- entry points ----
    def launch_count(self) -> int:
        return int(self.lib.acache_launch_count(self.h))

    def poll_status(self) -> int:
        flags = C.c_uint32(0)
        st = self.lib.acache_poll_status(self.h, _stream(), C.byref(flags))
        if st not in (OK, ERR_TIMEOUT):
            self._check(st)
        return int(flags.value)

    def poll_status_code(self):
        """(status code, flags) of acache_poll_status: ERR_TIMEOUT when a bounded device-side wait ran out."""
        flags = C.c_uint32(0)
        st = self.lib.acache_poll_status(self.h, _stream(), C.byref(flags))
        return int(st), int(flags.value)

    def debug_expire_next_wait(self):
        """Failure-detection self-test: the next Q/K/V projection's grid barrier is made to run out."""
        self._check(self.lib.acache_debug_expire_next_wait(self.h))

    def stage_timing(self, enable: bool):
        self._check(self.lib.acache_stage_timing(self.h, int(enable)))

    def read_stage_times(self) -> Dict[str, float]:
        """Milliseconds per stage of the last timed layer-step (synchronises)."""
        ms = (C.c_float * len(STAGES))()
        self._check(self.lib.acache_read_stage_times(self.h, ms))
        return {n: float(ms[i]) for i, n in enumerate(STAGES)}

    def score_anchors(self, req: Request, q_mask, kv: KV, scores, accumulate=False, norm_full=False):
        self._check(self.lib.acache_score_anchors(self.h, C.byref(req), _ptr(q_mask), C.byref(kv), _ptr(scores),
                                                  int(accumulate), int(norm_full), _stream()))

    def score_kv_deviation(self, req: Request, kv_ref: KV, kv_full: KV, scores, accumulate=False):
        self._check(self.lib.acache_score_kv_deviation(self.h, C.byref(req), C.byref(kv_ref), C.byref(kv_full), _ptr(scores),
                                                       int(accumulate), _stream()))

    def select_topk(self, scores, batch, affix_len, k, anchor_idx):
        self._check(self.lib.acache_select_topk(self.h, _ptr(scores), batch, affix_len, k, _ptr(anchor_idx), _stream()))

    def recompute_anchors(self, w: LayerWeights, req: Request, kv: KV, x, x_is_compact, anchor_idx, k,
                          k_new, v_new, y):
        self._check(self.lib.acache_recompute_anchors(self.h, C.byref(w), C.byref(req), C.byref(kv), _ptr(x),
                                                      int(x_is_compact), _ptr(anchor_idx), k, _ptr(k_new),
                                                      _ptr(v_new), _ptr(y), _stream()))

    def scatter_kv(self, req: Request, kv: KV, anchor_idx, k, k_new, v_new):
        self._check(self.lib.acache_scatter_kv(self.h, C.byref(req), C.byref(kv), _ptr(anchor_idx), k,
                                               _ptr(k_new), _ptr(v_new), _stream()))

    def layer_step(self, w: LayerWeights, req: Request, kv: KV, x, x_is_compact, ratio, flags, scores,
                   anchor_idx, y):
        self._check(self.lib.acache_layer_step(self.h, C.byref(w), C.byref(req), C.byref(kv), _ptr(x),
                                               int(x_is_compact), float(ratio), int(flags), _ptr(scores),
                                               _ptr(anchor_idx), _ptr(y), _stream()))

    # A call of the three below takes 6-8 us, more than many of their kernels, most of it here: tensors are asked for each property once.
    def kv8_write(self, cache: KV8, batch, ctx_len, k_rows, v_rows, start=0, pos=None):
        """Rows [B, n, Hkv, d] (bf16; requests may lie further apart) to positions start .. or pos [B, n] (int32)."""
        self._cache_fits(cache, batch)
        shape, stride = self._rows(k_rows, batch, pos)
        if self._rows(v_rows, batch, None) != (shape, stride):
            raise ValueError("k_rows and v_rows differ in shape or stride")
        self._check(self.lib.acache_kv8_write(self.h, C.byref(cache), batch, ctx_len, k_rows.data_ptr(), v_rows.data_ptr(), stride,
                                              shape[1], _ptr(pos), start, _stream()))

    def kv8_read(self, cache: KV8, batch, ctx_len, k_out, v_out, start=0, pos=None):
        """Rows at positions start .. or pos [B, n] into k_out, v_out [B, n, Hkv, d] (contiguous; either may be None)."""
        self._cache_fits(cache, batch)
        one = v_out if k_out is None else k_out
        if one is None:
            raise AcacheError(ERR_INVALID_ARG, "neither k_out nor v_out is given")
        shape, _ = self._rows(one, batch, pos)
        if not one.is_contiguous():
            raise ValueError("k_out and v_out are contiguous")
        if one is not v_out and v_out is not None:
            _check_tensor(v_out, one.dtype, shape)
        self._check(self.lib.acache_kv8_read(self.h, C.byref(cache), batch, ctx_len, _ptr(k_out), _ptr(v_out), shape[1], _ptr(pos), start,
                                             _stream()))

    def kv8_attention(self, cache: KV8, batch, ctx_len, q, o, lse=None, lens=None, key_drop=None):
        """q, o: bf16 [B, n, H, d]; lse: fp32 [B, n, H]; lens: int32 [B]; key_drop: int32 [B, ceil(ctx_len / 32)] (pack_key_drop)."""
        import torch
        self._cache_fits(cache, batch)
        shape = q.shape
        B, n, H, d = shape
        if B != batch or H != self.heads[0] or d != self.heads[2]:
            raise ValueError(f"q {tuple(shape)} is not [batch, n, H, d]")
        _check_tensor(q, torch.bfloat16, shape)
        _check_tensor(o, torch.bfloat16, shape)
        if lse is not None:
            _check_tensor(lse, torch.float32, shape[:3])
        if lens is not None:
            _check_tensor(lens, torch.int32, (B,))
        if key_drop is not None:
            _check_tensor(key_drop, torch.int32, (B, -(-ctx_len // 32)))
        self._check(self.lib.acache_kv8_attention(self.h, C.byref(cache), batch, n, ctx_len, q.data_ptr(), _ptr(lens), _ptr(key_drop),
                                                  o.data_ptr(), _ptr(lse), _stream()))

    def layer_step_kv8(self, w: LayerWeights, req: Request, cache: KV8, x, x_is_compact, ratio, flags, scores, anchor_idx, y):
        """The layer-step on an 8-bit cache."""
        self._cache_fits(cache, req.batch)
        self._check(self.lib.acache_layer_step_kv8(self.h, C.byref(w), C.byref(req), C.byref(cache), _ptr(x), int(x_is_compact),
                                                   float(ratio), int(flags), _ptr(scores), _ptr(anchor_idx), _ptr(y), _stream()))

    def _cache_fits(self, cache, batch):
        """What a call would read or write past the cache's tensors for (a KV8 filled in by hand is the caller's affair)."""
        m = cache.made_of
        if m is not None and (m[0] < batch or m[1:] != (self.heads[1], self.heads[2], True)):
            raise ValueError(f"a cache of {m[0]} requests, {m[1]} KV heads of {m[2]}, {'not ' if not m[3] else ''}all on a GPU, "
                             f"for {batch} requests and {self.heads[1]} KV heads of {self.heads[2]}")

    def _rows(self, t, batch, pos):
        """Shape of rows [B, n, Hkv, d], and elements between the requests."""
        import torch
        shape = t.shape
        B, n, hkv, d = shape
        if B != batch or hkv != self.heads[1] or d != self.heads[2] or t.dtype is not torch.bfloat16 or not t.is_cuda:
            raise ValueError(f"rows {tuple(shape)} of {t.dtype} on {t.device} are not bf16 [batch, n, Hkv, d] on a GPU")
        stride = t.stride()
        if stride[1:] != (hkv * d, d, 1) and not _dense(t, (hkv * d, d, 1)):
            raise ValueError("the rows of a request are contiguous")
        if pos is not None:
            _check_tensor(pos, torch.int32, (B, n))
        return shape, stride[0] if B > 1 else n * hkv * d

    def predict_commit(self, h, h_rows, block_rows, batch, n_blk, final_norm_g, w_lm, vocab, threshold, token,
                       confidence, commit):
        self._check(self.lib.acache_predict_commit(self.h, _ptr(h), h_rows, _ptr(block_rows), batch, n_blk,
                                                   _ptr(final_norm_g), _ptr(w_lm), vocab, float(threshold), _ptr(token),
                                                   _ptr(confidence), _ptr(commit), _stream()))

    def denoise_step(self, layers, kvs, req: Request, x0, anchor_idx, k, y_a, y_b, block_rows, n_blk, final_norm_g,
                     w_lm, vocab, threshold, token, confidence, commit) -> int:
        """layers: list of LayerWeights, kvs: list of KV.  Returns the device address of the last layer's output."""
        n = len(layers)
        la = (LayerWeights * n)(*layers)
        ka = (KV * n)(*kvs)
        last = C.c_void_p()
        self._check(self.lib.acache_denoise_step(self.h, n, la, ka, C.byref(req), _ptr(x0), _ptr(anchor_idx), k,
                                                 _ptr(y_a), _ptr(y_b), C.byref(last), _ptr(block_rows), n_blk,
                                                 _ptr(final_norm_g), _ptr(w_lm), vocab, float(threshold), _ptr(token),
                                                 _ptr(confidence), _ptr(commit), _stream()))
        return last.value

    def denoise_step_shared(self, layers, kvs, req: Request, x0, anchor_idx, k, k_new, v_new, y_a, y_b, block_rows, n_blk,
                            final_norm_g, w_lm, vocab, threshold, token, confidence, commit) -> int:
        """k_new, v_new: lists of per-layer tensors [B, K+e, Hkv, d].  Returns the device address of the last output."""
        n = len(layers)
        la = (LayerWeights * n)(*layers)
        ka = (KV * n)(*kvs)
        kn = (C.c_void_p * n)(*[_ptr(t) for t in k_new])
        vn = (C.c_void_p * n)(*[_ptr(t) for t in v_new])
        last = C.c_void_p()
        self._check(self.lib.acache_denoise_step_shared(self.h, n, la, ka, C.byref(req), _ptr(x0), _ptr(anchor_idx), k, kn, vn,
                                                        _ptr(y_a), _ptr(y_b), C.byref(last), _ptr(block_rows), n_blk,
                                                        _ptr(final_norm_g), _ptr(w_lm), vocab, float(threshold), _ptr(token),
                                                        _ptr(confidence), _ptr(commit), _stream()))
        return last.value

    def layer_step_shared(self, w: LayerWeights, req: Request, kv: KV, x, x_is_compact, ratio, flags, scores, anchor_idx,
                          k_new, v_new, y):
        """The fused layer-step over storage that is not written (the cache may be shared by the batch)."""
        self._check(self.lib.acache_layer_step_shared(self.h, C.byref(w), C.byref(req), C.byref(kv), _ptr(x), int(x_is_compact),
                                                      float(ratio), int(flags), _ptr(scores), _ptr(anchor_idx), _ptr(k_new),
                                                      _ptr(v_new), _ptr(y), _stream()))

    def recompute_rows_shared(self, w: LayerWeights, req_rows: Request, req_slots: Request, kv: KV, x, x_is_compact,
                              anchor_idx, k, slot_rows, k_slots, v_slots, y):
        self._check(self.lib.acache_recompute_rows_shared(self.h, C.byref(w), C.byref(req_rows), C.byref(req_slots),
                                                          C.byref(kv), _ptr(x), int(x_is_compact), _ptr(anchor_idx), k,
                                                          _ptr(slot_rows), _ptr(k_slots), _ptr(v_slots), _ptr(y), _stream()))

    def decode_step_shared(self, layers, kvs, req_rows: Request, req_slots: Request, x0, anchor_idx, k, slot_rows, k_slots,
                           v_slots, y_a, y_b, block_rows, n_blk, final_norm_g, w_lm, vocab, threshold, token, confidence,
                           commit) -> int:
        """k_slots, v_slots: lists of per-layer tensors [B, K+e, Hkv, d] as the refresh pass left them."""
        n = len(layers)
        la = (LayerWeights * n)(*layers)
        ka = (KV * n)(*kvs)
        kn = (C.c_void_p * n)(*[_ptr(t) for t in k_slots])
        vn = (C.c_void_p * n)(*[_ptr(t) for t in v_slots])
        last = C.c_void_p()
        self._check(self.lib.acache_decode_step_shared(self.h, n, la, ka, C.byref(req_rows), C.byref(req_slots), _ptr(x0),
                                                       _ptr(anchor_idx), k, _ptr(slot_rows), kn, vn, _ptr(y_a), _ptr(y_b),
                                                       C.byref(last), _ptr(block_rows), n_blk, _ptr(final_norm_g), _ptr(w_lm),
                                                       vocab, float(threshold), _ptr(token), _ptr(confidence), _ptr(commit),
                                                       _stream()))
        return last.value

    def generate_block_shared(self, layers, kvs, req_refresh: Request, req_decode: Request, embed, anchor_idx, k, k_slots,
                              v_slots, y_a, y_b, block_rows_refresh, block_rows_decode, n_blk, final_norm_g, w_lm, vocab,
                              threshold, mask_id, max_steps, token, confidence, commit, remaining) -> int:
        """acache_generate_block over shared affix storage; returns the number of model passes run."""
        n = len(layers)
        la = (LayerWeights * n)(*layers)
        ka = (KV * n)(*kvs)
        kn = (C.c_void_p * n)(*[_ptr(t) for t in k_slots])
        vn = (C.c_void_p * n)(*[_ptr(t) for t in v_slots])
        steps = C.c_int32(0)
        self._check(self.lib.acache_generate_block_shared(self.h, n, la, ka, C.byref(req_refresh), C.byref(req_decode),
                                                          _ptr(embed), _ptr(anchor_idx), k, kn, vn, _ptr(y_a), _ptr(y_b),
                                                          _ptr(block_rows_refresh), _ptr(block_rows_decode), n_blk,
                                                          _ptr(final_norm_g), _ptr(w_lm), vocab, float(threshold),
                                                          int(mask_id), int(max_steps), _ptr(token), _ptr(confidence),
                                                          _ptr(commit), _ptr(remaining), C.byref(steps), _stream()))
        return int(steps.value)

    def probe_select(self, layers, kvs, req: Request, x0, ratio, flags, y_a, y_b, scores, anchor_idx):
        n = len(layers)
        la = (LayerWeights * n)(*layers)
        ka = (KV * n)(*kvs)
        self._check(self.lib.acache_probe_select(self.h, n, la, ka, C.byref(req), _ptr(x0), float(ratio), int(flags),
                                                 _ptr(y_a), _ptr(y_b), _ptr(scores), _ptr(anchor_idx), _stream()))

    def commit_update(self, token_ids, ctx_len, block_pos, batch, n_blk, token, confidence, mask_id, threshold, remaining):
        self._check(self.lib.acache_commit_update(self.h, _ptr(token_ids), ctx_len, _ptr(block_pos), batch, n_blk,
                                                  _ptr(token), _ptr(confidence), int(mask_id), float(threshold),
                                                  _ptr(remaining), _stream()))

    def generate_block(self, layers, kvs, req_refresh: Request, req_decode: Request, embed, anchor_idx, k, y_a, y_b,
                       block_rows_refresh, block_rows_decode, n_blk, final_norm_g, w_lm, vocab, threshold, mask_id,
                       max_steps, token, confidence, commit, remaining) -> int:
        """Returns the number of model passes run (synchronises the stream once per pass)."""
        n = len(layers)
        la = (LayerWeights * n)(*layers)
        ka = (KV * n)(*kvs)
        steps = C.c_int32(0)
        self._check(self.lib.acache_generate_block(self.h, n, la, ka, C.byref(req_refresh), C.byref(req_decode), _ptr(embed),
                                                   _ptr(anchor_idx), k, _ptr(y_a), _ptr(y_b), _ptr(block_rows_refresh),
                                                   _ptr(block_rows_decode), n_blk, _ptr(final_norm_g), _ptr(w_lm), vocab,
                                                   float(threshold), int(mask_id), int(max_steps), _ptr(token),
                                                   _ptr(confidence), _ptr(commit), _ptr(remaining), C.byref(steps),
                                                   _stream()))
        return int(steps.value)

    def layer_step_host(self, w: LayerWeights, req: Request, kv: KV, x_host, ratio, flags, scores_host,
                        anchor_idx_host, y_host):
        self._check(self.lib.acache_layer_step_host(self.h, C.byref(w), C.byref(req), C.byref(kv), _ptr(x_host),
                                                    float(ratio), int(flags), _ptr(scores_host),
                                                    _ptr(anchor_idx_host), _ptr(y_host), _stream()))


    def host_x_in_place(self, x_host) -> bool:
        """True when layer_step_host reads this x in place (page-locked memory) instead of staging a copy."""
        return bool(self.lib.acache_host_x_in_place(_ptr(x_host)))


# --------------------------------------------------------------------------
# host <-> device conveniences for bf16-bit numpy arrays
# --------------------------------------------------------------------------
def to_device_bf16(bits, device="cuda:0"):
    """numpy uint16 bf16 bits -> torch.bfloat16 CUDA tensor (same bytes)."""
    import numpy as np
    import torch
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


def to_host_bits(t):
    """torch.bfloat16 tensor -> numpy uint16 bf16 bits."""
    import numpy as np
    import torch
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)
