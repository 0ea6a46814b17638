"""Thin ctypes binding over libpt.so (see include/pt.h for the contract of every call).

Only argument marshalling lives here; every step of the forward pass runs in the library's
CUDA kernels.  PyTorch is used for device memory and streams: the ``Model`` helper owns the
torch tensors that back the packed weights, the KV pool and the workspace, and hands their
raw pointers to the C ABI.  Without the compiled library every call raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpt.so")

PT_OK = 0
STATUS = {0: "PT_OK", 1: "PT_ERR_INVALID_ARG", 2: "PT_ERR_BAD_CONFIG", 3: "PT_ERR_UNSUPPORTED",
          4: "PT_ERR_BUFFER_TOO_SMALL", 5: "PT_ERR_CACHE_FULL", 6: "PT_ERR_MISALIGNED", 7: "PT_ERR_CUDA",
          8: "PT_ERR_DEVICE_BOUNDS", 9: "PT_ERR_DEVICE_TIMEOUT", 10: "PT_ERR_STATE"}
PT_F32, PT_BF16 = 0, 1
PT_KV_MODEL, PT_KV_E4M3, PT_KV_E2M1 = 0, 1, 2
KIND = {"wq": 0, "wk": 1, "wv": 2, "wo": 3, "wg": 4, "wu": 5, "wd": 6, "g1": 7, "g2": 8, "wr": 9}


class PtError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class pt_config(C.Structure):
    _fields_ = [("T", C.c_int32), ("D", C.c_int32), ("L", C.c_int32), ("hidden", C.c_int32),
                ("heads", C.c_int32), ("kv_heads", C.c_int32), ("ffn", C.c_int32),
                ("rope_base", C.c_float), ("rms_eps", C.c_float), ("dtype", C.c_int32),
                ("sync_op", C.c_int32), ("max_pos", C.c_int32), ("flags", C.c_int32),
                ("experts", C.c_int32), ("top_k", C.c_int32)]


class pt_sampling(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("u", "temperature", "top_k", "top_p", "min_p", "prob")]


_P, _I32, _I64, _SZ = C.c_void_p, C.c_int32, C.c_int64, C.c_size_t
_PROTOS = {
    "pt_model_create": (_I32, [C.POINTER(pt_config), C.POINTER(_P)]),
    "pt_model_destroy": (None, [_P]),
    "pt_model_weight_bytes": (_I32, [_P, C.POINTER(_SZ)]),
    "pt_model_bind_weights": (_I32, [_P, _P, _SZ]),
    "pt_model_set_weight": (_I32, [_P, _I32, _I32, _I32, _P, _P]),
    "pt_model_set_expert_weight": (_I32, [_P, _I32, _I32, _I32, _I32, _P, _P]),
    "pt_sync_count": (_I32, [_P]),
    "pt_model_set_track_group": (_I32, [_P, _I32, _P, _P]),
    "pt_kv_cache_bytes": (_I32, [_P, _I32, _I32, C.POINTER(_SZ)]),
    "pt_kv_cache_alloc": (_I32, [_P, _I32, _I32, _P, _SZ, C.POINTER(_P)]),
    "pt_kv_cache_bytes_ex": (_I32, [_P, _I32, _I32, _I32, C.POINTER(_SZ)]),
    "pt_kv_cache_alloc_ex": (_I32, [_P, _I32, _I32, _I32, _P, _SZ, C.POINTER(_P)]),
    "pt_kv_scale_slot": (_I32, [_P, _I32, _I32, _I32, _I32, _I32, _I32, C.POINTER(_I64)]),
    "pt_workspace_bytes_ex": (_I32, [_P, _I64, _I32, _I32, _I32, _I64, C.POINTER(_SZ)]),
    "pt_kernel_kv_quant_e4m3": (_I32, [_P, _P, _P, _I64, _P, _P]),
    "pt_kv_cache_free": (None, [_P]),
    "pt_kv_set_free_list": (_I32, [_P, C.POINTER(_I32), _I32]),
    "pt_kv_seq_reserve": (_I32, [_P, _I32, _I32]),
    "pt_kv_seq_release": (_I32, [_P, _I32]),
    "pt_kv_seq_len": (_I32, [_P, _I32, C.POINTER(_I32)]),
    "pt_kv_seq_truncate": (_I32, [_P, _I32, _I32]),
    "pt_kv_block_table": (_I32, [_P, _I32, C.POINTER(_I32), _I32, C.POINTER(_I32)]),
    "pt_kv_slot": (_I32, [_P, _I32, _I32, _I32, _I32, _I32, _I32, C.POINTER(_I64)]),
    "pt_workspace_bytes": (_I32, [_P, _I64, _I32, _I32, C.POINTER(_SZ)]),
    "pt_prefill": (_I32, [_P, _P, _P, _I64, _I32, _I32, C.POINTER(_I32), _P, _P, _SZ, _P]),
    "pt_decode_step": (_I32, [_P, _P, _P, _I64, _I32, C.POINTER(_I32), _P, _P, _SZ, _P]),
    "pt_lm_bytes": (_I32, [_P, _I32, C.POINTER(_SZ)]),
    "pt_lm_bind": (_I32, [_P, _I32, _P, _SZ]),
    "pt_lm_set": (_I32, [_P, _I32, _P, _P]),
    "pt_embed": (_I32, [_P, _P, _I64, _P, _P]),
    "pt_lm_workspace_bytes": (_I32, [_P, _I64, C.POINTER(_SZ)]),
    "pt_lm_head": (_I32, [_P, _P, _I64, _I64, _P, _P, _P, _SZ, _P]),
    "pt_generate_workspace_bytes": (_I32, [_P, _I32, _I32, _I32, C.POINTER(_SZ)]),
    "pt_generate": (_I32, [_P, _P, _P, _I32, _I32, _I32, C.POINTER(_I32), _P, _P, _P, _SZ, _P]),
    "pt_kv_seq_fork": (_I32, [_P, _I32, _I32, _I32]),
    "pt_kv_free_pages": (_I32, [_P, C.POINTER(_I32)]),
    "pt_kv_page_refs": (_I32, [_P, _I32, C.POINTER(_I32)]),
    "pt_kv_compact": (_I32, [_P, C.POINTER(_I32), _P]),
    "pt_kv_move_pool": (_I32, [_P, _I32, _P, _SZ, _P]),
    "pt_call_context": (_I32, [_P, _I32, C.POINTER(_I32), C.POINTER(_I32), C.POINTER(_I64), C.POINTER(_I32)]),
    "pt_extend_workspace_bytes": (_I32, [_P, _I64, _I32, _I32, _I32, _I64, C.POINTER(_SZ)]),
    "pt_extend": (_I32, [_P, _P, _P, _I64, _I32, C.POINTER(_I32), C.POINTER(_I32), _P, _P, _SZ, _P]),
    "pt_sample": (_I32, [_P, _I32, _I64, _I64, _I32, _P, _P, _P, _P, _P, _P, _P, _P]),
    "pt_generate_sample": (_I32, [_P, _P, _P, _I32, _I32, _I32, C.POINTER(_I32), C.POINTER(pt_sampling), _P, _P, _P, _SZ, _P]),
    "pt_set_debug_tap": (_I32, [_P, _I32, _P]),
    "pt_device_status": (_I32, [_P, _P, C.POINTER(_I32), C.POINTER(_I32)]),
    "pt_profile_enable": (_I32, [_P, _I32]),
    "pt_profile_read": (_I32, [_P, C.POINTER(C.c_float), C.POINTER(_I64)]),
    "pt_launch_count": (_I64, []),
    "pt_kernel_gemm_bf16": (_I32, [_P, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _P, _P]),
    "pt_kernel_prefill_attn": (_I32, [_P, _P, _I64, _P, _I32, _P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _P, _I32, _P, _P]),
    "pt_kernel_decode_attn_scratch_bytes": (_I32, [_I32, _I32, _I32, _I32, C.POINTER(_SZ)]),
    "pt_kernel_decode_attn": (_I32, [_P, _P, _I64, _P, _I32, C.POINTER(_I32), _I32, _I32, _I32, _I32, _I32, _I32, _I32,
                                     _P, _P, _SZ, _P, _P]),
    "pt_kernel_decode_attn_static": (_I32, [_P, _P, _I64, _P, _I32, C.POINTER(_I32), _I32, _I32, _I32, _I32, _I32, _I32, _I32,
                                            _P, _P, _P]),
    "pt_kernel_decode_attn_e4m3": (_I32, [_P, _P, _I64, _P, _I64, _P, _I32, C.POINTER(_I32), _I32, _I32, _I32, _I32, _I32, _I32,
                                          _P, _I32, _P, _SZ, _P, _P]),
    "pt_kernel_chunk_attn_scratch_bytes": (_I32, [_I32, _I32, _I32, _I32, C.POINTER(_SZ)]),
    "pt_kernel_chunk_attn": (_I32, [_P, _P, _I64, _P, _I32, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _I32,
                                    _P, _I32, _P, _SZ, _P, _P]),
    "pt_kernel_kv_copy_pages": (_I32, [_P, _I32, _P, _I32, _I64, _I64, _P, _P, _I32, _P]),
    "pt_kernel_kv_write_e2m1": (_I32, [_P, _P, _I64, _I64, _I32, _I32, _I32, _I32, _I32, _I32, _P, _I64, _P, _P, _P, _P, _P]),
    "pt_kernel_kv_read_e2m1": (_I32, [_P, _I64, _P, _I32, _P, _I32, _I32, _I32, _I32, _I32, _I32, _P, _I64, _P, _I32, _I32, _I32, _P, _P]),
    "pt_kernel_attn_e2m1_scratch_bytes": (_I32, [_I32, _I32, _I32, _I32, C.POINTER(_SZ)]),
    "pt_kernel_attn_e2m1": (_I32, [_P, _P, _I64, _P, _I32, _P, _P, _I32, _I32, _I32, _I32, _I32, _I32, _I32, _I32,
                                   _P, _P, _SZ, _P, _P]),
    "pt_kernel_wait_selftest": (_I32, [_P, C.c_uint64, _P]),
    "pt_last_error": (C.c_char_p, []),
}
EXPORTS = tuple(_PROTOS)
_lib = None


def lib() -> C.CDLL:
    """Load libpt.so once; raise if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2602_07306_b200.build` "
                               "(there is no CPU fallback)")
        l = C.CDLL(LIB_PATH)
        for name, (res, args) in _PROTOS.items():
            f = getattr(l, name)
            f.restype, f.argtypes = res, args
        _lib = l
    return _lib


def check(code: int) -> None:
    if code != PT_OK:
        raise PtError(code, lib().pt_last_error().decode())


def _i32arr(a):
    a = np.ascontiguousarray(a, dtype=np.int32)
    return a, a.ctypes.data_as(C.POINTER(_I32))


def _grown(have, want):
    """Sizes (tokens, sequences, page size, cache format, context) of the workspace that serves `want` and what `have` served
    (None: nothing); `have` itself where it serves.  A context that grows does so by a quarter at least: a decoding loop
    raises it by a few tokens at a time."""
    if have is None:
        return want
    most = (max(want[0], have[0]), max(want[1], have[1]), min(want[2], have[2]), max(want[3], have[3]))
    if most == have[:4] and want[4] <= have[4]:
        return have
    return most + (have[4] if want[4] <= have[4] else max(want[4], have[4] + have[4] // 4),)


class Model:
    """A PT model with its packed weights on one CUDA device (torch owns the memory)."""

    def __init__(self, *, T, D, L, hidden, heads, kv_heads, ffn, dtype="bf16", rope_base=10000.0,
                 rms_eps=1e-6, sync_op="sum", max_pos=4096, simt=False, flags=0, experts=0, top_k=0, device="cuda:0"):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        self.cfg = pt_config(T, D, L, hidden, heads, kv_heads, ffn, rope_base, rms_eps,
                             PT_BF16 if dtype == "bf16" else PT_F32, 1 if sync_op == "mean" else 0,
                             max_pos, (1 if simt else 0) | int(flags), experts, top_k)
        self.dtype = dtype
        self.tdtype = torch.bfloat16 if dtype == "bf16" else torch.float32
        self.h = _P()
        check(lib().pt_model_create(C.byref(self.cfg), C.byref(self.h)))
        if not torch.cuda.is_available():
            raise RuntimeError("a CUDA device is required: there is no CPU path")
        n = _SZ()
        check(lib().pt_model_weight_bytes(self.h, C.byref(n)))
        self.weight_bytes = n.value
        with torch.cuda.device(self.device):
            self.wbuf = torch.empty(n.value, dtype=torch.uint8, device=self.device)
            check(lib().pt_model_bind_weights(self.h, self.wbuf.data_ptr(), n.value))
        self.ws = None
        self.ws_key = (0, 0, 0)
        self.ext_ws = self.gen_ws = self.ext_key = None     # of ragged calls, of the generate loop
        self._tap = None

    def close(self):
        if self.h:
            lib().pt_model_destroy(self.h)
            self.h = _P()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _stream(self):
        return self.torch.cuda.current_stream(self.device).cuda_stream

    def _borrow(self, ws):
        """(address, bytes) of a workspace for a call on the current stream.  A larger one may replace it before that stream
        has come to the call: its memory must not be handed out meanwhile."""
        ws.record_stream(self.torch.cuda.current_stream(self.device))
        return ws.data_ptr(), ws.numel()

    def set_weight(self, t: int, l: int, kind: str, w) -> None:
        """w: numpy float32 array or torch tensor, [out, in] (gains: [hidden])."""
        torch = self.torch
        if isinstance(w, np.ndarray):
            w = torch.from_numpy(np.ascontiguousarray(w))
        want = torch.float32 if kind in ("g1", "g2", "wr") else self.tdtype
        w = w.to(device=self.device, dtype=want).contiguous()
        with torch.cuda.device(self.device):
            if self.cfg.experts and kind in ("wg", "wu", "wd"):       # PT-MoE: [experts, ...], one call per expert
                for e in range(self.cfg.experts):
                    check(lib().pt_model_set_expert_weight(self.h, t, l, e, KIND[kind], w[e].data_ptr(), self._stream()))
            else:
                check(lib().pt_model_set_weight(self.h, t, l, KIND[kind], w.data_ptr(), self._stream()))
            torch.cuda.current_stream().synchronize()      # w may be freed after return

    def load(self, source) -> None:
        """source.get(t, l) -> dict kind -> float32 numpy array."""
        for l in range(self.cfg.L):
            for t in range(self.cfg.T):
                for k, w in source.get(t, l).items():
                    self.set_weight(t, l, k, w)

    def init_random(self, seed: int = 0, std: float = 0.02) -> None:
        """Weights N(0, std), gains 1, drawn on the device (for timing runs)."""
        torch = self.torch
        c = self.cfg
        dh = c.hidden // c.heads
        g = torch.Generator(device=self.device).manual_seed(seed)
        shapes = {"wq": (c.heads * dh, c.hidden), "wk": (c.kv_heads * dh, c.hidden), "wv": (c.kv_heads * dh, c.hidden),
                  "wo": (c.hidden, c.heads * dh), "wg": (c.ffn, c.hidden), "wu": (c.ffn, c.hidden), "wd": (c.hidden, c.ffn)}
        ones = torch.ones(c.hidden, dtype=torch.float32, device=self.device)
        with torch.cuda.device(self.device):
            for l in range(c.L):
                for t in range(c.T):
                    for k, shp in shapes.items():
                        for e in range(c.experts if c.experts and k in ("wg", "wu", "wd") else 1):
                            w = (torch.randn(shp, generator=g, device=self.device, dtype=torch.float32) * std).to(self.tdtype)
                            if c.experts and k in ("wg", "wu", "wd"):
                                check(lib().pt_model_set_expert_weight(self.h, t, l, e, KIND[k], w.data_ptr(), self._stream()))
                            else:
                                check(lib().pt_model_set_weight(self.h, t, l, KIND[k], w.data_ptr(), self._stream()))
                    if c.experts:
                        wr = torch.randn((c.experts, c.hidden), generator=g, device=self.device, dtype=torch.float32) * std
                        check(lib().pt_model_set_weight(self.h, t, l, KIND["wr"], wr.data_ptr(), self._stream()))
                    for k in ("g1", "g2"):
                        check(lib().pt_model_set_weight(self.h, t, l, KIND[k], ones.data_ptr(), self._stream()))
            torch.cuda.synchronize()

    def set_track_group(self, world_tracks: int, allreduce) -> None:
        """This model holds cfg.T of `world_tracks` tracks; `allreduce(t)` must sum the fp32 CUDA tensor t in
        place over all ranks on the current stream (e.g. torch.distributed.all_reduce).  None clears it."""
        if allreduce is None:
            check(lib().pt_model_set_track_group(self.h, 0, None, None))
            self._ar_cb = None
            return
        torch = self.torch

        def hook(user, ptr, count, stream):
            try:
                # the buffer lies in the workspace of the call that runs: one of the model's three
                for ws in (self.ws, self.ext_ws, self.gen_ws):
                    off = -1 if ws is None else ptr - ws.data_ptr()
                    if 0 <= off and off + 4 * count <= ws.numel():
                        break
                else:
                    raise RuntimeError("buffer outside the workspaces")
                allreduce(ws[off:off + 4 * count].view(torch.float32))
                return 0
            except Exception as e:      # never let an exception cross the C boundary
                self._ar_error = e
                return 1
        self._ar_cb = C.CFUNCTYPE(_I32, _P, _P, _I64, _P)(hook)
        check(lib().pt_model_set_track_group(self.h, world_tracks, C.cast(self._ar_cb, _P), None))

    def sync_count(self) -> int:
        return lib().pt_sync_count(self.h)

    def new_cache(self, num_pages: int, page_size: int = 16, free_order=None, kv_dtype: str = "model") -> "Cache":
        """kv_dtype "model" keeps K and V in the model dtype, "e4m3" stores 8-bit codes and one scale per vector, "e2m1" 4-bit
        codes and one scale for 32 values (PT_KV_E2M1 in include/pt.h)."""
        return Cache(self, num_pages, page_size, free_order, kv_dtype=kv_dtype)

    def workspace(self, tokens: int, batch: int, page_size: int, kv_dtype: int = PT_KV_MODEL, context: int = 0):
        """Workspace for calls of up to `tokens` tokens / `batch` sequences; with an E4M3 or E2M1 cache `context` bounds the
        keys of which a prefill call makes a copy (Cache.call_context)."""
        key = self.ws_key + (0, 0) if len(self.ws_key) == 3 else self.ws_key
        if (self.ws is None or tokens > key[0] or batch > key[1] or page_size < key[2] or kv_dtype > key[3] or context > key[4]):
            tokens, batch, context = max(tokens, key[0]), max(batch, key[1]), max(context, key[4])
            kv_dtype = max(kv_dtype, key[3])
            page_size = min(page_size, key[2]) if key[2] else page_size
            n = _SZ()
            check(lib().pt_workspace_bytes_ex(self.h, tokens, batch, page_size, kv_dtype, context, C.byref(n)))
            self.ws = None
            self.ws = self.torch.empty(n.value, dtype=self.torch.uint8, device=self.device)
            self.ws_key = (tokens, batch, page_size, kv_dtype, context)
        return self.ws

    def set_tap(self, layer: int | None, tokens: int = 0):
        """layer None: off; -1: all layers.  Returns the tap tensor [nl, 2, T, tokens, hidden]."""
        torch = self.torch
        if layer is None:
            check(lib().pt_set_debug_tap(self.h, 0, None))
            self._tap = None
            return None
        nl = self.cfg.L if layer == -1 else 1
        self._tap = torch.zeros((nl, 2, self.cfg.T, tokens, self.cfg.hidden), dtype=torch.float32, device=self.device)
        check(lib().pt_set_debug_tap(self.h, layer, self._tap.data_ptr()))
        return self._tap

    def prefill(self, cache: "Cache", x, seq_ids, out=None):
        """x: torch tensor [T, B, S, H] (or [1, B, S, H] = shared input) in the model dtype."""
        torch = self.torch
        assert x.is_cuda and x.dtype == self.tdtype and x.is_contiguous()
        Tn, B, S, H = x.shape
        stride = 0 if Tn == 1 and self.cfg.T > 1 else B * S * H
        if out is None:
            out = torch.empty((B, S, H), dtype=torch.float32, device=self.device)
        ids, pids = _i32arr(seq_ids)
        assert len(ids) == B
        ctx = cache.call_context(np.full(B, S, np.int32), ids) if cache.kv_dtype != PT_KV_MODEL else 0
        ws = self.workspace(B * S, B, cache.page_size, cache.kv_dtype, ctx)
        with torch.cuda.device(self.device):
            check(lib().pt_prefill(self.h, cache.h, x.data_ptr(), stride, B, S, pids, out.data_ptr(),
                                   *self._borrow(ws), self._stream()))
        return out

    def extend(self, cache: "Cache", x, n_tokens, seq_ids, out=None):
        """A ragged batch: n_tokens[b] new tokens of sequence seq_ids[b], rows packed sequence by sequence.
        x: torch tensor [T, M, H] (or [1, M, H] = shared input) in the model dtype, M = sum(n_tokens) -> fp32 [M, H]."""
        torch = self.torch
        assert x.is_cuda and x.dtype == self.tdtype and x.is_contiguous()
        Tn, M, H = x.shape
        assert Tn in (1, self.cfg.T) and H == self.cfg.hidden
        stride = 0 if Tn == 1 and self.cfg.T > 1 else M * H
        cnt, pcnt = _i32arr(n_tokens)
        ids, pids = _i32arr(seq_ids)
        assert len(ids) == len(cnt) and int(cnt.sum()) == M
        if out is None:
            out = torch.empty((M, H), dtype=torch.float32, device=self.device)
        assert out.is_cuda and out.dtype == torch.float32 and out.is_contiguous() and out.numel() == M * H
        ctx = cache.call_context(cnt, ids) if cache.kv_dtype != PT_KV_MODEL else 0
        key = _grown(self.ext_key, (M, len(ids), cache.page_size, cache.kv_dtype, ctx))
        if self.ext_ws is None or key != self.ext_key:
            n = _SZ()
            check(lib().pt_extend_workspace_bytes(self.h, *key, C.byref(n)))
            self.ext_ws = None
            self.ext_ws = torch.empty(n.value, dtype=torch.uint8, device=self.device)
            self.ext_key = key
        with torch.cuda.device(self.device):
            check(lib().pt_extend(self.h, cache.h, x.data_ptr(), stride, len(ids), pcnt, pids, out.data_ptr(),
                                  *self._borrow(self.ext_ws), self._stream()))
        return out

    def decode_step(self, cache: "Cache", x, seq_ids, out=None):
        """x: torch tensor [T, B, H] (or [1, B, H]) in the model dtype -> fp32 [B, H]."""
        torch = self.torch
        assert x.is_cuda and x.dtype == self.tdtype and x.is_contiguous()
        Tn, B, H = x.shape
        stride = 0 if Tn == 1 and self.cfg.T > 1 else B * H
        if out is None:
            out = torch.empty((B, H), dtype=torch.float32, device=self.device)
        ws = self.workspace(B, B, cache.page_size, cache.kv_dtype, 0)
        ids, pids = _i32arr(seq_ids)
        assert len(ids) == B
        with torch.cuda.device(self.device):
            check(lib().pt_decode_step(self.h, cache.h, x.data_ptr(), stride, B, pids, out.data_ptr(),
                                       *self._borrow(ws), self._stream()))
        return out

    # ---- ends of the model -------------------------------------------------------------------
    def load_lm(self, table, head, gain) -> None:
        """table, head: [vocab, hidden]; gain: [hidden] (numpy or torch); stored in the model dtype / fp32."""
        torch = self.torch
        as_t = lambda a: torch.from_numpy(np.ascontiguousarray(a)) if isinstance(a, np.ndarray) else a
        table, head, gain = as_t(table), as_t(head), as_t(gain)
        self.vocab = table.shape[0]
        n = _SZ()
        check(lib().pt_lm_bytes(self.h, self.vocab, C.byref(n)))
        with torch.cuda.device(self.device):
            self.lm_buf = torch.empty(n.value, dtype=torch.uint8, device=self.device)
            check(lib().pt_lm_bind(self.h, self.vocab, self.lm_buf.data_ptr(), n.value))
            for kind, w, dt in ((0, table, self.tdtype), (1, head, self.tdtype), (2, gain, torch.float32)):
                w = w.to(device=self.device, dtype=dt).contiguous()
                check(lib().pt_lm_set(self.h, kind, w.data_ptr(), self._stream()))
                torch.cuda.current_stream().synchronize()

    def embed(self, tokens):
        """tokens: int32 CUDA tensor of any shape -> [..., hidden] in the model dtype."""
        torch = self.torch
        assert tokens.is_cuda and tokens.dtype == torch.int32 and tokens.is_contiguous()
        x = torch.empty(tuple(tokens.shape) + (self.cfg.hidden,), dtype=self.tdtype, device=self.device)
        with torch.cuda.device(self.device):
            check(lib().pt_embed(self.h, tokens.data_ptr(), tokens.numel(), x.data_ptr(), self._stream()))
        return x

    def lm_head(self, h, want_tokens=True):
        """h: fp32 CUDA [n, hidden] (contiguous) -> (logits fp32 [n, vocab], greedy tokens int32 [n] or None)."""
        torch = self.torch
        assert h.is_cuda and h.dtype == torch.float32 and h.is_contiguous() and h.dim() == 2
        n = h.shape[0]
        logits = torch.empty((n, self.vocab), dtype=torch.float32, device=self.device)
        tok = torch.empty(n, dtype=torch.int32, device=self.device) if want_tokens else None
        nb = _SZ()
        check(lib().pt_lm_workspace_bytes(self.h, n, C.byref(nb)))
        ws = torch.empty(nb.value, dtype=torch.uint8, device=self.device)
        with torch.cuda.device(self.device):
            check(lib().pt_lm_head(self.h, h.data_ptr(), h.shape[1], n, logits.data_ptr(), tok.data_ptr() if want_tokens else None,
                                   ws.data_ptr(), ws.numel(), self._stream()))
        return logits, tok

    def generate(self, cache: "Cache", prompt, n_new: int, seq_ids, want_logits=False, *, u=None, temperature=None,
                 top_k=None, top_p=None, min_p=None, prob=None):
        """prompt: int32 CUDA [B, S] -> (tokens int32 [B, n_new], logits fp32 [B, n_new, vocab] or None).
        Greedy, or with u (fp32 CUDA [n_new, B], uniform in [0, 1)) sampled: temperature, top_k, top_p, min_p are CUDA
        tensors [B] as for sample(); prob (fp32 CUDA [B, n_new]) receives the tokens' probabilities."""
        torch = self.torch
        assert prompt.is_cuda and prompt.dtype == torch.int32 and prompt.is_contiguous()
        B, S = prompt.shape
        out = torch.empty((B, n_new), dtype=torch.int32, device=self.device)
        logits = torch.empty((B, n_new, self.vocab), dtype=torch.float32, device=self.device) if want_logits else None
        nb = _SZ()
        check(lib().pt_generate_workspace_bytes(self.h, B, S, cache.page_size, C.byref(nb)))
        if self.gen_ws is None or self.gen_ws.numel() < nb.value:
            self.gen_ws = None
            self.gen_ws = torch.empty(nb.value, dtype=torch.uint8, device=self.device)
        ids, pids = _i32arr(seq_ids)
        if u is not None:
            index = prompt.get_device()
            _sampling_args(index, (n_new, B), u=u)
            _sampling_args(index, (B,), temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p)
            _sampling_args(index, (B, n_new), prob=prob)
            sp = pt_sampling(*(None if a is None else a.data_ptr() for a in (u, temperature, top_k, top_p, min_p, prob)))
            with torch.cuda.device(self.device):
                check(lib().pt_generate_sample(self.h, cache.h, prompt.data_ptr(), B, S, n_new, pids, C.byref(sp), out.data_ptr(),
                                               logits.data_ptr() if want_logits else None, *self._borrow(self.gen_ws), self._stream()))
            return out, logits
        assert temperature is None and top_k is None and top_p is None and min_p is None and prob is None, "sampling needs u"
        with torch.cuda.device(self.device):
            check(lib().pt_generate(self.h, cache.h, prompt.data_ptr(), B, S, n_new, pids, out.data_ptr(),
                                    logits.data_ptr() if want_logits else None, *self._borrow(self.gen_ws), self._stream()))
        return out, logits

    PROF_NAMES = ("attention", "gemm_qkv", "gemm_out", "gemm_gate_up", "gemm_down", "gemm_down_sync", "other")

    def profile(self, on, only=None) -> None:
        """on False / True: no launch / every launch bracketed with events; only=("attention", ...) brackets
        the launches of those categories alone."""
        code = int(bool(on))
        if on and only:
            code = sum(2 << self.PROF_NAMES.index(n) for n in only)
        check(lib().pt_profile_enable(self.h, code))

    def profile_read(self) -> dict:
        """Device milliseconds and launches per kernel category since the last read."""
        ms = (C.c_float * 7)()
        n = (_I64 * 7)()
        with self.torch.cuda.device(self.device):
            check(lib().pt_profile_read(self.h, ms, n))
        return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(self.PROF_NAMES)}

    def device_status(self) -> tuple[int, int]:
        code, detail = _I32(), _I32()
        with self.torch.cuda.device(self.device):
            check(lib().pt_device_status(self.h, self._stream(), C.byref(code), C.byref(detail)))
        return code.value, detail.value


class Cache:
    """Paged KV cache: torch owns the pool, the library's host allocator owns the page tables."""

    def __init__(self, model: Model, num_pages: int, page_size: int = 16, free_order=None, fill=None, kv_dtype: str = "model"):
        torch = model.torch
        self.model, self.num_pages, self.page_size = model, num_pages, page_size
        self.kv_dtype = {"model": PT_KV_MODEL, "e4m3": PT_KV_E4M3, "e2m1": PT_KV_E2M1}[kv_dtype]
        n = _SZ()
        check(lib().pt_kv_cache_bytes_ex(model.h, num_pages, page_size, self.kv_dtype, C.byref(n)))
        self.bytes = n.value
        self.pool, self.codes, self.scales = self._new_pool(num_pages, n.value)
        self.h = _P()
        check(lib().pt_kv_cache_alloc_ex(model.h, num_pages, page_size, self.kv_dtype, self.pool.data_ptr(), n.value, C.byref(self.h)))
        if free_order is not None:
            a, p = _i32arr(free_order)
            check(lib().pt_kv_set_free_list(self.h, p, len(a)))

    def _new_pool(self, num_pages: int, nbytes: int):
        """(pool, codes, scales) of a pool in the cache's format; codes and scales are None in the model dtype.  E2M1: codes
        has the blocks [T, L, pages, kv_heads, page / 16, bytes], scales is None."""
        model, torch = self.model, self.model.torch
        if self.kv_dtype == PT_KV_E2M1:
            c = model.cfg
            pool = torch.empty(nbytes, dtype=torch.uint8, device=model.device)
            return pool, pool.view(c.T, c.L, num_pages, c.kv_heads, self.page_size // 16, 17 * (c.hidden // c.heads)), None
        if self.kv_dtype != PT_KV_E4M3:
            return torch.empty(nbytes // (2 if model.dtype == "bf16" else 4), dtype=model.tdtype, device=model.device), None, None
        # one byte buffer: the codes, then the fp32 scales (views)
        pool = torch.empty(nbytes, dtype=torch.uint8, device=model.device)
        c = model.cfg
        vecs = c.T * c.L * num_pages * 2 * c.kv_heads * self.page_size
        return pool, pool[: vecs * (c.hidden // c.heads)], pool[nbytes - vecs * 4:].view(torch.float32)

    def close(self):
        if self.h:
            lib().pt_kv_cache_free(self.h)
            self.h = _P()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def reserve(self, seq: int, new_len: int):
        check(lib().pt_kv_seq_reserve(self.h, seq, new_len))

    def release(self, seq: int):
        check(lib().pt_kv_seq_release(self.h, seq))

    def call_context(self, n_tokens, seq_ids) -> int:
        """Keys of the bf16 copy that Model.prefill or Model.extend would make for n_tokens[b] new tokens of sequence seq_ids[b]; 0: none."""
        cnt, pcnt = _i32arr(n_tokens)
        ids, pids = _i32arr(seq_ids)
        assert len(ids) == len(cnt)
        v = _I64()
        check(lib().pt_call_context(self.h, len(ids), pcnt, pids, C.byref(v), None))
        return v.value

    def truncate(self, seq: int, n: int):
        check(lib().pt_kv_seq_truncate(self.h, seq, n))

    def fork(self, src: int, dst: int, length: int | None = None):
        """A new sequence dst that shares the first `length` (default: all) tokens of src; pages are copied on write."""
        check(lib().pt_kv_seq_fork(self.h, src, dst, self.length(src) if length is None else length))

    def free_pages(self) -> int:
        v = _I32()
        check(lib().pt_kv_free_pages(self.h, C.byref(v)))
        return v.value

    def page_refs(self, page: int) -> int:
        v = _I32()
        check(lib().pt_kv_page_refs(self.h, page, C.byref(v)))
        return v.value

    def compact(self) -> int:
        """Move every page in use to the front of the pool (current stream); returns the pages copied."""
        v = _I32()
        with self.model.torch.cuda.device(self.model.device):
            check(lib().pt_kv_compact(self.h, C.byref(v), self.model._stream()))
        return v.value

    def resize(self, num_pages: int) -> None:
        """Continue in a new pool of num_pages pages, those in use at its front (current stream)."""
        n = _SZ()
        check(lib().pt_kv_cache_bytes_ex(self.model.h, num_pages, self.page_size, self.kv_dtype, C.byref(n)))
        pool, codes, scales = self._new_pool(num_pages, n.value)
        with self.model.torch.cuda.device(self.model.device):
            check(lib().pt_kv_move_pool(self.h, num_pages, pool.data_ptr(), n.value, self.model._stream()))
            self.pool.record_stream(self.model.torch.cuda.current_stream(self.model.device))
        self.pool, self.codes, self.scales = pool, codes, scales
        self.num_pages, self.bytes = num_pages, n.value

    def length(self, seq: int) -> int:
        v = _I32()
        check(lib().pt_kv_seq_len(self.h, seq, C.byref(v)))
        return v.value

    def block_table(self, seq: int) -> list[int]:
        n = _I32()
        check(lib().pt_kv_block_table(self.h, seq, None, 0, C.byref(n)))
        buf = (_I32 * max(1, n.value))()
        check(lib().pt_kv_block_table(self.h, seq, buf, n.value, C.byref(n)))
        return list(buf[: n.value])

    def slot(self, t: int, l: int, seq: int, pos: int, kv: int, head: int) -> int:
        v = _I64()
        check(lib().pt_kv_slot(self.h, t, l, seq, pos, kv, head, C.byref(v)))
        return v.value

    def scale_slot(self, t: int, l: int, seq: int, pos: int, kv: int, head: int) -> int:
        """E4M3 caches: byte offset inside the pool of the fp32 scale of the vector `slot` addresses (E2M1: of the scales of its
        16 tokens)."""
        v = _I64()
        check(lib().pt_kv_scale_slot(self.h, t, l, seq, pos, kv, head, C.byref(v)))
        return v.value

    def dequantized(self):
        """E4M3 and E2M1 caches: code * scale of the whole pool as a float32 CUDA tensor [T, L, pages, 2, kv_heads, page, dh]."""
        torch = self.model.torch
        c = self.model.cfg
        dh = c.hidden // c.heads
        if self.kv_dtype == PT_KV_E2M1:
            dev = dict(dtype=torch.int32, device=self.model.device)
            pages = torch.arange(self.num_pages, **dev)[:, None]
            out = torch.empty((c.T * c.L, self.num_pages, 2, c.kv_heads, self.page_size, dh), dtype=torch.bfloat16, device=self.model.device)
            kernel_kv_read_e2m1(self.codes.flatten(0, 1), pages, torch.full((self.num_pages,), self.page_size, **dev), out, pages,
                                nkv=c.kv_heads, dh=dh, ps=self.page_size)
            return out.float().view((c.T, c.L) + out.shape[1:])
        shape = (c.T, c.L, self.num_pages, 2, c.kv_heads, self.page_size)
        codes = self.codes.view(torch.float8_e4m3fn).to(torch.float32).view(shape + (dh,))
        return codes * self.scales.view(shape + (1,))


def _raw_stream(index: int) -> int:
    """Handle of torch's current stream of a device."""
    import torch
    return torch._C._cuda_getCurrentRawStream(index)


def _call(index: int, fn, *args) -> None:
    """fn(*args, current stream) with device `index` current, checked.  The device is switched only where it has to be: a
    guard costs as much as a small call."""
    import torch
    if torch._C._cuda_getDevice() == index:
        check(fn(*args, _raw_stream(index)))
    else:
        with torch.cuda.device(index):
            check(fn(*args, _raw_stream(index)))


_status_blocks = {}


def _capturing(index: int) -> bool:
    """Whether torch's current stream of a device is being captured into a graph."""
    import torch
    if torch._C._cuda_getDevice() == index:
        return torch.cuda.is_current_stream_capturing()
    with torch.cuda.device(index):
        return torch.cuda.is_current_stream_capturing()


def _new_status(index: int):
    """A zeroed int32[16] of its own on the device, for a call on its current stream: cut from a block that one fill zeroes
    for 256 calls of that stream (inside a capture, whose memory belongs to the graph: from none)."""
    import torch
    if _capturing(index):
        return torch.zeros(16, dtype=torch.int32, device=index)
    key = (index, _raw_stream(index))
    try:
        return _status_blocks[key].pop()            # one step: another thread may take the last
    except (KeyError, IndexError):
        left = list(torch.zeros((256, 16), dtype=torch.int32, device=index).unbind(0))
        mine = left.pop()
        _status_blocks[key] = left
        return mine


def _sampling_args(index, shape, **arrays):
    import torch
    for name, a in arrays.items():
        if a is None:
            continue
        want = torch.int32 if name == "top_k" or name == "token" else torch.float32
        if a.dtype is not want or a.shape != shape or a.get_device() != index or not a.is_contiguous():
            raise ValueError(f"{name}: a contiguous {want} tensor of shape {shape} on CUDA device {index} is wanted")


def sample(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, *, out=None, prob=None):
    """One token per row of logits (fp32 or bf16 CUDA [n, vocab], rows may be strided) from the random numbers u (fp32 [n]):
    temperature, then top_k, top_p and min_p, each a CUDA tensor [n] or None; see pt_sample in include/pt.h.
    Returns (tokens int32 [n], probabilities fp32 [n]) in `out` and `prob` where given."""
    import torch
    dt = logits.dtype
    if not logits.is_cuda or logits.dim() != 2 or (dt is not torch.float32 and dt is not torch.bfloat16) or logits.stride(1) != 1:
        raise ValueError("logits: an fp32 or bf16 CUDA tensor [n, vocab] with contiguous rows is wanted")
    n, vocab = logits.shape
    index = logits.get_device()
    if out is None:
        out = torch.empty(n, dtype=torch.int32, device=logits.device)
    if prob is None:
        prob = torch.empty(n, dtype=torch.float32, device=logits.device)
    if u is None:
        raise ValueError("u: random numbers are wanted")
    _sampling_args(index, (n,), u=u, temperature=temperature, top_k=top_k, top_p=top_p, min_p=min_p, token=out, prob=prob)
    _call(index, lib().pt_sample, logits.data_ptr(), PT_F32 if dt is torch.float32 else PT_BF16, logits.stride(0) if n > 1 else vocab, n, vocab,
          u.data_ptr(), None if temperature is None else temperature.data_ptr(), None if top_k is None else top_k.data_ptr(),
          None if top_p is None else top_p.data_ptr(), None if min_p is None else min_p.data_ptr(), out.data_ptr(), prob.data_ptr())
    return out, prob


def _page_ids(ids):
    """ids as a contiguous int32 array; numbers that are not whole or do not fit are refused, not cut."""
    if type(ids) is np.ndarray and ids.dtype == np.int32 and ids.flags.c_contiguous:
        return ids
    a = np.asarray(ids)
    b = np.ascontiguousarray(a, np.int32)
    if a.dtype != np.int32 and not np.array_equal(a, b):
        raise ValueError("page numbers: whole numbers of 32 bits are wanted")
    return b


def _host_ptr(a):
    """A call's argument for the data of a contiguous int32 array (which the caller keeps)."""
    try:
        return C.byref(_I32.from_buffer(a))      # a third of the time of a.ctypes
    except (TypeError, ValueError, BufferError):  # read-only, or empty
        return a.ctypes.data


def _plane_args(index, a, b):
    """Arguments of a page copy from pool a to pool b in front of its pairs, checked as far as shapes go."""
    sa, sb = a.shape, b.shape
    if a.get_device() != index or not a.is_contiguous() or index < 0 or b is not a and \
            (not b.is_contiguous() or a.dtype != b.dtype or b.get_device() != index or sa[:2] != sb[:2] or sa[3:] != sb[3:]):
        raise ValueError("pools: contiguous CUDA tensors [T, L, pages, ...] that differ in their pages alone are wanted")
    slabs = sa[0] * sa[1]
    if a.numel() == 0 or sb[2] == 0:
        raise ValueError("pools: at least one page is wanted")
    return a.data_ptr(), sa[2], b.data_ptr(), sb[2], slabs, a.nbytes // (slabs * sa[2])


def kernel_kv_copy_pages(pool, src, dst, *, scales=None, out=None, out_scales=None):
    """Pages src[i] of pool [T, L, pages, ...] (any type) to its pages dst[i] in every (track, layer) slab; `scales`
    [T, L, pages, ...] likewise.  src, dst: host integers.  `out`, `out_scales`: another pool to copy to (with scales: both).
    A call that is refused has copied nothing."""
    src, dst = _page_ids(src), _page_ids(dst)
    if src.ndim != 1 or src.shape != dst.shape:
        raise ValueError("src and dst: two lists of the same length are wanted")
    index, ps, pd, n, fn = pool.get_device(), _host_ptr(src), _host_ptr(dst), len(src), lib().pt_kernel_kv_copy_pages
    codes = _plane_args(index, pool, pool if out is None else out)
    if scales is None:
        if out_scales is not None:
            raise ValueError("out_scales without scales")
        _call(index, fn, *codes, ps, pd, n)
        return
    if (out is None) != (out_scales is None):
        raise ValueError("scales: out and out_scales are wanted together")
    fine = _plane_args(index, scales, scales if out_scales is None else out_scales)
    if tuple(scales.shape[:2]) != tuple(pool.shape[:2]) or fine[1] != codes[1] or fine[3] != codes[3]:
        raise ValueError("scales: the tracks, layers and pages of the pool are wanted")
    _call(index, fn, *fine, None, None, 0)          # without pairs: checks alignment, sizes and overlap, and launches nothing
    _call(index, fn, *codes, ps, pd, n)
    _call(index, fn, *fine, ps, pd, n)


def chunk_attn_scratch(T: int, B: int, nq: int, dh: int, device="cuda:0"):
    """Scratch buffer for kernel_chunk_attn calls of up to B sequences (one per stream that calls at the same time)."""
    import torch
    n = _SZ()
    check(lib().pt_kernel_chunk_attn_scratch_bytes(T, B, nq, dh, C.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=device)


def kernel_chunk_attn(q, pool_l, block_table, q_len, kv_len, *, nq, nkv, dh, ps, out=None, scratch=None, status=None, impl=None):
    """q bf16 [T, M, nq*dh], rows packed by sequence; pool_l bf16 [T, pages, 2, nkv, ps, dh]; block_table int32 [B, maxp],
    q_len, kv_len int32 [B] (all CUDA); impl 0 = tcgen05 kernel, 1 = plain kernel, None = the first where it serves the shape.
    Returns (out bf16 [T, M, nq*dh], status int32[16])."""
    import torch
    T, M, width = q.shape
    B, maxp = block_table.shape
    pages = pool_l.shape[1]
    index = q.get_device()
    i32, bf16 = torch.int32, torch.bfloat16
    assert q.is_cuda and q.is_contiguous() and block_table.is_contiguous() and q_len.is_contiguous() and kv_len.is_contiguous()
    assert q.dtype is bf16 and pool_l.dtype is bf16 and block_table.dtype is i32 and q_len.dtype is i32 and kv_len.dtype is i32
    assert width == nq * dh and pool_l.shape == (T, pages, 2, nkv, ps, dh) and q_len.numel() == kv_len.numel() == B
    assert pool_l.stride()[1:] == (2 * nkv * ps * dh, nkv * ps * dh, ps * dh, dh, 1) or pool_l[0].is_contiguous()
    assert index == pool_l.get_device() == block_table.get_device() == q_len.get_device() == kv_len.get_device()
    if out is None:
        out = torch.empty_like(q)
    if scratch is None:
        scratch = chunk_attn_scratch(T, B, nq, dh, q.device)
    if status is None:
        status = _new_status(index)
    assert out.get_device() == index and out.dtype is bf16 and out.shape == q.shape and out.is_contiguous()
    assert scratch.get_device() == index and status.get_device() == index and status.dtype is i32 and status.numel() >= 16
    assert scratch.is_contiguous() and status.is_contiguous()
    if impl is None:
        impl = 0 if dh in (64, 128) and ps % 16 == 0 else 1
    _call(index, lib().pt_kernel_chunk_attn, q.data_ptr(), pool_l.data_ptr(), pool_l.stride(0), block_table.data_ptr(), maxp,
          q_len.data_ptr(), kv_len.data_ptr(), T, B, M, nq, nkv, dh, ps, pages, out.data_ptr(), impl,
          scratch.data_ptr(), scratch.numel() * scratch.element_size(), status.data_ptr())
    return out, status


def _kv4_pool(torch, pool_l, T, nkv, dh, ps, index):
    """Checks one layer of an E2M1 pool: uint8 [T, pages, nkv, ps // 16, 17 * dh], contiguous but for the track stride.
    Returns (pages, bytes between tracks).  (torch is handed on: an import in every helper costs as much as its checks.)"""
    shape = pool_l.shape
    if len(shape) == 5:
        tracks, pages, heads, blocks, size = shape
        if pool_l.is_contiguous():
            stride = pages * heads * blocks * size
        else:
            stride, *rest = pool_l.stride()
            if rest != [heads * blocks * size, blocks * size, size, 1]:
                tracks = -1
        if tracks == T and heads == nkv and blocks * 16 == ps and size == 17 * dh and pages and pool_l.dtype is torch.uint8 and pool_l.get_device() == index:
            return pages, stride if T > 1 else 0
    raise ValueError(f"pool: a uint8 CUDA tensor [{T}, pages, {nkv}, {ps // 16}, {17 * dh}] with contiguous tracks on the call's device is wanted")


def _kv4_int(name, a, shape, dtype, index):
    if a.shape != shape or a.dtype is not dtype or a.get_device() != index or not a.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor of shape {tuple(shape)} on CUDA device {index} is wanted")
    return a.data_ptr()


def _kv4_table(torch, name, a, rows, index):
    shape = a.shape
    if len(shape) != 2 or shape[0] != rows or a.dtype is not torch.int32 or a.get_device() != index or not a.is_contiguous():
        raise ValueError(f"{name}: a contiguous int32 tensor [{rows}, columns] on CUDA device {index} is wanted")
    return a.data_ptr(), shape[1]


def _kv4_status(torch, status, index):
    if status is None:
        return _new_status(index)
    if status.dtype is not torch.int32 or status.numel() < 16 or not status.is_contiguous() or status.get_device() != index:
        raise ValueError(f"status: a contiguous int32 tensor of 16 on CUDA device {index} is wanted")
    return status


def kernel_kv_write_e2m1(k, v, pool_l, slots, *, nkv, dh, ps, k_out=None, v_out=None, status=None):
    """K and V of new tokens (bf16 CUDA [T, M, nkv*dh], rows and tracks may be strided, both alike) into the 4-bit pages pool_l
    (uint8 [T, pages, nkv, ps/16, 17*dh]): row r to token slots[r] % ps of page slots[r] // ps (int64 CUDA [M]; negative:
    not cached).  k_out, v_out (bf16 [T, M, nkv*dh]) receive the values that the cache then returns.  Returns status int32[16]."""
    import torch
    bf16, index, shape, stride = torch.bfloat16, k.get_device(), k.shape, k.stride()
    if len(shape) != 3 or shape[2] != nkv * dh or stride[2] != 1 or k.dtype is not bf16 or index < 0 \
            or v.dtype is not bf16 or v.shape != shape or v.stride() != stride or v.get_device() != index:
        raise ValueError("k, v: bf16 CUDA tensors [T, M, nkv*dh] of the same strides with contiguous values are wanted")
    T, M, _ = shape
    pages, pstride = _kv4_pool(torch, pool_l, T, nkv, dh, ps, index)
    at = _kv4_int("slots", slots, (M,), torch.int64, index)
    ko = vo = None
    if k_out is not None or v_out is not None:
        for a in (k_out, v_out):
            if a is None or a.dtype is not bf16 or a.shape != shape or not a.is_contiguous() or a.get_device() != index:
                raise ValueError("k_out, v_out: both or neither, contiguous bf16 CUDA tensors of k's shape")
        ko, vo = k_out.data_ptr(), v_out.data_ptr()
    status = _kv4_status(torch, status, index)
    if M:
        _call(index, lib().pt_kernel_kv_write_e2m1, k.data_ptr(), v.data_ptr(), stride[0] if T > 1 else 0, stride[1] if M > 1 else 0, T, M, nkv, dh, ps,
              pages, pool_l.data_ptr(), pstride, at, ko, vo, status.data_ptr())
    return status


def kernel_kv_read_e2m1(pool_l, block_table, kv_len, out, out_table, *, nkv, dh, ps, status=None):
    """The first kv_len[b] cached tokens of every sequence from 4-bit pages (pool_l as for kernel_kv_write_e2m1, block_table
    int32 [B, maxp], kv_len int32 [B], all CUDA) into bf16 pages out [T, pages, 2, nkv, out_ps, dh] at out_table int32
    [B, out_maxp].  Returns (out, status int32[16])."""
    import torch
    index, shape = pool_l.get_device(), out.shape
    if len(shape) != 6 or out.dtype is not torch.bfloat16 or out.get_device() != index or index < 0:
        raise ValueError("out: a bf16 CUDA tensor [T, pages, 2, nkv, out_ps, dh] on the pool's device is wanted")
    T, opages, two, heads, ops, width = shape
    if out.is_contiguous():
        ostride = 2 * opages * heads * ops * width
    else:
        ostride, *rest = out.stride()
        if rest != [2 * heads * ops * width, heads * ops * width, ops * width, width, 1]:
            two = 0
    if two != 2 or heads != nkv or width != dh or not T or not opages:
        raise ValueError("out: a bf16 CUDA tensor [T, pages, 2, nkv, out_ps, dh] with contiguous tracks is wanted")
    pages, pstride = _kv4_pool(torch, pool_l, T, nkv, dh, ps, index)
    B = kv_len.numel()
    lens = _kv4_int("kv_len", kv_len, (B,), torch.int32, index)
    bt, maxp = _kv4_table(torch, "block_table", block_table, B, index)
    obt, omaxp = _kv4_table(torch, "out_table", out_table, B, index)
    status = _kv4_status(torch, status, index)
    if B:
        _call(index, lib().pt_kernel_kv_read_e2m1, pool_l.data_ptr(), pstride, bt, maxp, lens, T, B, nkv, dh, ps, pages, out.data_ptr(),
              ostride if T > 1 else 0, obt, omaxp, ops, opages, status.data_ptr())
    return out, status


def attn_e2m1_scratch(T: int, nq: int, nkv: int, dh: int, device="cuda:0"):
    """Scratch buffer for kernel_attn_e2m1 calls (one per stream that calls at the same time)."""
    import torch
    n = _SZ()
    check(lib().pt_kernel_attn_e2m1_scratch_bytes(T, nq, nkv, dh, C.byref(n)))
    return torch.empty(n.value, dtype=torch.uint8, device=device)


def kernel_attn_e2m1(q, pool_l, block_table, kv_len, q_len=None, *, nq, nkv, dh, ps, out=None, scratch=None, status=None):
    """Attention straight from 4-bit pages: q bf16 [T, M, nq*dh], rows packed by sequence; pool_l uint8 [T, pages, nkv, ps/16,
    17*dh]; block_table int32 [B, maxp], kv_len int32 [B], q_len int32 [B] or None (one new token each), all CUDA.
    Returns (out bf16 [T, M, nq*dh], status int32[16])."""
    import torch
    bf16, index, shape = torch.bfloat16, q.get_device(), q.shape
    if len(shape) != 3 or shape[2] != nq * dh or q.dtype is not bf16 or not q.is_contiguous() or index < 0:
        raise ValueError("q: a contiguous bf16 CUDA tensor [T, M, nq*dh] is wanted")
    T, M, _ = shape
    pages, pstride = _kv4_pool(torch, pool_l, T, nkv, dh, ps, index)
    B = kv_len.numel()
    lens = _kv4_int("kv_len", kv_len, (B,), torch.int32, index)
    news = None if q_len is None else _kv4_int("q_len", q_len, (B,), torch.int32, index)
    bt, maxp = _kv4_table(torch, "block_table", block_table, B, index)
    if out is None:
        out = torch.empty_like(q)
    elif out.dtype is not bf16 or out.shape != shape or not out.is_contiguous() or out.get_device() != index:
        raise ValueError("out: a contiguous bf16 CUDA tensor of q's shape is wanted, apart from q")
    if scratch is None:
        scratch = attn_e2m1_scratch(T, nq, nkv, dh, q.device)
    elif scratch.get_device() != index or not scratch.is_contiguous():
        raise ValueError("scratch: a contiguous tensor on the call's device is wanted")
    status = _kv4_status(torch, status, index)
    if M:
        _call(index, lib().pt_kernel_attn_e2m1, q.data_ptr(), pool_l.data_ptr(), pstride, bt, maxp, news, lens, T, B, M, nq, nkv, dh, ps, pages,
              out.data_ptr(), scratch.data_ptr(), scratch.nbytes, status.data_ptr())
    return out, status


def kernel_gemm_bf16(a, w, bn: int = 0, fold_tracks: bool = False):
    """a [T, M, K], w [T, N, K] bf16 CUDA tensors -> fp32 [T, M, N] ([1, M, N] when folding tracks)."""
    import torch
    T, M, K = a.shape
    N = w.shape[1]
    assert a.is_contiguous() and w.is_contiguous() and a.dtype == w.dtype == torch.bfloat16
    c = torch.empty((1 if fold_tracks else T, M, N), dtype=torch.float32, device=a.device)
    status = torch.zeros(16, dtype=torch.int32, device=a.device)
    with torch.cuda.device(a.device):
        check(lib().pt_kernel_gemm_bf16(a.data_ptr(), w.data_ptr(), c.data_ptr(), T, M, N, K, bn, int(fold_tracks),
                                        status.data_ptr(), torch.cuda.current_stream().cuda_stream))
    return c, status


def kernel_kv_quant_e4m3(src):
    """src: bf16 CUDA tensor [n, 128] -> (codes uint8 [n, 128], scales fp32 [n], status int32[16])."""
    import torch
    assert src.is_cuda and src.dtype == torch.bfloat16 and src.is_contiguous() and src.shape[1] == 128
    n = src.shape[0]
    codes = torch.empty((n, 128), dtype=torch.uint8, device=src.device)
    scales = torch.empty(n, dtype=torch.float32, device=src.device)
    status = torch.zeros(16, dtype=torch.int32, device=src.device)
    with torch.cuda.device(src.device):
        check(lib().pt_kernel_kv_quant_e4m3(src.data_ptr(), codes.data_ptr(), scales.data_ptr(), n, status.data_ptr(),
                                            torch.cuda.current_stream().cuda_stream))
    return codes, scales, status


def kernel_wait_selftest(limit_ns: int, device="cuda:0"):
    """Run the library's bounded wait on a barrier nothing arrives at; returns the status block (int32[16], CUDA)."""
    import torch
    status = torch.zeros(16, dtype=torch.int32, device=device)
    with torch.cuda.device(status.device):
        check(lib().pt_kernel_wait_selftest(status.data_ptr(), int(limit_ns), torch.cuda.current_stream().cuda_stream))
    return status


def kernel_decode_attn(q, pool_l, block_table, kv_len, *, nq, nkv, dh, ps, scratch=None):
    """q bf16 [T, B, nq*dh]; pool_l bf16 [T, pages, 2, nkv, ps, dh]; block_table int32 [B, maxp] (CUDA);
    kv_len: host ints [B].  Returns (out bf16 [T, B, nq*dh], status int32[16])."""
    import torch
    T, B, _ = q.shape
    pages = pool_l.shape[1]
    assert q.is_contiguous() and pool_l.is_contiguous() and block_table.is_contiguous()
    assert q.dtype == pool_l.dtype == torch.bfloat16 and block_table.dtype == torch.int32
    out = torch.empty_like(q)
    status = torch.zeros(16, dtype=torch.int32, device=q.device)
    n = _SZ()
    check(lib().pt_kernel_decode_attn_scratch_bytes(T, B, nq, dh, C.byref(n)))
    if scratch is None:
        scratch = torch.empty(n.value, dtype=torch.uint8, device=q.device)
    lens, plens = _i32arr(kv_len)
    with torch.cuda.device(q.device):
        check(lib().pt_kernel_decode_attn(q.data_ptr(), pool_l.data_ptr(), pool_l.stride(0), block_table.data_ptr(),
                                          block_table.shape[1], plens, T, B, nq, nkv, dh, ps, pages, out.data_ptr(),
                                          scratch.data_ptr(), scratch.numel(), status.data_ptr(),
                                          torch.cuda.current_stream().cuda_stream))
    return out, status


def kernel_decode_attn_e4m3(q, codes_l, scales_l, block_table, kv_len, *, nq, nkv, ps, impl=0):
    """q bf16 [T, B, nq*128]; codes_l uint8 [T, pages, 2, nkv, ps, 128]; scales_l fp32 [T, pages, 2, nkv, ps];
    block_table int32 [B, maxp] (CUDA); kv_len: host ints [B]; impl 0 = tcgen05 kernel, 1 = mma.sync kernel.
    Returns (out bf16 [T, B, nq*128], status int32[16])."""
    import torch
    T, B, _ = q.shape
    pages = codes_l.shape[1]
    assert q.is_contiguous() and codes_l.is_contiguous() and scales_l.is_contiguous() and block_table.is_contiguous()
    assert q.dtype == torch.bfloat16 and codes_l.dtype == torch.uint8 and scales_l.dtype == torch.float32
    assert block_table.dtype == torch.int32 and tuple(scales_l.shape) == tuple(codes_l.shape[:-1])
    out = torch.empty_like(q)
    status = torch.zeros(16, dtype=torch.int32, device=q.device)
    n = _SZ()
    check(lib().pt_kernel_decode_attn_scratch_bytes(T, B, nq, 128, C.byref(n)))
    scratch = torch.empty(n.value, dtype=torch.uint8, device=q.device)
    lens, plens = _i32arr(kv_len)
    with torch.cuda.device(q.device):
        check(lib().pt_kernel_decode_attn_e4m3(q.data_ptr(), codes_l.data_ptr(), codes_l.stride(0), scales_l.data_ptr(),
                                               scales_l.stride(0), block_table.data_ptr(), block_table.shape[1], plens,
                                               T, B, nq, nkv, ps, pages, out.data_ptr(), impl, scratch.data_ptr(),
                                               scratch.numel(), status.data_ptr(), torch.cuda.current_stream().cuda_stream))
    return out, status


def kernel_prefill_attn(q, pool_l, block_table, kv_len, *, S, nq, nkv, dh, ps, impl=0):
    """q bf16 [T, B*S, nq*dh]; pool_l bf16 [T, pages, 2, nkv, ps, dh]; block_table int32 [B, maxp] and kv_len
    int32 [B] on the device (keys cached per sequence, the S new ones included).
    Returns (out bf16 [T, B*S, nq*dh], status int32[16])."""
    import torch
    T, M, _ = q.shape
    B = M // S
    assert q.is_contiguous() and pool_l.is_contiguous() and block_table.is_contiguous() and kv_len.is_cuda
    assert q.dtype == pool_l.dtype == torch.bfloat16 and block_table.dtype == kv_len.dtype == torch.int32
    out = torch.empty_like(q)
    status = torch.zeros(16, dtype=torch.int32, device=q.device)
    with torch.cuda.device(q.device):
        check(lib().pt_kernel_prefill_attn(q.data_ptr(), pool_l.data_ptr(), pool_l.stride(0), block_table.data_ptr(),
                                           block_table.shape[1], kv_len.data_ptr(), T, B, S, nq, nkv, dh, ps, pool_l.shape[1],
                                           out.data_ptr(), impl, status.data_ptr(), torch.cuda.current_stream().cuda_stream))
    return out, status


def kernel_decode_attn_static(q, pool_l, block_table, kv_len, *, nq, nkv, dh, ps, out=None, status=None):
    """pt_kernel_decode_attn for callers that may not allocate device memory: the scratch is an
    8 MiB array built into the library.  Pass preallocated ``out`` / ``status`` tensors to keep the
    call itself free of allocations; calls on one device must not overlap on the GPU."""
    import torch
    T, B, _ = q.shape
    if out is None:
        out = torch.empty_like(q)
    if status is None:
        status = torch.zeros(16, dtype=torch.int32, device=q.device)
    lens, plens = _i32arr(kv_len)
    with torch.cuda.device(q.device):
        check(lib().pt_kernel_decode_attn_static(q.data_ptr(), pool_l.data_ptr(), pool_l.stride(0), block_table.data_ptr(),
                                                 block_table.shape[1], plens, T, B, nq, nkv, dh, ps, pool_l.shape[1],
                                                 out.data_ptr(), status.data_ptr(), torch.cuda.current_stream().cuda_stream))
    return out, status
