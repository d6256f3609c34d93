"""ctypes binding of the C ABI declared in include/kvrebuild.h (argument marshalling only)."""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB = None

KV_OP_PREFILL, KV_OP_DECODE = 0, 1
KV_WIRE_BLOCK_MAJOR, KV_WIRE_LAYER_MAJOR = 0, 1

# every symbol include/kvrebuild.h declares
EXPORTS = [
    "kv_model_create", "kv_model_destroy", "kv_workspace_bytes", "kv_status_string", "kv_last_cuda_error",
    "kv_bytes_per_token", "kv_check_device_status", "kv_prefill_prefix", "kv_pack_blocks",
    "kv_unpack_assemble", "kv_decode_step", "kv_pack_blocks_batched", "kv_unpack_blocks_batched",
    "kv_op_gemm", "kv_gemm_plan", "kv_op_rmsnorm",
    "kv_op_attention_prefill", "kv_paged_attention_scratch_bytes", "kv_op_paged_attention", "kv_fill_pattern",
    "kv_profile_enable", "kv_profile_read", "kv_launch_count", "kv_op_paged_attention_noalloc", "kv_check_copy_status", "kv_op_gemv",
    "kv_window_evaluate", "kv_window_select", "kv_window_waste_bound", "kv_ewma", "kv_prefill_prefix_batched",
    "kv_selftest_bounded_wait", "kv_workspace_residual", "kv_cache_page_bytes", "kv_rope_create", "kv_rope_destroy",
    "kv_rope_frequencies", "kv_op_rope", "kv_op_cache_write", "kv_op_cache_read",
    "kv_paged_attention_batched_scratch_bytes", "kv_op_paged_attention_batched", "kv_op_cache_append", "kv_op_block_bounds",
    "kv_select_blocks_scratch_bytes", "kv_op_select_blocks", "kv_op_paged_attention_selected",
]

PROFILE_KINDS = ("embed", "rmsnorm", "gemm_qkv", "rope_store", "attention", "gemm_o", "gemm_gate_up", "gemm_down",
                 "lm_head", "pack", "unpack", "decode_gemv", "decode_attention", "decode_other")


class KVError(RuntimeError):
    def __init__(self, status: int, what: str = ""):
        self.status = status
        detail = ""
        if _LIB is not None:
            detail = _LIB.kv_status_string(status).decode()
            if status in (-13, -14):
                detail += " [" + _LIB.kv_last_cuda_error().decode() + "]"
        super().__init__(f"{what}: status {status} ({detail})")


class ModelDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("n_layers", "hidden", "n_q_heads", "n_kv_heads", "head_dim", "ffn", "vocab")] \
        + [("rope_base", C.c_float), ("rms_eps", C.c_float)]


class Weights(C.Structure):
    _fields_ = [("embed_dev", C.c_void_p), ("lm_head_dev", C.c_void_p), ("final_norm_dev", C.c_void_p)] + \
        [(n, C.POINTER(C.c_void_p)) for n in ("attn_norm_dev", "w_qkv_dev", "w_o_dev", "ffn_norm_dev",
                                              "w_gate_up_dev", "w_down_dev")]


class WindowInputs(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("k_curr", "r_p", "r_d", "goodput", "s_kv", "t0", "t_load", "alpha", "t_remain")]


class WindowEval(C.Structure):
    _fields_ = [(n, C.c_double) for n in ("t_w", "l_hist", "t_hist", "t_res", "t_sit", "t_early", "cost")]

    def as_dict(self):
        return {n: getattr(self, n) for n, _ in self._fields_}


class RopeDesc(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("rotary_dim", "layout", "scaling")] + \
        [(n, C.c_double) for n in ("base", "factor", "original_ctx", "low", "high", "gain")]


class CacheDesc(C.Structure):
    _fields_ = [("base_dev", C.c_void_p), ("layer_stride", C.c_int64), ("kv_stride", C.c_int64),
                ("block_stride", C.c_int64)] + \
        [(n, C.c_int32) for n in ("num_blocks", "block_size", "n_layers", "n_kv_heads", "head_dim", "elem_bytes")]


def lib_path() -> str:
    return os.path.join(_PKG, "libkvrebuild.so")


def load(build_if_missing: bool = True):
    """Loads libkvrebuild.so.  Raises if it is missing and cannot be built: there is no fallback path."""
    global _LIB
    if _LIB is not None:
        return _LIB
    path = lib_path()
    if not os.path.exists(path):
        if not build_if_missing:
            raise RuntimeError(f"{path} is missing: run __graft_entry__.build() (no CPU fallback exists)")
        from . import build as _build
        _build.build()
    lib = C.CDLL(path)
    i32, i64, vp = C.c_int32, C.c_int64, C.c_void_p
    pi32 = C.POINTER(C.c_int32)
    sig = {
        "kv_model_create": (i32, [C.POINTER(ModelDesc), C.POINTER(Weights), C.POINTER(vp)]),
        "kv_model_destroy": (i32, [vp]),
        "kv_workspace_bytes": (i64, [vp, i32, i32]),
        "kv_workspace_residual": (i32, [vp, i32, i32, C.POINTER(C.c_int64), C.POINTER(C.c_int64)]),
        "kv_status_string": (C.c_char_p, [i32]),
        "kv_last_cuda_error": (C.c_char_p, []),
        "kv_bytes_per_token": (i64, [i32, i32, i32, i32]),
        "kv_check_device_status": (i32, [vp, vp]),
        "kv_prefill_prefix": (i32, [vp, C.POINTER(CacheDesc), pi32, i32, i32, pi32, i32, vp, i64, vp, vp]),
        "kv_prefill_prefix_batched": (i32, [vp, C.POINTER(CacheDesc), i32, pi32, pi32, pi32, pi32, vp, i64, vp, vp]),
        "kv_pack_blocks": (i32, [C.POINTER(CacheDesc), pi32, i32, vp, i64, i32, vp]),
        "kv_unpack_assemble": (i32, [C.POINTER(CacheDesc), vp, i64, i32, pi32, pi32, i32, pi32, i32, i32,
                                     C.c_uint32, C.c_uint32, pi32, vp]),
        "kv_decode_step": (i32, [vp, C.POINTER(CacheDesc), i32, i32, pi32, i32, vp, i64, vp, vp]),
        "kv_pack_blocks_batched": (i32, [C.POINTER(CacheDesc), i32, pi32, pi32, C.POINTER(vp), i32, vp]),
        "kv_unpack_blocks_batched": (i32, [C.POINTER(CacheDesc), i32, pi32, pi32, C.POINTER(vp), i32, vp]),
        "kv_op_gemm": (i32, [vp, i32, vp, i32, i32, i32, i32, vp, vp, vp, vp]),
        "kv_gemm_plan": (i32, [i32, i32, i32, i32, pi32, pi32]),
        "kv_op_rmsnorm": (i32, [vp, vp, i32, i32, C.c_float, vp, vp]),
        "kv_op_attention_prefill": (i32, [vp, i32, i32, i32, i32, i32, C.POINTER(CacheDesc), i32, vp, vp, vp, vp]),
        "kv_paged_attention_scratch_bytes": (i64, [i32, i32, i32]),
        "kv_op_paged_attention": (i32, [vp, i32, C.POINTER(CacheDesc), i32, vp, i32, vp, i64, vp, vp]),
        "kv_fill_pattern": (i32, [vp, i64, C.c_uint64, i64, vp]),
        "kv_op_paged_attention_noalloc": (i32, [vp, i32, C.POINTER(CacheDesc), i32, vp, i32, vp, vp]),
        "kv_check_copy_status": (i32, [vp]),
        "kv_selftest_bounded_wait": (i32, [vp, i32, vp]),
        "kv_window_evaluate": (i32, [C.POINTER(WindowInputs), C.c_double, C.POINTER(WindowEval)]),
        "kv_window_select": (i32, [C.POINTER(WindowInputs), C.c_double, C.c_double, C.POINTER(WindowEval),
                                   C.POINTER(C.c_int32)]),
        "kv_window_waste_bound": (C.c_double, [C.c_double, C.c_double, C.c_double]),
        "kv_ewma": (C.c_double, [C.c_double, C.c_double, C.c_double]),
        "kv_op_gemv": (i32, [vp, vp, i32, i32, i32, vp, C.c_float, vp, vp]),
        "kv_profile_enable": (i32, [i32]),
        "kv_profile_read": (i32, [C.POINTER(C.c_float), C.POINTER(C.c_int64), i32]),
        "kv_launch_count": (i64, []),
        "kv_cache_page_bytes": (i64, [i32, i32, i32, i32]),
        "kv_rope_create": (i32, [C.POINTER(RopeDesc), C.POINTER(vp)]),
        "kv_rope_destroy": (i32, [vp]),
        "kv_rope_frequencies": (i32, [vp, C.POINTER(C.c_double), i32]),
        "kv_op_rope": (i32, [vp, vp, i64, i64, i32, i32, i32, i32, vp, i32, vp, i64, i64, vp]),
        "kv_op_cache_write": (i32, [C.POINTER(CacheDesc), i32, vp, i64, i64, vp, i64, i64, i32, i32, vp, vp]),
        "kv_op_cache_read": (i32, [C.POINTER(CacheDesc), i32, vp, i32, vp, i64, i64, vp, i64, i64, i32, vp]),
        "kv_paged_attention_batched_scratch_bytes": (i64, [i32, i32, i32, i32, i32]),
        "kv_op_paged_attention_batched": (i32, [vp, i64, i32, i32, i32, C.POINTER(CacheDesc), i32, vp, i64, vp, i32,
                                                C.c_float, vp, i64, vp, i64, vp, vp]),
        "kv_op_cache_append": (i32, [vp, C.POINTER(CacheDesc), i32, vp, i64, i64, i32, vp, i64, i64, vp, i64, i64, vp, i64, i64,
                                     i32, i32, vp, vp, vp]),
        "kv_op_block_bounds": (i32, [C.POINTER(CacheDesc), i32, vp, vp, i32, vp, vp, vp]),
        "kv_select_blocks_scratch_bytes": (i64, [i32, i32, i32, i32]),
        "kv_op_select_blocks": (i32, [vp, i64, i32, i32, i32, i32, i32, vp, vp, i32, i32, vp, i64, vp, i32, i32, i32, i32, vp, i64,
                                      vp, vp, vp]),
        "kv_op_paged_attention_selected": (i32, [vp, i64, i32, i32, i32, C.POINTER(CacheDesc), i32, vp, i64, i64, vp, i32,
                                                 C.c_float, vp, i64, vp, i64, vp, vp]),
    }
    for name, (res, args) in sig.items():
        fn = getattr(lib, name)
        fn.restype, fn.argtypes = res, args
    _LIB = lib
    return lib


def status_string(status: int) -> str:
    return load().kv_status_string(status).decode()


def _check(status: int, what: str) -> None:
    if status != 0:
        raise KVError(status, what)


def _i32(a):
    arr = np.ascontiguousarray(a, dtype=np.int32)
    return arr, arr.ctypes.data_as(C.POINTER(C.c_int32))


def _stream(stream) -> int:
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    return getattr(stream, "cuda_stream", stream)


def _ptr(t) -> int:
    return 0 if t is None else (t.data_ptr() if hasattr(t, "data_ptr") else int(t))


KV_ELEM_E2M1 = -2


def _elem(elem_bytes) -> int:
    """kv_cache_desc.elem_bytes of 2 (bf16), 1 (e4m3) or 0.5 (e2m1)."""
    return KV_ELEM_E2M1 if elem_bytes == 0.5 else elem_bytes


class PagedCache:
    """A paged KV cache in device memory plus its descriptor: a torch tensor of bf16 bit patterns (elem_bytes 2, int16),
    of e4m3 pages with their scale bytes (elem_bytes 1, uint8) or of e2m1 pages with their scales (elem_bytes 0.5, uint8).

    layout "layer_major": [L][2][num_blocks][page]; "block_major": [num_blocks][L][2][page].  `data` gives the cache
    memory that is there already (contiguous, of exactly the pool's size) instead of allocating it.
    """

    def __init__(self, shape, num_blocks: int, layout: str = "layer_major", device="cuda", fill=None,
                 elem_bytes: float = 2, data=None):
        import torch
        self.n_layers, self.n_kv_heads, self.head_dim = shape.n_layers, shape.n_kv_heads, shape.head_dim
        self.block_size, self.num_blocks, self.layout = shape.block_size, num_blocks, layout
        self.elem_bytes = elem_bytes
        if elem_bytes not in (0.5, 1, 2):
            raise ValueError(f"elem_bytes {elem_bytes}: 2 (bf16), 1 (e4m3) or 0.5 (e2m1)")
        if elem_bytes == 0.5:
            self.page_bytes = self.n_kv_heads * (-(-self.block_size * (self.head_dim // 2 + self.head_dim // 16 + 1) // 16) * 16)
        else:
            self.page_bytes = self.block_size * self.n_kv_heads * self.head_dim * elem_bytes
        if elem_bytes == 1:
            self.page_bytes += -(-self.block_size * self.n_kv_heads // 16) * 16
        item = 2 if elem_bytes == 2 else 1
        page_elems = self.page_bytes // item
        if layout == "layer_major":
            dims = (self.n_layers, 2, num_blocks, page_elems)
            strides = (2 * num_blocks * self.page_bytes, num_blocks * self.page_bytes, self.page_bytes)
        elif layout == "block_major":
            dims = (num_blocks, self.n_layers, 2, page_elems)
            strides = (2 * self.page_bytes, self.page_bytes, 2 * self.n_layers * self.page_bytes)
        else:
            raise ValueError(layout)
        if data is None:
            self.data = torch.empty(dims, dtype=torch.int16 if elem_bytes == 2 else torch.uint8, device=device)
        elif not data.is_contiguous() or data.numel() * data.element_size() != int(np.prod(dims)) * item:
            raise ValueError("data: a contiguous tensor of the pool's size is wanted")
        else:
            self.data = data.view(torch.int16 if elem_bytes == 2 else torch.uint8).view(dims)
        if fill is not None:
            self.data.fill_(fill)
        self.desc = CacheDesc(self.data.data_ptr(), strides[0], strides[1], strides[2], num_blocks, self.block_size,
                              self.n_layers, self.n_kv_heads, self.head_dim, _elem(elem_bytes))
        self._desc_ref = C.byref(self.desc)

    def pages(self, block_ids):
        """int16 (bf16) or uint8 (e4m3, e2m1) tensor [len(ids), L, 2, page] of the given blocks (torch indexing; test helper)."""
        import torch
        idx = torch.as_tensor(np.asarray(block_ids, dtype=np.int64), device=self.data.device)
        if self.layout == "layer_major":
            return self.data[:, :, idx].permute(2, 0, 1, 3)
        return self.data[idx]

    def as_logical_numpy(self) -> np.ndarray:
        """uint16 array [L, 2, num_blocks, Bs, Hkv, d] of a bf16 cache on the host."""
        if self.elem_bytes != 2:
            raise ValueError("as_logical_numpy: bf16 caches only (kv_op_cache_read decodes the others)")
        d = self.data if self.layout == "layer_major" else self.data.permute(1, 2, 0, 3)
        return d.contiguous().cpu().numpy().view(np.uint16).reshape(
            self.n_layers, 2, self.num_blocks, self.block_size, self.n_kv_heads, self.head_dim)


class Model:
    """Uploads bf16 weights to the device and creates the library handle."""

    def __init__(self, shape, head: dict | None = None, layers=None, device="cuda"):
        import torch
        self.shape = shape
        self._lib = load()
        self._keep = []
        self.device = device

        def up(arr):
            if isinstance(arr, torch.Tensor):
                t = arr.to(device=device, dtype=torch.bfloat16).contiguous()
            else:
                t = torch.from_numpy(np.ascontiguousarray(arr, dtype=np.float32)).to(device).to(torch.bfloat16)
            self._keep.append(t)
            return t.data_ptr()

        names = ("attn_norm", "w_qkv", "w_o", "ffn_norm", "w_gate_up", "w_down")
        arrays = {n: (C.c_void_p * shape.n_layers)() for n in names}
        for l in range(shape.n_layers):
            w = layers(l)
            for n in names:
                arrays[n][l] = up(w[n])
        self._arrays = arrays
        self._w = Weights(up(head["embed"]), up(head["lm_head"]), up(head["final_norm"]),
                          *[C.cast(arrays[n], C.POINTER(C.c_void_p)) for n in names])
        self._desc = ModelDesc(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim,
                               shape.ffn, shape.vocab, shape.rope_base, shape.rms_eps)
        handle = C.c_void_p()
        _check(self._lib.kv_model_create(C.byref(self._desc), C.byref(self._w), C.byref(handle)), "kv_model_create")
        self.handle = handle
        self._ws = {}

    def workspace(self, op: int, max_tokens: int):
        """A cached, caller-side (torch) workspace tensor large enough for `op` over max_tokens."""
        import torch
        need = kv_workspace_bytes(self, op, max_tokens)
        cur = self._ws.get(op)
        if cur is None or cur.numel() - ((-cur.data_ptr()) % 1024) < need:
            cur = torch.empty(need + 1024, dtype=torch.uint8, device=self.device)
            self._ws[op] = cur
        off = (-cur.data_ptr()) % 1024            # the library wants a 1 KiB-aligned base
        return cur[off:off + need]

    def __del__(self):
        try:
            if getattr(self, "handle", None):
                self._lib.kv_model_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


def kv_bytes_per_token(n_layers, n_kv_heads, head_dim, elem_bytes=2) -> int:
    return load().kv_bytes_per_token(n_layers, n_kv_heads, head_dim, _elem(elem_bytes))


def kv_cache_page_bytes(block_size: int, n_kv_heads: int, head_dim: int, elem_bytes: float) -> int:
    r = load().kv_cache_page_bytes(block_size, n_kv_heads, head_dim, _elem(elem_bytes))
    if r < 0:
        raise KVError(int(r), "kv_cache_page_bytes")
    return int(r)


def kv_workspace_bytes(model: Model, op: int, max_tokens: int) -> int:
    r = load().kv_workspace_bytes(model.handle, op, max_tokens)
    if r < 0:
        raise KVError(int(r), "kv_workspace_bytes")
    return int(r)


def kv_workspace_residual(model: Model, op: int, max_tokens: int):
    """(offset, bytes) of the fp32 residual stream inside a workspace sized for (op, max_tokens)."""
    off, nbytes = C.c_int64(), C.c_int64()
    _check(load().kv_workspace_residual(model.handle, op, max_tokens, C.byref(off), C.byref(nbytes)), "kv_workspace_residual")
    return int(off.value), int(nbytes.value)


def kv_check_device_status(workspace, stream=None) -> None:
    _check(load().kv_check_device_status(_ptr(workspace), _stream(stream)), "kv_check_device_status")


def kv_prefill_prefix(model: Model, cache: PagedCache, token_ids, block_table, pos0: int = 0, logits_out=None,
                      workspace=None, stream=None):
    ids, pids = _i32(token_ids)
    tab, ptab = _i32(block_table)
    ws = workspace if workspace is not None else model.workspace(KV_OP_PREFILL, pos0 + len(ids))
    _check(load().kv_prefill_prefix(model.handle, C.byref(cache.desc), pids, len(ids), pos0, ptab, len(tab),
                                    _ptr(ws), ws.numel(), _ptr(logits_out), _stream(stream)), "kv_prefill_prefix")
    return ws


def kv_decode_step(model: Model, cache: PagedCache, token_id: int, pos: int, block_table, logits_out,
                   workspace=None, stream=None):
    tab, ptab = _i32(block_table)
    ws = workspace if workspace is not None else model.workspace(KV_OP_DECODE, pos + 1)
    _check(load().kv_decode_step(model.handle, C.byref(cache.desc), int(token_id), int(pos), ptab, len(tab),
                                 _ptr(ws), ws.numel(), _ptr(logits_out), _stream(stream)), "kv_decode_step")
    return ws


def kv_pack_blocks(cache: PagedCache, block_ids, wire, wire_layout: int = KV_WIRE_BLOCK_MAJOR, stream=None,
                   wire_bytes=None):
    ids, pids = _i32(block_ids)
    nbytes = wire.numel() * wire.element_size() if wire_bytes is None else wire_bytes
    _check(load().kv_pack_blocks(C.byref(cache.desc), pids, len(ids), _ptr(wire), nbytes, wire_layout,
                                 _stream(stream)), "kv_pack_blocks")


def kv_unpack_assemble(cache: PagedCache, wire, logical_blocks, dst_block_ids, prefix_block_table,
                       n_tokens_total: int, epoch: int = 0, expected_epoch: int = 0,
                       wire_layout: int = KV_WIRE_BLOCK_MAJOR, stream=None, wire_bytes=None) -> np.ndarray:
    lg, plg = _i32(logical_blocks)
    ds, pds = _i32(dst_block_ids)
    pf, ppf = _i32(prefix_block_table)
    bs = cache.block_size
    merged = np.full(max(-(-n_tokens_total // bs), len(pf) + len(ds), 1), -1, dtype=np.int32)
    nbytes = (wire.numel() * wire.element_size() if wire is not None else 0) if wire_bytes is None else wire_bytes
    _check(load().kv_unpack_assemble(C.byref(cache.desc), _ptr(wire), nbytes, wire_layout, plg, pds, len(ds), ppf,
                                     len(pf), n_tokens_total, epoch, expected_epoch,
                                     merged.ctypes.data_as(C.POINTER(C.c_int32)), _stream(stream)),
           "kv_unpack_assemble")
    return merged[: -(-n_tokens_total // bs)]


def _batched(fn_name, cache, blk_offsets, block_ids, wires, wire_layout, stream):
    offs, poffs = _i32(blk_offsets)
    ids, pids = _i32(block_ids)
    ptrs = (C.c_void_p * len(wires))(*[_ptr(w) for w in wires])
    _check(getattr(load(), fn_name)(C.byref(cache.desc), len(wires), poffs, pids, ptrs, wire_layout,
                                    _stream(stream)), fn_name)


def kv_pack_blocks_batched(cache, blk_offsets, block_ids, wires, wire_layout=KV_WIRE_BLOCK_MAJOR, stream=None):
    _batched("kv_pack_blocks_batched", cache, blk_offsets, block_ids, wires, wire_layout, stream)


def kv_unpack_blocks_batched(cache, blk_offsets, dst_block_ids, wires, wire_layout=KV_WIRE_BLOCK_MAJOR, stream=None):
    _batched("kv_unpack_blocks_batched", cache, blk_offsets, dst_block_ids, wires, wire_layout, stream)


KV_GEMM_CTA_PAIR = 0x100


def kv_op_gemm(a, w, mode: int, out=None, resid=None, status=None, stream=None, n=None):
    """mode 0 store / 1 residual add / 2 SwiGLU, optionally | KV_GEMM_CTA_PAIR for the two-SM kernel."""
    m, k = a.shape
    base_mode = mode & ~KV_GEMM_CTA_PAIR
    n = n if n is not None else (w.shape[0] // 2 if base_mode == 2 else w.shape[0])
    want = (m, n)
    for t in (out, resid):
        if t is not None and hasattr(t, "shape") and tuple(t.shape) != want:
            raise ValueError(f"output shape {tuple(t.shape)} does not match the product's {want}")
    _check(load().kv_op_gemm(_ptr(a), a.stride(0), _ptr(w), m, n, k, mode, _ptr(out), _ptr(resid), _ptr(status),
                             _stream(stream)), "kv_op_gemm")


def kv_gemm_plan(m: int, n: int, mode: int, head_dim: int = 0):
    """(cta_pair, tile_width) the projection launcher picks for an m x n problem (mode 3 = fused QKV)."""
    pair, bn = C.c_int32(), C.c_int32()
    _check(load().kv_gemm_plan(m, n, mode, head_dim, C.byref(pair), C.byref(bn)), "kv_gemm_plan")
    return bool(pair.value), int(bn.value)


def kv_op_rmsnorm(x, gain, eps: float, out, stream=None):
    _check(load().kv_op_rmsnorm(_ptr(x), _ptr(gain), x.shape[0], x.shape[1], eps, _ptr(out), _stream(stream)),
           "kv_op_rmsnorm")


def kv_op_attention_prefill(qkv_ctx, n_q_heads, n_kv_heads, head_dim, out, pos0=0, cache=None, layer=0,
                            block_table_dev=None, status=None, stream=None):
    """qkv_ctx has pos0 + T rows (the chunk's rows last); with pos0 > 0 the call fills the K/V columns of the first
    pos0 rows from the cache."""
    _check(load().kv_op_attention_prefill(_ptr(qkv_ctx), qkv_ctx.shape[0] - pos0, pos0, n_q_heads, n_kv_heads, head_dim,
                                          C.byref(cache.desc) if cache is not None else None, layer,
                                          _ptr(block_table_dev), _ptr(out), _ptr(status), _stream(stream)),
           "kv_op_attention_prefill")


def kv_paged_attention_scratch_bytes(n_q_heads, head_dim, n_ctx) -> int:
    return int(load().kv_paged_attention_scratch_bytes(n_q_heads, head_dim, n_ctx))


def kv_op_paged_attention(q, cache: PagedCache, layer, block_table_dev, n_ctx, scratch, out, stream=None):
    _check(load().kv_op_paged_attention(_ptr(q), q.shape[0], C.byref(cache.desc), layer, _ptr(block_table_dev), n_ctx,
                                        _ptr(scratch), scratch.numel() * scratch.element_size(), _ptr(out),
                                        _stream(stream)), "kv_op_paged_attention")


def kv_fill_pattern(dst, nbytes: int, seed: int, pattern_offset: int = 0, stream=None):
    _check(load().kv_fill_pattern(_ptr(dst), nbytes, seed, pattern_offset, _stream(stream)), "kv_fill_pattern")


def kv_profile_enable(on: bool) -> None:
    _check(load().kv_profile_enable(int(on)), "kv_profile_enable")


def kv_profile_read() -> dict:
    """{kind: (milliseconds, kernel launches)} accumulated since the last read."""
    n = len(PROFILE_KINDS)
    ms = (C.c_float * n)()
    cnt = (C.c_int64 * n)()
    _check(load().kv_profile_read(ms, cnt, n), "kv_profile_read")
    return {k: (float(ms[i]), int(cnt[i])) for i, k in enumerate(PROFILE_KINDS)}


def kv_launch_count() -> int:
    return int(load().kv_launch_count())


def kv_op_paged_attention_noalloc(q, cache: PagedCache, layer, block_table_dev, n_ctx, out, stream=None):
    """kv_op_paged_attention for callers that cannot provide scratch memory: the partial results live in a
    fixed array inside the library (limit KV_NOALLOC_SCRATCH_BYTES; larger contexts raise KVError)."""
    _check(load().kv_op_paged_attention_noalloc(_ptr(q), q.shape[0], C.byref(cache.desc), layer,
                                                _ptr(block_table_dev), n_ctx, _ptr(out), _stream(stream)),
           "kv_op_paged_attention_noalloc")


def kv_selftest_bounded_wait(status_buf, limit_us: int = 200, stream=None) -> None:
    """Launches the bounded-wait self-test into `status_buf`; kv_check_device_status(status_buf) then raises KVError(-14)."""
    _check(load().kv_selftest_bounded_wait(_ptr(status_buf), limit_us, _stream(stream)), "kv_selftest_bounded_wait")


def kv_check_copy_status(stream=None) -> None:
    _check(load().kv_check_copy_status(_stream(stream)), "kv_check_copy_status")


def kv_op_gemv(w, x, mode: int, y, gain=None, eps: float = 0.0, stream=None, n=None):
    rows, k = w.shape
    n = n if n is not None else (rows // 2 if mode == 2 else rows)
    _check(load().kv_op_gemv(_ptr(w), _ptr(x), n, k, mode, _ptr(gain), eps, _ptr(y), _stream(stream)), "kv_op_gemv")


def kv_window_evaluate(t_w: float, **inputs) -> dict:
    win, out = WindowInputs(**inputs), WindowEval()
    _check(load().kv_window_evaluate(C.byref(win), t_w, C.byref(out)), "kv_window_evaluate")
    return out.as_dict()


def kv_window_select(t_max: float, d_t: float, **inputs):
    """Returns (evaluation at T_w*, trigger)."""
    win, out, trig = WindowInputs(**inputs), WindowEval(), C.c_int32()
    _check(load().kv_window_select(C.byref(win), t_max, d_t, C.byref(out), C.byref(trig)), "kv_window_select")
    return out.as_dict(), bool(trig.value)


def kv_window_waste_bound(t_max: float, e_early: float, t_avail: float) -> float:
    return float(load().kv_window_waste_bound(t_max, e_early, t_avail))


def kv_ewma(old: float, sample: float, beta: float) -> float:
    return float(load().kv_ewma(old, sample, beta))


def kv_prefill_prefix_batched(model: Model, cache: PagedCache, token_id_lists, block_tables, logits_out=None,
                              workspace=None, stream=None):
    """Prefix reconstruction of several requests in one call (lists of per-request token ids / block tables)."""
    tok_off = np.concatenate([[0], np.cumsum([len(t) for t in token_id_lists])]).astype(np.int32)
    tab_off = np.concatenate([[0], np.cumsum([len(t) for t in block_tables])]).astype(np.int32)
    ids, pids = _i32(np.concatenate([np.asarray(t, dtype=np.int32) for t in token_id_lists]))
    tabs, ptabs = _i32(np.concatenate([np.asarray(t, dtype=np.int32) for t in block_tables]))
    toff, ptoff = _i32(tok_off)
    boff, pboff = _i32(tab_off)
    ws = workspace if workspace is not None else model.workspace(KV_OP_PREFILL, int(tok_off[-1]))
    _check(load().kv_prefill_prefix_batched(model.handle, C.byref(cache.desc), len(token_id_lists), ptoff, pids, pboff,
                                            ptabs, _ptr(ws), ws.numel(), _ptr(logits_out), _stream(stream)),
           "kv_prefill_prefix_batched")
    return ws


# ---- serving a batch of requests: rotary positions, rows into and out of pages, attention of one new token each.
# A decode step makes these calls for every layer, so their checks are written out instead of shared.
KV_ROPE_LAYOUTS = {"half": 0, "interleaved": 1}
KV_ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "parts": 3}
_TORCH = None


def _torch():
    global _TORCH
    if _TORCH is None:
        import torch
        _TORCH = torch
    return _TORCH


def _dtype(name, dtype):
    torch = _torch()
    if dtype is torch.bfloat16:
        return 0
    if dtype is torch.float32:
        return 1
    raise ValueError(f"{name}: bfloat16 or float32 is wanted, not {dtype}")


def _refuse(name, what):
    raise ValueError(f"{name}: {what}")


_INT32 = (1 << 31) - 1


def _int32(name, *values):
    """The library counts in 32 bits, and ctypes passes what is left of a larger number."""
    for v in values:
        if not -_INT32 <= v <= _INT32:
            _refuse(name, f"{v} is past the library's 32-bit counts")


def _on_device(name, stream, tensors):
    """(device index, raw stream) of a call on `tensors`, which all have to be on one CUDA device."""
    index = tensors[0].get_device()                 # -1 on the host
    for t in tensors:
        if t.get_device() != index or index < 0:
            _refuse(name, f"tensors on one CUDA device are wanted, not on {[str(t.device) for t in tensors]}")
    if stream is None:
        return index, _torch()._C._cuda_getCurrentRawStream(index)
    return index, getattr(stream, "cuda_stream", stream)


def _launch(name, index, args):
    """Calls the library with `index` as the current device (it need not be that of the caller)."""
    torch, call = _torch(), getattr(_LIB or load(), name)
    if index == torch._C._cuda_getDevice():
        status = call(*args)
    else:
        with torch.cuda.device(index):
            status = call(*args)
    if status != 0:
        raise KVError(status, name)


class Rope:
    """Rotary plan (kv_rope): which pairs turn, how fast, and the factor on the result.  scaling "none", "linear", "ntk"
    or "parts" (frequencies blended between theta and theta / factor by how often a pair turns in original_ctx)."""

    def __init__(self, rotary_dim: int, layout: str = "half", base: float = 1.0e6, scaling: str = "none",
                 factor: float = 1.0, original_ctx: float = 0.0, low: float = 1.0, high: float = 32.0, gain: float = 1.0):
        self.handle = None
        if layout not in KV_ROPE_LAYOUTS:
            _refuse("Rope", f"layout {layout!r}: one of {sorted(KV_ROPE_LAYOUTS)}")
        if scaling not in KV_ROPE_SCALINGS:
            _refuse("Rope", f"scaling {scaling!r}: one of {sorted(KV_ROPE_SCALINGS)}")
        _int32("Rope", rotary_dim)
        self._lib = load()
        self.rotary_dim = rotary_dim
        desc = RopeDesc(rotary_dim, KV_ROPE_LAYOUTS[layout], KV_ROPE_SCALINGS[scaling], base, factor, original_ctx, low,
                        high, gain)
        handle = C.c_void_p()
        _check(self._lib.kv_rope_create(C.byref(desc), C.byref(handle)), "kv_rope_create")
        self.handle = handle

    def frequencies(self) -> np.ndarray:
        """theta_j of the rotary_dim / 2 pairs (radians per position, float64)."""
        out = np.empty(self.rotary_dim // 2, dtype=np.float64)
        _check(self._lib.kv_rope_frequencies(self.handle, out.ctypes.data_as(C.POINTER(C.c_double)), len(out)),
               "kv_rope_frequencies")
        return out

    def __del__(self):
        try:
            if self.handle:
                self._lib.kv_rope_destroy(self.handle)
                self.handle = None
        except Exception:
            pass


def kv_op_rope(rope: Rope, x, positions, out, backward: bool = False, stream=None):
    """out[t, h] = x[t, h] rotated at positions[t]; x and out [T, heads, head_dim] (bf16 or fp32, any strides whose last is
    1; out may be x), positions int32 [T].  backward: the gradient of x from the gradient of out."""
    name, shape = "kv_op_rope", x.shape
    if len(shape) != 3 or out.shape != shape or out.dtype is not x.dtype:
        _refuse(name, "x and out are [tokens, heads, head_dim] of one type")
    t, h, d = shape
    (xt, xh, xd), (ot, oh, od) = x.stride(), out.stride()
    if t * h * d and d > 1 and (xd != 1 or od != 1):
        _refuse(name, "head_dim has to be contiguous")
    if positions.shape != (t,) or positions.dtype is not _torch().int32 or not positions.is_contiguous():
        _refuse(name, "positions is a contiguous int32 vector, one per token")
    dtype = _dtype(name, x.dtype)
    if t > _INT32 or h > _INT32 or d > _INT32:
        _int32(name, t, h, d)
    index, stream = _on_device(name, stream, (x, positions, out))
    _launch(name, index, (rope.handle, x.data_ptr(), xt if t > 1 else 0, xh if h > 1 else 0, dtype, t, h, d,
                          positions.data_ptr(), 1 if backward else 0, out.data_ptr(), ot if t > 1 else 0,
                          oh if h > 1 else 0, stream))


def _rows(name, cache, layer, k, v, slots):
    """(tokens, dtype, strides of K, strides of V) of rows [tokens, n_kv_heads, head_dim]."""
    if slots.dim() != 1 or slots.dtype is not _torch().int64 or not slots.is_contiguous():
        _refuse(name, "slots is a contiguous int64 vector, one per token")
    t, h, d = slots.shape[0], cache.n_kv_heads, cache.head_dim
    if k.shape != (t, h, d) or v.shape != (t, h, d) or k.dtype is not v.dtype:
        _refuse(name, f"rows are [tokens, n_kv_heads, head_dim] = {(t, h, d)} of one type")
    (kt, kh, kd), (vt, vh, vd) = k.stride(), v.stride()
    if t and (kd != 1 or vd != 1):
        _refuse(name, "head_dim has to be contiguous")
    if t > _INT32 or layer > _INT32 or layer < 0:
        _int32(name, t, layer)
    if t < 2:
        kt = vt = 0
    if h < 2:
        kh = vh = 0
    return t, _dtype(name, k.dtype), kt, kh, vt, vh


def kv_op_cache_write(cache: PagedCache, layer: int, k, v, slots, stream=None):
    """K and V rows [T, n_kv_heads, head_dim] (bf16 or fp32) into the cache's slots (int64 [T], block * block_size +
    offset; -1 skips a token).  An e4m3 or e2m1 cache quantises them on the way."""
    name = "kv_op_cache_write"
    t, dtype, kt, kh, vt, vh = _rows(name, cache, layer, k, v, slots)
    index, stream = _on_device(name, stream, (cache.data, k, v, slots))
    _launch(name, index, (cache._desc_ref, layer, k.data_ptr(), kt, kh, v.data_ptr(), vt, vh, dtype, t, slots.data_ptr(),
                          stream))


def kv_op_cache_read(cache: PagedCache, layer: int, slots, k_out, v_out, stream=None):
    """The cache's rows at `slots` into k_out and v_out [T, n_kv_heads, head_dim] (bf16 or fp32); rows whose slot is
    outside the pool stay as they were."""
    name = "kv_op_cache_read"
    t, dtype, kt, kh, vt, vh = _rows(name, cache, layer, k_out, v_out, slots)
    index, stream = _on_device(name, stream, (cache.data, slots, k_out, v_out))
    _launch(name, index, (cache._desc_ref, layer, slots.data_ptr(), t, k_out.data_ptr(), kt, kh, v_out.data_ptr(), vt, vh,
                          dtype, stream))


def kv_paged_attention_batched_scratch_bytes(n_req: int, n_q_heads: int, cache: PagedCache, max_ctx: int) -> int:
    _int32("kv_paged_attention_batched_scratch_bytes", n_req, n_q_heads, max_ctx)
    r = load().kv_paged_attention_batched_scratch_bytes(n_req, n_q_heads, cache.n_kv_heads, cache.head_dim, max_ctx)
    if r < 0:
        raise KVError(int(r), "kv_paged_attention_batched_scratch_bytes")
    return int(r)


def kv_op_paged_attention_batched(q, cache: PagedCache, layer: int, block_tables, context_lens, max_ctx: int, out,
                                  scratch, lse=None, softmax_scale=None, stream=None):
    """Attention of one new token per request: q and out [R, n_q_heads, head_dim] (bf16 or fp32, heads contiguous),
    block_tables int32 [R, B], context_lens int32 [R] (clamped to max_ctx), scratch of
    kv_paged_attention_batched_scratch_bytes(R, ...) bytes, lse fp32 [R, n_q_heads] or None; softmax_scale defaults to
    head_dim ** -0.5."""
    name, torch, shape = "kv_op_paged_attention_batched", _torch(), q.shape
    if len(shape) != 3 or shape[2] != cache.head_dim or out.shape != shape or out.dtype is not q.dtype:
        _refuse(name, "q and out are [requests, heads, head_dim] of one type")
    r, hq, d = shape
    (qr, qh, qd), (outr, outh, outd) = q.stride(), out.stride()
    if r and (qd != 1 or outd != 1 or (hq > 1 and (qh != d or outh != d))):
        _refuse(name, "a request's heads have to be contiguous")
    columns = block_tables.shape[1] if block_tables.dim() == 2 else -1
    if columns < 0 or block_tables.shape[0] != r or block_tables.dtype is not torch.int32:
        _refuse(name, "block_tables is int32 [requests, blocks]")
    # one row may have any row stride: what counts is its length
    row, step = (block_tables.stride() if r > 1 else (columns, block_tables.stride(1)))
    if (r and columns > 1 and step != 1) or (r > 1 and row < columns):
        _refuse(name, "rows of block_tables have to be contiguous, and not to overlap")
    if context_lens.shape != (r,) or context_lens.dtype is not torch.int32 or not context_lens.is_contiguous():
        _refuse(name, "context_lens is a contiguous int32 vector, one per request")
    if columns * cache.block_size < max_ctx:
        raise KVError(-8, name)
    tensors = [cache.data, q, block_tables, context_lens, out]
    lse_ptr = scratch_ptr = scratch_bytes = 0
    if lse is not None:
        if lse.shape != (r, hq) or lse.dtype is not torch.float32 or not lse.is_contiguous():
            _refuse(name, "lse is contiguous float32 [requests, heads]")
        tensors.append(lse)
        lse_ptr = lse.data_ptr()
    if scratch is not None:
        if not scratch.is_contiguous():
            _refuse(name, "scratch has to be contiguous")
        tensors.append(scratch)
        scratch_ptr, scratch_bytes = scratch.data_ptr(), scratch.numel() * scratch.element_size()
    dtype = _dtype(name, q.dtype)
    if r > _INT32 or hq > _INT32 or max_ctx > _INT32 or layer > _INT32 or max_ctx < 0 or layer < 0:
        _int32(name, r, hq, max_ctx, layer)
    index, stream = _on_device(name, stream, tensors)
    _launch(name, index, (q.data_ptr(), qr if r > 1 else 0, dtype, r, hq, cache._desc_ref, layer, block_tables.data_ptr(),
                          row, context_lens.data_ptr(), max_ctx, d ** -0.5 if softmax_scale is None else softmax_scale,
                          scratch_ptr, scratch_bytes, out.data_ptr(), outr if r > 1 else 0, lse_ptr, stream))


def kv_op_cache_append(rope: Rope, cache: PagedCache, layer: int, k, v, positions, slots, q=None, q_out=None, stream=None):
    """kv_op_rope on k (and on q, into q_out) and kv_op_cache_write of the result in one launch: k and v [T, n_kv_heads, head_dim]
    (left as they were), q and q_out [T, heads, head_dim] or None (q_out may be q), positions int32 [T], slots int64 [T]."""
    name, torch = "kv_op_cache_append", _torch()
    t, dtype, kt, kh, vt, vh = _rows(name, cache, layer, k, v, slots)
    if positions.shape != (t,) or positions.dtype is not torch.int32 or not positions.is_contiguous():
        _refuse(name, "positions is a contiguous int32 vector, one per token")
    if (q is None) != (q_out is None):
        _refuse(name, "q and q_out come together")
    tensors = (cache.data, k, v, positions, slots)
    hq = q_ptr = q_to = qt = qh = ot = oh = 0
    if q is not None:
        shape, kind = q.shape, k.dtype
        if len(shape) != 3 or shape[0] != t or shape[2] != cache.head_dim or q_out.shape != shape or q.dtype is not kind or \
                q_out.dtype is not kind:
            _refuse(name, "q and q_out are [tokens, heads, head_dim], of the type of k")
        hq = shape[1]
        (qt, qh, qd), (ot, oh, od) = q.stride(), q_out.stride()
        if t and hq and (qd != 1 or od != 1):
            _refuse(name, "head_dim has to be contiguous")
        if hq > _INT32:
            _int32(name, hq)
        if t < 2:
            qt = ot = 0
        if hq < 2:
            qh = oh = 0
        tensors = (cache.data, k, v, positions, slots, q, q_out)
        q_ptr, q_to = q.data_ptr(), q_out.data_ptr()
    index, stream = _on_device(name, stream, tensors)
    _launch(name, index, (rope.handle, cache._desc_ref, layer, q_ptr, qt, qh, hq, q_to, ot, oh, k.data_ptr(), kt, kh, v.data_ptr(), vt,
                          vh, dtype, t, positions.data_ptr(), slots.data_ptr(), stream))


class BlockBounds:
    """What the keys of every block of a cache span, per layer and KV head: codes int8 [layers, blocks, n_kv_heads, 2, head_dim] and
    scales uint8 [layers, blocks, n_kv_heads], written by kv_op_block_bounds.  codes and scales give memory that is there already."""

    def __init__(self, cache: PagedCache, codes=None, scales=None):
        torch = _torch()
        self.n_layers, self.num_blocks, self.n_kv_heads = cache.n_layers, cache.num_blocks, cache.n_kv_heads
        self.head_dim, self.block_size = cache.head_dim, cache.block_size
        shape = (cache.n_layers, cache.num_blocks, cache.n_kv_heads)
        if codes is None:
            codes = torch.zeros(*shape, 2, cache.head_dim, dtype=torch.int8, device=cache.data.device)
        if scales is None:
            scales = torch.zeros(shape, dtype=torch.uint8, device=cache.data.device)
        if codes.shape != (*shape, 2, cache.head_dim) or codes.dtype is not torch.int8 or not codes.is_contiguous():
            _refuse("BlockBounds", "codes is contiguous int8 [layers, blocks, n_kv_heads, 2, head_dim]")
        if scales.shape != shape or scales.dtype is not torch.uint8 or not scales.is_contiguous():
            _refuse("BlockBounds", "scales is contiguous uint8 [layers, blocks, n_kv_heads]")
        self.codes, self.scales = codes, scales

    def _layer(self, name, layer):
        """Addresses of a layer's codes and scales."""
        if not 0 <= layer < self.n_layers:
            raise KVError(-2, name)
        blocks = self.num_blocks * self.n_kv_heads
        return self.codes.data_ptr() + layer * blocks * 2 * self.head_dim, self.scales.data_ptr() + layer * blocks


def kv_op_block_bounds(cache: PagedCache, layer: int, blocks, counts, bounds: BlockBounds, stream=None):
    """Bounds of the blocks (int32 [n], each once) from the keys in their first counts (int32 [n]) slots; a block of -1 is left out."""
    name, torch = "kv_op_block_bounds", _torch()
    if blocks.dim() != 1 or blocks.dtype is not torch.int32 or not blocks.is_contiguous():
        _refuse(name, "blocks is a contiguous int32 vector")
    n = blocks.shape[0]
    if counts.shape != (n,) or counts.dtype is not torch.int32 or not counts.is_contiguous():
        _refuse(name, "counts is a contiguous int32 vector, one per block")
    if (bounds.num_blocks, bounds.n_kv_heads, bounds.head_dim, bounds.n_layers) != \
            (cache.num_blocks, cache.n_kv_heads, cache.head_dim, cache.n_layers):
        _refuse(name, "bounds of another cache")
    if n > _INT32:
        _int32(name, n)
    codes, scales = bounds._layer(name, layer)
    index, stream = _on_device(name, stream, (cache.data, blocks, counts, bounds.codes, bounds.scales))
    _launch(name, index, (cache._desc_ref, layer, blocks.data_ptr(), counts.data_ptr(), n, codes, scales, stream))


def kv_select_blocks_scratch_bytes(n_req: int, cache, max_ctx: int) -> int:
    """cache: the PagedCache or its BlockBounds."""
    _int32("kv_select_blocks_scratch_bytes", n_req, max_ctx)
    r = load().kv_select_blocks_scratch_bytes(n_req, cache.n_kv_heads, cache.block_size, max_ctx)
    if r < 0:
        raise KVError(int(r), "kv_select_blocks_scratch_bytes")
    return int(r)


def _vector(name, what, x, n, torch):
    """x is a contiguous int32 vector of n."""
    if x.shape != (n,) or x.dtype is not torch.int32 or not x.is_contiguous():
        _refuse(name, f"{what} is a contiguous int32 vector, one per request")


def kv_op_select_blocks(q, bounds: BlockBounds, layer: int, block_tables, context_lens, max_ctx: int, kept, kept_lens, scratch,
                        first: int = 1, last: int = 2, stream=None):
    """Chooses kept.shape[2] blocks for each request and KV head: q [R, heads, head_dim] (bf16 or fp32, heads contiguous), block_tables
    int32 [R, B], context_lens int32 [R] (clamped to max_ctx); writes kept int32 [R, n_kv_heads, keep] and kept_lens int32 [R].  The
    first `first` and last `last` blocks of a context are always among them.  scratch: kv_select_blocks_scratch_bytes(R, ...) bytes."""
    name, torch, shape = "kv_op_select_blocks", _torch(), q.shape
    if len(shape) != 3 or shape[2] != bounds.head_dim:
        _refuse(name, "q is [requests, heads, head_dim]")
    r, hq, d = shape
    qr, qh, qd = q.stride()
    if r and (qd != 1 or (hq > 1 and qh != d)):
        _refuse(name, "a request's heads have to be contiguous")
    if len(block_tables.shape) != 2 or block_tables.shape[0] != r or block_tables.dtype is not torch.int32:
        _refuse(name, "block_tables is int32 [requests, blocks]")
    columns, (row, step) = block_tables.shape[1], block_tables.stride()
    if r < 2:
        qr, row = 0, columns                        # one row may have any row stride: what counts is its length
    if (r and columns > 1 and step != 1) or row < columns:
        _refuse(name, "rows of block_tables have to be contiguous, and not to overlap")
    _vector(name, "context_lens", context_lens, r, torch)
    _vector(name, "kept_lens", kept_lens, r, torch)
    heads, keep = bounds.n_kv_heads, kept.shape[-1] if kept.dim() else 0
    if kept.shape != (r, heads, keep) or kept.dtype is not torch.int32 or not kept.is_contiguous():
        _refuse(name, "kept is contiguous int32 [requests, n_kv_heads, keep]")
    if r > _INT32 or hq > _INT32 or max_ctx > _INT32 or keep > _INT32 or not 0 <= first <= _INT32 or not 0 <= last <= _INT32 or max_ctx < 0:
        _int32(name, r, hq, max_ctx, first, last, keep)
    if columns * bounds.block_size < max_ctx:
        raise KVError(-8, name)
    dtype = _dtype(name, q.dtype)
    codes, scales = bounds._layer(name, layer)
    scratch_ptr = scratch_bytes = 0
    tensors = [q, bounds.codes, bounds.scales, block_tables, context_lens, kept, kept_lens]
    if scratch is not None:
        if not scratch.is_contiguous():
            _refuse(name, "scratch has to be contiguous")
        tensors.append(scratch)
        scratch_ptr, scratch_bytes = scratch.data_ptr(), scratch.nbytes
    index, stream = _on_device(name, stream, tensors)
    _launch(name, index, (q.data_ptr(), qr, dtype, r, hq, heads, d, codes, scales, bounds.num_blocks, bounds.block_size,
                          block_tables.data_ptr(), row, context_lens.data_ptr(), max_ctx, first, last, keep, scratch_ptr, scratch_bytes,
                          kept.data_ptr(), kept_lens.data_ptr(), stream))


def kv_op_paged_attention_selected(q, cache: PagedCache, layer: int, kept, kept_lens, out, scratch, lse=None, softmax_scale=None,
                                   stream=None):
    """kv_op_paged_attention_batched over the blocks that kv_op_select_blocks chose: kept int32 [R, n_kv_heads, keep], kept_lens
    int32 [R]; scratch of kv_paged_attention_batched_scratch_bytes(R, heads, cache, keep * block_size) bytes."""
    name, torch, shape = "kv_op_paged_attention_selected", _torch(), q.shape
    if len(shape) != 3 or shape[2] != cache.head_dim or out.shape != shape or out.dtype is not q.dtype:
        _refuse(name, "q and out are [requests, heads, head_dim] of one type")
    r, hq, d = shape
    (qr, qh, qd), (outr, outh, outd) = q.stride(), out.stride()
    if r and (qd != 1 or outd != 1 or (hq > 1 and (qh != d or outh != d))):
        _refuse(name, "a request's heads have to be contiguous")
    heads, columns = cache.n_kv_heads, kept.shape[-1] if kept.dim() else 0
    if kept.shape != (r, heads, columns) or kept.dtype is not torch.int32:
        _refuse(name, "kept is int32 [requests, n_kv_heads, blocks]")
    of_req, of_head, step = kept.stride()
    if heads < 2:
        of_head = columns
    if r < 2:
        of_req = max(columns, of_head * heads)
    if (r and columns > 1 and step != 1) or of_head < columns or of_req < columns:
        _refuse(name, "rows of kept have to be contiguous, and not to overlap")
    _vector(name, "kept_lens", kept_lens, r, torch)
    tensors = [cache.data, q, kept, kept_lens, out]
    lse_ptr = scratch_ptr = scratch_bytes = 0
    if lse is not None:
        if lse.shape != (r, hq) or lse.dtype is not torch.float32 or not lse.is_contiguous():
            _refuse(name, "lse is contiguous float32 [requests, heads]")
        tensors.append(lse)
        lse_ptr = lse.data_ptr()
    if scratch is not None:
        if not scratch.is_contiguous():
            _refuse(name, "scratch has to be contiguous")
        tensors.append(scratch)
        scratch_ptr, scratch_bytes = scratch.data_ptr(), scratch.nbytes
    dtype = _dtype(name, q.dtype)
    longest = columns * cache.block_size
    if r > _INT32 or hq > _INT32 or longest > _INT32 or not 0 <= layer <= _INT32:
        _int32(name, r, hq, longest, layer)
    index, stream = _on_device(name, stream, tensors)
    _launch(name, index, (q.data_ptr(), qr if r > 1 else 0, dtype, r, hq, cache._desc_ref, layer, kept.data_ptr(), of_req, of_head,
                          kept_lens.data_ptr(), longest, d ** -0.5 if softmax_scale is None else softmax_scale, scratch_ptr, scratch_bytes,
                          out.data_ptr(), outr if r > 1 else 0, lse_ptr, stream))
