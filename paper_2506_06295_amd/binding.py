"""ctypes binding of libdllmc.so: argument marshalling only.

Every step of the cached denoising path runs inside the HIP library; torch is used
here for device memory and the stream handle.  Loading fails loudly when the library has
not been built (``python -c "import __graft_entry__ as g; g.build()"``): there is no
fallback path.
"""
from __future__ import annotations

import ctypes as C
import functools
import os
from typing import Dict, List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libdllmc.so")

DLLMC_F32, DLLMC_BF16 = 0, 1
DLLMC_KV4 = 2
_DTYPES = {"f32": (DLLMC_F32, torch.float32), "bf16": (DLLMC_BF16, torch.bfloat16)}
_ERR = {-1: "EINVAL", -2: "ESTATE", -3: "EHIP", -4: "ENOMEM", -5: "ETOOBIG"}

EXPORTS = (
    "dllmc_workspace_bytes", "dllmc_create", "dllmc_num_selected", "dllmc_step",
    "dllmc_read_cache", "dllmc_read_scores", "dllmc_destroy", "dllmc_strerror",
    "dllmc_last_hip_error", "dllmc_op_select", "dllmc_op_vverify", "dllmc_op_linear",
    "dllmc_op_attention", "dllmc_profile_enable", "dllmc_profile_read", "dllmc_kernel_class_name",
    "dllmc_set_gemm_tuning", "dllmc_op_attention_scratch_bytes", "dllmc_plan_gemm_slices", "dllmc_plan_attention", "dllmc_plan_vverify", "dllmc_plan_gate_up", "dllmc_plan_tile",
    "dllmc_gen_workspace_bytes", "dllmc_gen_create", "dllmc_gen_step", "dllmc_gen_read",
    "dllmc_gen_destroy", "dllmc_op_head_scratch_bytes", "dllmc_op_head", "dllmc_set_policy",
    "dllmc_set_layer_rho", "dllmc_layer_num_selected", "dllmc_probe_copy", "dllmc_probe_read", "dllmc_probe_mfma",
    "dllmc_op_linear_static", "dllmc_op_linear_static_max_elements", "dllmc_op_linear_rows",
    "dllmc_pool_bytes", "dllmc_workspace_bytes_paged", "dllmc_create_paged", "dllmc_set_page_table",
    "dllmc_pool_create", "dllmc_pool_available", "dllmc_pool_alloc", "dllmc_pool_free", "dllmc_pool_destroy",
    "dllmc_kv4_bytes", "dllmc_op_kv4_store", "dllmc_op_kv4_load", "dllmc_op_attention_kv4_scratch_bytes",
    "dllmc_op_attention_kv4", "dllmc_op_attention_weights_scratch_bytes", "dllmc_op_attention_weights", "dllmc_op_evict",
    "dllmc_op_compact", "dllmc_i8_row_bytes", "dllmc_op_quant8", "dllmc_op_linear_i8_scratch_bytes", "dllmc_op_linear_i8",
    "dllmc_plan_linear_i8", "dllmc_plan_attention_kv4", "dllmc_plan_attention_weights",
)
NUM_KERNEL_CLASSES = 13


class dllmc_model(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("d_model", C.c_int32), ("n_q_heads", C.c_int32),
                ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32), ("d_ffn", C.c_int32),
                ("batch", C.c_int32), ("dtype", C.c_int32), ("rms_eps", C.c_float),
                ("rope_theta", C.c_float)]


class dllmc_layer_weights(C.Structure):
    _fields_ = [(k, C.c_void_p) for k in ("attn_norm_g", "wq", "wk", "wv", "wo", "ffn_norm_g",
                                          "w_gate", "w_up", "w_down")]


class dllmc_paging(C.Structure):
    _fields_ = [("page_rows", C.c_int32), ("pool_pages", C.c_int32), ("page_table", C.POINTER(C.c_int32)),
                ("pool", C.c_void_p), ("pool_bytes", C.c_size_t)]


class dllmc_gen_config(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("final_norm_g", C.c_void_p), ("lm_head", C.c_void_p),
                ("vocab", C.c_int32), ("steps", C.c_int32), ("block_len", C.c_int32)]


class dllmc_kernel_stat(C.Structure):
    _fields_ = [("launches", C.c_int64), ("ms", C.c_double), ("alg_bytes", C.c_double),
                ("flops", C.c_double)]


class DllmcError(RuntimeError):
    pass


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise DllmcError(f"{LIB_PATH} is missing: build it first (__graft_entry__.build())")
        L = C.CDLL(LIB_PATH)
        L.dllmc_workspace_bytes.restype = C.c_size_t
        L.dllmc_workspace_bytes.argtypes = [C.POINTER(dllmc_model), C.c_int32, C.c_int32]
        L.dllmc_create.restype = C.c_int
        L.dllmc_create.argtypes = [C.POINTER(C.c_void_p), C.POINTER(dllmc_model),
                                   C.POINTER(dllmc_layer_weights), C.c_int32, C.c_int32, C.c_float,
                                   C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]
        L.dllmc_pool_bytes.restype = C.c_size_t
        L.dllmc_pool_bytes.argtypes = [C.POINTER(dllmc_model), C.c_int32, C.c_int32]
        L.dllmc_workspace_bytes_paged.restype = C.c_size_t
        L.dllmc_workspace_bytes_paged.argtypes = [C.POINTER(dllmc_model), C.c_int32, C.c_int32,
                                                  C.POINTER(dllmc_paging)]
        L.dllmc_create_paged.restype = C.c_int
        L.dllmc_create_paged.argtypes = [C.POINTER(C.c_void_p), C.POINTER(dllmc_model),
                                         C.POINTER(dllmc_layer_weights), C.c_int32, C.c_int32, C.c_float,
                                         C.c_int32, C.c_int32, C.POINTER(dllmc_paging), C.c_void_p,
                                         C.c_size_t, C.c_void_p]
        L.dllmc_set_page_table.restype = C.c_int
        L.dllmc_set_page_table.argtypes = [C.c_void_p, C.POINTER(C.c_int32)]
        L.dllmc_pool_create.restype = C.c_int
        L.dllmc_pool_create.argtypes = [C.POINTER(C.c_void_p), C.c_int32]
        L.dllmc_pool_available.restype = C.c_int32
        L.dllmc_pool_available.argtypes = [C.c_void_p]
        L.dllmc_pool_alloc.restype = C.c_int
        L.dllmc_pool_alloc.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_int32)]
        L.dllmc_pool_free.restype = C.c_int
        L.dllmc_pool_free.argtypes = [C.c_void_p, C.POINTER(C.c_int32), C.c_int32]
        L.dllmc_pool_destroy.restype = C.c_int
        L.dllmc_pool_destroy.argtypes = [C.c_void_p]
        L.dllmc_num_selected.restype = C.c_int32
        L.dllmc_num_selected.argtypes = [C.c_void_p]
        L.dllmc_step.restype = C.c_int
        L.dllmc_step.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p,
                                 C.POINTER(C.c_int32)]
        L.dllmc_read_cache.restype = C.c_int
        L.dllmc_read_cache.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p]
        L.dllmc_read_scores.restype = C.c_int
        L.dllmc_read_scores.argtypes = [C.c_void_p, C.c_void_p]
        L.dllmc_destroy.restype = C.c_int
        L.dllmc_destroy.argtypes = [C.c_void_p]
        L.dllmc_strerror.restype = C.c_char_p
        L.dllmc_strerror.argtypes = [C.c_int]
        L.dllmc_last_hip_error.restype = C.c_int
        L.dllmc_op_select.restype = C.c_int
        L.dllmc_op_select.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p,
                                      C.c_void_p]
        L.dllmc_op_vverify.restype = C.c_int
        L.dllmc_op_vverify.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                       C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.dllmc_op_linear.restype = C.c_int
        L.dllmc_op_linear.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                      C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.dllmc_op_linear_rows.restype = C.c_int
        L.dllmc_op_linear_rows.argtypes = [C.c_int32, C.c_void_p, C.c_int32, C.c_void_p, C.c_int32, C.c_void_p,
                                           C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.dllmc_op_linear_static.restype = C.c_int
        L.dllmc_op_linear_static.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                             C.c_int32, C.c_int32, C.c_void_p, C.c_void_p]
        L.dllmc_op_linear_static_max_elements.restype = C.c_size_t
        L.dllmc_op_linear_static_max_elements.argtypes = []
        L.dllmc_op_attention.restype = C.c_int
        L.dllmc_op_attention.argtypes = [C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_void_p,
                                         C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32,
                                         C.c_void_p, C.c_void_p, C.c_void_p]
        L.dllmc_op_attention_scratch_bytes.restype = C.c_size_t
        L.dllmc_set_policy.restype = C.c_int
        L.dllmc_set_policy.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_int32, C.c_uint32]
        L.dllmc_gen_workspace_bytes.restype = C.c_size_t
        L.dllmc_gen_workspace_bytes.argtypes = [C.c_void_p, C.POINTER(dllmc_gen_config)]
        L.dllmc_gen_create.restype = C.c_int
        L.dllmc_gen_create.argtypes = [C.POINTER(C.c_void_p), C.c_void_p, C.POINTER(dllmc_gen_config),
                                       C.c_void_p, C.c_size_t]
        L.dllmc_gen_step.restype = C.c_int
        L.dllmc_gen_step.argtypes = [C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p,
                                     C.POINTER(C.c_int32), C.POINTER(C.c_int32)]
        L.dllmc_gen_read.restype = C.c_int
        L.dllmc_gen_read.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.dllmc_gen_destroy.restype = C.c_int
        L.dllmc_gen_destroy.argtypes = [C.c_void_p]
        L.dllmc_op_head_scratch_bytes.restype = C.c_size_t
        L.dllmc_op_head_scratch_bytes.argtypes = [C.c_int32] * 4
        L.dllmc_op_head.restype = C.c_int
        L.dllmc_op_head.argtypes = [C.c_int32, C.c_void_p, C.c_void_p, C.c_int32, C.c_void_p, C.c_float,
                                    C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p,
                                    C.c_void_p, C.c_void_p]
        L.dllmc_op_attention_scratch_bytes.argtypes = []
        L.dllmc_profile_enable.restype = C.c_int
        L.dllmc_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        L.dllmc_profile_read.restype = C.c_int
        L.dllmc_profile_read.argtypes = [C.c_void_p, C.POINTER(dllmc_kernel_stat), C.c_int32]
        L.dllmc_kernel_class_name.restype = C.c_char_p
        L.dllmc_kernel_class_name.argtypes = [C.c_int32]
        L.dllmc_plan_gemm_slices.restype = C.c_int32
        L.dllmc_plan_gemm_slices.argtypes = [C.c_int32] * 5 + [C.c_size_t]
        L.dllmc_plan_gate_up.restype = C.c_int32
        L.dllmc_plan_gate_up.argtypes = [C.c_int32] * 3 + [C.POINTER(C.c_int32)]
        L.dllmc_plan_tile.restype = C.c_int32
        L.dllmc_plan_tile.argtypes = [C.c_int32] * 5 + [C.POINTER(C.c_int32)]
        L.dllmc_plan_vverify.restype = C.c_int32
        L.dllmc_plan_vverify.argtypes = [C.c_int32] * 4
        L.dllmc_plan_attention.restype = C.c_int32
        L.dllmc_plan_attention.argtypes = [C.c_int32] * 6 + [C.POINTER(C.c_int32)]
        L.dllmc_set_gemm_tuning.restype = C.c_int
        L.dllmc_set_gemm_tuning.argtypes = [C.c_int32] * 7
        L.dllmc_set_layer_rho.restype = C.c_int
        L.dllmc_set_layer_rho.argtypes = [C.c_void_p, C.POINTER(C.c_float), C.c_int32]
        L.dllmc_layer_num_selected.restype = C.c_int32
        L.dllmc_layer_num_selected.argtypes = [C.c_void_p, C.c_int32]
        L.dllmc_probe_copy.restype = C.c_int
        L.dllmc_probe_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.dllmc_probe_read.restype = C.c_int
        L.dllmc_probe_read.argtypes = [C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.dllmc_probe_mfma.restype = C.c_int
        L.dllmc_probe_mfma.argtypes = [C.c_int32, C.c_int32, C.c_void_p, C.POINTER(C.c_double), C.c_void_p]
        i32, ptr, size = C.c_int32, C.c_void_p, C.c_size_t
        for name, res, args in (
                ("dllmc_kv4_bytes", size, [i32] * 3),
                ("dllmc_op_kv4_store", C.c_int, [i32, ptr, i32, ptr, ptr, i32, i32, i32, ptr]),
                ("dllmc_op_kv4_load", C.c_int, [i32, ptr, i32, i32, i32, ptr, i32, ptr, ptr]),
                ("dllmc_op_attention_kv4_scratch_bytes", size, [i32] * 7),
                ("dllmc_op_attention_kv4", C.c_int, [i32, ptr, i32, i32, ptr, ptr, i32, ptr, ptr, i32, i32, i32, i32, ptr, ptr,
                                                     ptr, size, ptr]),
                ("dllmc_op_attention_weights_scratch_bytes", size, [i32] * 8),
                ("dllmc_op_attention_weights", C.c_int, [i32, i32, ptr, i32, i32, ptr, i32, ptr, ptr, i32, i32, i32, i32, ptr,
                                                         ptr, ptr, ptr, size, ptr]),
                ("dllmc_op_evict", C.c_int, [ptr, i32, i32, ptr, ptr, i32, i32, i32, i32, ptr, ptr, ptr, ptr, ptr]),
                ("dllmc_op_compact", C.c_int, [i32, ptr, i32, i32, i32, i32, i32, ptr, ptr, ptr, ptr, ptr]),
                ("dllmc_i8_row_bytes", size, [i32]),
                ("dllmc_op_quant8", C.c_int, [i32, ptr, i32, ptr, i32, i32, ptr, ptr, ptr]),
                ("dllmc_op_linear_i8_scratch_bytes", size, [i32] * 3),
                ("dllmc_plan_attention_kv4", i32, [i32] * 7 + [C.POINTER(i32)] * 3),
                ("dllmc_plan_attention_weights", i32, [i32] * 8 + [C.POINTER(i32)] * 3),
                ("dllmc_plan_linear_i8", i32, [i32] * 3 + [C.POINTER(i32)] * 3),
                ("dllmc_op_linear_i8", C.c_int, [i32, ptr, ptr, i32, ptr, ptr, i32, i32, ptr, ptr, size, ptr])):
            fn = getattr(L, name)
            fn.restype, fn.argtypes = res, args
        _lib = L
    return _lib


def _check(rc: int, what: str) -> None:
    if rc != 0:
        L = lib()
        msg = L.dllmc_strerror(rc).decode()
        extra = f" (hipError {L.dllmc_last_hip_error()})" if rc == -3 else ""
        raise DllmcError(f"{what}: {_ERR.get(rc, rc)} {msg}{extra}")


def _stream_handle() -> int:
    # (the handle alone: 0.3 us, torch.cuda.current_stream().cuda_stream makes an object for 3)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device())


def _stream(device: int) -> int:
    return torch._C._cuda_getCurrentRawStream(device)


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


class CachedDenoiser:
    """dllmc_create / dllmc_step / dllmc_destroy around torch-owned device memory."""

    def __init__(self, *, n_layers: int, d_model: int, n_q_heads: int, n_kv_heads: int,
                 head_dim: int, d_ffn: int, batch: int, dtype: str,
                 weights: Sequence[Dict[str, torch.Tensor]], L_p: int, L_r: int, rho: float,
                 K_p: int, K_r: int, rms_eps: float = 1e-5, rope_theta: float = 10000.0,
                 paging: Optional[Dict] = None):
        """paging: None for the flat cache layout, else dict(page_rows, pool_pages, page_table
        [B][pages per sequence] of ints[, pool: uint8 device tensor shared between contexts])."""
        self._h = None
        L = lib()
        code, tdt = _DTYPES[dtype]
        self.torch_dtype = tdt
        self.B, self.L_p, self.L_r, self.n, self.d, self.T = batch, L_p, L_r, L_p + L_r, d_model, n_layers
        self.d_kv = n_kv_heads * head_dim
        self.model = dllmc_model(n_layers, d_model, n_q_heads, n_kv_heads, head_dim, d_ffn, batch,
                                 code, rms_eps, rope_theta)
        if len(weights) != n_layers:
            raise DllmcError("one weight dict per layer expected")
        self._weights = weights  # keep the tensors alive: the library borrows the pointers
        arr = (dllmc_layer_weights * n_layers)()
        for l, w in enumerate(weights):
            for name, _ in dllmc_layer_weights._fields_:
                t = w[name]
                if not (t.is_cuda and t.is_contiguous() and t.dtype == tdt):
                    raise DllmcError(f"layer {l} {name}: need a contiguous {tdt} device tensor")
                setattr(arr[l], name, t.data_ptr())
        self.stream = _stream_handle()
        h = C.c_void_p()
        self.paging = None
        if paging is None:
            nbytes = L.dllmc_workspace_bytes(C.byref(self.model), L_p, L_r)
            if nbytes == 0:
                raise DllmcError("dllmc_workspace_bytes: invalid model description")
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
            _check(L.dllmc_create(C.byref(h), C.byref(self.model), arr, L_p, L_r, rho, K_p, K_r,
                                  self.workspace.data_ptr(), nbytes, self.stream), "dllmc_create")
        else:
            table = self._table(paging["page_table"])
            pool = paging.get("pool")
            self._pool = pool   # keep a shared pool alive
            pg = dllmc_paging(int(paging["page_rows"]), int(paging["pool_pages"]), table,
                              None if pool is None else pool.data_ptr(),
                              0 if pool is None else pool.numel() * pool.element_size())
            nbytes = L.dllmc_workspace_bytes_paged(C.byref(self.model), L_p, L_r, C.byref(pg))
            if nbytes == 0:
                raise DllmcError("dllmc_workspace_bytes_paged: invalid model or paging description")
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
            _check(L.dllmc_create_paged(C.byref(h), C.byref(self.model), arr, L_p, L_r, rho, K_p, K_r,
                                        C.byref(pg), self.workspace.data_ptr(), nbytes, self.stream),
                   "dllmc_create_paged")
            self.paging = dict(paging)
        self._h = h
        self.num_selected = L.dllmc_num_selected(h)
        self.sel_idx = torch.full((n_layers, batch, L_r), -1, dtype=torch.int32, device="cuda")

    @staticmethod
    def _table(page_table):
        flat = [int(p) for row in page_table for p in row]
        return (C.c_int32 * len(flat))(*flat)

    def set_page_table(self, page_table) -> None:
        """New page table for a paged context; the next step must be step 0."""
        _check(lib().dllmc_set_page_table(self._h, self._table(page_table)), "dllmc_set_page_table")

    def step(self, hidden_in: torch.Tensor, step_idx: int, hidden_out: Optional[torch.Tensor] = None):
        """Enqueue one denoising step; returns (hidden_out, n_sel).  self.sel_idx[:, :, :n_sel]
        holds the recomputed response rows per layer and sequence once the stream is synced."""
        if hidden_out is None:
            hidden_out = torch.empty_like(hidden_in)
        for t in (hidden_in, hidden_out):
            if not (t.is_cuda and t.is_contiguous() and t.dtype == self.torch_dtype
                    and tuple(t.shape) == (self.B, self.n, self.d)):
                raise DllmcError("hidden states must be contiguous [B, n, d] device tensors of the model dtype")
        n_sel = C.c_int32(0)
        _check(lib().dllmc_step(self._h, hidden_in.data_ptr(), step_idx, hidden_out.data_ptr(),
                                self.sel_idx.data_ptr(), C.byref(n_sel)), "dllmc_step")
        return hidden_out, n_sel.value

    def set_policy(self, metric: str = "cosine", selection: str = "verify", v_update: str = "all",
                   seed: int = 0, source: str = "v") -> None:
        """Variants of the paper's ablations; see dllmc_set_policy."""
        _check(lib().dllmc_set_policy(self._h, {"v": 0, "k": 1}[source], {"cosine": 0, "l2": 1}[metric],
                                      {"verify": 0, "random": 1}[selection],
                                      {"all": 0, "selected": 1}[v_update], seed & 0xFFFFFFFF),
               "dllmc_set_policy")

    def set_layer_rho(self, rho_layers) -> None:
        """One update ratio per layer, or None for the single ratio given at creation."""
        if rho_layers is None:
            _check(lib().dllmc_set_layer_rho(self._h, None, 0), "dllmc_set_layer_rho")
            return
        arr = (C.c_float * len(rho_layers))(*[float(r) for r in rho_layers])
        _check(lib().dllmc_set_layer_rho(self._h, arr, len(rho_layers)), "dllmc_set_layer_rho")

    def layer_num_selected(self, layer: int) -> int:
        k = lib().dllmc_layer_num_selected(self._h, layer)
        if k < 0:
            raise DllmcError("dllmc_layer_num_selected: invalid argument")
        return k

    def read_cache(self, layer: int, which: int) -> torch.Tensor:
        width = self.d_kv if which < 2 else self.d
        out = torch.empty((self.B, self.n, width), dtype=self.torch_dtype, device="cuda")
        _check(lib().dllmc_read_cache(self._h, layer, which, out.data_ptr()), "dllmc_read_cache")
        return out

    def read_scores(self) -> torch.Tensor:
        out = torch.empty((self.T, self.B, self.L_r), dtype=torch.float32, device="cuda")
        _check(lib().dllmc_read_scores(self._h, out.data_ptr()), "dllmc_read_scores")
        return out

    def profile_enable(self, on: bool) -> None:
        _check(lib().dllmc_profile_enable(self._h, 1 if on else 0), "dllmc_profile_enable")

    def profile_read(self, reset: bool = True) -> Dict[str, Dict[str, float]]:
        arr = (dllmc_kernel_stat * NUM_KERNEL_CLASSES)()
        _check(lib().dllmc_profile_read(self._h, arr, 1 if reset else 0), "dllmc_profile_read")
        return {lib().dllmc_kernel_class_name(i).decode(): {
            "launches": int(arr[i].launches), "ms": arr[i].ms, "alg_bytes": arr[i].alg_bytes,
            "flops": arr[i].flops} for i in range(NUM_KERNEL_CLASSES)}

    def close(self) -> None:
        if self._h is not None:
            h, self._h = self._h, None
            _check(lib().dllmc_destroy(h), "dllmc_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def pool_bytes(model: dllmc_model, page_rows: int, pool_pages: int) -> int:
    return lib().dllmc_pool_bytes(C.byref(model), page_rows, pool_pages)


class PagePool:
    """dllmc_pool_*: host-side allocator of page ids."""

    def __init__(self, pool_pages: int):
        self._h = None
        h = C.c_void_p()
        _check(lib().dllmc_pool_create(C.byref(h), pool_pages), "dllmc_pool_create")
        self._h = h

    @property
    def available(self) -> int:
        return lib().dllmc_pool_available(self._h)

    def alloc(self, count: int) -> List[int]:
        ids = (C.c_int32 * max(count, 1))()
        _check(lib().dllmc_pool_alloc(self._h, count, ids), "dllmc_pool_alloc")
        return list(ids[:count])

    def free(self, ids: Sequence[int]) -> None:
        arr = (C.c_int32 * max(len(ids), 1))(*[int(i) for i in ids])
        _check(lib().dllmc_pool_free(self._h, arr, len(ids)), "dllmc_pool_free")

    def close(self) -> None:
        if self._h is not None:
            h, self._h = self._h, None
            _check(lib().dllmc_pool_destroy(h), "dllmc_pool_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Generator:
    """dllmc_gen_* around a CachedDenoiser: the closed denoising loop, tokens stay on the device."""

    def __init__(self, den: CachedDenoiser, embed: torch.Tensor, final_norm_g: torch.Tensor,
                 lm_head: torch.Tensor, steps: int, block_len: int = 0):
        self._h = None
        self.den = den
        vocab = lm_head.shape[0]
        for name, t, shape in (("embed", embed, (vocab + 1, den.d)), ("final_norm_g", final_norm_g, (den.d,)),
                               ("lm_head", lm_head, (vocab, den.d))):
            if not (t.is_cuda and t.is_contiguous() and t.dtype == den.torch_dtype and tuple(t.shape) == shape):
                raise DllmcError(f"{name}: need a contiguous {den.torch_dtype} device tensor of shape {shape}")
        self._keep = (embed, final_norm_g, lm_head)
        self.vocab, self.steps = vocab, steps
        self.cfg = dllmc_gen_config(embed.data_ptr(), final_norm_g.data_ptr(), lm_head.data_ptr(),
                                    vocab, steps, block_len)
        L = lib()
        nbytes = L.dllmc_gen_workspace_bytes(den._h, C.byref(self.cfg))
        if nbytes == 0:
            raise DllmcError("dllmc_gen_workspace_bytes: invalid configuration")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device="cuda")
        h = C.c_void_p()
        _check(L.dllmc_gen_create(C.byref(h), den._h, C.byref(self.cfg), self.workspace.data_ptr(), nbytes),
               "dllmc_gen_create")
        self._h = h

    def step(self, tokens: torch.Tensor, step_idx: int):
        """Enqueue one step of the loop on tokens [B, n] int32 (updated in place); returns
        (positions revealed per sequence, n_sel); den.sel_idx is filled as by den.step."""
        den = self.den
        if not (tokens.is_cuda and tokens.is_contiguous() and tokens.dtype == torch.int32
                and tuple(tokens.shape) == (den.B, den.n)):
            raise DllmcError("tokens must be a contiguous int32 [B, n] device tensor")
        n_rev, n_sel = C.c_int32(0), C.c_int32(0)
        _check(lib().dllmc_gen_step(self._h, tokens.data_ptr(), step_idx, den.sel_idx.data_ptr(),
                                    C.byref(n_sel), C.byref(n_rev)), "dllmc_gen_step")
        return n_rev.value, n_sel.value

    def read(self, hidden: bool = False):
        """(x0 [B, L_r] int32, conf [B, L_r] float32, chosen [B, L_r] int32[, hidden_out]) of the
        most recent step."""
        den = self.den
        x0 = torch.empty((den.B, den.L_r), dtype=torch.int32, device="cuda")
        conf = torch.empty((den.B, den.L_r), dtype=torch.float32, device="cuda")
        chosen = torch.empty((den.B, den.L_r), dtype=torch.int32, device="cuda")
        hout = torch.empty((den.B, den.n, den.d), dtype=den.torch_dtype, device="cuda") if hidden else None
        _check(lib().dllmc_gen_read(self._h, x0.data_ptr(), conf.data_ptr(), chosen.data_ptr(), _ptr(hout)),
               "dllmc_gen_read")
        return (x0, conf, chosen, hout) if hidden else (x0, conf, chosen)

    def close(self) -> None:
        if self._h is not None:
            h, self._h = self._h, None
            _check(lib().dllmc_gen_destroy(h), "dllmc_gen_destroy")

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def op_head(dtype: str, hidden: torch.Tensor, final_norm_g: torch.Tensor, lm_head: torch.Tensor,
            eps: float, rows: Optional[torch.Tensor] = None):
    """(x0 [M] int32, conf [M] float32) of the listed rows of hidden [*, d]."""
    d = hidden.shape[1]
    vocab = lm_head.shape[0]
    M = hidden.shape[0] if rows is None else rows.numel()
    code = _DTYPES[dtype][0]
    scratch = torch.empty(lib().dllmc_op_head_scratch_bytes(code, M, vocab, d), dtype=torch.uint8, device="cuda")
    x0 = torch.empty(M, dtype=torch.int32, device="cuda")
    conf = torch.empty(M, dtype=torch.float32, device="cuda")
    _check(lib().dllmc_op_head(code, hidden.data_ptr(), _ptr(rows), M, final_norm_g.data_ptr(), eps,
                               lm_head.data_ptr(), vocab, d, scratch.data_ptr(), x0.data_ptr(),
                               conf.data_ptr(), _stream_handle()), "dllmc_op_head")
    return x0, conf


def set_gemm_tuning(nw: int = -1, nw_dual: int = -1, force_s: int = -1, target_wg: int = -1,
                    tile_min_m: int = -1, fat_min_m: int = -1, tall_max_m: int = -1) -> None:
    _check(lib().dllmc_set_gemm_tuning(nw, nw_dual, force_s, target_wg, tile_min_m, fat_min_m,
                                       tall_max_m),
           "dllmc_set_gemm_tuning")


def op_select(scores: torch.Tensor, k: int) -> torch.Tensor:
    B, Lr = scores.shape
    out = torch.empty((B, max(k, 1)), dtype=torch.int32, device="cuda")
    _check(lib().dllmc_op_select(scores.data_ptr(), B, Lr, k, out.data_ptr(), _stream_handle()),
           "dllmc_op_select")
    return out[:, :k]


def op_vverify(dtype: str, h: torch.Tensor, wv: torch.Tensor, v_cache: torch.Tensor) -> torch.Tensor:
    """Scores [rows]; v_cache is overwritten with the new V rows."""
    rows, d = h.shape
    d_kv = wv.shape[0]
    scores = torch.empty(rows, dtype=torch.float32, device="cuda")
    scratch = torch.empty(rows * d_kv * 8, dtype=torch.float32, device="cuda")
    _check(lib().dllmc_op_vverify(_DTYPES[dtype][0], h.data_ptr(), wv.data_ptr(), v_cache.data_ptr(),
                                  scores.data_ptr(), rows, d, d_kv, scratch.data_ptr(),
                                  _stream_handle()), "dllmc_op_vverify")
    return scores


def op_linear(dtype: str, a: torch.Tensor, w: torch.Tensor, row_idx: Optional[torch.Tensor] = None) -> torch.Tensor:
    K = a.shape[1]
    N = w.shape[0]
    M = a.shape[0] if row_idx is None else row_idx.numel()
    out = torch.empty((M, N), dtype=torch.float32, device="cuda")
    scratch = torch.empty(M * N * 8, dtype=torch.float32, device="cuda")
    _check(lib().dllmc_op_linear_rows(_DTYPES[dtype][0], a.data_ptr(), a.shape[0], _ptr(row_idx), M, w.data_ptr(),
                                      N, K, out.data_ptr(), scratch.data_ptr(), _stream_handle()),
           "dllmc_op_linear_rows")
    return out


def op_linear_static(dtype: str, a: torch.Tensor, w: torch.Tensor, out: torch.Tensor,
                     row_idx: Optional[torch.Tensor] = None) -> torch.Tensor:
    """dllmc_op_linear_static into the caller's `out` (float32 [M, N]); allocates nothing."""
    M = a.shape[0] if row_idx is None else row_idx.numel()
    _check(lib().dllmc_op_linear_static(_DTYPES[dtype][0], a.data_ptr(), _ptr(row_idx), M, w.data_ptr(),
                                        w.shape[0], a.shape[1], out.data_ptr(), _stream_handle()),
           "dllmc_op_linear_static")
    return out


def op_attention(dtype: str, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                 H_q: int, H_kv: int, d_h: int, split_keys: bool = True) -> torch.Tensor:
    B, Mq, _ = q.shape
    n = k_cache.shape[1]
    # (the library takes sizes, not tensors: what is smaller than they say would be read past its end)
    for name, t, numel in (("q", q, B * Mq * H_q * d_h), ("k_cache", k_cache, B * n * H_kv * d_h), ("v_cache", v_cache, B * n * H_kv * d_h)):
        if t.numel() != numel or t.dtype is not _DTYPES[dtype][1] or not t.is_contiguous():
            raise DllmcError(f"op_attention: {name} has to be a contiguous {dtype} tensor of {numel} elements, got {t.dtype} {tuple(t.shape)}")
    if not (q.is_cuda and k_cache.is_cuda and v_cache.is_cuda):
        raise DllmcError("op_attention: the tensors have to be on the device")
    out = torch.empty_like(q)
    scratch = None
    if split_keys:
        scratch = torch.empty(lib().dllmc_op_attention_scratch_bytes(), dtype=torch.uint8, device="cuda")
    _check(lib().dllmc_op_attention(_DTYPES[dtype][0], q.data_ptr(), B, Mq, k_cache.data_ptr(),
                                    v_cache.data_ptr(), n, H_q, H_kv, d_h, out.data_ptr(),
                                    _ptr(scratch), _stream_handle()), "dllmc_op_attention")
    return out


# ---- the step's pieces in fewer bits ------------------------------------------------------------
def _device(name: str, t: torch.Tensor) -> int:
    """Index of the current device, which t has to be on."""
    d = t.get_device()  # (-1: host memory; a device tensor's runtime is up)
    if d < 0 or d != torch._C._cuda_getDevice():
        raise DllmcError(f"{name}: need a tensor on the current device, got one on {t.device}")
    return d


def _need(name: str, t: Optional[torch.Tensor], dtype: torch.dtype, shape: tuple, device: int) -> Optional[int]:
    """Address of a contiguous tensor of this device, dtype and shape (None stays None)."""
    if t is None:
        return None
    if t.get_device() != device or t.dtype is not dtype or t.shape != shape or not t.is_contiguous():
        raise DllmcError(f"{name}: need a contiguous {dtype} tensor of shape {tuple(shape)} on the current device, got "
                         f"{t.dtype} {tuple(t.shape)} on {t.device}{'' if t.is_contiguous() else ', not contiguous'}")
    return t.data_ptr()


@functools.lru_cache(maxsize=4096)
def _scratch_bytes(what: str, *shape: int) -> int:
    """dllmc_op_<what>_scratch_bytes, a function of its arguments alone (the choice of a kernel takes a microsecond or two)."""
    return getattr(lib(), f"dllmc_op_{what}_scratch_bytes")(*shape)


def _scratch(nbytes: int, like: torch.Tensor) -> Optional[torch.Tensor]:
    # (new_empty: 1.5 us, torch.empty with a device 1.7)
    return like.new_empty(nbytes, dtype=torch.uint8) if nbytes else None


def _need_cache(name: str, fmt: str, t: torch.Tensor, cache_rows: int, H: int, d_h: int, device: int) -> int:
    if fmt == "kv4":
        return _need(name, t, torch.uint8, (kv4_bytes(cache_rows, H, d_h),), device)
    return _need(name, t, _DTYPES[fmt][1], (cache_rows, H * d_h), device)


def _need_positions(n: int) -> None:
    # (no tensor's shape need say n, and the calls take 32 bits of it)
    if not 0 < n < 1 << 31:
        raise DllmcError(f"n: no {n} positions")


def _format(fmt: str) -> int:
    return DLLMC_KV4 if fmt == "kv4" else _DTYPES[fmt][0]


@functools.lru_cache(maxsize=1024)
def kv4_bytes(cache_rows: int, H: int, d_h: int) -> int:
    """Bytes of a 4-bit cache tensor (a uint8 tensor of that size holds it)."""
    n = lib().dllmc_kv4_bytes(cache_rows, H, d_h) if all(0 < v < 1 << 31 for v in (cache_rows, H, d_h)) else 0  # (of 32 bits)
    if n == 0:
        raise DllmcError(f"dllmc_kv4_bytes: no 4-bit tensor of {cache_rows} rows, {H} heads of {d_h}")
    return n


def op_kv4_store(dtype: str, x: torch.Tensor, cache: torch.Tensor, cache_rows: int, H: int, d_h: int,
                 rows: Optional[torch.Tensor] = None) -> None:
    """Rows of x [M, H * d_h] into rows `rows` (int32 [M], distinct; 0 .. M - 1 if None) of a 4-bit cache tensor."""
    M = x.shape[0]
    code, tdt = _DTYPES[dtype]
    dev = _device("x", x)
    _check(lib().dllmc_op_kv4_store(code, _need("x", x, tdt, (M, H * d_h), dev), M, _need("rows", rows, torch.int32, (M,), dev),
                                    _need_cache("cache", "kv4", cache, cache_rows, H, d_h, dev), cache_rows, H, d_h,
                                    _stream(dev)), "dllmc_op_kv4_store")


def op_kv4_load(dtype: str, cache: torch.Tensor, cache_rows: int, H: int, d_h: int,
                rows: Optional[torch.Tensor] = None) -> torch.Tensor:
    """[M, H * d_h]: the values of rows `rows` (int32 [M]; all if None) of a 4-bit cache tensor."""
    M = cache_rows if rows is None else rows.numel()
    code, tdt = _DTYPES[dtype]
    dev = _device("cache", cache)
    at = _need_cache("cache", "kv4", cache, cache_rows, H, d_h, dev)
    out = cache.new_empty((M, H * d_h), dtype=tdt)
    _check(lib().dllmc_op_kv4_load(code, at, cache_rows, H, d_h, _need("rows", rows, torch.int32, (M,), dev), M, out.data_ptr(),
                                   _stream(dev)), "dllmc_op_kv4_load")
    return out


def op_attention_kv4(dtype: str, q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor, cache_rows: int, n: int,
                     H_q: int, H_kv: int, d_h: int, lens: Optional[torch.Tensor] = None,
                     row_map: Optional[torch.Tensor] = None, with_lse: bool = False):
    """Attention rows [B, Mq, H_q * d_h] of q over a 4-bit cache, with with_lse also float32 [B, Mq, H_q] log-sum-exps.
    lens int32 [B]: keys of each sequence (n if None); row_map int32 [B, n]: cache row of each (b * n + j if None; an entry
    that is no row: no such key)."""
    code, tdt = _DTYPES[dtype]
    B, Mq = q.shape[:2]
    dev = _device("q", q)
    _need_positions(n)
    qp = _need("q", q, tdt, (B, Mq, H_q * d_h), dev)
    kp = _need_cache("k_cache", "kv4", k_cache, cache_rows, H_kv, d_h, dev)
    vp = _need_cache("v_cache", "kv4", v_cache, cache_rows, H_kv, d_h, dev)
    lp, rp = _need("lens", lens, torch.int32, (B,), dev), _need("row_map", row_map, torch.int32, (B, n), dev)
    out = torch.empty_like(q)
    lse = q.new_empty((B, Mq, H_q), dtype=torch.float32) if with_lse else None
    nbytes = _scratch_bytes("attention_kv4", code, B, Mq, n, H_q, H_kv, d_h)
    scratch = _scratch(nbytes, q)
    _check(lib().dllmc_op_attention_kv4(code, qp, B, Mq, kp, vp, cache_rows, rp, lp, n, H_q, H_kv, d_h, out.data_ptr(),
                                        _ptr(lse), _ptr(scratch), nbytes, _stream(dev)), "dllmc_op_attention_kv4")
    return (out, lse) if with_lse else out


def op_attention_weights(dtype: str, cache_format: str, q: torch.Tensor, k_cache: torch.Tensor, cache_rows: int, n: int,
                         H_q: int, H_kv: int, d_h: int, lens: Optional[torch.Tensor] = None,
                         row_map: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         acc: Optional[torch.Tensor] = None, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """float32 [B, n]: acc (0 if None) plus the attention weight that q gives to every cached position.  cache_format: the
    dtype, or "kv4".  lse: the rows' log-sum-exps over these operands (of op_attention_kv4 for "kv4"), if there are any.  out: where it
    goes (may be acc)."""
    code, tdt = _DTYPES[dtype]
    fmt = _format(cache_format)
    B, Mq = q.shape[:2]
    dev = _device("q", q)
    _need_positions(n)
    qp = _need("q", q, tdt, (B, Mq, H_q * d_h), dev)
    kp = _need_cache("k_cache", cache_format, k_cache, cache_rows, H_kv, d_h, dev)
    lp, rp = _need("lens", lens, torch.int32, (B,), dev), _need("row_map", row_map, torch.int32, (B, n), dev)
    sp, ap = _need("lse", lse, torch.float32, (B, Mq, H_q), dev), _need("acc", acc, torch.float32, (B, n), dev)
    if out is None:
        out = q.new_empty((B, n), dtype=torch.float32)
    op = _need("out", out, torch.float32, (B, n), dev)
    nbytes = _scratch_bytes("attention_weights", code, fmt, B, Mq, n, H_q, H_kv, d_h)
    scratch = _scratch(nbytes, q)
    _check(lib().dllmc_op_attention_weights(code, fmt, qp, B, Mq, kp, cache_rows, rp, lp, n, H_q, H_kv, d_h, sp, ap, op,
                                            _ptr(scratch), nbytes, _stream(dev)), "dllmc_op_attention_weights")
    return out


def op_evict(acc: torch.Tensor, keep: int, cache_rows: int, first: int = 0, last: int = 0,
             lens: Optional[torch.Tensor] = None, row_map: Optional[torch.Tensor] = None):
    """(kept [B, keep], kept_rows [B, keep], new_lens [B] int32, acc [B, keep] float32): the positions that stay, see
    dllmc_op_evict."""
    B, n = acc.shape
    dev = _device("acc", acc)
    if not (1 <= keep <= n and first >= 0 and last >= 0 and first + last <= keep and 1 <= cache_rows < 1 << 31):
        # (what is allocated goes by keep, and the call takes 32 bits of each)
        raise DllmcError(f"op_evict: cannot keep {keep} of {n} positions, the first {first} and last {last} among them, of a cache of "
                         f"{cache_rows} rows")
    ap = _need("acc", acc, torch.float32, (B, n), dev)
    lp, rp = _need("lens", lens, torch.int32, (B,), dev), _need("row_map", row_map, torch.int32, (B, n), dev)
    left = acc.new_empty((B, keep))
    kept = torch.empty_like(left, dtype=torch.int32)
    kept_rows, new_lens = torch.empty_like(kept), acc.new_empty(B, dtype=torch.int32)
    _check(lib().dllmc_op_evict(ap, B, n, lp, rp, cache_rows, keep, first, last, kept.data_ptr(), kept_rows.data_ptr(),
                                new_lens.data_ptr(), left.data_ptr(), _stream(dev)), "dllmc_op_evict")
    return kept, kept_rows, new_lens, left


def op_compact(cache_format: str, rows: torch.Tensor, src_rows: int, H: int, d_h: int, k_src: torch.Tensor,
               k_dst: torch.Tensor, v_src: Optional[torch.Tensor] = None, v_dst: Optional[torch.Tensor] = None,
               dst_rows: Optional[int] = None) -> None:
    """Row i of the destinations (dst_rows rows, as many as `rows` has if None) = row rows[i] of the sources; an entry that
    is no row leaves row i as it was.  rows: int32 of any shape, taken flat.  Formats: "f32", "bf16", "kv4"."""
    M = rows.numel()
    dst_rows = M if dst_rows is None else dst_rows
    dev = _device("rows", rows)
    rp = _need("rows", rows, torch.int32, rows.shape, dev)
    ks = _need_cache("k_src", cache_format, k_src, src_rows, H, d_h, dev)
    kd = _need_cache("k_dst", cache_format, k_dst, dst_rows, H, d_h, dev)
    vs = None if v_src is None else _need_cache("v_src", cache_format, v_src, src_rows, H, d_h, dev)
    vd = None if v_dst is None else _need_cache("v_dst", cache_format, v_dst, dst_rows, H, d_h, dev)
    _check(lib().dllmc_op_compact(_format(cache_format), rp, M, src_rows, dst_rows, H, d_h, ks, kd, vs, vd, _stream(dev)),
           "dllmc_op_compact")


@functools.lru_cache(maxsize=1024)
def i8_row_bytes(K: int) -> int:
    """Bytes of a row of K 8-bit integers: K rounded up to 128."""
    n = lib().dllmc_i8_row_bytes(K) if 0 < K < 1 << 31 else 0  # (of 32 bits)
    if n == 0:
        raise DllmcError(f"dllmc_i8_row_bytes: no 8-bit rows of {K}")
    return n


def plan_attention_kv4(dtype: str, B: int, Mq: int, n: int, H_q: int, H_kv: int, d_h: int):
    """(rows and wavefronts of a workgroup, key ranges, tiles that are not cut) of op_attention_kv4; no GPU needed."""
    rows, waves, whole = C.c_int32(), C.c_int32(), C.c_int32()
    ks = lib().dllmc_plan_attention_kv4(_DTYPES[dtype][0], B, Mq, n, H_q, H_kv, d_h, C.byref(rows), C.byref(waves), C.byref(whole))
    if ks < 1:
        raise DllmcError("dllmc_plan_attention_kv4: invalid argument")
    return rows.value, waves.value, ks, whole.value


def plan_attention_weights(dtype: str, cache_format: str, B: int, Mq: int, n: int, H_q: int, H_kv: int, d_h: int):
    """(keys a wavefront holds, key ranges of the row sums or 0 where one launch does both, their rows, row shares) of
    op_attention_weights; no GPU needed."""
    ranges, rows, shares = C.c_int32(), C.c_int32(), C.c_int32()
    keys = lib().dllmc_plan_attention_weights(_DTYPES[dtype][0], _format(cache_format), B, Mq, n, H_q, H_kv, d_h, C.byref(ranges),
                                              C.byref(rows), C.byref(shares))
    if keys < 1:
        raise DllmcError("dllmc_plan_attention_weights: invalid argument")
    return keys, ranges.value, rows.value, shares.value


def plan_linear_i8(M: int, N: int, K: int):
    """(rows, columns) of op_linear_i8's tiles, slices of the contraction, whether it takes the tile kernels; no GPU needed."""
    cols, slices, whole = C.c_int32(), C.c_int32(), C.c_int32()
    rows = lib().dllmc_plan_linear_i8(M, N, K, C.byref(cols), C.byref(slices), C.byref(whole))
    if rows < 1:
        raise DllmcError("dllmc_plan_linear_i8: invalid argument")
    return (rows, cols.value), slices.value, bool(whole.value)


def op_quant8(dtype: str, x: torch.Tensor, row_idx: Optional[torch.Tensor] = None):
    """(int8 [M, i8_row_bytes(K)], float32 [M]): rows of x [*, K] (those that row_idx int32 [M] names, zeros where it names none) and
    their scales."""
    code, tdt = _DTYPES[dtype]
    K = x.shape[1]
    M = x.shape[0] if row_idx is None else row_idx.numel()
    dev = _device("x", x)
    xp, rp = _need("x", x, tdt, x.shape, dev), _need("row_idx", row_idx, torch.int32, (M,), dev)
    q, scale = x.new_empty((M, i8_row_bytes(K)), dtype=torch.int8), x.new_empty(M, dtype=torch.float32)
    _check(lib().dllmc_op_quant8(code, xp, x.shape[0], rp, M, K, q.data_ptr(), scale.data_ptr(), _stream(dev)), "dllmc_op_quant8")
    return q, scale


def op_linear_i8(dtype: str, a: torch.Tensor, a_scale: torch.Tensor, w: torch.Tensor, w_scale: torch.Tensor,
                 K: int) -> torch.Tensor:
    """[M, N] of dtype: rows a times rows w (both as op_quant8 gives them, K integers each), scales multiplied in."""
    code, tdt = _DTYPES[dtype]
    M, N, kp = a.shape[0], w.shape[0], i8_row_bytes(K)
    dev = _device("a", a)
    ap, wp = _need("a", a, torch.int8, (M, kp), dev), _need("w", w, torch.int8, (N, kp), dev)
    sa, sw = _need("a_scale", a_scale, torch.float32, (M,), dev), _need("w_scale", w_scale, torch.float32, (N,), dev)
    out = a.new_empty((M, N), dtype=tdt)
    nbytes = _scratch_bytes("linear_i8", M, N, K)
    scratch = _scratch(nbytes, out)
    _check(lib().dllmc_op_linear_i8(code, ap, sa, M, wp, sw, N, K, out.data_ptr(), _ptr(scratch), nbytes, _stream(dev)),
           "dllmc_op_linear_i8")
    return out


def probe_copy(src: torch.Tensor, dst: torch.Tensor) -> None:
    """dst = src with the library's plain copy kernel (achievable-bandwidth probe)."""
    nbytes = src.numel() * src.element_size()
    if dst.numel() * dst.element_size() != nbytes:
        raise DllmcError("probe_copy: size mismatch")
    _check(lib().dllmc_probe_copy(src.data_ptr(), dst.data_ptr(), nbytes, _stream_handle()),
           "dllmc_probe_copy")


def probe_read(src: torch.Tensor, sink: torch.Tensor) -> None:
    _check(lib().dllmc_probe_read(src.data_ptr(), src.numel() * src.element_size(), sink.data_ptr(),
                                  _stream_handle()), "dllmc_probe_read")


def probe_mfma(iters: int, sink: torch.Tensor, shape: int = 0) -> float:
    """Enqueues the MFMA loop (shape 0: 16x16x32, 1: 32x32x16); returns the flops of the launch."""
    f = C.c_double(0.0)
    _check(lib().dllmc_probe_mfma(iters, shape, sink.data_ptr(), C.byref(f), _stream_handle()),
           "dllmc_probe_mfma")
    return f.value
