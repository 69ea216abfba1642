"""Thin ctypes binding of libsun (argument marshalling only; every step of the decode path
runs in the HIP kernels).  Function names follow include/sun.h.  PyTorch tensors are used
as device-memory owners; their data_ptr() is what crosses the boundary.

There is no CPU fallback: if the HIP library is missing the import of a function fails."""
from __future__ import annotations

import ctypes as C
import os
from typing import Dict, List, Optional, Sequence

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.environ.get("SUN_LIB_PATH", os.path.join(_HERE, "libsun.so"))  # override: another build of libsun

SUN_F32, SUN_BF16 = 0, 1
SUN_VALIDATE, SUN_PROFILE, SUN_SERVE_RESET = 1, 2, 4


def SUN_WAIT_POLLS(n: int) -> int:
    """Step flag for tests: a wait inside the launch of a small batch gives up after n polls."""
    return (n + 1) << 16


STATUS = {0: "SUN_OK", 1: "SUN_ERR_NULL", 2: "SUN_ERR_SHAPE", 3: "SUN_ERR_POOL_SIZE", 4: "SUN_ERR_WORKSPACE",
          5: "SUN_ERR_PAGE_RANGE", 6: "SUN_ERR_SEQ_LEN", 7: "SUN_ERR_MODEL_ID", 8: "SUN_ERR_HIP", 9: "SUN_ERR_TOKEN"}
PROFILE_KINDS = ("attn_split", "attn_combine", "qkv_proj", "o_proj", "gate_up_proj", "down_proj", "lm_head", "other")

EXPORTS = [
    "sun_kv_pool_bytes", "sun_kv_pool_create", "sun_kv_pool_layout", "sun_kv_pool_destroy",
    "sun_kv_pool_ingest", "sun_kv_pool_model_tokens",
    "sun_weights_pack_bytes", "sun_weights_create", "sun_weights_destroy",
    "sun_qweights_pack_bytes", "sun_qweights_create", "sun_quantize_w4",
    "sun_workspace_bytes", "sun_decode_step", "sun_qdecode_step", "sun_decode_run",
    "sun_prefill_workspace_bytes", "sun_prefill", "sun_serve_workspace_bytes", "sun_decode_serve",
    "sun_paged_attention", "sun_paged_attention_static", "sun_paged_attention_static_bytes",
    "sun_paged_attention_static_limit", "sun_linear",
    "sun_kv8_pool_bytes", "sun_kv8_pool_create", "sun_kv8_pool_layout", "sun_kv8_pool_destroy", "sun_kv8_append",
    "sun_kv8_attention", "sun_kv8_attention_workspace_bytes", "sun_kv8_attention_window_workspace_bytes",
    "sun_mx4_quantize", "sun_mx4_dequantize", "sun_mx4_linear", "sun_mx4_linear_workspace_bytes",
    "sun_hbm_read_probe", "sun_profile_read", "sun_profile_reset", "sun_last_error", "sun_version",
]


class ServeState(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("token_ids", "page_tables", "seq_lens", "model_ids", "slot_req", "slot_left",
                                          "w_req", "w_token", "w_tables", "w_lens", "w_model", "w_budget", "ring",
                                          "counters")] + \
               [(n, C.c_int32) for n in ("n_wait", "ring_cap", "idle_page", "eos_id")]


class SunError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS.get(status, status)}: {message}")
        self.status = status


class ModelCfg(C.Structure):
    _fields_ = [("n_layers", C.c_int32), ("hidden", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("ffn", C.c_int32), ("vocab", C.c_int32), ("rms_eps", C.c_float),
                ("rope_base", C.c_float), ("act_dtype", C.c_int32), ("qk_norm", C.c_int32), ("rope_scaling", C.c_int32),
                ("rope_original_max_position", C.c_int32), ("rope_factor", C.c_float),
                ("rope_low_freq_factor", C.c_float), ("rope_high_freq_factor", C.c_float), ("qkv_bias", C.c_int32)]


class KvLayout(C.Structure):
    _fields_ = [("n_pages", C.c_int64), ("page_tokens", C.c_int32), ("reserved", C.c_int32),
                ("k_off", C.c_int64), ("k_layer", C.c_int64), ("k_page", C.c_int64), ("k_head", C.c_int64),
                ("k_token", C.c_int64), ("k_dim", C.c_int64),
                ("v_off", C.c_int64), ("v_layer", C.c_int64), ("v_page", C.c_int64), ("v_head", C.c_int64),
                ("v_token", C.c_int64), ("v_dim", C.c_int64), ("total_elems", C.c_int64)]


class Kv8Layout(C.Structure):
    _fields_ = [("n_pages", C.c_int64), ("page_tokens", C.c_int32), ("reserved", C.c_int32)] + \
               [(n, C.c_int64) for n in ("k_off", "k_layer", "k_page", "k_head", "k_token", "k_dim",
                                         "v_off", "v_layer", "v_page", "v_head", "v_token", "v_dim",
                                         "ks_off", "vs_off", "s_layer", "s_page", "s_head", "total_bytes")]


class WeightPtrs(C.Structure):
    _fields_ = [("embed", C.c_void_p)] + [(k, C.POINTER(C.c_void_p)) for k in
                                          ("g1", "wq", "wk", "wv", "wo", "g2", "wg", "wu", "wd")] + \
               [("gf", C.c_void_p), ("wlm", C.c_void_p), ("q_norm", C.POINTER(C.c_void_p)), ("k_norm", C.POINTER(C.c_void_p)),
                ("bq", C.POINTER(C.c_void_p)), ("bk", C.POINTER(C.c_void_p)), ("bv", C.POINTER(C.c_void_p))]


class QMat(C.Structure):
    _fields_ = [("q", C.c_void_p), ("s", C.c_void_p), ("z", C.c_void_p)]


class QWeightPtrs(C.Structure):
    _fields_ = [("embed", C.c_void_p), ("g1", C.POINTER(C.c_void_p)),
                ("wq", C.POINTER(QMat)), ("wk", C.POINTER(QMat)), ("wv", C.POINTER(QMat)), ("wo", C.POINTER(QMat)),
                ("g2", C.POINTER(C.c_void_p)),
                ("wg", C.POINTER(QMat)), ("wu", C.POINTER(QMat)), ("wd", C.POINTER(QMat)),
                ("gf", C.c_void_p), ("wlm", C.c_void_p),
                ("q_norm", C.POINTER(C.c_void_p)), ("k_norm", C.POINTER(C.c_void_p)),
                ("bq", C.POINTER(C.c_void_p)), ("bk", C.POINTER(C.c_void_p)), ("bv", C.POINTER(C.c_void_p))]


_lib = None


def lib() -> C.CDLL:
    """Loads the in-tree HIP library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} is missing: build it with `python -m paper_2603_02599_amd.build`")
        L = C.CDLL(LIB_PATH)
        L.sun_last_error.restype = C.c_char_p
        L.sun_version.restype = C.c_char_p
        for f in ("sun_kv_pool_bytes", "sun_weights_pack_bytes", "sun_qweights_pack_bytes", "sun_workspace_bytes",
                  "sun_prefill_workspace_bytes", "sun_serve_workspace_bytes", "sun_paged_attention_static_bytes",
                  "sun_paged_attention_static_limit", "sun_kv8_pool_bytes", "sun_kv8_attention_workspace_bytes",
                  "sun_kv8_attention_window_workspace_bytes", "sun_mx4_linear_workspace_bytes"):
            getattr(L, f).restype = C.c_size_t
        L.sun_kv_pool_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int64, C.c_int]
        L.sun_kv_pool_create.argtypes = [C.POINTER(ModelCfg), C.c_void_p, C.c_size_t, C.c_int, C.c_int,
                                         C.POINTER(C.c_void_p)]
        L.sun_kv_pool_layout.argtypes = [C.c_void_p, C.POINTER(KvLayout)]
        L.sun_kv_pool_destroy.argtypes = [C.c_void_p]
        L.sun_kv_pool_destroy.restype = None
        L.sun_weights_pack_bytes.argtypes = [C.POINTER(ModelCfg)]
        L.sun_weights_create.argtypes = [C.POINTER(ModelCfg), C.POINTER(WeightPtrs), C.c_void_p, C.c_size_t,
                                         C.c_void_p, C.POINTER(C.c_void_p)]
        L.sun_weights_destroy.argtypes = [C.c_void_p]
        L.sun_weights_destroy.restype = None
        L.sun_qweights_pack_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int]
        L.sun_qweights_create.argtypes = [C.POINTER(ModelCfg), C.POINTER(QWeightPtrs), C.c_int, C.c_void_p,
                                          C.c_size_t, C.c_void_p, C.POINTER(C.c_void_p)]
        L.sun_quantize_w4.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_int, C.c_int, C.c_void_p,
                                      C.c_void_p, C.c_void_p, C.c_void_p]
        L.sun_kv_pool_ingest.argtypes = [C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p,
                                         C.c_int, C.c_void_p, C.c_uint]
        L.sun_kv_pool_model_tokens.argtypes = [C.c_void_p, C.c_int, C.POINTER(C.c_int64)]
        L.sun_workspace_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
        step_args = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p,
                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint]
        L.sun_decode_step.argtypes = step_args
        L.sun_qdecode_step.argtypes = step_args
        L.sun_decode_run.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint]
        L.sun_serve_workspace_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
        L.sun_decode_serve.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.POINTER(ServeState),
                                       C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint]
        L.sun_prefill_workspace_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
        L.sun_prefill.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int,
                                  C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint]
        L.sun_paged_attention.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                          C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.sun_paged_attention_static.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int,
                                                 C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sun_paged_attention_static_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
        L.sun_paged_attention_static_limit.argtypes = []
        L.sun_linear.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_size_t, C.c_void_p]
        L.sun_kv8_pool_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int64, C.c_int]
        L.sun_kv8_pool_create.argtypes = [C.POINTER(ModelCfg), C.c_void_p, C.c_size_t, C.c_int, C.POINTER(C.c_void_p)]
        L.sun_kv8_pool_layout.argtypes = [C.c_void_p, C.POINTER(Kv8Layout)]
        L.sun_kv8_pool_destroy.argtypes = [C.c_void_p]
        L.sun_kv8_pool_destroy.restype = None
        L.sun_kv8_append.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                     C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_void_p,
                                     C.c_void_p, C.c_void_p, C.c_void_p, C.c_uint]
        L.sun_kv8_attention_workspace_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int]
        L.sun_kv8_attention_window_workspace_bytes.argtypes = [C.POINTER(ModelCfg), C.c_int, C.c_int, C.c_int]
        L.sun_kv8_attention.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_int, C.c_void_p,
                                        C.c_int, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p, C.c_uint]
        L.sun_mx4_quantize.argtypes = [C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p, C.c_void_p]
        L.sun_mx4_dequantize.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
        L.sun_mx4_linear_workspace_bytes.argtypes = [C.c_int, C.c_int, C.c_int]
        L.sun_mx4_linear.argtypes = [C.c_void_p, C.c_void_p, C.c_int, C.c_int, C.c_int, C.c_void_p, C.c_int, C.c_int64,
                                     C.c_void_p, C.c_int, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
        L.sun_hbm_read_probe.argtypes = [C.c_void_p, C.c_size_t, C.c_int, C.c_void_p, C.c_int, C.c_int, C.c_void_p, C.c_void_p]
        L.sun_profile_read.argtypes = [C.c_int, C.POINTER(C.c_double), C.POINTER(C.c_int64)]
        L.sun_profile_reset.restype = None
        _lib = L
    return _lib


def _check(rc: int):
    if rc != 0:
        raise SunError(rc, lib().sun_last_error().decode())


def _p(t) -> Optional[int]:
    if t is None:
        return None
    if isinstance(t, torch.Tensor):
        assert t.is_contiguous()
        return t.data_ptr()
    return int(t)


def _stream(stream) -> Optional[int]:
    if stream is None:
        return torch.cuda.current_stream().cuda_stream
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _aside(device, stream, shape, dtype) -> torch.Tensor:
    """An empty tensor of the pool of `stream`, which is about to fill it.  A block of the current stream's pool may still be read by work that is
    queued there.  Nor is it handed out again before what the current stream, whose work may use it, has queued by then is done."""
    here = torch.cuda.current_stream(device)
    with torch.cuda.stream(torch.cuda.ExternalStream(_stream(stream), device=device)):
        t = torch.empty(shape, dtype=dtype, device=device)
    t.record_stream(here)
    return t


def _pack_buffer(cfg: ModelCfg, nbytes: int, device, stream) -> Optional[torch.Tensor]:
    if cfg.act_dtype != SUN_BF16:
        return None
    n = max(nbytes, 256)
    return torch.empty(n, dtype=torch.uint8, device=device) if stream is None else _aside(device, stream, n, torch.uint8)


def make_cfg(shape, act_dtype: str) -> ModelCfg:
    """shape: object with n_layers, hidden, n_q_heads, n_kv_heads, head_dim, ffn, vocab, rms_eps, rope_base and
    optionally qk_norm (bool), qkv_bias (bool) and rope_scaling = (factor, low_freq_factor, high_freq_factor, original_max_position)."""
    rs = getattr(shape, "rope_scaling", None)
    return ModelCfg(shape.n_layers, shape.hidden, shape.n_q_heads, shape.n_kv_heads, shape.head_dim, shape.ffn,
                    shape.vocab, float(shape.rms_eps), float(shape.rope_base),
                    {"f32": SUN_F32, "bf16": SUN_BF16}[act_dtype], int(bool(getattr(shape, "qk_norm", False))),
                    1 if rs else 0, int(rs[3]) if rs else 0, float(rs[0]) if rs else 0.0, float(rs[1]) if rs else 0.0,
                    float(rs[2]) if rs else 0.0, int(bool(getattr(shape, "qkv_bias", False))))


# ------------------------------------------------------------------ pool
def sun_kv_pool_bytes(cfg: ModelCfg, n_pages: int, page_tokens: int = 16) -> int:
    return int(lib().sun_kv_pool_bytes(C.byref(cfg), n_pages, page_tokens))


class KvPool:
    """Owner of the pool handle; `mem` (a torch uint8/bf16 CUDA tensor) is borrowed and kept alive."""

    def __init__(self, handle: int, mem: torch.Tensor):
        self.handle, self.mem = handle, mem

    def layout(self) -> KvLayout:
        return sun_kv_pool_layout(self)

    def __del__(self):
        # at interpreter shutdown the module globals may already be gone; the handle is host memory only
        if getattr(self, "handle", None) and _lib is not None:
            _lib.sun_kv_pool_destroy(self.handle)
            self.handle = None


def sun_kv_pool_create(cfg: ModelCfg, mem: torch.Tensor, page_tokens: int = 16, n_source_models: int = 1) -> KvPool:
    out = C.c_void_p()
    nbytes = mem.numel() * mem.element_size() if isinstance(mem, torch.Tensor) else 0
    _check(lib().sun_kv_pool_create(C.byref(cfg), _p(mem), nbytes, page_tokens, n_source_models, C.byref(out)))
    return KvPool(out.value, mem)


def sun_kv_pool_layout(pool: KvPool) -> KvLayout:
    lay = KvLayout()
    _check(lib().sun_kv_pool_layout(pool.handle, C.byref(lay)))
    return lay


# ------------------------------------------------------------------ weights
LAYER_KEYS = ("g1", "wq", "wk", "wv", "wo", "g2", "wg", "wu", "wd")
QUANT_KEYS = ("wq", "wk", "wv", "wo", "wg", "wu", "wd")


class Weights:
    def __init__(self, handle: int, keep: list, quant: bool):
        self.handle, self.keep, self.quant = handle, keep, quant

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.sun_weights_destroy(self.handle)
            self.handle = None


def _ptr_array(tensors: Sequence[torch.Tensor]):
    arr = (C.c_void_p * len(tensors))(*[t.data_ptr() for t in tensors])
    return arr


def _set_head_norms(ptrs, w, cfg: ModelCfg, keep: List[object]):
    """Per-layer vectors of the backbone options: head-norm gains (w["qn"], w["kn"]) and projection biases
    (w["bq"], w["bk"], w["bv"])."""
    fields = ((("q_norm", "qn"), ("k_norm", "kn")) if cfg.qk_norm else ()) + \
             ((("bq", "bq"), ("bk", "bk"), ("bv", "bv")) if cfg.qkv_bias else ())
    for field, key in fields:
        arr = _ptr_array(w[key])
        keep.extend([arr, w[key]])
        setattr(ptrs, field, C.cast(arr, C.POINTER(C.c_void_p)))


def sun_weights_pack_bytes(cfg: ModelCfg) -> int:
    return int(lib().sun_weights_pack_bytes(C.byref(cfg)))


def sun_weights_create(cfg: ModelCfg, w: Dict[str, object], stream=None, keep_sources: bool = True) -> Weights:
    """w: dict from workloads.make_weights (torch CUDA tensors).  Allocates the pack buffer with torch, from the pool of the stream that packs."""
    ptrs = WeightPtrs()
    keep: List[object] = []
    ptrs.embed = w["embed"].data_ptr()
    for k in LAYER_KEYS:
        arr = _ptr_array(w[k])
        keep.append(arr)
        setattr(ptrs, k, C.cast(arr, C.POINTER(C.c_void_p)))
    ptrs.gf, ptrs.wlm = w["gf"].data_ptr(), w["wlm"].data_ptr()
    _set_head_norms(ptrs, w, cfg, keep)
    nbytes = sun_weights_pack_bytes(cfg)
    pack = _pack_buffer(cfg, nbytes, w["embed"].device, stream)
    out = C.c_void_p()
    _check(lib().sun_weights_create(C.byref(cfg), C.byref(ptrs), _p(pack), nbytes, _stream(stream), C.byref(out)))
    keep.append(pack)
    if keep_sources or cfg.act_dtype == SUN_F32:
        keep.append(w)
    else:
        keep.extend([w["embed"], w["g1"], w["g2"], w["gf"], w.get("qn"), w.get("kn")])
    return Weights(out.value, keep, False)


def sun_qweights_pack_bytes(cfg: ModelCfg, group: int = 128) -> int:
    return int(lib().sun_qweights_pack_bytes(C.byref(cfg), group))


def sun_qweights_create(cfg: ModelCfg, w: Dict[str, object], quant: Dict[str, list], group: int = 128,
                        stream=None) -> Weights:
    """quant[key][layer] = (q uint8 [out, in/2], s fp16 [out, in/128], z fp16 [out, in/128]) CUDA tensors;
    w supplies embed, g1, g2, gf, wlm.  The pack buffer is from the pool of the stream that packs."""
    ptrs = QWeightPtrs()
    keep: List[object] = [w["embed"], w["g1"], w["g2"], w["gf"], w["wlm"], quant]
    ptrs.embed = w["embed"].data_ptr()
    for k in ("g1", "g2"):
        arr = _ptr_array(w[k])
        keep.append(arr)
        setattr(ptrs, k, C.cast(arr, C.POINTER(C.c_void_p)))
    for k in QUANT_KEYS:
        arr = (QMat * len(quant[k]))(*[QMat(q.data_ptr(), s.data_ptr(), z.data_ptr() if z is not None else None)
                                       for (q, s, z) in quant[k]])
        keep.append(arr)
        setattr(ptrs, k, C.cast(arr, C.POINTER(QMat)))
    ptrs.gf, ptrs.wlm = w["gf"].data_ptr(), w["wlm"].data_ptr()
    _set_head_norms(ptrs, w, cfg, keep)
    nbytes = sun_qweights_pack_bytes(cfg, group)
    pack = _pack_buffer(cfg, nbytes, w["embed"].device, stream)
    out = C.c_void_p()
    _check(lib().sun_qweights_create(C.byref(cfg), C.byref(ptrs), group, _p(pack), nbytes, _stream(stream), C.byref(out)))
    keep.append(pack)
    return Weights(out.value, keep, True)


def sun_quantize_w4(w: torch.Tensor, group: int = 128, mode: str = "asym", stream=None):
    """Returns (q uint8 [rows, cols/2], s fp16 [rows, cols/group], z fp16 [rows, cols/group]); mode "sym_noz" is
    the symmetric grid without stored zero points (z is None: 8 everywhere).  They belong to the stream that fills them."""
    rows, cols = w.shape
    dt = {torch.float32: SUN_F32, torch.bfloat16: SUN_BF16}[w.dtype]
    new = (lambda shape, t: torch.empty(shape, dtype=t, device=w.device)) if stream is None else (lambda shape, t: _aside(w.device, stream, shape, t))
    q, s = new((rows, cols // 2), torch.uint8), new((rows, cols // group), torch.float16)
    z = new(s.shape, torch.float16) if mode != "sym_noz" else None
    _check(lib().sun_quantize_w4(_p(w), dt, rows, cols, group, {"asym": 0, "sym": 1, "sym_noz": 1}[mode], _p(q), _p(s),
                                 _p(z), _stream(stream)))
    return q, s, z


# ------------------------------------------------------------------ step
def sun_workspace_bytes(cfg: ModelCfg, max_batch: int, max_pages: int) -> int:
    return int(lib().sun_workspace_bytes(C.byref(cfg), max_batch, max_pages))


def _host_i32(a):
    if a is None:
        return None, None
    import numpy as np
    arr = np.ascontiguousarray(a, dtype=np.int32)
    return arr, arr.ctypes.data


def _step(fn, pool, weights, token_ids, page_tables, seq_lens, model_ids, logits_out, next_tokens_out, workspace,
          seq_lens_host, stream, flags):
    batch, max_pages = page_tables.shape
    keep, host_ptr = _host_i32(seq_lens_host)
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(fn(pool.handle if pool is not None else None, weights.handle if weights is not None else None, batch,
              _p(token_ids), _p(page_tables), max_pages, _p(seq_lens), host_ptr, _p(model_ids), _p(logits_out),
              _p(next_tokens_out), _p(workspace), ws_bytes, _stream(stream), flags))


def sun_decode_step(pool, weights, token_ids, page_tables, seq_lens, model_ids, logits_out, next_tokens_out,
                    workspace, seq_lens_host=None, stream=None, flags: int = 0):
    _step(lib().sun_decode_step, pool, weights, token_ids, page_tables, seq_lens, model_ids, logits_out,
          next_tokens_out, workspace, seq_lens_host, stream, flags)


def sun_qdecode_step(pool, weights, token_ids, page_tables, seq_lens, model_ids, logits_out, next_tokens_out,
                     workspace, seq_lens_host=None, stream=None, flags: int = 0):
    _step(lib().sun_qdecode_step, pool, weights, token_ids, page_tables, seq_lens, model_ids, logits_out,
          next_tokens_out, workspace, seq_lens_host, stream, flags)


def sun_kv_pool_ingest(pool, model_id: int, k_src, v_src, first_pos: int, page_table_row, stream=None, flags: int = 0):
    """k_src, v_src: bf16 tensors [n_layers, n_tokens, n_kv_heads, head_dim]; page_table_row: int32 [max_pages]."""
    _check(lib().sun_kv_pool_ingest(pool.handle, model_id, _p(k_src), _p(v_src), int(k_src.shape[1]), first_pos,
                                    _p(page_table_row), int(page_table_row.numel()), _stream(stream), flags))


def sun_kv_pool_model_tokens(pool, model_id: int) -> int:
    n = C.c_int64()
    _check(lib().sun_kv_pool_model_tokens(pool.handle, model_id, C.byref(n)))
    return int(n.value)


def sun_decode_run(pool, weights, n_steps: int, token_ids, page_tables, seq_lens, model_ids, free_pages, free_head,
                   run_status, tokens_out, logits_out, workspace, stream=None, flags: int = 0):
    """n_steps greedy steps in a row; token_ids, page_tables, seq_lens and free_head are updated on the device."""
    batch, max_pages = page_tables.shape
    n_free = int(free_pages.numel()) if free_pages is not None else 0
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    _check(lib().sun_decode_run(pool.handle if pool is not None else None,
                                weights.handle if weights is not None else None, batch, n_steps, _p(token_ids),
                                _p(page_tables), max_pages, _p(seq_lens), _p(model_ids), _p(free_pages), n_free,
                                _p(free_head), _p(run_status), _p(tokens_out), _p(logits_out), _p(workspace), ws_bytes,
                                _stream(stream), flags))


def sun_serve_workspace_bytes(cfg: ModelCfg, slots: int, max_pages: int) -> int:
    return int(lib().sun_serve_workspace_bytes(C.byref(cfg), slots, max_pages))


class ServeTensors:
    """Device tensors of a continuous-batching decode worker (the fields of sun_serve_state), kept alive
    together with the struct handed to the library."""

    def __init__(self, slots: int, max_pages: int, waiting, ring_pages, ring_cap: int, idle_page: int,
                 eos_id: int = -1, device="cuda"):
        import torch
        i32 = dict(dtype=torch.int32, device=device)
        self.slots, self.max_pages = slots, max_pages
        self.token_ids = torch.zeros(slots, **i32)
        self.page_tables = torch.full((slots, max_pages), -1, **i32)
        self.seq_lens = torch.zeros(slots, **i32)
        self.model_ids = torch.zeros(slots, **i32)
        self.slot_req = torch.full((slots,), -1, **i32)
        self.slot_left = torch.zeros(slots, **i32)
        n = len(waiting["req"])
        self.n_wait = n
        self.w = {k: torch.as_tensor(waiting[k], dtype=torch.int32).to(device).contiguous()
                  for k in ("req", "token", "tables", "lens", "model", "budget")}
        assert self.w["tables"].shape == (n, max_pages) or n == 0
        ring = torch.zeros(ring_cap, **i32)
        ring[:len(ring_pages)] = torch.as_tensor(ring_pages, dtype=torch.int32)
        self.ring, self.ring_cap = ring, ring_cap
        self.counters = torch.zeros(8, **i32)
        self.counters[2] = len(ring_pages)
        self.idle_page, self.eos_id = idle_page, eos_id

    def struct(self) -> "ServeState":
        s = ServeState()
        for name in ("token_ids", "page_tables", "seq_lens", "model_ids", "slot_req", "slot_left", "ring", "counters"):
            setattr(s, name, _p(getattr(self, name)))
        for k in ("req", "token", "tables", "lens", "model", "budget"):
            setattr(s, "w_" + k, _p(self.w[k]) if self.n_wait else None)
        s.n_wait, s.ring_cap, s.idle_page, s.eos_id = self.n_wait, self.ring_cap, self.idle_page, self.eos_id
        return s


def sun_decode_serve(pool, weights, n_steps: int, state: ServeTensors, tokens_out, req_out, logits_out, workspace,
                     stream=None, flags: int = 0):
    """n_steps iterations of decode + retire/advance/admit on the device; `state` is updated in place."""
    st = state.struct()
    _check(lib().sun_decode_serve(pool.handle, weights.handle, state.slots, state.max_pages, n_steps, C.byref(st),
                                  _p(tokens_out), _p(req_out), _p(logits_out), _p(workspace),
                                  workspace.numel() * workspace.element_size(), _stream(stream), flags))


def sun_prefill_workspace_bytes(cfg: ModelCfg, n_tokens: int, max_pages: int) -> int:
    return int(lib().sun_prefill_workspace_bytes(C.byref(cfg), n_tokens, max_pages))


def sun_prefill(pool, weights, token_ids, page_table_row, first_pos: int, model_id: int, logits_out, next_token_out,
                workspace, stream=None, flags: int = 0):
    """Causal forward of `weights` over the prompt tokens (int32 [n_tokens]) of one request; fills its pages."""
    ws_bytes = workspace.numel() * workspace.element_size() if workspace is not None else 0
    n_tokens = int(token_ids.numel()) if token_ids is not None else 0
    max_pages = int(page_table_row.numel()) if page_table_row is not None else 0
    _check(lib().sun_prefill(pool.handle if pool is not None else None,
                             weights.handle if weights is not None else None, n_tokens, _p(token_ids),
                             _p(page_table_row), max_pages, first_pos, model_id, _p(logits_out), _p(next_token_out),
                             _p(workspace), ws_bytes, _stream(stream), flags))


def sun_paged_attention(pool, layer: int, q, page_tables, n_tokens, out, workspace, n_tokens_host=None, stream=None):
    batch, max_pages = page_tables.shape
    keep, host_ptr = _host_i32(n_tokens_host)
    _check(lib().sun_paged_attention(pool.handle, layer, batch, _p(q), _p(page_tables), max_pages, _p(n_tokens),
                                     host_ptr, _p(out), _p(workspace), workspace.numel() * workspace.element_size(),
                                     _stream(stream)))


def sun_paged_attention_static(pool, layer: int, q, page_tables, n_tokens, out, n_tokens_host=None, stream=None):
    batch, max_pages = page_tables.shape
    keep, host_ptr = _host_i32(n_tokens_host)
    _check(lib().sun_paged_attention_static(pool.handle, layer, batch, _p(q), _p(page_tables), max_pages, _p(n_tokens),
                                            host_ptr, _p(out), _stream(stream)))


def sun_paged_attention_static_bytes(cfg, batch: int, max_pages: int) -> int:
    return int(lib().sun_paged_attention_static_bytes(C.byref(cfg), batch, max_pages))


def sun_paged_attention_static_limit() -> int:
    return int(lib().sun_paged_attention_static_limit())


def sun_linear(weights, layer: int, mat: int, x, out, workspace, stream=None):
    _check(lib().sun_linear(weights.handle, layer, mat, x.shape[0], _p(x), _p(out), _p(workspace),
                            workspace.numel() * workspace.element_size(), _stream(stream)))


# ------------------------------------------------------------------ 8-bit cache, microscaled 4-bit floats
# Tensors of these calls live on one GPU, which need not be the current one: the work goes to that GPU's current stream unless
# `stream` names another.  Wrong types, shapes and strides raise SunError (SUN_ERR_SHAPE) before anything is enqueued.
_DTYPES = {torch.float32: SUN_F32, torch.bfloat16: SUN_BF16}


def _refuse(message: str):
    raise SunError(2, message)


def _dtype(t: torch.Tensor, name: str) -> int:
    dt = _DTYPES.get(t.dtype)
    if dt is None:
        _refuse(f"{name} must be float32 or bfloat16, is {t.dtype}")
    return dt


def _want(name: str, t: torch.Tensor, device: int, dtype, shape, rows: bool = False) -> int:
    """The address of a tensor of this type and shape on GPU `device`: contiguous, or with rows any stride between rows."""
    if t.dtype is dtype and t.shape == shape and t.get_device() == device and (t.is_contiguous() or (rows and t.stride(1) == 1)):
        return t.data_ptr()
    _refuse(f"{name} must be {dtype} {tuple(shape)} on GPU {device}, " + ("contiguous within a row" if rows else "contiguous")
            + f"; is {t.dtype} {tuple(t.shape)} on {t.device}, strides {t.stride()}")


def _row_stride(t: torch.Tensor) -> int:
    rows, cols = t.shape
    return t.stride(0) if rows > 1 else cols


def _workspace(t: torch.Tensor, device: int):
    if t.get_device() != device or not t.is_contiguous():
        _refuse(f"workspace must be contiguous and on GPU {device}")
    return t.data_ptr(), t.numel() * t.element_size()


def _gpu(t: torch.Tensor) -> int:
    device = t.get_device()
    if device < 0:
        _refuse(f"tensors must be on a GPU, are on {t.device}")
    return device


def _table(page_tables: torch.Tensor):
    if page_tables.dim() != 2:
        _refuse("page_tables must be [requests, max_pages]")
    return page_tables.shape


# torch.cuda.current_stream(), an object, takes longer than a launch.  A torch build without GPUs has neither name, nor tensors that get as far.
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)
_current_gpu = getattr(torch._C, "_cuda_getDevice", None)


def _int32(**values):
    """Counts that the library takes in 32 bits, which a conversion would cut without a word."""
    for name, v in values.items():
        if not -1 << 31 <= v < 1 << 31:
            _refuse(f"{name} = {v} is beyond 32 bits")


def _fits(*values) -> bool:
    return all(-1 << 31 <= v < 1 << 31 for v in values)


def _call(device: int, stream, fn, args, behind=()):
    """fn(*args, stream, *behind) with GPU `device` current."""
    if device != _current_gpu():
        with torch.cuda.device(device):
            return _call(device, stream, fn, args, behind)
    rc = fn(*args, _raw_stream(device) if stream is None else _stream(stream), *behind)
    if rc:
        _check(rc)


def sun_kv8_pool_bytes(cfg: ModelCfg, n_pages: int, page_tokens: int = 16) -> int:
    return int(lib().sun_kv8_pool_bytes(C.byref(cfg), n_pages, page_tokens)) if _fits(page_tokens) else 0


class Kv8Pool:
    """Owner of the handle of an 8-bit pool; `mem` (a torch uint8 tensor on the GPU) is borrowed and kept alive."""

    def __init__(self, handle: int, mem: torch.Tensor, cfg: ModelCfg):
        self.handle, self.mem, self.cfg = handle, mem, cfg
        self.head_dim, self.q_dim, self.kv_dim = cfg.head_dim, cfg.n_q_heads * cfg.head_dim, cfg.n_kv_heads * cfg.head_dim

    def layout(self) -> Kv8Layout:
        return sun_kv8_pool_layout(self)

    def __del__(self):
        if getattr(self, "handle", None) and _lib is not None:
            _lib.sun_kv8_pool_destroy(self.handle)
            self.handle = None


def sun_kv8_pool_create(cfg: ModelCfg, mem: torch.Tensor, page_tokens: int = 16) -> Kv8Pool:
    out = C.c_void_p()
    nbytes = mem.numel() * mem.element_size() if isinstance(mem, torch.Tensor) else 0
    _check(lib().sun_kv8_pool_create(C.byref(cfg), _p(mem), nbytes, page_tokens, C.byref(out)))
    kept = ModelCfg()
    C.pointer(kept)[0] = cfg
    return Kv8Pool(out.value, mem, kept)


def sun_kv8_pool_layout(pool: Kv8Pool) -> Kv8Layout:
    lay = Kv8Layout()
    _check(lib().sun_kv8_pool_layout(pool.handle, C.byref(lay)))
    return lay


def sun_kv8_append(pool: Kv8Pool, layer: int, q, k, v, positions, requests, page_tables, q_out, q_norm=None, k_norm=None,
                   stream=None, flags: int = 0):
    """k, v [rows, Hkv*d] (and q [rows, Hq*d], or None with q_out None), rows at any stride; positions, requests int32 [rows];
    page_tables int32 [n_requests, max_pages]; gains [d] of the same type as q, k and v."""
    dev, t, i32, kd = _gpu(pool.mem), k.dtype, torch.int32, pool.kv_dim
    if k.dim() != 2:
        _refuse("k must be [rows, Hkv*d]")
    rows, (n_requests, max_pages) = k.shape[0], _table(page_tables)
    _int32(layer=layer, rows=rows, n_requests=n_requests)
    if q is None:
        pq = lq = None
    else:
        pq, lq = _want("q", q, dev, t, (rows, pool.q_dim), True), _row_stride(q)
    _call(dev, stream, lib().sun_kv8_append, (
        pool.handle, layer, rows, _dtype(k, "k"), pq, lq or 0, _want("k", k, dev, t, (rows, kd), True), _row_stride(k),
        _want("v", v, dev, t, (rows, kd), True), _row_stride(v), _want("positions", positions, dev, i32, (rows,)),
        _want("requests", requests, dev, i32, (rows,)), _want("page_tables", page_tables, dev, i32, (n_requests, max_pages)), n_requests, max_pages,
        None if q_norm is None else _want("q_norm", q_norm, dev, t, (pool.head_dim,)),
        None if k_norm is None else _want("k_norm", k_norm, dev, t, (pool.head_dim,)),
        None if q_out is None else _want("q_out", q_out, dev, t, (rows, pool.q_dim))), (flags,))


def sun_kv8_attention_workspace_bytes(cfg: ModelCfg, batch: int, max_pages: int) -> int:
    return int(lib().sun_kv8_attention_workspace_bytes(C.byref(cfg), batch, max_pages)) if _fits(batch, max_pages) else 0


def sun_kv8_attention_window_workspace_bytes(cfg: ModelCfg, batch: int, max_pages: int, window: int) -> int:
    """For calls with a window in [1, window] alone (0: any)."""
    return int(lib().sun_kv8_attention_window_workspace_bytes(C.byref(cfg), batch, max_pages, window)) if _fits(batch, max_pages, window) else 0


def sun_kv8_attention(pool: Kv8Pool, layer: int, q, page_tables, n_tokens, out, workspace, window: int = 0, stream=None,
                      flags: int = 0):
    """q, out [batch, Hq*d]; page_tables int32 [batch, max_pages]; n_tokens int32 [batch]."""
    dev, t, i32 = _gpu(pool.mem), q.dtype, torch.int32
    batch, max_pages = _table(page_tables)
    shape = (batch, pool.q_dim)
    _int32(layer=layer, max_pages=max_pages, window=window)
    _call(dev, stream, lib().sun_kv8_attention, (
        pool.handle, layer, batch, _dtype(q, "q"), _want("q", q, dev, t, shape), _want("page_tables", page_tables, dev, i32, (batch, max_pages)),
        max_pages, _want("n_tokens", n_tokens, dev, i32, (batch,)), window, _want("out", out, dev, t, shape), *_workspace(workspace, dev)), (flags,))


def sun_mx4_quantize(w: torch.Tensor, stream=None):
    """Returns (codes uint8 [rows, cols/2], scales uint8 [rows, cols/32]), which belong to the stream that fills them."""
    if w.dim() != 2 or w.shape[1] % 32:
        _refuse("w must be [rows, cols], cols a multiple of 32")
    (rows, cols), dev = w.shape, _gpu(w)
    _int32(rows=rows, cols=cols)
    if stream is None:
        codes, scales = w.new_empty((rows, cols // 2), dtype=torch.uint8), w.new_empty((rows, cols // 32), dtype=torch.uint8)
    else:
        codes, scales = _aside(dev, stream, (rows, cols // 2), torch.uint8), _aside(dev, stream, (rows, cols // 32), torch.uint8)
    _call(dev, stream, lib().sun_mx4_quantize, (_want("w", w, dev, w.dtype, w.shape), _dtype(w, "w"), rows, cols, codes.data_ptr(), scales.data_ptr()))
    return codes, scales


def _mx4(codes: torch.Tensor, scales: torch.Tensor, device: int):
    if codes.dim() != 2:
        _refuse("codes must be [rows, cols/2]")
    n, half = codes.shape
    _int32(rows=n, cols=2 * half)
    return (_want("codes", codes, device, torch.uint8, (n, half)), _want("scales", scales, device, torch.uint8, (n, half // 16)), n, 2 * half)


def sun_mx4_dequantize(codes: torch.Tensor, scales: torch.Tensor, dtype: torch.dtype = torch.bfloat16, stream=None) -> torch.Tensor:
    """The values [rows, cols], float32 or bfloat16, which belong to the stream that fills them."""
    dev = _gpu(codes)
    pc, ps, n, k = _mx4(codes, scales, dev)
    out = codes.new_empty((n, k), dtype=dtype) if stream is None else _aside(dev, stream, (n, k), dtype)
    _call(dev, stream, lib().sun_mx4_dequantize, (pc, ps, n, k, _dtype(out, "dtype"), out.data_ptr()))
    return out


def sun_mx4_linear_workspace_bytes(N: int, K: int, rows: int) -> int:
    return int(lib().sun_mx4_linear_workspace_bytes(N, K, rows)) if _fits(N, K, rows) else 0


def sun_mx4_linear(codes, scales, x, out, workspace, stream=None):
    """out [rows, N] = x [rows, K] W^T; x and out float32 or bfloat16 each, rows at any stride."""
    dev = _gpu(codes)
    pc, ps, n, k = _mx4(codes, scales, dev)
    if x.dim() != 2:
        _refuse("x must be [rows, K]")
    rows, tx, to = x.shape[0], x.dtype, out.dtype
    _int32(rows=rows)
    _call(dev, stream, lib().sun_mx4_linear, (
        pc, ps, n, k, rows, _want("x", x, dev, tx, (rows, k), True), _dtype(x, "x"), _row_stride(x),
        _want("out", out, dev, to, (rows, n), True), _dtype(out, "out"), _row_stride(out), *_workspace(workspace, dev)))


def sun_hbm_read_probe(src, block_bytes: int, perm, workgroups: int, sink, streaming_loads: bool = False, stream=None):
    _check(lib().sun_hbm_read_probe(_p(src), src.numel() * src.element_size(), block_bytes, _p(perm) if perm is not None else None,
                                    workgroups, 1 if streaming_loads else 0, _p(sink), _stream(stream)))


def sun_profile_reset():
    lib().sun_profile_reset()


def sun_profile_read() -> Dict[str, Dict[str, float]]:
    out = {}
    for k, name in enumerate(PROFILE_KINDS):
        ms, n = C.c_double(), C.c_int64()
        _check(lib().sun_profile_read(k, C.byref(ms), C.byref(n)))
        out[name] = {"ms": ms.value, "launches": int(n.value)}
    return out


def sun_version() -> str:
    return lib().sun_version().decode()
