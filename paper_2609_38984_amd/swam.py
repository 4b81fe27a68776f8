"""Thin ctypes binding of libswam (include/swam.h, swam_ops.h and swam_cache.h).

Argument marshalling only: tensors are checked for device, dtype, size and
contiguity, then their device pointers are passed to the C ABI.  Every step of
the path runs in the HIP kernels of libswam.so; if the library is missing the
binding raises instead of computing anything itself.
"""
from __future__ import annotations

import ctypes as C
import os

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libswam.so")

SWAM_F32, SWAM_BF16 = 0, 1
STATUS = {0: "SWAM_OK", -1: "SWAM_E_INVALID", -2: "SWAM_E_SHAPE", -3: "SWAM_E_DTYPE",
          -4: "SWAM_E_STATE", -5: "SWAM_E_HIP", -6: "SWAM_E_NOMEM", -7: "SWAM_E_UNSUPPORTED"}
FORCE_DENSE, FORCE_REFRESH = 1, 2
KIND_DENSE, KIND_REFRESH, KIND_SPARSE = 0, 1, 2
KIND_NONE, KIND_ANY = -1, -2   # timer slots outside any step / every slot
TIMERS = ["ADALN", "LNMOD", "GEMM_QKV", "ATTN", "GEMM_OUT", "GEMM_UP", "GEMM_DOWN", "SCORE",
          "REDUCE", "SELECT", "PACK", "UNPACK", "COPY", "SAMPLE", "QK_POST", "QUANT", "GEMM_I8",
          "CROSS", "HEAD_POST", "APPEND", "CACHE_ATTN"]
T = {name: i for i, name in enumerate(TIMERS)}

EXPORTS = ["swam_create", "swam_destroy", "swam_set_stream", "swam_plan", "swam_status_str",
           "swam_last_error", "swam_score", "swam_score_reduce", "swam_select",
           "swam_set_selection", "swam_packed_rows", "swam_export", "swam_pack", "swam_unpack",
           "swam_block", "swam_step", "swam_step_graph", "swam_graph_clear", "swam_timer_enable",
           "swam_timer_reset", "swam_timer_read", "swam_timer_stride",
           "swam_timer_read_kind", "swam_embed", "swam_velocity",
           "swam_sample_update", "swam_sample_step", "swam_overlap", "swam_select_random",
           "swam_flow_sigmas", "swam_select_noalloc"]

# include/swam_ops.h
OP_EXPORTS = ["swam_rms_norm_i8", "swam_quantize_i8", "swam_gemm_i8", "swam_cross_attention"]
I8_MAX_WIDTH, I8_MAX_K = 32768, 131056   # SWAM_I8_MAX_WIDTH, SWAM_I8_MAX_K
GEMM_GELU = 1                            # SWAM_GEMM_GELU

# include/swam_cache.h
CACHE_EXPORTS = ["swam_rope_frequencies", "swam_qk_norm_rope", "swam_cache_append", "swam_cache_attention"]
CACHE_MAX_SEQS, CACHE_MAX_PAGE, QK_MAX_DIM = 1024, 4096, 512   # SWAM_CACHE_MAX_SEQS, ...
ROPE_LAYOUTS = {"interleaved": 0, "half": 1}                     # SWAM_ROPE_INTERLEAVED, ...
ROPE_SCALINGS = {"plain": 0, "linear": 1, "ntk": 2, "yarn": 3}   # SWAM_ROPE_PLAIN, ...

# the flow-schedule shift of the paper's backbones (App. B.2)
SCHEDULE_SHIFT = 5.0


def flow_sigmas(n_steps: int, shift: float = SCHEDULE_SHIFT) -> list[float]:
    """The n_steps + 1 noise levels of the shifted flow schedule, computed by
    swam_flow_sigmas in the library (a host call, no GPU needed)."""
    lib = load_library()
    out = (C.c_double * (n_steps + 1))()
    _check(lib, None, lib.swam_flow_sigmas(int(n_steps), float(shift), out))
    return list(out)


def rope_frequencies(dims: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0,
                     trained: float = 0.0) -> tuple[list[float], float]:
    """The dims / 2 frequencies of a rotation (radians per position) and the factor of the rotated
    elements, for a context `factor` times longer than the `trained` positions by the rule
    `scaling`: "plain" (none), "linear", "ntk" or "yarn".  Computed by swam_rope_frequencies in
    the library (a host call, no GPU needed)."""
    lib = load_library()
    if scaling not in ROPE_SCALINGS:
        raise ValueError(f"scaling must be one of {list(ROPE_SCALINGS)}, got {scaling!r}")
    out, m = (C.c_double * max(1, int(dims) // 2))(), C.c_float()
    _check(lib, None, lib.swam_rope_frequencies(int(dims), float(base), ROPE_SCALINGS[scaling], float(factor),
                                                float(trained), out, C.byref(m)))
    return list(out), m.value


class SwamError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"{STATUS.get(code, code)}: {msg}")
        self.code = code


class Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in (
        "batch", "d_model", "n_heads", "head_dim", "mlp_ratio", "n_blocks", "d_temb", "n_ctx",
        "n_frames", "frame_h", "frame_w", "n_act", "k_core", "k_anchor", "k_layer")] + [
        ("cv_penalty", C.c_float), ("mass_threshold", C.c_float), ("reuse_R", C.c_int32),
        ("dtype", C.c_int32), ("rope", C.c_int32), ("qk_norm", C.c_int32),
        ("cfg_pairs", C.c_int32), ("guidance", C.c_float)]

    @classmethod
    def from_obj(cls, o) -> "Config":
        """Build from any object with the workload attributes (dtype 'f32'/'bf16')."""
        c = cls()
        for n, _ in cls._fields_:
            if n == "dtype":
                c.dtype = SWAM_BF16 if o.dtype == "bf16" else SWAM_F32
            elif n in ("rope", "qk_norm", "cfg_pairs"):
                setattr(c, n, int(getattr(o, n, 0)))
            elif n == "guidance":
                c.guidance = float(getattr(o, n, 1.0))
            else:
                setattr(c, n, getattr(o, n))
        return c


class PlanInfo(C.Structure):
    _fields_ = [(n, C.c_int64) for n in ("n_s", "group_size", "l_full", "rows_full", "k_max",
                                         "t_pack_fixed", "k_layer_eff", "workspace_bytes")]


WEIGHT_NAMES = ["w_ada", "b_ada", "w_qkv", "b_qkv", "w_o", "b_o", "w_1", "b_1", "w_2", "b_2"]


class BlockWeights(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in WEIGHT_NAMES]


class ModelStruct(C.Structure):
    _fields_ = [("n_blocks", C.c_int32), ("blocks", C.POINTER(BlockWeights))]


LATENT_NAMES = ["w_in", "b_in", "w_v", "b_v"]


class LatentIOStruct(C.Structure):
    _fields_ = [("d_latent", C.c_int32)] + [(n, C.c_void_p) for n in LATENT_NAMES]


class QkPostStruct(C.Structure):
    _fields_ = [("norm", C.c_int32), ("eps", C.c_float), ("q_gain", C.c_void_p), ("k_gain", C.c_void_p),
                ("rope_dims", C.c_int32), ("rope_layout", C.c_int32), ("rope_freq", C.c_void_p),
                ("rope_magnitude", C.c_float)]


class CacheStruct(C.Structure):
    _fields_ = [(n, C.c_void_p) for n in ("k", "v")] + [(n, C.c_int64) for n in (
        "k_page", "k_token", "k_head", "v_page", "v_token", "v_head", "n_pages")] + [(n, C.c_int32) for n in (
            "page_size", "n_kv_heads", "head_dim", "n_seqs", "max_pages")] + [
        ("table_stride", C.c_int64), ("table", C.c_void_p), ("length", C.c_void_p)]


_lib = None


def load_library(path: str = LIB_PATH):
    """Load libswam.so (raises if it has not been built)."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(the HIP library is required; there is no fallback)")
    lib = C.CDLL(path)
    P, I32, I64, F = C.c_void_p, C.c_int32, C.c_int64, C.c_float
    sig = {
        "swam_create": [C.POINTER(Config), P, C.POINTER(P)],
        "swam_destroy": [P], "swam_set_stream": [P, P],
        "swam_plan": [C.POINTER(Config), C.POINTER(PlanInfo)],
        "swam_score": [P, P, I64, I64, P, I64, I64, P, P, I64, P],
        "swam_score_reduce": [P, P, P, P, P, P],
        "swam_select": [P, P, P, P, P, P, P, P],
        "swam_select_random": [P, C.c_uint64, P, P, P, P, P],
        "swam_set_selection": [P, P, P],
        "swam_packed_rows": [P, C.POINTER(I64)],
        "swam_export": [P, P, P, P, P, P, P, P, P, P],
        "swam_pack": [P, P, P], "swam_unpack": [P, P, P, P],
        "swam_block": [P, C.POINTER(BlockWeights), P, P, I64, P, I32, P, P],
        "swam_step": [P, C.POINTER(ModelStruct), P, P, I32, P, I32, C.POINTER(I32)],
        "swam_step_graph": [P, C.POINTER(ModelStruct), P, P, I32, P, I32, C.POINTER(I32)],
        "swam_graph_clear": [P],
        "swam_timer_enable": [P, C.c_uint32, I32], "swam_timer_reset": [P],
        "swam_timer_read": [P, I32, C.POINTER(I64), C.POINTER(C.c_double)],
        "swam_timer_stride": [P, I32],
        "swam_timer_read_kind": [P, I32, I32, C.POINTER(I64), C.POINTER(C.c_double)],
        "swam_overlap": [P, P, P, I64, I64, P],
        "swam_flow_sigmas": [I32, C.c_double, C.POINTER(C.c_double)],
        "swam_select_noalloc": [I32, I32, I32, I32, I32, I32, I32, F, P, P, P, P, P, P, P, P],
        "swam_embed": [P, C.POINTER(LatentIOStruct), P, P],
        "swam_velocity": [P, C.POINTER(LatentIOStruct), P, I32, P],
        "swam_sample_update": [P, I32, P, P, P, F, I32],
        "swam_sample_step": [P, C.POINTER(ModelStruct), C.POINTER(LatentIOStruct), P, P, P, P, P,
                             P, I32, F, I32, C.POINTER(I32)],
        "swam_rms_norm_i8": [P, P, I64, P, I64, P, P, P, F, I64, I64, P, I64, P, I64, P],
        "swam_quantize_i8": [P, P, I64, I64, I64, P, I64, P],
        "swam_gemm_i8": [P, P, I64, P, P, I64, P, P, P, I64, P, I32, P, I64, I64, I64, I64],
        "swam_cross_attention": [P, P, I64, P, I64, P, I64, P, P, P, P, I32, I32, I64, I64, I32, I32,
                                 I32, F, P, I64, P],
        "swam_rope_frequencies": [I32, C.c_double, I32, C.c_double, C.c_double, C.POINTER(C.c_double),
                                  C.POINTER(C.c_float)],
        "swam_qk_norm_rope": [P, C.POINTER(QkPostStruct), P, P, I64, P, I64, I64, I32, I32, I32, P, I64, P, I64],
        "swam_cache_append": [P, C.POINTER(CacheStruct), C.POINTER(QkPostStruct), P, P, P, I64, P, I64, P, I64, I64,
                              I32, P, I64],
        "swam_cache_attention": [P, C.POINTER(CacheStruct), P, P, I64, I64, I32, I32, I32, F, P, I64, P],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = C.c_int
    lib.swam_status_str.argtypes = [C.c_int]
    lib.swam_status_str.restype = C.c_char_p
    lib.swam_last_error.argtypes = [P]
    lib.swam_last_error.restype = C.c_char_p
    _lib = lib
    return lib


def _check(lib, ctx, rc):
    if rc != 0:
        raise SwamError(rc, lib.swam_last_error(ctx).decode())


def plan(cfg) -> PlanInfo:
    lib = load_library()
    c = cfg if isinstance(cfg, Config) else Config.from_obj(cfg)
    info = PlanInfo()
    _check(lib, None, lib.swam_plan(C.byref(c), C.byref(info)))
    return info


def _ptr(t, dtype=None, numel=None, name="tensor"):
    """Device pointer of a contiguous CUDA tensor (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if numel is not None and t.numel() < numel:
        raise ValueError(f"{name} has {t.numel()} elements, needs {numel}")
    return t.data_ptr()


def _refuse(t, dtype, name, device):
    """The error for a tensor of another kind, type or GPU."""
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a GPU tensor")
    if t.dtype is not dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.get_device() != device:
        raise ValueError(f"{name} is on GPU {t.get_device()}, the context on {device}")


def _rows(t, dtype, shape, name, device):
    """Device pointer and row stride of a tensor of `shape` on GPU `device` whose
    rows are contiguous (None -> NULL); the rows themselves may lie further
    apart."""
    if t is None:
        return None, 0
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device:
        _refuse(t, dtype, name, device)
    if t.shape != shape:
        raise ValueError(f"{name} has shape {tuple(t.shape)}, needs {tuple(shape)}")
    width = shape[1] if len(shape) == 2 else shape[1] * shape[2]
    if t.is_contiguous():
        return t.data_ptr(), width
    run = 1
    for n, step in zip(reversed(shape[1:]), reversed(t.stride()[1:])):
        if n != 1 and step != run:
            raise ValueError(f"{name} must have contiguous rows")
        run *= n
    return t.data_ptr(), t.stride(0) if shape[0] > 1 else width


def _vec(t, dtype, numel, name, device):
    """Device pointer of a contiguous tensor of at least `numel` elements on GPU
    `device` (None -> NULL)."""
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or t.dtype is not dtype or t.get_device() != device:
        _refuse(t, dtype, name, device)
    if t.numel() < numel or not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous, with {numel} elements (it has {t.numel()})")
    return t.data_ptr()


class Model:
    """Device weights of every block, kept alive with their C descriptors."""

    def __init__(self, blocks: list[dict], act_dtype: torch.dtype):
        self.blocks = blocks
        self._arr = (BlockWeights * len(blocks))()
        for i, w in enumerate(blocks):
            for n in WEIGHT_NAMES:
                setattr(self._arr[i], n, _ptr(w[n], act_dtype, name=n))
        self.struct = ModelStruct(len(blocks), self._arr)


class LatentIO:
    """Device latent embedding / velocity head weights with their C descriptor."""

    def __init__(self, weights: dict, act_dtype: torch.dtype):
        self.weights = weights
        self.d_latent = int(weights["w_in"].shape[1])
        self.struct = LatentIOStruct(self.d_latent, *[_ptr(weights[n], act_dtype, name=n)
                                                      for n in LATENT_NAMES])


class Rope:
    """Rotation of the first 2 len(freq) elements of a head by position times freq (float64 GPU
    tensor, radians per position; rope_frequencies makes them).  layout "interleaved": pairs
    (2i, 2i + 1), "half": (i, i + len(freq)); magnitude: factor of the rotated elements."""

    def __init__(self, freq: torch.Tensor, layout: str = "interleaved", magnitude: float = 1.0):
        if layout not in ROPE_LAYOUTS:
            raise ValueError(f"layout must be one of {list(ROPE_LAYOUTS)}, got {layout!r}")
        _ptr(freq, torch.float64, name="freq")
        self.freq, self.layout, self.magnitude = freq, layout, float(magnitude)


class QkPost:
    """What is done to query and key heads: RMS norm (norm, eps, gains [head_dim] in the context's
    dtype or None) and rotation (rope, or None), with the C descriptor."""

    def __init__(self, norm: bool = True, eps: float = 1e-6, q_gain=None, k_gain=None, rope: Rope | None = None):
        self.q_gain, self.k_gain, self.rope = q_gain, k_gain, rope
        self.struct = QkPostStruct(int(bool(norm)), float(eps), _ptr(q_gain, name="q_gain"), _ptr(k_gain, name="k_gain"))
        if rope is not None:
            self.struct.rope_dims = 2 * rope.freq.numel()
            self.struct.rope_layout = ROPE_LAYOUTS[rope.layout]
            self.struct.rope_freq = rope.freq.data_ptr()
            self.struct.rope_magnitude = rope.magnitude
        self._ref, self._fits = C.byref(self.struct), None

    def _for(self, act, dim, device):
        """The descriptor, once its tensors fit the call (what fitted the last one does)."""
        if self._fits != (act, dim, device):
            for name in ("q_gain", "k_gain"):
                t = getattr(self, name)
                if t is not None:
                    if t.dtype is not act or t.get_device() != device:
                        _refuse(t, act, name, device)
                    if t.numel() != dim:
                        raise ValueError(f"{name} has {t.numel()} elements, needs {dim}")
            if self.rope is not None and self.rope.freq.get_device() != device:
                _refuse(self.rope.freq, torch.float64, "freq", device)
            self._fits = (act, dim, device)
        return self._ref


class Cache:
    """A paged cache with its C descriptor.  k, v [n_pages][page_size][kv_heads][head_dim] in the
    context's dtype, any strides with contiguous heads; table int32 [n_seqs][max_pages]: the
    pages of each sequence (outside [0, n_pages): none); length int32 [n_seqs]: tokens before the
    chunk.  The caller keeps and updates table and length in place."""

    def __init__(self, k: torch.Tensor, v: torch.Tensor, table: torch.Tensor, length: torch.Tensor):
        if not isinstance(k, torch.Tensor) or k.dim() != 4:
            raise ValueError("k must be a tensor [n_pages][page_size][kv_heads][head_dim]")
        self.device, self.act_dtype = k.get_device(), k.dtype
        n_pages, page, self.kv_heads, self.head_dim = k.shape
        for name, t in (("k", k), ("v", v)):
            if not isinstance(t, torch.Tensor) or t.dtype is not k.dtype or t.get_device() != self.device or self.device < 0:
                _refuse(t, k.dtype, name, self.device)
            if t.shape != k.shape:
                raise ValueError(f"{name} has shape {tuple(t.shape)}, needs {tuple(k.shape)}")
            if t.numel() and t.stride(3) != 1:
                raise ValueError(f"{name} must have contiguous heads")
        if not isinstance(table, torch.Tensor) or table.dim() != 2:
            raise ValueError("table must be a tensor [n_seqs][max_pages]")
        n_seqs, max_pages = table.shape
        tp, ts = _rows(table, torch.int32, table.shape, "table", self.device)
        lp = _vec(length, torch.int32, n_seqs, "length", self.device)
        if length.numel() != n_seqs:
            raise ValueError(f"length has {length.numel()} elements, needs {n_seqs}")
        self.k, self.v, self.table, self.length, self.n_seqs = k, v, table, length, n_seqs
        # (a dimension of one has no second element to reach)
        ks, vs = ([st if n > 1 else 0 for n, st in zip(t.shape, t.stride())] for t in (k, v))
        self.struct = CacheStruct(k.data_ptr(), v.data_ptr(), *ks[:3], *vs[:3], n_pages, page, self.kv_heads,
                                  self.head_dim, n_seqs, max_pages, ts, tp, lp)
        self._ref = C.byref(self.struct)

    def _for(self, act, device, cu):
        """The descriptor, once the cache and the offsets fit the call."""
        if self.act_dtype is not act:
            raise TypeError(f"the cache must be {act}, got {self.act_dtype}")
        if self.device != device:
            raise ValueError(f"the cache is on GPU {self.device}, the context on {device}")
        if cu is not None and cu.numel() != self.n_seqs + 1:
            raise ValueError(f"cu has {cu.numel()} elements, needs {self.n_seqs + 1}")
        return self._ref


NOALLOC_SCRATCH_BYTES = 1 << 20   # SWAM_NOALLOC_SCRATCH_BYTES


def select_noalloc(batch, n_frames, n_s, n_ctx, n_act, k_core, k_anchor, mass_threshold,
                   v, a, keep_idx, keep_cnt, pack_pos, gather, cu_seqlens,
                   stream: torch.cuda.Stream | None = None):
    """swam_select_noalloc: the selection and pack map for explicit sizes,
    without a context and without any allocation (scratch in the library's
    static device array), on `stream` (default: torch's current stream)."""
    lib = load_library()
    l_full = n_ctx + n_frames * n_s + n_act
    k_max = n_s if mass_threshold > 0 else max(1, k_core + k_anchor)
    i32 = torch.int32
    args = [_ptr(v, torch.float32, batch * n_frames * n_s, "v"),
            _ptr(a, torch.float32, batch * n_s, "a"),
            _ptr(keep_idx, i32, batch * n_frames * k_max, "keep_idx"),
            _ptr(keep_cnt, i32, batch * n_frames, "keep_cnt"),
            _ptr(pack_pos, i32, batch * l_full, "pack_pos"),
            _ptr(gather, i32, batch * l_full, "gather"),
            _ptr(cu_seqlens, i32, batch + 1, "cu_seqlens")]
    st = (stream or torch.cuda.current_stream()).cuda_stream
    _check(lib, None, lib.swam_select_noalloc(int(batch), int(n_frames), int(n_s), int(n_ctx),
                                              int(n_act), int(k_core), int(k_anchor),
                                              float(mass_threshold), *args, C.c_void_p(st)))


class Context:
    """One libswam context bound to a stream (default: torch's current stream)."""

    def __init__(self, cfg, stream: torch.cuda.Stream | None = None):
        self.lib = load_library()
        self.cfg = cfg
        self.c_cfg = cfg if isinstance(cfg, Config) else Config.from_obj(cfg)
        self.plan = plan(self.c_cfg)
        self.act_dtype = torch.bfloat16 if self.c_cfg.dtype == SWAM_BF16 else torch.float32
        self.stream = stream or torch.cuda.current_stream()
        self.device = self.stream.device.index   # the GPU that the operators' tensors lie on
        h = C.c_void_p()
        # the workspace comes from the current device: the stream's, whatever the caller's is
        with torch.cuda.device(self.device):
            _check(self.lib, None, self.lib.swam_create(C.byref(self.c_cfg),
                                                        C.c_void_p(self.stream.cuda_stream),
                                                        C.byref(h)))
        self.h = h

    def close(self):
        if getattr(self, "h", None):
            self.lib.swam_destroy(self.h)
            self.h = None

    def __del__(self):
        self.close()

    def _ok(self, rc):
        _check(self.lib, self.h, rc)

    def set_stream(self, stream: torch.cuda.Stream):
        """swam_set_stream: later calls run on `stream`, of the same GPU, after the
        work already queued on the previous one."""
        if stream.device.index != self.device:
            raise ValueError(f"the stream is on GPU {stream.device.index}, the context on {self.device}")
        self._ok(self.lib.swam_set_stream(self.h, C.c_void_p(stream.cuda_stream)))
        self.stream = stream

    # -- sizes -----------------------------------------------------------------
    @property
    def n_s(self):
        return self.plan.n_s

    @property
    def rows_full(self):
        return self.plan.rows_full

    @property
    def k_max(self):
        return self.plan.k_max

    @property
    def n_scored(self):
        """Sequences that are scored and selected (the conditional half with
        guidance pairs)."""
        c = self.c_cfg
        return c.batch // 2 if c.cfg_pairs else c.batch

    # -- (1) scoring -----------------------------------------------------------
    def score(self, q_act, q_seq, q_row, k_fut, k_seq, k_row, s_out, lse_act=None, k_all=None,
              kall_seq=0):
        c = self.c_cfg
        n_s = self.n_s
        _ptr(s_out, torch.float32, self.n_scored * c.n_frames * n_s, "s_out")
        self._ok(self.lib.swam_score(
            self.h, _ptr(q_act, self.act_dtype, name="q_act"), q_seq, q_row,
            _ptr(k_fut, self.act_dtype, name="k_fut"), k_seq, k_row,
            _ptr(lse_act, torch.float32, self.n_scored * c.n_act * c.n_heads, "lse_act"),
            _ptr(k_all, self.act_dtype, name="k_all"), kall_seq, s_out.data_ptr()))

    def score_reduce(self, s_all, v_out, a_out, q_out=None, core_out=None):
        c = self.c_cfg
        self._ok(self.lib.swam_score_reduce(
            self.h, _ptr(s_all, torch.float32, self.n_scored * c.n_blocks * c.n_frames * self.n_s, "s_all"),
            _ptr(q_out, torch.float32, self.n_scored * c.n_blocks, "q_out"),
            _ptr(v_out, torch.float32, self.n_scored * c.n_frames * self.n_s, "v_out"),
            _ptr(a_out, torch.float32, self.n_scored * self.n_s, "a_out"),
            _ptr(core_out, torch.int32, self.n_scored * self.plan.k_layer_eff, "core_out")))

    # -- (2) selection ---------------------------------------------------------
    def select(self, v=None, a=None, keep_idx=None, keep_cnt=None, pack_pos=None, gather=None,
               cu_seqlens=None):
        c = self.c_cfg
        self._ok(self.lib.swam_select(
            self.h, _ptr(v, torch.float32, self.n_scored * c.n_frames * self.n_s, "v"),
            _ptr(a, torch.float32, self.n_scored * self.n_s, "a"),
            _ptr(keep_idx, torch.int32, c.batch * c.n_frames * self.k_max, "keep_idx"),
            _ptr(keep_cnt, torch.int32, c.batch * c.n_frames, "keep_cnt"),
            _ptr(pack_pos, torch.int32, self.rows_full, "pack_pos"),
            _ptr(gather, torch.int32, self.rows_full, "gather"),
            _ptr(cu_seqlens, torch.int32, c.batch + 1, "cu_seqlens")))

    def select_random(self, seed: int, keep_idx=None, keep_cnt=None, pack_pos=None, gather=None,
                      cu_seqlens=None):
        """Random-selection baseline at the configured budget K_c + K_s."""
        c = self.c_cfg
        self._ok(self.lib.swam_select_random(
            self.h, int(seed) & ((1 << 64) - 1),
            _ptr(keep_idx, torch.int32, c.batch * c.n_frames * self.k_max, "keep_idx"),
            _ptr(keep_cnt, torch.int32, c.batch * c.n_frames, "keep_cnt"),
            _ptr(pack_pos, torch.int32, self.rows_full, "pack_pos"),
            _ptr(gather, torch.int32, self.rows_full, "gather"),
            _ptr(cu_seqlens, torch.int32, c.batch + 1, "cu_seqlens")))

    def set_selection(self, keep_idx, keep_cnt=None):
        c = self.c_cfg
        self._ok(self.lib.swam_set_selection(
            self.h, _ptr(keep_idx, torch.int32, c.batch * c.n_frames * self.k_max, "keep_idx"),
            _ptr(keep_cnt, torch.int32, c.batch * c.n_frames, "keep_cnt")))

    def packed_rows(self) -> int:
        r = C.c_int64()
        self._ok(self.lib.swam_packed_rows(self.h, C.byref(r)))
        return r.value

    def export(self, s_all=None, q=None, v=None, a=None, keep_idx=None, keep_cnt=None,
               pack_pos=None, gather=None, cu_seqlens=None):
        c = self.c_cfg
        n_s = self.n_s
        self._ok(self.lib.swam_export(
            self.h, _ptr(s_all, torch.float32, self.n_scored * c.n_blocks * c.n_frames * n_s, "s_all"),
            _ptr(q, torch.float32, self.n_scored * c.n_blocks, "q"),
            _ptr(v, torch.float32, self.n_scored * c.n_frames * n_s, "v"),
            _ptr(a, torch.float32, self.n_scored * n_s, "a"),
            _ptr(keep_idx, torch.int32, c.batch * c.n_frames * self.k_max, "keep_idx"),
            _ptr(keep_cnt, torch.int32, c.batch * c.n_frames, "keep_cnt"),
            _ptr(pack_pos, torch.int32, self.rows_full, "pack_pos"),
            _ptr(gather, torch.int32, self.rows_full, "gather"),
            _ptr(cu_seqlens, torch.int32, c.batch + 1, "cu_seqlens")))

    # -- (3) pack / (5) unpack ---------------------------------------------------
    def pack(self, x_full, x_packed):
        d = self.c_cfg.d_model
        self._ok(self.lib.swam_pack(self.h, _ptr(x_full, self.act_dtype, self.rows_full * d, "x_full"),
                                    _ptr(x_packed, self.act_dtype, self.packed_rows() * d, "x_packed")))

    def unpack(self, y_packed, x_full, y_full):
        d = self.c_cfg.d_model
        self._ok(self.lib.swam_unpack(
            self.h, _ptr(y_packed, self.act_dtype, self.packed_rows() * d, "y_packed"),
            _ptr(x_full, self.act_dtype, self.rows_full * d, "x_full"),
            _ptr(y_full, self.act_dtype, self.rows_full * d, "y_full")))

    # -- (4) block ---------------------------------------------------------------
    def block(self, weights: dict, temb, x, n_rows=None, cu_seqlens=None, n_seqs=0, lse_out=None,
              qkv_out=None):
        c = self.c_cfg
        d = c.d_model
        n_rows = self.rows_full if n_rows is None else int(n_rows)
        bw = BlockWeights()
        for n in WEIGHT_NAMES:
            setattr(bw, n, _ptr(weights[n], self.act_dtype, name=n))
        self._ok(self.lib.swam_block(
            self.h, C.byref(bw), _ptr(temb, torch.float32, c.d_temb, "temb"),
            _ptr(x, self.act_dtype, n_rows * d, "x"), n_rows,
            _ptr(cu_seqlens, torch.int32, None, "cu_seqlens"), n_seqs,
            _ptr(lse_out, torch.float32, n_rows * c.n_heads, "lse_out"),
            _ptr(qkv_out, self.act_dtype, n_rows * 3 * d, "qkv_out")))

    # -- step --------------------------------------------------------------------
    def step(self, model: Model, x_full, temb, tau: int, y_full, flags: int = 0) -> int:
        c = self.c_cfg
        n = self.rows_full * c.d_model
        kind = C.c_int32(-1)
        self._ok(self.lib.swam_step(
            self.h, C.byref(model.struct), _ptr(x_full, self.act_dtype, n, "x_full"),
            _ptr(temb, torch.float32, c.d_temb, "temb"), int(tau),
            _ptr(y_full, self.act_dtype, n, "y_full"), int(flags), C.byref(kind)))
        return kind.value

    def step_graph(self, model: Model, x_full, temb, tau: int, y_full, flags: int = 0) -> int:
        """swam_step through cached HIP graphs (needs a non-default stream)."""
        c = self.c_cfg
        n = self.rows_full * c.d_model
        kind = C.c_int32(-1)
        self._ok(self.lib.swam_step_graph(
            self.h, C.byref(model.struct), _ptr(x_full, self.act_dtype, n, "x_full"),
            _ptr(temb, torch.float32, c.d_temb, "temb"), int(tau),
            _ptr(y_full, self.act_dtype, n, "y_full"), int(flags), C.byref(kind)))
        return kind.value

    def graph_clear(self):
        self._ok(self.lib.swam_graph_clear(self.h))

    # -- diagnostics ---------------------------------------------------------------
    def overlap(self, p, q, out):
        """out[m] = Overlap(p[m], q[m]) of normalised maps (rows of p and q)."""
        n_maps, n = int(p.shape[0]), int(p[0].numel())
        self._ok(self.lib.swam_overlap(self.h, _ptr(p, torch.float32, n_maps * n, "p"),
                                       _ptr(q, torch.float32, n_maps * n, "q"), n_maps, n,
                                       _ptr(out, torch.float32, n_maps, "out")))

    # -- sampling update -----------------------------------------------------------
    def _n_lat(self):
        """Latent rows of every sequence (the rows of v)."""
        c = self.c_cfg
        return c.batch * (self.plan.l_full - c.n_ctx)

    def _n_state(self):
        """Latent rows of the state z and the velocity cache (one per pair
        with guidance)."""
        return self.n_scored * (self.plan.l_full - self.c_cfg.n_ctx)

    def embed(self, io: LatentIO, z, x_full):
        n = self._n_state() * io.d_latent
        self._ok(self.lib.swam_embed(self.h, C.byref(io.struct), _ptr(z, torch.float32, n, "z"),
                                     _ptr(x_full, self.act_dtype, self.rows_full * self.c_cfg.d_model,
                                          "x_full")))

    def velocity(self, io: LatentIO, y_full, v, retained_only: bool = False):
        self._ok(self.lib.swam_velocity(
            self.h, C.byref(io.struct),
            _ptr(y_full, self.act_dtype, self.rows_full * self.c_cfg.d_model, "y_full"),
            int(bool(retained_only)), _ptr(v, torch.float32, self._n_lat() * io.d_latent, "v")))

    def sample_update(self, d_latent: int, v, v_cache, z, dsigma: float, kind: int):
        n = self._n_state() * d_latent
        self._ok(self.lib.swam_sample_update(
            self.h, int(d_latent), _ptr(v, torch.float32, self._n_lat() * d_latent, "v"),
            _ptr(v_cache, torch.float32, n, "v_cache"), _ptr(z, torch.float32, n, "z"),
            float(dsigma), int(kind)))

    def sample_step(self, model: Model, io: LatentIO, z, v, v_cache, x_full, y_full, temb,
                    tau: int, dsigma: float, flags: int = 0) -> int:
        c = self.c_cfg
        n = self._n_state() * io.d_latent
        nt = self.rows_full * c.d_model
        kind = C.c_int32(-1)
        self._ok(self.lib.swam_sample_step(
            self.h, C.byref(model.struct), C.byref(io.struct), _ptr(z, torch.float32, n, "z"),
            _ptr(v, torch.float32, self._n_lat() * io.d_latent, "v"),
            _ptr(v_cache, torch.float32, n, "v_cache"),
            _ptr(x_full, self.act_dtype, nt, "x_full"), _ptr(y_full, self.act_dtype, nt, "y_full"),
            _ptr(temb, torch.float32, c.d_temb, "temb"), int(tau), float(dsigma), int(flags),
            C.byref(kind)))
        return kind.value

    # -- 8-bit, encoder-conditioned block (include/swam_ops.h) -------------------------
    def rms_norm_i8(self, x, q, q_scale, residual=None, sum_out=None, gain=None, shift=None,
                    scale=None, eps: float = 1e-6):
        """q, q_scale = 8-bit codes of RMSnorm(x + residual) gain (1 + scale) + shift, a scale
        per row.  x, residual, sum_out [rows][d] (sum_out receives x + residual and may be
        either of them), gain [d] in the context's dtype; shift, scale float [d]; q int8
        [rows][d]; q_scale float [rows]."""
        shape, act, f32, dev = x.shape, self.act_dtype, torch.float32, self.device
        rows, d = shape
        xp, xs = _rows(x, act, shape, "x", dev)
        rp, rs = _rows(residual, act, shape, "residual", dev)
        sp, ss = _rows(sum_out, act, shape, "sum_out", dev)
        qp, qs = _rows(q, torch.int8, shape, "q", dev)
        rc = self.lib.swam_rms_norm_i8(
            self.h, xp, xs, rp, rs, _vec(gain, act, d, "gain", dev), _vec(shift, f32, d, "shift", dev),
            _vec(scale, f32, d, "scale", dev), eps, rows, d, sp, ss, qp, qs,
            _vec(q_scale, f32, rows, "q_scale", dev))
        if rc:
            self._ok(rc)

    def quantize_i8(self, x, q, q_scale):
        """q int8 [rows][d], q_scale float [rows] = 8-bit codes of the rows of x with a scale
        each: activations per token, a weight [out][in] per output channel."""
        shape, dev = x.shape, self.device
        rows, d = shape
        xp, xs = _rows(x, self.act_dtype, shape, "x", dev)
        qp, qs = _rows(q, torch.int8, shape, "q", dev)
        rc = self.lib.swam_quantize_i8(self.h, xp, xs, rows, d, qp, qs,
                                       _vec(q_scale, torch.float32, rows, "q_scale", dev))
        if rc:
            self._ok(rc)

    def gemm_i8(self, a, a_scale, w, w_scale, c, bias=None, residual=None, gate=None, gelu: bool = False):
        """c [m][n] = z, GELU(z) or residual + gate z with z = (a_scale a) (w_scale w)^T + bias:
        a int8 [m][k], w int8 [n][k], a_scale float [m], w_scale float [n], bias [n] and
        residual [m][n] (may be c) in the context's dtype, gate float [n]."""
        act, i8, f32, dev = self.act_dtype, torch.int8, torch.float32, self.device
        (m, k), n = a.shape, w.shape[0]
        out = (m, n)
        ap, lda = _rows(a, i8, (m, k), "a", dev)
        wp, ldw = _rows(w, i8, (n, k), "w", dev)
        rp, ldr = _rows(residual, act, out, "residual", dev)
        cp, ldc = _rows(c, act, out, "c", dev)
        rc = self.lib.swam_gemm_i8(
            self.h, ap, lda, _vec(a_scale, f32, m, "a_scale", dev), wp, ldw, _vec(w_scale, f32, n, "w_scale", dev),
            _vec(bias, act, n, "bias", dev), rp, ldr, _vec(gate, f32, n, "gate", dev),
            GEMM_GELU if gelu else 0, cp, ldc, m, n, k)
        if rc:
            self._ok(rc)

    def cross_attention(self, q, k, v, o, cu_q=None, cu_k=None, kv_seq=None, key_mask=None,
                        scale: float | None = None, lse=None):
        """o [n_q][heads][head_dim] = attention of the tokens q to the encoder states k, v
        [n_k][kv_heads][head_dim].  cu_q, cu_k: int32 row offsets of the sequences (None: one
        sequence); kv_seq: int32, the key sequence of each query sequence (None: its own);
        key_mask: bool or uint8 [n_k], 0 hides a key; scale: 1 / sqrt(head_dim) by default;
        lse float [n_q][heads] receives the normalisers."""
        act, i32, dev = self.act_dtype, torch.int32, self.device
        (n_q, heads, dim), (n_k, kv_heads, _) = q.shape, k.shape
        keys = (n_k, kv_heads, dim)
        qp, qs = _rows(q, act, q.shape, "q", dev)
        kp, ks = _rows(k, act, keys, "k", dev)
        vp, vs = _rows(v, act, keys, "v", dev)
        op, os_ = _rows(o, act, q.shape, "o", dev)
        mp = None
        if key_mask is not None:
            mp = _vec(key_mask, torch.uint8 if key_mask.dtype is torch.uint8 else torch.bool, n_k, "key_mask", dev)
        n_kv = 1 if cu_k is None else cu_k.numel() - 1
        n_seqs = 1 if cu_q is None else cu_q.numel() - 1
        if kv_seq is not None and kv_seq.numel() != n_seqs:
            raise ValueError(f"kv_seq has {kv_seq.numel()} elements, needs {n_seqs}")
        rc = self.lib.swam_cross_attention(
            self.h, qp, qs, kp, ks, vp, vs, mp, _vec(cu_q, i32, 0, "cu_q", dev), _vec(cu_k, i32, 0, "cu_k", dev),
            _vec(kv_seq, i32, 0, "kv_seq", dev), n_seqs, n_kv, n_q, n_k, heads, kv_heads, dim,
            dim ** -0.5 if scale is None else scale, op, os_, _vec(lse, torch.float32, n_q * heads, "lse", dev))
        if rc:
            self._ok(rc)

    # -- streaming block on a paged cache (include/swam_cache.h) -----------------------
    def qk_norm_rope(self, q, k, post: QkPost, pos=None, q_out=None, k_out=None):
        """Norm and rotation (post) of the heads of q [rows][heads][head_dim] and k
        [rows][kv_heads][head_dim] (either may be None), in place or to q_out, k_out.  pos int32
        [rows]: positions (None: the row's index)."""
        act, dev = self.act_dtype, self.device
        some = q if q is not None else k
        if some is None:
            raise ValueError("q or k required")
        rows, _, dim = some.shape
        heads, kv_heads = (0 if t is None else t.shape[1] for t in (q, k))
        qp, qs = _rows(q, act, (rows, heads, dim), "q", dev)
        kp, ks = _rows(k, act, (rows, kv_heads, dim), "k", dev)
        qo, qos = (qp, qs) if q_out is None else _rows(q_out, act, (rows, heads, dim), "q_out", dev)
        ko, kos = (kp, ks) if k_out is None else _rows(k_out, act, (rows, kv_heads, dim), "k_out", dev)
        rc = self.lib.swam_qk_norm_rope(self.h, post._for(act, dim, dev), _vec(pos, torch.int32, rows, "pos", dev), qp, qs,
                                        kp, ks, rows, heads, kv_heads, dim, qo, qos, ko, kos)
        if rc:
            self._ok(rc)

    def cache_append(self, cache: Cache, k, v, cu=None, q=None, q_out=None, post: QkPost | None = None, pos=None):
        """Append a chunk to the cache: k (after norm and rotation, post) and v [rows][kv_heads][head_dim]
        of token i of sequence s at cache.length[s] + i.  cu int32 [n_seqs + 1]: row offsets of the
        sequences (None: one sequence); q [rows][heads][head_dim] gets the same norm and rotation, in
        place or to q_out; pos int32 [rows]: positions of the rotation (None: the token's in its
        sequence)."""
        act, dev, dim = self.act_dtype, self.device, cache.head_dim
        rows = k.shape[0]
        heads = 0 if q is None else q.shape[1]
        keys = (rows, cache.kv_heads, dim)
        kp, ks = _rows(k, act, keys, "k", dev)
        vp, vs = _rows(v, act, keys, "v", dev)
        qp, qs = _rows(q, act, (rows, heads, dim), "q", dev)
        qo, qos = (qp, qs) if q_out is None else _rows(q_out, act, (rows, heads, dim), "q_out", dev)
        rc = self.lib.swam_cache_append(
            self.h, cache._for(act, dev, cu), None if post is None else post._for(act, dim, dev),
            _vec(pos, torch.int32, rows, "pos", dev), _vec(cu, torch.int32, 0, "cu", dev), qp, qs, kp, ks, vp, vs, rows,
            heads, qo, qos)
        if rc:
            self._ok(rc)

    def cache_attention(self, cache: Cache, q, o, cu=None, causal: bool = True, window: int = 0,
                        scale: float | None = None, lse=None):
        """o [rows][heads][head_dim] = attention of a chunk's tokens q to everything in the cache, the
        appended chunk included.  cu as for cache_append; causal: a token sees the chunk up to
        itself (else all of it); window: keys up to its own that a token sees at most (0: all); scale:
        1 / sqrt(head_dim) by default; lse float [rows][heads] receives the normalisers."""
        act, dev, dim = self.act_dtype, self.device, cache.head_dim
        rows, heads = q.shape[:2]
        qp, qs = _rows(q, act, (rows, heads, dim), "q", dev)
        op, os_ = _rows(o, act, (rows, heads, dim), "o", dev)
        rc = self.lib.swam_cache_attention(
            self.h, cache._for(act, dev, cu), _vec(cu, torch.int32, 0, "cu", dev), qp, qs, rows, heads,
            1 if causal else 0, window, dim ** -0.5 if scale is None else scale, op, os_,
            _vec(lse, torch.float32, rows * heads, "lse", dev))
        if rc:
            self._ok(rc)

    # -- timers ------------------------------------------------------------------
    def timer_enable(self, classes, capacity=8192):
        mask = 0
        for cls in classes:
            mask |= 1 << (T[cls] if isinstance(cls, str) else int(cls))
        self._ok(self.lib.swam_timer_enable(self.h, mask, capacity))

    def timer_reset(self):
        self._ok(self.lib.swam_timer_reset(self.h))

    def timer_stride(self, stride: int):
        self._ok(self.lib.swam_timer_stride(self.h, int(stride)))

    def timer_read(self, cls, kind: int = KIND_ANY) -> tuple[int, float]:
        n, ms = C.c_int64(), C.c_double()
        self._ok(self.lib.swam_timer_read_kind(self.h, T[cls] if isinstance(cls, str) else int(cls),
                                               int(kind), C.byref(n), C.byref(ms)))
        return n.value, ms.value
