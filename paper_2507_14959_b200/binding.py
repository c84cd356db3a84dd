"""ctypes binding of libpolymorph.so: argument marshalling only.

Every function mirrors the C entry point of the same name (include/polymorph.h).  Device buffers
are torch CUDA tensors (torch is used for device memory and streams, nothing else); model
weights are numpy float32 arrays on the host.  There is no CPU fallback: if the shared library
is missing or a call fails, an exception is raised.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libpolymorph.so")

PM_OK, PM_ERR_ARG, PM_ERR_STATE, PM_ERR_CAPACITY, PM_ERR_CUDA, PM_ERR_TIMEOUT, PM_ERR_OOM = 0, -1, -2, -3, -4, -5, -6
ERROR_NAMES = {0: "PM_OK", -1: "PM_ERR_ARG", -2: "PM_ERR_STATE", -3: "PM_ERR_CAPACITY",
               -4: "PM_ERR_CUDA", -5: "PM_ERR_TIMEOUT", -6: "PM_ERR_OOM"}

EXPORTS = [
    "pm_create", "pm_register_adapter", "pm_set_cover", "pm_destroy", "pm_forward", "pm_forward_branched", "pm_forward_device_sets", "pm_select",
    "pm_select_static", "pm_metrics_reset", "pm_metrics_read", "pm_status", "pm_last_error", "pm_launch_count", "pm_set_graphs", "pm_set_small_batch_kernel", "pm_profile_enable", "pm_profile_read", "pm_plan_stats", "pm_linear_create", "pm_linear_register",
    "pm_linear_forward", "pm_linear_status", "pm_linear_last_error", "pm_linear_destroy",
    "pm_layernorm", "pm_attention", "pm_selftest_wait_timeout", "pm_linear_kernel", "pm_cooccurrence", "pm_build_contexts", "pm_intra_coherence",
    "pm_rope_init", "pm_rope", "pm_qk_norm_rope", "pm_attention_packed", "pm_attention_packed_workspace",
]


class PolymorphError(RuntimeError):
    def __init__(self, code, where, detail=""):
        self.code = code
        super().__init__(f"{where}: {ERROR_NAMES.get(code, code)} {detail}".strip())


class pm_config(C.Structure):
    _fields_ = [("img", C.c_int), ("patch", C.c_int), ("d", C.c_int), ("layers", C.c_int),
                ("heads", C.c_int), ("mlp", C.c_int), ("n_classes", C.c_int), ("ln_eps", C.c_float),
                ("max_adapters", C.c_int), ("max_rank", C.c_int), ("max_set", C.c_int),
                ("max_frames", C.c_int), ("dtype", C.c_int)]


_FP = C.POINTER(C.c_float)
BACKBONE_FIELDS = ["patch_w", "patch_b", "cls", "pos", "ln1_g", "ln1_b", "qkv_w", "qkv_b", "proj_w",
                   "proj_b", "ln2_g", "ln2_b", "fc1_w", "fc1_b", "fc2_w", "fc2_b", "lnf_g", "lnf_b",
                   "head_w", "head_b"]


class pm_backbone(C.Structure):
    _fields_ = [(n, _FP) for n in BACKBONE_FIELDS]


class pm_adapter(C.Structure):
    _fields_ = [("rank", C.c_int), ("scale", C.c_float), ("A", C.POINTER(_FP)), ("B", C.POINTER(_FP)),
                ("n_cls", C.c_int), ("class_ids", C.POINTER(C.c_int32)), ("head_w", _FP),
                ("head_b", _FP), ("acc", _FP)]


ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "bands": 3}
NORMS = {"rms": 0, "layer": 1}
ROPE_MAX_DIM = 256


class pm_rope_config(C.Structure):
    _fields_ = [("head_dim", C.c_int), ("rot_dim", C.c_int), ("interleaved", C.c_int), ("axes", C.c_int), ("scaling", C.c_int),
                ("amplitude", C.c_float), ("base", C.c_double), ("factor", C.c_double), ("original", C.c_double),
                ("low_turns", C.c_double), ("high_turns", C.c_double)]


class pm_rope_table(C.Structure):
    _fields_ = [("head_dim", C.c_int), ("rot_dim", C.c_int), ("interleaved", C.c_int), ("axes", C.c_int), ("amplitude", C.c_float),
                ("reserved", C.c_int), ("step", C.c_ulonglong * (ROPE_MAX_DIM // 2))]


class pm_qk_norm_rope_args(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "q_out", "k_out")] +
                [(n, C.c_longlong) for n in ("q_stride", "k_stride", "q_out_stride", "k_out_stride")] +
                [(n, C.c_void_p) for n in ("q_gamma", "k_gamma", "q_beta", "k_beta", "positions", "table")] +
                [(n, C.c_int) for n in ("rows", "heads", "kv_heads", "head_dim", "norm", "per_head")] +
                [("eps", C.c_float), ("dtype", C.c_int)])


class pm_packed_attention(C.Structure):
    _fields_ = ([(n, C.c_void_p) for n in ("q", "k", "v", "out")] +
                [(n, C.c_longlong) for n in ("q_stride", "k_stride", "v_stride", "out_stride")] +
                [(n, C.c_void_p) for n in ("q_offsets", "kv_offsets", "kv_lengths")] +
                [(n, C.c_int) for n in ("q_rows", "kv_rows", "n_seqs", "max_q", "max_kv", "heads", "kv_heads", "head_dim", "causal")] +
                [("scale", C.c_float), ("dtype", C.c_int), ("status_out", C.c_void_p), ("workspace", C.c_void_p), ("workspace_bytes", C.c_size_t)])


_lib = None


def load():
    """Loads the shared library (building nothing).  Raises if it is not there."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise RuntimeError(f"{LIB_PATH} is missing: run `python -m paper_2507_14959_b200.build` "
                           "(there is no fallback path)")
    lib = C.CDLL(LIB_PATH)
    vp, ip = C.c_void_p, C.c_int
    lib.pm_create.argtypes = [C.POINTER(pm_config), C.POINTER(pm_backbone), C.POINTER(vp)]
    lib.pm_register_adapter.argtypes = [vp, ip, C.POINTER(pm_adapter)]
    lib.pm_set_cover.argtypes = [vp, C.c_float]
    lib.pm_destroy.argtypes = [vp]
    lib.pm_destroy.restype = None
    lib.pm_forward.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp]
    lib.pm_forward_device_sets.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp]
    lib.pm_forward_branched.argtypes = [vp, vp, ip, vp, vp, ip, vp, vp, vp]
    lib.pm_select.argtypes = [vp, vp, ip, C.c_float, ip, ip, vp, vp, vp, vp, vp, ip, vp]
    lib.pm_select_static.argtypes = [vp, ip, ip, ip, C.c_float, ip, ip, vp, vp, vp, vp, vp, vp, vp, ip, vp, vp]
    lib.pm_status.argtypes = [vp, vp]
    lib.pm_metrics_reset.argtypes = [vp, vp]
    lib.pm_metrics_read.argtypes = [vp, vp, C.POINTER(C.c_longlong), C.POINTER(C.c_longlong), C.POINTER(C.c_longlong)]
    lib.pm_last_error.argtypes = [vp]
    lib.pm_last_error.restype = C.c_char_p
    lib.pm_launch_count.argtypes = [vp]
    lib.pm_cooccurrence.argtypes = [vp, ip, ip, vp, vp, vp]
    lib.pm_build_contexts.argtypes = [vp, ip, ip, ip, ip, vp, vp, C.POINTER(C.c_int)]
    lib.pm_intra_coherence.argtypes = [_FP, ip, C.POINTER(C.c_int32), C.POINTER(C.c_int32), ip, C.POINTER(C.c_double)]
    lib.pm_set_graphs.argtypes = [vp, ip]
    lib.pm_set_small_batch_kernel.argtypes = [vp, ip]
    lib.pm_launch_count.restype = C.c_longlong
    lib.pm_profile_enable.argtypes = [vp, ip]
    lib.pm_profile_read.argtypes = [vp, vp, C.POINTER(C.c_double), C.POINTER(C.c_longlong)]
    lib.pm_plan_stats.argtypes = [vp, C.POINTER(C.c_longlong), C.POINTER(C.c_double)]
    lib.pm_linear_create.argtypes = [ip, ip, _FP, _FP, ip, ip, ip, ip, ip, ip, ip, C.POINTER(vp)]
    lib.pm_linear_register.argtypes = [vp, ip, ip, C.c_float, _FP, _FP]
    lib.pm_linear_forward.argtypes = [vp, vp, ip, vp, vp, vp, vp, vp]
    lib.pm_linear_status.argtypes = [vp, vp]
    lib.pm_linear_last_error.argtypes = [vp]
    lib.pm_linear_last_error.restype = C.c_char_p
    lib.pm_linear_destroy.argtypes = [vp]
    lib.pm_linear_destroy.restype = None
    lib.pm_layernorm.argtypes = [vp, vp, vp, vp, ip, ip, C.c_float, ip, vp]
    lib.pm_attention.argtypes = [vp, vp, ip, ip, ip, ip, vp]
    lib.pm_selftest_wait_timeout.argtypes = [C.c_longlong, vp, vp, vp]
    lib.pm_linear_kernel.argtypes = [ip, ip, ip, ip, ip, ip, C.POINTER(C.c_int32)]
    lib.pm_rope_init.argtypes = [C.POINTER(pm_rope_config), C.POINTER(pm_rope_table)]
    lib.pm_rope.argtypes = [vp, C.c_longlong, vp, C.c_longlong, vp, ip, ip, vp, ip, vp]
    lib.pm_qk_norm_rope.argtypes = [vp, vp]
    lib.pm_attention_packed.argtypes = [vp, vp]
    lib.pm_attention_packed_workspace.argtypes = [vp, ip, C.POINTER(C.c_size_t)]
    _lib = lib
    return lib


def _f32(a):
    return np.ascontiguousarray(a, dtype=np.float32)


def _fp(a):
    return a.ctypes.data_as(_FP)


def _ptr(t):
    """Address of a torch tensor / numpy array / None as a void pointer value."""
    if t is None:
        return None
    if isinstance(t, np.ndarray):
        try:
            return C.addressof(_Start.from_buffer(t))      # a third of the time of the array's own attributes
        except (TypeError, ValueError, BufferError):       # read-only
            return t.ctypes.data
    return t.data_ptr()


_Start = C.c_byte * 0


def _i32(a):
    """The array itself if it is contiguous int32 already (the usual case, and cheaper to see than to convert)."""
    if a.dtype == _INT32 and a.flags.c_contiguous:
        return a
    return np.ascontiguousarray(a, dtype=np.int32)


_INT32 = np.dtype(np.int32)
_raw_stream = None             # () -> cudaStream_t of the current device's current stream


def _stream_ptr(stream):
    if stream is None:
        global _raw_stream
        if _raw_stream is None:
            import torch
            torch.cuda.current_stream()                    # initialises CUDA
            get, device = getattr(torch._C, "_cuda_getCurrentRawStream", None), getattr(torch._C, "_cuda_getDevice", None)
            # the Stream object that torch.cuda.current_stream() builds costs more than a kernel launch
            _raw_stream = (lambda: get(device())) if get and device else (lambda: torch.cuda.current_stream().cuda_stream)
        return _raw_stream()
    return getattr(stream, "cuda_stream", stream)


class Model:
    """Owner of a pm_handle.  Methods are the C calls with the handle bound."""

    def __init__(self, *, img, d, layers, heads, mlp, n_classes, backbone, max_adapters, max_rank,
                 max_set, max_frames, dtype=0, patch=16, ln_eps=1e-6):
        lib = load()
        self.lib = lib
        self.cfg = pm_config(img, patch, d, layers, heads, mlp, n_classes, ln_eps, max_adapters,
                             max_rank, max_set, max_frames, dtype)
        keep = {k: _f32(backbone[k]) for k in BACKBONE_FIELDS}
        bb = pm_backbone(**{k: _fp(v) for k, v in keep.items()})
        self.handle = C.c_void_p()
        rc = lib.pm_create(C.byref(self.cfg), C.byref(bb), C.byref(self.handle))
        if rc != PM_OK:
            self.handle = None
            raise PolymorphError(rc, "pm_create")
        self.n_classes = n_classes
        self.dtype = dtype

    def _check(self, rc, where):
        if rc != PM_OK:
            raise PolymorphError(rc, where, self.lib.pm_last_error(self.handle).decode())

    def register_adapter(self, adapter_id, *, rank, scale, A, B, class_ids, head_w, head_b, acc=None):
        n = len(A)
        keepA = [None if m is None else _f32(m) for m in A]
        keepB = [None if m is None else _f32(m) for m in B]
        arrA = (_FP * n)(*[None if m is None else _fp(m) for m in keepA])
        arrB = (_FP * n)(*[None if m is None else _fp(m) for m in keepB])
        cls = np.ascontiguousarray(class_ids, dtype=np.int32)
        hw, hb = _f32(head_w), _f32(head_b)
        ac = None if acc is None else _f32(acc)
        ad = pm_adapter(rank, scale, arrA, arrB, len(cls), cls.ctypes.data_as(C.POINTER(C.c_int32)),
                        _fp(hw), _fp(hb), None if ac is None else _fp(ac))
        self._check(self.lib.pm_register_adapter(self.handle, adapter_id, C.byref(ad)), "pm_register_adapter")

    def set_cover(self, tau):
        self._check(self.lib.pm_set_cover(self.handle, tau), "pm_set_cover")

    def forward(self, frames, set_offsets, set_ids, scores_out, base_out=None, stream=None):
        """frames/scores_out/base_out: torch CUDA tensors; set lists: numpy int32 (host) or torch
        CUDA int32 tensors."""
        n = len(frames)
        if isinstance(set_offsets, np.ndarray):
            set_offsets = _i32(set_offsets)
        if isinstance(set_ids, np.ndarray):
            set_ids = _i32(set_ids)
        self._check(self.lib.pm_forward(self.handle, _ptr(frames), n, _ptr(set_offsets), _ptr(set_ids),
                                        _ptr(scores_out), _ptr(base_out), _stream_ptr(stream)), "pm_forward")

    def forward_device_sets(self, frames, set_offsets, set_ids, scores_out, base_out=None, stream=None):
        """pm_forward_device_sets: the set lists are torch CUDA int32 tensors (e.g. written by
        select()); the plan is built on the device, nothing synchronises."""
        self._check(self.lib.pm_forward_device_sets(self.handle, _ptr(frames), len(frames),
                                                    _ptr(set_offsets), _ptr(set_ids), _ptr(scores_out),
                                                    _ptr(base_out), _stream_ptr(stream)), "pm_forward_device_sets")

    def forward_branched(self, frames, set_offsets, set_ids, trunk_layers, scores_out, base_out=None, stream=None):
        """pm_forward_branched: shared trunk of `trunk_layers` blocks, then one branch per active
        adapter (and the base branch if base_out is given).  Arguments as for forward()."""
        n = len(frames)
        if isinstance(set_offsets, np.ndarray):
            set_offsets = _i32(set_offsets)
        if isinstance(set_ids, np.ndarray):
            set_ids = _i32(set_ids)
        self._check(self.lib.pm_forward_branched(self.handle, _ptr(frames), n, _ptr(set_offsets), _ptr(set_ids),
                                                 int(trunk_layers), _ptr(scores_out), _ptr(base_out),
                                                 _stream_ptr(stream)), "pm_forward_branched")

    def select(self, scores, score_thr, context_copy, has_prev, prev_labels, prev_offsets, prev_ids,
               next_offsets, next_ids, stream=None):
        n = len(scores)
        cap = 0 if next_ids is None else next_ids.numel()
        self._check(self.lib.pm_select(self.handle, _ptr(scores), n, score_thr, int(context_copy),
                                       int(has_prev), _ptr(prev_labels), _ptr(prev_offsets), _ptr(prev_ids),
                                       _ptr(next_offsets), _ptr(next_ids), cap, _stream_ptr(stream)), "pm_select")

    def status(self, stream=None):
        return self.lib.pm_status(self.handle, _stream_ptr(stream))

    def metrics_reset(self, stream=None):
        self._check(self.lib.pm_metrics_reset(self.handle, _stream_ptr(stream)), "pm_metrics_reset")

    def metrics_read(self, stream=None):
        """(frames, contexts, switches) counted by select() since the last reset; synchronises."""
        f, c, s = C.c_longlong(0), C.c_longlong(0), C.c_longlong(0)
        self._check(self.lib.pm_metrics_read(self.handle, _stream_ptr(stream), C.byref(f), C.byref(c), C.byref(s)),
                    "pm_metrics_read")
        return int(f.value), int(c.value), int(s.value)

    def set_graphs(self, on):
        """Switches the recording / replaying of the forward's launch sequence as CUDA graphs."""
        self._check(self.lib.pm_set_graphs(self.handle, int(on)), "pm_set_graphs")

    def set_small_batch_kernel(self, on):
        """Whether small batches of small models run as the one whole-network kernel (default on)."""
        self._check(self.lib.pm_set_small_batch_kernel(self.handle, int(on)), "pm_set_small_batch_kernel")

    KERNEL_CLASSES = ("gemm", "shrink", "attention", "layernorm", "other", "heads", "select", "plan")

    def profile_enable(self, on):
        self._check(self.lib.pm_profile_enable(self.handle, int(on)), "pm_profile_enable")

    def profile_read(self, stream=None):
        """{class: (total_ms, launch_sites)} since the last read; synchronises the stream."""
        ms = (C.c_double * len(self.KERNEL_CLASSES))()
        n = (C.c_longlong * len(self.KERNEL_CLASSES))()
        self._check(self.lib.pm_profile_read(self.handle, _stream_ptr(stream), ms, n), "pm_profile_read")
        return {k: (ms[i], int(n[i])) for i, k in enumerate(self.KERNEL_CLASSES)}

    def plan_stats(self):
        """(plans built on the host, total host milliseconds spent building them)."""
        n, ms = C.c_longlong(0), C.c_double(0.0)
        self._check(self.lib.pm_plan_stats(self.handle, C.byref(n), C.byref(ms)), "pm_plan_stats")
        return int(n.value), float(ms.value)

    def launch_count(self):
        return int(self.lib.pm_launch_count(self.handle))

    def close(self):
        if getattr(self, "handle", None):
            self.lib.pm_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Linear:
    """Owner of a pm_linear (one isolated base + multi-LoRA linear)."""

    def __init__(self, w, bias, *, max_adapters, max_rank, max_set, max_frames, tokens, epilogue=0, dtype=0):
        lib = load()
        self.lib = lib
        w, bias = _f32(w), _f32(bias)
        self.k_in, self.n_out = w.shape
        self.tokens = tokens
        self.handle = C.c_void_p()
        rc = lib.pm_linear_create(self.k_in, self.n_out, _fp(w), _fp(bias), max_adapters, max_rank, max_set,
                                  max_frames, tokens, epilogue, dtype, C.byref(self.handle))
        if rc != PM_OK:
            self.handle = None
            raise PolymorphError(rc, "pm_linear_create")

    def _check(self, rc, where):
        if rc != PM_OK:
            raise PolymorphError(rc, where, self.lib.pm_linear_last_error(self.handle).decode())

    def register(self, adapter_id, rank, scale, A, B):
        A, B = _f32(A), _f32(B)
        self._check(self.lib.pm_linear_register(self.handle, adapter_id, rank, scale, _fp(A), _fp(B)),
                    "pm_linear_register")

    def forward(self, x, n_frames, set_offsets, set_ids, y, residual=None, stream=None):
        so = _i32(set_offsets) if isinstance(set_offsets, np.ndarray) else np.ascontiguousarray(set_offsets, dtype=np.int32)
        si = _i32(set_ids) if isinstance(set_ids, np.ndarray) else np.ascontiguousarray(set_ids, dtype=np.int32)
        self._check(self.lib.pm_linear_forward(self.handle, _ptr(x), n_frames, _ptr(so), _ptr(si),
                                               _ptr(residual), _ptr(y), _stream_ptr(stream)), "pm_linear_forward")

    def status(self, stream=None):
        return self.lib.pm_linear_status(self.handle, _stream_ptr(stream))

    def close(self):
        if getattr(self, "handle", None):
            self.lib.pm_linear_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def layernorm(x, gamma, beta, y, eps, dtype, stream=None):
    rc = load().pm_layernorm(_ptr(x), _ptr(gamma), _ptr(beta), _ptr(y), int(x.shape[0]), int(x.shape[1]),
                             eps, dtype, _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_layernorm")


def attention(qkv, out, n_frames, tokens, heads, dtype, stream=None):
    rc = load().pm_attention(_ptr(qkv), _ptr(out), n_frames, tokens, heads, dtype, _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_attention")


def selftest_wait_timeout(limit_cycles, status, trace, stream=None):
    """pm_selftest_wait_timeout: status = torch CUDA int32 [1], trace = torch CUDA int32 [3]."""
    rc = load().pm_selftest_wait_timeout(int(limit_cycles), _ptr(status), _ptr(trace), _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_selftest_wait_timeout")


def linear_kernel(k_in, n_out, rows, epilogue, adapters, n_sms=148):
    """pm_linear_kernel: (kernel, columns of a tile, CTAs that share K, threads per CTA); kernel is "few rows", "pair" or "single"."""
    form = (C.c_int32 * 4)()
    rc = load().pm_linear_kernel(int(k_in), int(n_out), int(rows), int(epilogue), int(bool(adapters)), int(n_sms), form)
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_linear_kernel")
    return ("few rows", "pair", "single")[form[0]], form[1], form[2], form[3]


def select_static(scores, n_adapters, score_thr, context_copy, has_prev, prev_labels, prev_offsets, prev_ids,
                  first, provider, next_offsets, next_ids, status_out=None, stream=None):
    """pm_select_static: Algorithm 2 with caller-provided cover tables and no device allocation."""
    n, k = int(scores.shape[0]), int(scores.shape[1])
    cap = 0 if next_ids is None else int(next_ids.numel())
    rc = load().pm_select_static(_ptr(scores), n, k, int(n_adapters), score_thr, int(context_copy), int(has_prev),
                                 _ptr(prev_labels), _ptr(prev_offsets), _ptr(prev_ids), _ptr(first),
                                 _ptr(provider), _ptr(next_offsets), _ptr(next_ids), cap, _ptr(status_out),
                                 _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_select_static")


def model_from_workload(w, *, dtype=0, max_frames=None, max_set=None):
    """Builds a Model from a workloads.Workload-shaped object (duck-typed: .spec, .backbone,
    .adapters) and registers all its adapters."""
    spec = w.spec
    ads = w.adapters
    if max_set is None:
        sizes = np.diff(w.set_offsets)
        max_set = max(3, int(sizes.max()) if len(sizes) else 0)
    m = Model(img=spec.img, d=spec.d, layers=spec.layers, heads=spec.heads, mlp=spec.mlp,
              n_classes=spec.n_classes, backbone=w.backbone, max_adapters=max(1, len(ads)),
              max_rank=max([a.rank for a in ads] + [1]), max_set=max_set,
              max_frames=max_frames or max(1, int(w.frames.shape[0])), dtype=dtype, patch=spec.patch,
              ln_eps=spec.ln_eps)
    for i, a in enumerate(ads):
        m.register_adapter(i, rank=a.rank, scale=a.scale, A=a.A, B=a.B, class_ids=a.class_ids,
                           head_w=a.head_w, head_b=a.head_b, acc=a.acc)
    return m


def cooccurrence(labels, n_labels, co, status=None, stream=None):
    """pm_cooccurrence: labels = torch CUDA int32 [T, ceil(K/32)] bit sets, co = torch CUDA fp32 [K, K]."""
    rc = load().pm_cooccurrence(_ptr(labels), int(labels.shape[0]), int(n_labels), _ptr(co), _ptr(status),
                                _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_cooccurrence")


def build_contexts(co, max_size, max_contexts, allow_overlap):
    """pm_build_contexts (Algorithm 1) on a host matrix; returns the contexts as lists of label ids."""
    co = np.ascontiguousarray(co, dtype=np.float32)
    K = co.shape[0]
    off = np.zeros(max(0, max_contexts) + 1, dtype=np.int32)
    ids = np.zeros(max(0, max_contexts * max_size), dtype=np.int32)
    n = C.c_int(0)
    rc = load().pm_build_contexts(_ptr(co), K, int(max_size), int(max_contexts), int(bool(allow_overlap)), _ptr(off), _ptr(ids),
                                  C.byref(n))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_build_contexts")
    bounds = off[:n.value + 1].tolist()
    flat = ids[:bounds[-1]].tolist()
    return [flat[b:e] for b, e in zip(bounds, bounds[1:])]


def intra_coherence(contexts, co_norm):
    """pm_intra_coherence (Eq. 6)."""
    co_norm = np.ascontiguousarray(co_norm, dtype=np.float32)
    off, ids = [0], []
    for c in contexts:
        ids.extend(int(i) for i in c)
        off.append(len(ids))
    off = np.asarray(off, dtype=np.int32)
    ids = np.asarray(ids if ids else [0], dtype=np.int32)
    out = C.c_double(0.0)
    i32 = C.POINTER(C.c_int32)
    rc = load().pm_intra_coherence(co_norm.ctypes.data_as(_FP), co_norm.shape[0], off.ctypes.data_as(i32),
                                   ids.ctypes.data_as(i32), len(contexts), C.byref(out))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_intra_coherence")
    return out.value


# ---- encoders that pack sequences of different lengths ----------------------------------------------
def _here(where, dtype_name, *tensors):
    """Refuses tensors of another element type, on the host or on another device than the current one."""
    import torch
    here = torch.cuda.current_device() if torch.cuda.is_available() else None
    for name, t, want in tensors:
        if t is None:
            continue
        if not t.is_cuda or t.get_device() != here:
            raise PolymorphError(PM_ERR_ARG, where, f"{name} is not on the current device")
        if t.dtype != (getattr(torch, dtype_name) if want is None else getattr(torch, want)):
            raise PolymorphError(PM_ERR_ARG, where, f"{name} has type {t.dtype}")


def _heads(where, name, t):
    """(rows, heads, head_dim, elements between rows) of [rows, heads, head_dim] whose heads lie side by side in a row."""
    if t.dim() != 3:
        raise PolymorphError(PM_ERR_ARG, where, f"{name} is not [rows, heads, head_dim]")
    (rows, heads, dim), (row, head, element) = t.shape, t.stride()
    if (dim > 1 and element != 1) or (heads > 1 and head != dim):
        raise PolymorphError(PM_ERR_ARG, where, f"the heads of a row of {name} do not lie side by side")
    return rows, heads, dim, row if rows > 1 else max(row, heads * dim)


def _ints_of(where, name, t, *shapes):
    """Refuses an index tensor that is not contiguous or has none of the shapes."""
    if not t.is_contiguous() or tuple(t.shape) not in shapes:
        raise PolymorphError(PM_ERR_ARG, where, f"{name} has shape {tuple(t.shape)} or is not contiguous")


def _type_name(where, dtype):
    if dtype not in (0, 1):
        raise PolymorphError(PM_ERR_ARG, where, "dtype is 0 (bf16) or 1 (fp32)")
    return "bfloat16" if dtype == 0 else "float32"


class RopeTable:
    """pm_rope_init: rotation by position for heads of head_dim, kept by the caller and passed to rope() and qk_norm_rope()."""

    def __init__(self, head_dim, *, rot_dim=None, base=10000.0, interleaved=False, axes=1, scaling="none", factor=1.0, original=0.0,
                 low_turns=1.0, high_turns=4.0, amplitude=1.0):
        if scaling not in ROPE_SCALINGS:
            raise PolymorphError(PM_ERR_ARG, "pm_rope_init", f"scaling is one of {', '.join(ROPE_SCALINGS)}")
        cfg = pm_rope_config(head_dim, head_dim if rot_dim is None else rot_dim, int(bool(interleaved)), axes, ROPE_SCALINGS[scaling], amplitude,
                             base, factor, original, low_turns, high_turns)
        self.table = pm_rope_table()
        rc = load().pm_rope_init(C.byref(cfg), C.byref(self.table))
        if rc != PM_OK:
            raise PolymorphError(rc, "pm_rope_init")
        self.head_dim, self.axes, self.address = head_dim, axes, C.addressof(self.table)


def _positions(where, positions, rows, axes):
    _ints_of(where, "positions", positions, *([(rows,), (rows, 1)] if axes == 1 else [(rows, axes)]))


def rope(x, y, positions, table, dtype, stream=None):
    """pm_rope: x, y = torch CUDA [rows, heads, head_dim] (y may be x), positions = torch CUDA int32 [rows] or [rows, 2]."""
    lib, where = load(), "pm_rope"
    name = _type_name(where, dtype)
    _here(where, name, ("x", x, None), ("y", y, None), ("positions", positions, "int32"))
    rows, heads, dim, xs = _heads(where, "x", x)
    ys = _heads(where, "y", y)[3]
    if y.shape != x.shape or dim != table.head_dim:
        raise PolymorphError(PM_ERR_ARG, where, "shapes differ")
    _positions(where, positions, rows, table.axes)
    rc = lib.pm_rope(_ptr(x), xs, _ptr(y), ys, _ptr(positions), rows, heads, table.address, dtype, _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, where)


def qk_norm_rope(q, k, q_out, k_out, q_gamma, k_gamma, *, norm, eps, dtype, q_beta=None, k_beta=None, positions=None, table=None, stream=None):
    """pm_qk_norm_rope: q, k and their outputs = torch CUDA [rows, heads, head_dim] (an output may be its input; k may be None);
    gamma, beta = torch CUDA fp32 [head_dim], or [heads, head_dim] for weights of each head; norm "rms" or "layer"."""
    lib, where = load(), "pm_qk_norm_rope"
    name = _type_name(where, dtype)
    if norm not in NORMS:
        raise PolymorphError(PM_ERR_ARG, where, "norm is rms or layer")
    if (table is None) != (positions is None):
        raise PolymorphError(PM_ERR_ARG, where, "positions and table go together")
    _here(where, name, ("q", q, None), ("k", k, None), ("q_out", q_out, None), ("k_out", k_out, None), ("positions", positions, "int32"),
          *((n, t, "float32") for n, t in (("q_gamma", q_gamma), ("k_gamma", k_gamma), ("q_beta", q_beta), ("k_beta", k_beta))))
    rows, heads, dim, qs = _heads(where, "q", q)
    qos = _heads(where, "q_out", q_out)[3]
    kv_heads = ks = kos = 0
    if k is not None:
        _, kv_heads, _, ks = _heads(where, "k", k)
        kos = _heads(where, "k_out", k_out)[3]
        if k.shape != (rows, kv_heads, dim) or k_out.shape != k.shape:
            raise PolymorphError(PM_ERR_ARG, where, "shapes differ")
    if q_out.shape != q.shape or (table is not None and dim != table.head_dim):
        raise PolymorphError(PM_ERR_ARG, where, "shapes differ")
    per_head = q_gamma.dim() == 2
    for n, t, h in (("q_gamma", q_gamma, heads), ("q_beta", q_beta, heads), ("k_gamma", k_gamma, kv_heads), ("k_beta", k_beta, kv_heads)):
        if t is not None:
            _ints_of(where, n, t, (h, dim) if per_head else (dim,))
    if table is not None:
        _positions(where, positions, rows, table.axes)
    args = pm_qk_norm_rope_args(_ptr(q), _ptr(k), _ptr(q_out), _ptr(k_out), qs, ks, qos, kos, _ptr(q_gamma), _ptr(k_gamma), _ptr(q_beta), _ptr(k_beta),
                                _ptr(positions), None if table is None else table.address, rows, heads, kv_heads, dim, NORMS[norm], int(per_head), eps, dtype)
    rc = lib.pm_qk_norm_rope(C.byref(args), _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, where)


LONG_HISTORY = 4096            # keys below which no call has a use for a workspace


def _lend_workspace(lib, args, like, stream):
    """Memory of torch's for the time of the call on its stream."""
    import torch
    need = C.c_size_t(0)
    sms = torch.cuda.get_device_properties(like.device).multi_processor_count
    rc = lib.pm_attention_packed_workspace(C.byref(args), sms, C.byref(need))
    if rc != PM_OK:
        raise PolymorphError(rc, "pm_attention_packed_workspace")
    if need.value:
        space = torch.empty(need.value, dtype=torch.uint8, device=like.device)
        if stream is not None:
            space.record_stream(stream if isinstance(stream, torch.cuda.Stream) else torch.cuda.ExternalStream(_stream_ptr(stream)))
        args.workspace, args.workspace_bytes = space.data_ptr(), need.value


def attention_packed(q, k, v, out, q_offsets, max_q, max_kv, dtype, *, kv_offsets=None, kv_lengths=None, causal=False, scale=None, status=None,
                     stream=None):
    """pm_attention_packed: q, out = torch CUDA [rows, heads, head_dim], k, v = [kv rows, kv_heads, head_dim]; q_offsets = torch CUDA int32
    [n + 1]; kv_offsets = the same for keys ([n] suffices with kv_lengths = [n]); status = torch CUDA int32 [1] or None."""
    lib, where = load(), "pm_attention_packed"
    name = _type_name(where, dtype)
    _here(where, name, ("q", q, None), ("k", k, None), ("v", v, None), ("out", out, None),
          *((n, t, "int32") for n, t in (("q_offsets", q_offsets), ("kv_offsets", kv_offsets), ("kv_lengths", kv_lengths), ("status", status))))
    rows, heads, dim, qs = _heads(where, "q", q)
    kv_rows, kv_heads, _, ks = _heads(where, "k", k)
    vs, os_ = _heads(where, "v", v)[3], _heads(where, "out", out)[3]
    if k.shape != v.shape or out.shape != q.shape or k.shape[2] != dim:
        raise PolymorphError(PM_ERR_ARG, where, "shapes differ")
    n = q_offsets.numel() - 1
    _ints_of(where, "q_offsets", q_offsets, (n + 1,))
    if kv_offsets is not None:
        _ints_of(where, "kv_offsets", kv_offsets, (n + 1,), *([(n,)] if kv_lengths is not None else []))
    if kv_lengths is not None:
        _ints_of(where, "kv_lengths", kv_lengths, (n,))
    args = pm_packed_attention(_ptr(q), _ptr(k), _ptr(v), _ptr(out), qs, ks, vs, os_, _ptr(q_offsets), _ptr(kv_offsets), _ptr(kv_lengths), rows, kv_rows, n,
                               int(max_q), int(max_kv), heads, kv_heads, dim, int(bool(causal)), 0.0 if scale is None else scale, dtype, _ptr(status))
    if dtype == 0 and max_kv >= LONG_HISTORY and max_q * heads <= 64 * kv_heads:
        _lend_workspace(lib, args, q, stream)
    rc = lib.pm_attention_packed(C.byref(args), _stream_ptr(stream))
    if rc != PM_OK:
        raise PolymorphError(rc, where)
