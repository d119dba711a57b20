"""Python binding of librv (include/rv.h): argument marshalling only.

Every step of the hot path runs in librv's HIP kernels; this module checks tensor
shapes/dtypes/devices the C ABI cannot see (it receives raw pointers), converts
handles, and raises RVError on any non-zero rv_status.  Tensors are torch CUDA
(HIP) tensors; bf16 tensors may be any 2-byte dtype (bfloat16, int16, uint16) since
only their bits matter (the calls for projections and sequences refuse others, float16
among them; the per-frame ones look at the size alone).  PyTorch supplies device memory
and streams, nothing else.  There is no fallback: if librv.so or the marshalling module _rv_bind.so is missing the
import of this module fails.
"""
import ctypes
import importlib.util
import os
import re
import sys

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
BIND_PATH = os.path.join(_HERE, "_rv_bind.so")
LIB_PATH = os.path.join(_HERE, "librv.so")
SYNTH_LIB_PATH = os.path.join(_HERE, "librv_synth.so")

RV_OK, RV_ERR_INVALID, RV_ERR_OOM, RV_ERR_CAPACITY, RV_ERR_HIP, RV_ERR_IO = range(6)
HEAD_DIM = 64


class RVError(RuntimeError):
    def __init__(self, status, message):
        super().__init__(f"librv status {status}: {message}")
        self.status = status


class rv_qsub(ctypes.Structure):
    _fields_ = [("grid_h", ctypes.c_int32), ("grid_w", ctypes.c_int32),
                ("n_special", ctypes.c_int32), ("stride", ctypes.c_int32)]


class rv_qkv_prep(ctypes.Structure):
    _fields_ = [("n_q_heads", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("norm", ctypes.c_int32),
                ("n_axes", ctypes.c_int32), ("eps", ctypes.c_float), ("base", ctypes.c_double)] + [
        (n, ctypes.c_void_p) for n in ("q_weight", "q_bias", "k_weight", "k_bias")]


class rv_attn_plan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("n_units", "q_tiles", "T", "U", "E", "E1", "n_first",
                                               "n_queues", "grid", "total_chunks")] + [
        ("unit_base", ctypes.c_int32 * 17), ("n_chunks", ctypes.c_int32 * 16), ("chunk_base", ctypes.c_int32 * 16)]


def _load():
    if not os.path.exists(LIB_PATH):
        raise ImportError(f"{LIB_PATH} is not built; run __graft_entry__.build() "
                          "(hipcc --offload-arch=gfx950)")
    lib = ctypes.CDLL(LIB_PATH)
    # (an array of pointers is a vp: it goes as the bytes that _rv_bind packs, or as a ctypes array)
    vp, i32, i64 = ctypes.c_void_p, ctypes.c_int, ctypes.c_int64
    P = ctypes.POINTER
    sigs = {
        "rv_last_error": ([], ctypes.c_char_p),
        "rv_version": ([], ctypes.c_char_p),
        "rv_init": ([], i32),
        "rv_mem_create": ([i32, i32, i64, i64, P(vp)], i32),
        "rv_mem_destroy": ([vp], i32),
        "rv_mem_len": ([vp], i64),
        "rv_mem_capacity": ([vp], i64),
        "rv_mem_view": ([vp, P(vp), P(vp), P(i64)], i32),
        "rv_mem_reserve": ([vp, i64, vp], i32),
        "rv_mem_reset": ([vp], i32),
        "rv_mem_truncate": ([vp, i64], i32),
        "rv_mem_write": ([vp, vp, vp, i64, i32, vp], i32),
        "rv_mem_read": ([vp, vp, vp, vp, vp], i32),
        "rv_mem_save": ([vp, ctypes.c_char_p], i32),
        "rv_mem_load": ([vp, ctypes.c_char_p], i32),
        "rv_attend_frame": ([vp, vp, vp, i32, vp, vp, i64, i64, i32, i32, P(rv_qsub), vp, vp, vp, vp], i32),
        "rv_attend_frame_fused": ([vp, vp, vp, i32, vp, vp, i64, i64, i32, i32, P(rv_qsub), vp, vp, vp, vp], i32),
        "rv_admit_layers_tiled": ([i32, vp, i32, i32, vp, vp, vp, i32, vp, vp, vp], i32),
        "rv_attend_frame_noalloc": ([vp, vp, vp, i32, vp, vp, i64, i64, i32, i32, P(rv_qsub), vp, vp, vp, vp],
                                    i32),
        "rv_admit": ([vp, i32, vp, vp, i32, vp, i32, vp, vp], i32),
        "rv_admit_layers": ([i32, vp, vp, vp, vp, i32, P(rv_qsub), i32, vp, i32, vp, vp, vp], i32),
        "rv_admit_layers_shared": ([i32, vp, vp, vp, vp, i32, P(rv_qsub), i32, vp, i32, vp, vp,
                                    vp], i32),
        "rv_mem_stage": ([vp, i32, P(vp), P(vp), P(i64), vp], i32),
        "rv_mem_stage_frame": ([vp, vp, vp, i32, vp], i32),
        "rv_mem_stage_frames": ([i32, vp, vp, vp, i32, vp], i32),
        "rv_attend_staged": ([vp, i32, vp, P(rv_qsub), vp, vp, vp, vp], i32),
        "rv_admit_staged_layers": ([i32, vp, vp, i32, P(rv_qsub), i32, vp, i32, vp, vp, vp], i32),
        "rv_reserve_workspace": ([i32, i32, i64, i32], i32),
        "rv_attention_plan": ([i32, i32, i64, i32, i32, i32, P(rv_attn_plan)], i32),
        "rv_attention_plan_long": ([P(rv_attn_plan)], i32),
        "rv_device_status": ([], i32),
        "rv_prepare_qkv": ([P(rv_qkv_prep), vp, i64, vp, i64, vp, i64, i32, i32, vp, vp, vp, vp, vp], i32),
        "rv_mem_stage_qkv": ([vp, P(rv_qkv_prep), vp, i64, vp, i64, vp, i64, i32, i32, vp, vp, vp], i32),
        "rv_prepare_qkv_bwd": ([P(rv_qkv_prep), vp, i64, vp, i64, i32, i32, vp, vp, vp, vp, vp, i64, vp, i64, vp, i64,
                                vp, vp, vp, vp, vp], i32),
        "rv_pool_create": ([i32, i32, i32, i32, i64, P(vp)], i32),
        "rv_pool_destroy": ([vp], i32),
        "rv_pool_free_pages": ([vp], i32),
        "rv_pool_open": ([vp, P(i32)], i32),
        "rv_pool_len": ([vp, i32], i64),
        "rv_pool_fork": ([vp, i32, i64, i32, vp, vp], i32),
        "rv_pool_close": ([vp, i32, vp], i32),
        "rv_pool_truncate": ([vp, i32, i64], i32),
        "rv_pool_append": ([vp, i32, vp, vp, vp, vp, vp], i32),
        "rv_pool_gather": ([vp, i32, vp, vp, vp, vp, vp, vp], i32),
        "rv_pool_compact": ([vp, i32, vp, vp, vp, vp, vp], i32),
        "rv_attend_seqs": ([vp, i32, vp, vp, vp, vp, vp, i32, vp, vp, vp], i32),
        "rv_admit_seqs": ([vp, i32, vp, vp, vp, vp, vp, i32, P(rv_qsub), i32, vp, vp, vp], i32),
    }
    for name, (args, res) in sigs.items():
        f = getattr(lib, name)
        f.argtypes = args
        f.restype = res
    return lib


def _load_bind():
    if not os.path.exists(BIND_PATH):
        raise ImportError(f"{BIND_PATH} is not built; run __graft_entry__.build()")
    here = (re.match(r"[\d.]+\d", torch.__version__).group(), *sys.version_info[:2])
    spec = importlib.util.spec_from_file_location("paper_2609_23286_amd._rv_bind", BIND_PATH)
    try:
        mod = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(mod)
        built_for = mod.built_for
    except (ImportError, AttributeError) as e:
        built_for = e
    if built_for != here:
        raise ImportError(f"{BIND_PATH} was built for another torch or Python than {here}: {built_for}; "
                          "run __graft_entry__.build()")
    return mod


_lib = _load()
_bind = _load_bind()


def lib():
    return _lib


def _check(status):
    if status != RV_OK:
        raise RVError(status, _lib.rv_last_error().decode(errors="replace"))


# (the same handle as torch.cuda.current_stream().cuda_stream, without the stream object: 1 us a call)
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None)


def _stream(stream):
    if stream is None:
        if _raw_stream is None:
            return torch.cuda.current_stream().cuda_stream
        return _raw_stream(torch.cuda.current_device())
    if isinstance(stream, torch.cuda.Stream):
        return ctypes.c_void_p(stream.cuda_stream)
    return ctypes.c_void_p(int(stream))


def _ptr_python(t, shape=None, itemsize=None, what="tensor"):
    """Address of a device tensor argument, or None; raises on one the C ABI cannot take."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{what}: must be a device tensor")
    if not t.is_contiguous():
        raise ValueError(f"{what}: must be contiguous")
    if itemsize is not None and t.element_size() != itemsize:
        raise TypeError(f"{what}: element size {t.element_size()}, expected {itemsize}")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {tuple(shape)}")
    return t.data_ptr()


# The same checks on plain tensors without Python's attribute calls: one address, and the
# addresses of a list of tensors (one per layer) as bytes.
_bind.setup(_ptr_python, ctypes.cast(_lib.rv_mem_view, ctypes.c_void_p).value,
            ctypes.cast(_lib.rv_mem_len, ctypes.c_void_p).value)
_ptr, _ptrs = _bind.ptr, _bind.ptrs
_bind.setup_calls(*(ctypes.cast(getattr(_lib, f), ctypes.c_void_p).value for f in (
    "rv_prepare_qkv", "rv_prepare_qkv_bwd", "rv_pool_fork", "rv_pool_close", "rv_pool_append", "rv_pool_gather",
    "rv_pool_compact", "rv_attend_seqs")))


def _made(status):
    """Whether a call made through _rv_bind went through; None: it was not made."""
    if status is None:
        return False
    if status != RV_OK:
        _check(status)
    return True


_BF16_BITS = (torch.bfloat16, torch.int16, torch.uint16)


def _typed(t, types, shape, what):
    if isinstance(t, torch.Tensor) and t.dtype not in types:
        raise TypeError(f"{what}: dtype {t.dtype}, expected {types[0]}")
    return _ptr(t, shape, types[0].itemsize, what)


def _bf16(t, shape, what):
    """_ptr of bf16 values, or of their bits as whole numbers."""
    return _typed(t, _BF16_BITS, shape, what)


def _fp32(t, shape, what):
    return _typed(t, (torch.float32,), shape, what)


def _int32(t, shape, what):
    return _typed(t, (torch.int32,), shape, what)


def _where(stream):
    """(current device, stream handle) as integers."""
    device = torch.cuda.current_device()
    if stream is None and _raw_stream is not None:
        return device, _raw_stream(device)
    s = _stream(stream)
    return device, s if isinstance(s, int) else s.value or 0


def _same_device(device, *tensors):
    for t in tensors:
        if isinstance(t, torch.Tensor) and t.is_cuda and t.get_device() != device:
            raise ValueError(f"a tensor on device {t.get_device()} while device {device} is current")


def _mem_state(mem):
    """(memK, memV, head stride, length) of a memory, as rv_mem_view and rv_mem_len give them."""
    if type(mem) is not Memory:
        return (*mem.view(), mem.len)
    st = _bind.mem_state(mem.handle.value if mem.handle else None)
    if isinstance(st, int):
        _check(st)
    return st


def version():
    return _lib.rv_version().decode()


def qsub(grid_h, grid_w, n_special, stride):
    return rv_qsub(grid_h, grid_w, n_special, stride)


def init():
    """rv_init: set up librv on the current device (limits, XCD count, workspace)."""
    _check(_lib.rv_init())


def reserve_workspace(n_tokens, n_heads, max_mem_len=0, n_layers=1):
    """rv_reserve_workspace: partial slots for forced work plans up to max_mem_len memory
    rows, saliency staging for n_layers layers."""
    _check(_lib.rv_reserve_workspace(n_tokens, n_heads, max_mem_len, n_layers))


def attention_plan(n_tokens, n_fkeys, mem_len, n_heads, n_cus, n_queues):
    """The attention work plan for a frame on a device of n_cus CUs and n_queues XCDs
    (rv_attention_plan; no device work), as an rv_attn_plan structure."""
    out = rv_attn_plan()
    _check(_lib.rv_attention_plan(n_tokens, n_fkeys, mem_len, n_heads, n_cus, n_queues, ctypes.byref(out)))
    return out


def attention_plan_long(plan):
    """Whether a launch of this rv_attn_plan takes the forward kernel for long chunks
    (rv_attention_plan_long)."""
    return bool(_lib.rv_attention_plan_long(ctypes.byref(plan)))


def device_status():
    """Synchronise the device; raise RVError if a kernel raised a status bit."""
    _check(_lib.rv_device_status())


class Memory:
    """One layer's regulated KV memory (rv_mem)."""

    def __init__(self, n_heads, head_dim=HEAD_DIM, reserve_tokens=0, max_tokens=1 << 31):
        h = ctypes.c_void_p()
        _check(_lib.rv_mem_create(n_heads, head_dim, reserve_tokens, max_tokens, ctypes.byref(h)))
        self.handle = h
        self.n_heads = n_heads

    def close(self):
        if self.handle:
            _lib.rv_mem_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def len(self):
        return _lib.rv_mem_len(self.handle)

    @property
    def capacity(self):
        return _lib.rv_mem_capacity(self.handle)

    def view(self):
        """(memK pointer, memV pointer, head stride in tokens)."""
        k, v, s = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
        _check(_lib.rv_mem_view(self.handle, ctypes.byref(k), ctypes.byref(v), ctypes.byref(s)))
        return k.value or 0, v.value or 0, s.value

    def reserve(self, tokens, stream=None):
        _check(_lib.rv_mem_reserve(self.handle, tokens, _stream(stream)))

    def reset(self):
        _check(_lib.rv_mem_reset(self.handle))

    def truncate(self, n_rows):
        """rv_mem_truncate: drop the newest rows (host-side length change only)."""
        _check(_lib.rv_mem_truncate(self.handle, n_rows))

    def write(self, K, V, frame_id=-1, stream=None):
        """Overwrite rows 0..n-1 with K, V ([H, n, 64], 2-byte elements, host or device)."""
        if K.shape != V.shape or K.shape[0] != self.n_heads or K.shape[2] != HEAD_DIM:
            raise ValueError("K, V must both be [n_heads, n_rows, 64]")
        kp, vp = _host_or_dev_ptr(K), _host_or_dev_ptr(V)
        _check(_lib.rv_mem_write(self.handle, kp, vp, K.shape[1], frame_id, _stream(stream)))

    def read(self, stream=None):
        """(K, V, prov) of the valid rows as CPU torch tensors (int16 bits / int32)."""
        n = self.len
        K = torch.empty((self.n_heads, n, HEAD_DIM), dtype=torch.int16, pin_memory=True)
        V = torch.empty_like(K, pin_memory=True)
        prov = torch.empty((self.n_heads, n, 2), dtype=torch.int32, pin_memory=True)
        _check(_lib.rv_mem_read(self.handle, ctypes.c_void_p(K.data_ptr()), ctypes.c_void_p(V.data_ptr()),
                                ctypes.c_void_p(prov.data_ptr()), _stream(stream)))
        return K, V, prov

    def stage(self, n_tokens, stream=None):
        """rv_mem_stage: room for a frame of n_tokens rows past the valid ones; returns
        (K_tail, V_tail, head_stride) device addresses / row stride."""
        k, v, hs = ctypes.c_void_p(), ctypes.c_void_p(), ctypes.c_int64()
        _check(_lib.rv_mem_stage(self.handle, n_tokens, ctypes.byref(k), ctypes.byref(v), ctypes.byref(hs),
                                 _stream(stream)))
        return k.value, v.value, hs.value

    def stage_frame(self, K, V, stream=None):
        """rv_mem_stage_frame: stage a frame given as [N, H, 64] bf16 K, V tensors."""
        N = K.shape[0]
        shp = (N, self.n_heads, HEAD_DIM)
        _check(_lib.rv_mem_stage_frame(self.handle, _ptr(K, shp, 2, "K"), _ptr(V, shp, 2, "V"), N,
                                       _stream(stream)))

    def save(self, path):
        """Write a snapshot (rows and provenance) to `path`."""
        _check(_lib.rv_mem_save(self.handle, os.fsencode(path)))

    def load(self, path):
        """Replace the contents with a snapshot written by save()."""
        _check(_lib.rv_mem_load(self.handle, os.fsencode(path)))


def _host_or_dev_ptr(t):
    if not isinstance(t, torch.Tensor) or not t.is_contiguous() or t.element_size() != 2:
        raise TypeError("expected a contiguous torch tensor with 2-byte elements")
    return ctypes.c_void_p(t.data_ptr())


def attend_frame(Q, K, V, mem, out, lse, saliency=None, qs=None, stream=None,
                 memK=None, memV=None, mem_len=None, head_stride=None):
    """rv_attend_frame.  Q, K, V, out: [N, H, 64] bf16; lse/saliency: [H, N] fp32.

    The memory is given either as a Memory (``mem``) or, with mem=None, as raw
    ``memK``/``memV`` device pointers (int or tensor), ``mem_len`` and ``head_stride``."""
    N, H, d = Q.shape
    if mem is not None:
        mk, mv, hs, ml = _mem_state(mem)
    else:
        mk = memK.data_ptr() if isinstance(memK, torch.Tensor) else (memK or 0)
        mv = memV.data_ptr() if isinstance(memV, torch.Tensor) else (memV or 0)
        ml, hs = int(mem_len or 0), int(head_stride or 0)
    shp = (N, H, d)
    q = qs if qs is None or isinstance(qs, rv_qsub) else rv_qsub(*qs)
    _check(_lib.rv_attend_frame(
        _ptr(Q, shp, 2, "Q"), _ptr(K, shp, 2, "K"), _ptr(V, shp, 2, "V"), N, mk, mv, ml, hs, H, d,
        ctypes.byref(q) if q is not None else None,
        _ptr(out, shp, 2, "out"), _ptr(lse, (H, N), 4, "lse"),
        _ptr(saliency, (H, N), 4, "saliency"), _stream(stream)))


QUERY_BLOCK = 128


def attend_frame_fused(Q, K, V, mem, out, lse, sal_tiles, qs, stream=None):
    """rv_attend_frame_fused: attention with the saliency formed in its epilogue, per
    128-query block: sal_tiles [H, ceil(N / 128), N] fp32."""
    N, H, d = Q.shape
    mk, mv, hs, ml = _mem_state(mem)
    shp = (N, H, d)
    q = qs if isinstance(qs, rv_qsub) else rv_qsub(*qs)
    _check(_lib.rv_attend_frame_fused(
        _ptr(Q, shp, 2, "Q"), _ptr(K, shp, 2, "K"), _ptr(V, shp, 2, "V"), N, mk, mv, ml, hs, H, d, ctypes.byref(q), _ptr(out, shp, 2, "out"),
        _ptr(lse, (H, N), 4, "lse"), _ptr(sal_tiles, (H, -(-N // QUERY_BLOCK), N), 4, "sal_tiles"),
        _stream(stream)))


def admit_layers_tiled(sal_tiles, budget, K, V, mems, frame_id, saliency_out=None, idx_out=None, stream=None):
    """rv_admit_layers_tiled over lists of per-layer sal_tiles [H, ceil(N / 128), N], K, V
    [N, H, 64] and Memory objects."""
    L = len(mems)
    N, H, d = K[0].shape
    arr = ctypes.c_void_p * L

    def pack(ts, shape, itemsize, what):
        return _ptrs(ts, L, shape, itemsize, what)

    sal = pack(saliency_out, (H, N), 4, "saliency_out") if saliency_out is not None else None
    idx = pack(idx_out, (H, budget), 4, "idx_out") if idx_out is not None else None
    _check(_lib.rv_admit_layers_tiled(
        L, pack(sal_tiles, (H, -(-N // QUERY_BLOCK), N), 4, "sal_tiles"), N, budget, pack(K, (N, H, d), 2, "K"),
        pack(V, (N, H, d), 2, "V"), arr(*[m.handle for m in mems]), frame_id, sal, idx, _stream(stream)))


def attend_staged(Q, mem, out, lse, saliency=None, qs=None, stream=None):
    """rv_attend_staged: attention of Q [N, H, 64] over mem's rows and its staged frame."""
    N, H, d = Q.shape
    q = qs if qs is None or isinstance(qs, rv_qsub) else rv_qsub(*qs)
    _check(_lib.rv_attend_staged(
        _ptr(Q, (N, H, d), 2, "Q"), N, mem.handle, ctypes.byref(q) if q is not None else None,
        _ptr(out, (N, H, d), 2, "out"), _ptr(lse, (H, N), 4, "lse"), _ptr(saliency, (H, N), 4, "saliency"),
        _stream(stream)))


def admit_staged_layers(Q, lse, qs, budget, mems, frame_id, saliency_out=None, idx_out=None, stream=None):
    """rv_admit_staged_layers over lists of per-layer Q [N, H, 64], lse [H, N] and Memory
    objects whose frames are staged."""
    L = len(mems)
    N, H, d = Q[0].shape
    arr = ctypes.c_void_p * L

    def pack(ts, shape, itemsize, what):
        return _ptrs(ts, L, shape, itemsize, what)

    q = qs if isinstance(qs, rv_qsub) else rv_qsub(*qs)
    sal = pack(saliency_out, (H, N), 4, "saliency_out") if saliency_out is not None else None
    idx = pack(idx_out, (H, budget), 4, "idx_out") if idx_out is not None else None
    _check(_lib.rv_admit_staged_layers(
        L, pack(Q, (N, H, d), 2, "Q"), pack(lse, (H, N), 4, "lse"), N, ctypes.byref(q), budget,
        arr(*[m.handle for m in mems]), frame_id, sal, idx, _stream(stream)))


def admit(saliency, budget, K, V, mem, frame_id, idx_out=None, stream=None):
    """rv_admit: per-head top-`budget` of saliency [H, N], append K/V rows to mem."""
    N, H, d = K.shape
    _check(_lib.rv_admit(_ptr(saliency, (H, N), 4, "saliency"), budget, _ptr(K, (N, H, d), 2, "K"),
                         _ptr(V, (N, H, d), 2, "V"), N, mem.handle, frame_id,
                         _ptr(idx_out, (H, budget), 4, "idx_out"), _stream(stream)))


def admit_layers(Q, K, V, lse, qs, budget, mems, frame_id, saliency_out=None, idx_out=None,
                 stream=None, shared=False):
    """rv_admit_layers (shared=False: head-specific retention) or rv_admit_layers_shared
    (shared=True: one selection per layer on the head-summed saliency) over lists of
    per-layer tensors and Memory objects."""
    L = len(mems)
    N, H, d = K[0].shape
    shp = (N, H, d)
    arr = ctypes.c_void_p * L

    def pack(ts, shape, itemsize, what):
        return _ptrs(ts, L, shape, itemsize, what)

    q = qs if isinstance(qs, rv_qsub) else rv_qsub(*qs)
    sal = pack(saliency_out, (H, N), 4, "saliency_out") if saliency_out is not None else None
    idx = pack(idx_out, (H, budget), 4, "idx_out") if idx_out is not None else None
    fn = _lib.rv_admit_layers_shared if shared else _lib.rv_admit_layers
    _check(fn(
        L, pack(Q, shp, 2, "Q"), pack(K, shp, 2, "K"), pack(V, shp, 2, "V"), pack(lse, (H, N), 4, "lse"),
        N, ctypes.byref(q), budget, arr(*[m.handle for m in mems]), frame_id, sal, idx, _stream(stream)))



def stage_frames(mems, K, V, stream=None):
    """rv_mem_stage_frames: stage each layer's frame (K[l], V[l]: [N, H, 64] bf16) in
    mems[l], one copy launch for up to 24 layers."""
    L = len(mems)
    N = K[0].shape[0]
    shp = (N, mems[0].n_heads, HEAD_DIM)
    arr = ctypes.c_void_p * L
    _check(_lib.rv_mem_stage_frames(L, arr(*[m.handle for m in mems]),
                                    _ptrs(K, L, shp, 2, "K"), _ptrs(V, L, shp, 2, "V"), N,
                                    _stream(stream)))

# ---- a layer's projections to frame tensors ----------------------------------------

RV_BF16, RV_F32 = range(2)
_NORMS = {None: 0, "rms": 1, "layer": 2}


class QKVPrep:
    """What rv_prepare_qkv does to a layer's projections (rv_qkv_prep): the norm of query and key
    heads (None, "rms" or "layer") with fp32 [64] weights and biases (each may be None), and the
    rotation by `axes` position axes (0: none) of frequency base `base`."""

    def __init__(self, n_q_heads, n_kv_heads, norm="layer", eps=1e-5, axes=2, base=100.0, q_weight=None, q_bias=None,
                 k_weight=None, k_bias=None):
        if norm not in _NORMS:
            raise ValueError(f"norm: {norm!r} is not one of None, 'rms', 'layer'")
        self.vectors = (q_weight, q_bias, k_weight, k_bias)  # (kept alive: the struct holds addresses)
        ptrs = [_fp32(t, (HEAD_DIM,), name)
                for t, name in zip(self.vectors, ("q_weight", "q_bias", "k_weight", "k_bias"))]
        devices = {t.get_device() for t in self.vectors if t is not None}
        if len(devices) > 1:
            raise ValueError("weights and biases on different devices")
        self.device = devices.pop() if devices else None
        self.c = rv_qkv_prep(n_q_heads, n_kv_heads, _NORMS[norm], axes, eps, base, *ptrs)
        self.n_q_heads, self.n_kv_heads, self.axes = n_q_heads, n_kv_heads, axes
        self._args = (ctypes.addressof(self.c), axes, n_q_heads, n_kv_heads)

    def _check_device(self, device):
        if self.device is not None and self.device != device:
            raise ValueError(f"weights and biases on device {self.device} while device {device} is current")


def _rows(t, heads, what):
    """(address, elements between rows, rv_dtype) of [N, heads * 64] or [N, heads, 64] rows at any
    distance, or (None, 0, None)."""
    if t is None:
        return None, 0, None
    if not isinstance(t, torch.Tensor):
        raise TypeError(f"{what}: expected a torch tensor")
    if not t.is_cuda:
        raise ValueError(f"{what}: must be a device tensor")
    n = t.shape[0] if t.dim() else 0
    width = heads * HEAD_DIM
    if tuple(t.shape) not in ((n, width), (n, heads, HEAD_DIM)):
        raise ValueError(f"{what}: shape {tuple(t.shape)}, expected {(n, width)} or {(n, heads, HEAD_DIM)}")
    if t.stride(-1) != 1 or (t.dim() == 3 and heads > 1 and t.stride(1) != HEAD_DIM):
        raise ValueError(f"{what}: the elements of a row must be contiguous")
    if t.dtype == torch.float32:
        dtype = RV_F32
    elif t.dtype in _BF16_BITS:
        dtype = RV_BF16
    else:
        raise TypeError(f"{what}: dtype {t.dtype}, expected bfloat16 or float32")
    return t.data_ptr(), t.stride(0) if n > 1 else width, dtype


def _prep_rows(ts, n):
    """_rows of several (tensor, heads, name), which must hold n rows of one dtype."""
    out, dtype = [], None
    for t, heads, what in ts:
        p, stride, d = _rows(t, heads, what)
        if t is not None:
            if t.shape[0] != n:
                raise ValueError(f"{what}: {t.shape[0]} rows, expected {n}")
            if dtype not in (None, d):
                raise TypeError(f"{what}: {t.dtype} beside another dtype")
            dtype = d
        out += [p, stride]
    return out, dtype


def _positions(prep, pos, n):
    if prep.axes == 0:
        return None
    return _int32(pos, (n,) if prep.axes == 1 and pos is not None and pos.dim() == 1 else (n, prep.axes), "pos")


def prepare_qkv(prep, q, k, v, pos, Q, K, V, stream=None):
    """rv_prepare_qkv: q [N, Hq * 64], k, v [N, Hk * 64] (bf16 or fp32, rows at any distance) to the frame
    tensors Q [N, Hq, 64], K, V [N, Hk, 64] bf16; pos [N, axes] int32.  v and V may be None."""
    device, s = _where(stream)
    prep._check_device(device)
    if _made(_bind.prepare(*prep._args, device, s, q, k, v, pos, Q, K, V)):
        return
    _same_device(device, q, k, v, pos, Q, K, V)
    N, Hq, Hk = q.shape[0], prep.n_q_heads, prep.n_kv_heads
    src, dtype = _prep_rows(((q, Hq, "q"), (k, Hk, "k"), (v, Hk, "v")), N)
    _check(_lib.rv_prepare_qkv(ctypes.byref(prep.c), *src, dtype, N, _positions(prep, pos, N),
                               _bf16(Q, (N, Hq, HEAD_DIM), "Q"), _bf16(K, (N, Hk, HEAD_DIM), "K"),
                               _bf16(V, (N, Hk, HEAD_DIM), "V"), s))


def stage_qkv(prep, q, k, v, pos, Q, mem, stream=None):
    """rv_mem_stage_qkv: prepare_qkv whose K and V become the frame staged in mem."""
    device = torch.cuda.current_device()
    prep._check_device(device)
    _same_device(device, q, k, v, pos, Q)
    N, Hq, Hk = q.shape[0], prep.n_q_heads, prep.n_kv_heads
    src, dtype = _prep_rows(((q, Hq, "q"), (k, Hk, "k"), (v, Hk, "v")), N)
    _check(_lib.rv_mem_stage_qkv(mem.handle, ctypes.byref(prep.c), *src, dtype, N, _positions(prep, pos, N),
                                 _bf16(Q, (N, Hq, HEAD_DIM), "Q"), _stream(stream)))


def prepare_qkv_bwd(prep, q, k, pos, dQ, dK, dV, dq, dk, dv, dq_weight=None, dq_bias=None, dk_weight=None,
                    dk_bias=None, stream=None):
    """rv_prepare_qkv_bwd: the gradients dq, dk, dv of prepare_qkv's inputs (their dtype, rows at any
    distance) and, where given, of the weights and biases ([64] fp32, overwritten), from dQ [N, Hq, 64]
    and dK, dV [N, Hk, 64] bf16.  dV and dv may be None.  No call here is recorded by autograd: a program's own
    torch.autograd.Function calls this one."""
    device, s = _where(stream)
    prep._check_device(device)
    if _made(_bind.prepare_bwd(*prep._args, device, s, q, k, pos, dQ, dK, dV, dq, dk, dv, dq_weight, dq_bias,
                               dk_weight, dk_bias)):
        return
    _same_device(device, q, k, pos, dQ, dK, dV, dq, dk, dv, dq_weight, dq_bias, dk_weight, dk_bias)
    N, Hq, Hk = q.shape[0], prep.n_q_heads, prep.n_kv_heads
    rows, dtype = _prep_rows(((q, Hq, "q"), (k, Hk, "k"), (dq, Hq, "dq"), (dk, Hk, "dk"), (dv, Hk, "dv")), N)
    sums = [_fp32(t, (HEAD_DIM,), name) for t, name in (
        (dq_weight, "dq_weight"), (dq_bias, "dq_bias"), (dk_weight, "dk_weight"), (dk_bias, "dk_bias"))]
    _check(_lib.rv_prepare_qkv_bwd(ctypes.byref(prep.c), *rows[:4], dtype, N, _positions(prep, pos, N),
                                   _bf16(dQ, (N, Hq, HEAD_DIM), "dQ"), _bf16(dK, (N, Hk, HEAD_DIM), "dK"),
                                   _bf16(dV, (N, Hk, HEAD_DIM), "dV"), *rows[4:], *sums, s))


# ---- sequences in pages ----------------------------------------------------------------

PAGE_ROWS = 64


def _ints(values, n, what, ctype=ctypes.c_int):
    if values is None:
        return None
    if len(values) != n:
        raise ValueError(f"{what}: {len(values)} values for {n} sequences")
    return (ctype * n)(*values)


class Pool:
    """Sequences of rows in pages of 64 rows, shared between forks (rv_pool).  Sequences are
    numbers that open() and fork() give."""

    def __init__(self, n_heads, n_pages, max_seqs, max_rows, head_dim=HEAD_DIM):
        self.handle = None
        h = ctypes.c_void_p()
        _check(_lib.rv_pool_create(n_heads, head_dim, n_pages, max_seqs, max_rows, ctypes.byref(h)))
        self.handle = h
        self.n_heads = n_heads

    @property
    def _address(self):
        return self.handle.value if self.handle else 0

    def close(self):
        if self.handle:
            _lib.rv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    @property
    def free_pages(self):
        return _lib.rv_pool_free_pages(self.handle)

    def open(self):
        """rv_pool_open: a new, empty sequence."""
        s = ctypes.c_int()
        _check(_lib.rv_pool_open(self.handle, ctypes.byref(s)))
        return s.value

    def len(self, seq):
        """Rows of a sequence; -1 if it is not open."""
        return _lib.rv_pool_len(self.handle, seq)

    def fork(self, seq, n_rows=None, n=1, stream=None):
        """rv_pool_fork: a list of n new sequences that share the first n_rows rows (default: all)."""
        rows = self.len(seq) if n_rows is None else n_rows
        s = _where(stream)[1]
        out = _bind.fork(self._address, s, seq, rows, n)
        if isinstance(out, list):
            return out
        if not _made(out):
            out = (ctypes.c_int * n)()
            _check(_lib.rv_pool_fork(self.handle, seq, rows, n, out, s))
        return list(out)

    def release(self, seqs):
        """rv_pool_close: close sequences; pages without another user are free."""
        if _made(_bind.release(self._address, seqs)):
            return
        _check(_lib.rv_pool_close(self.handle, len(seqs), _ints(seqs, len(seqs), "seqs")))

    def truncate(self, seq, n_rows):
        """rv_pool_truncate: drop the newest rows (host-side only)."""
        _check(_lib.rv_pool_truncate(self.handle, seq, n_rows))

    def append(self, seqs, K, V, n_rows, stream=None):
        """rv_pool_append: n_rows[i] rows of K, V [sum of n_rows, H, 64] to seqs[i]."""
        device, s = _where(stream)
        if _made(_bind.append(self._address, self.n_heads, device, s, seqs, K, V, n_rows)):
            return
        _same_device(device, K, V)
        n = len(seqs)
        shp = (sum(n_rows), self.n_heads, HEAD_DIM)
        _check(_lib.rv_pool_append(self.handle, n, _ints(seqs, n, "seqs"), _bf16(K, shp, "K"), _bf16(V, shp, "V"),
                                   _ints(n_rows, n, "n_rows"), s))

    def gather(self, seqs, K, V, n_rows, first=None, stream=None):
        """rv_pool_gather: rows first[i] (default 0) .. + n_rows[i] of seqs[i] to the next [H, n_rows[i], 64] of K
        and V (contiguous, sum of n_rows * H rows in all; either may be None)."""
        device, s = _where(stream)
        if _made(_bind.gather(self._address, self.n_heads, device, s, seqs, n_rows, first, K, V)):
            return
        _same_device(device, K, V)
        n, size = len(seqs), sum(n_rows) * self.n_heads * HEAD_DIM
        for t, what in ((K, "K"), (V, "V")):
            if t is not None and t.numel() != size:
                raise ValueError(f"{what}: {t.numel()} elements, expected {size}")
        _check(_lib.rv_pool_gather(
            self.handle, n, _ints(seqs, n, "seqs"), _ints(first, n, "first", ctypes.c_int64),
            _ints(n_rows, n, "n_rows", ctypes.c_int64), K if K is None else _bf16(K, tuple(K.shape), "K"),
            V if V is None else _bf16(V, tuple(V.shape), "V"), s))

    def compact(self, seqs, keep, n_keep, first=None, stream=None):
        """rv_pool_compact: seqs[i] keeps its rows before first[i] (default 0) and the n_keep[i] rows of each
        head that keep (int32, [H, n_keep[i]] for each i in turn) names."""
        device, s = _where(stream)
        if _made(_bind.compact(self._address, self.n_heads, device, s, seqs, n_keep, first, keep)):
            return
        _same_device(device, keep)
        n, size = len(seqs), sum(n_keep) * self.n_heads
        if keep is not None and (keep.numel() != size or keep.dtype != torch.int32):
            raise ValueError(f"keep: {keep.numel()} values of {keep.dtype}, expected {size} of torch.int32")
        _check(_lib.rv_pool_compact(self.handle, n, _ints(seqs, n, "seqs"), _ints(first, n, "first", ctypes.c_int64),
                                    _ints(n_keep, n, "n_keep", ctypes.c_int64),
                                    keep if keep is None else _ptr(keep, tuple(keep.shape), 4, "keep"), s))


def attend_seqs(Q, K, V, pool, seqs, n_tokens, out, lse, stream=None):
    """rv_attend_seqs: the queries of several sequences, Q, out [sum of n_tokens, Hq, 64] bf16, over the
    sequences' rows and (unless None) their own keys K, V [sum of n_tokens, H, 64]; lse: fp32,
    [Hq, n_tokens[i]] for each i in turn ([n, Hq, N] where all have N tokens)."""
    device, s = _where(stream)
    if _made(_bind.attend(pool._address, pool.n_heads, device, s, seqs, n_tokens, Q, K, V, out, lse)):
        return
    _same_device(device, Q, K, V, out, lse)
    n, total = len(seqs), sum(n_tokens)
    Hq = Q.shape[1]
    shp, kv = (total, Hq, HEAD_DIM), (total, pool.n_heads, HEAD_DIM)
    if lse.numel() != total * Hq:
        raise ValueError(f"lse: {lse.numel()} elements, expected {total * Hq}")
    _check(_lib.rv_attend_seqs(pool.handle, n, _ints(seqs, n, "seqs"), _ints(n_tokens, n, "n_tokens"),
                               _bf16(Q, shp, "Q"), _bf16(K, kv, "K"), _bf16(V, kv, "V"), Hq,
                               _bf16(out, shp, "out"), _fp32(lse, tuple(lse.shape), "lse"), s))


def admit_seqs(Q, K, V, lse, qs, budget, pool, seqs, saliency_out, idx_out, stream=None):
    """rv_admit_seqs: each frame's `budget` most salient rows per head to its sequence.  Q, K, V
    [n, N, H, 64] bf16; lse, saliency_out [n, H, N] fp32; idx_out [n, H, budget] int32."""
    _same_device(torch.cuda.current_device(), Q, K, V, lse, saliency_out, idx_out)
    n, N, H, d = Q.shape
    if (n, H) != (len(seqs), pool.n_heads):
        raise ValueError(f"Q: {n} frames of {H} heads for {len(seqs)} sequences of {pool.n_heads} heads")
    shp = (n, N, H, d)
    q = qs if isinstance(qs, rv_qsub) else rv_qsub(*qs)
    _check(_lib.rv_admit_seqs(pool.handle, n, _ints(seqs, n, "seqs"), _bf16(Q, shp, "Q"), _bf16(K, shp, "K"),
                              _bf16(V, shp, "V"), _fp32(lse, (n, H, N), "lse"), N, ctypes.byref(q), budget,
                              _fp32(saliency_out, (n, H, N), "saliency_out"),
                              _int32(idx_out, (n, H, budget), "idx_out"), _stream(stream)))


# ---- seeded stream generator on the GPU (benchmark inputs) -------------------------
_synth = None


def _load_synth():
    global _synth
    if _synth is None:
        if not os.path.exists(SYNTH_LIB_PATH):
            raise ImportError(f"{SYNTH_LIB_PATH} is not built; run __graft_entry__.build()")
        s = ctypes.CDLL(SYNTH_LIB_PATH)
        s.rvs_frame_qkv.argtypes = [ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                    ctypes.c_int, ctypes.c_int, ctypes.c_float, ctypes.c_int, ctypes.c_double,
                                    ctypes.c_double, ctypes.c_void_p, ctypes.c_void_p]
        s.rvs_frame_qkv.restype = ctypes.c_int
        s.rvs_normal_bf16.argtypes = [ctypes.c_uint64, ctypes.c_uint32, ctypes.c_int, ctypes.c_int,
                                      ctypes.c_int64, ctypes.c_float, ctypes.c_void_p, ctypes.c_void_p]
        s.rvs_normal_bf16.restype = ctypes.c_int
        _synth = s
    return _synth


def gpu_frame_qkv(cfg, frame, out, layer0=0, n_layers=None, stream=None):
    """Fill out = [n_layers, 3, N, H, 64] (2-byte) with frame `frame` of cfg's stream."""
    n_layers = cfg.n_layers if n_layers is None else n_layers
    shape = (n_layers, 3, cfg.n_tokens, cfg.n_heads, cfg.head_dim)
    rc = _load_synth().rvs_frame_qkv(cfg.seed, frame & 0xFFFFFFFF, layer0, n_layers, cfg.n_tokens, cfg.n_heads,
                                     cfg.head_dim, cfg.sigma, cfg.n_plant, cfg.alpha, cfg.lognormal_sigma,
                                     _ptr_python(out, shape, 2, "out"), _stream(stream))
    if rc != 0:
        raise RVError(rc, "rvs_frame_qkv failed")


def gpu_normal(seed, frame, layer, tag, out, sigma, stream=None):
    rc = _load_synth().rvs_normal_bf16(seed, frame & 0xFFFFFFFF, layer, tag, out.numel(), sigma,
                                       _ptr_python(out, None, 2, "out"), _stream(stream))
    if rc != 0:
        raise RVError(rc, "rvs_normal_bf16 failed")
