"""ctypes binding of libburst.so: same names as the C ABI, argument marshalling only.

Every step of the path runs inside the library's HIP kernels; nothing here computes.
PyTorch tensors are used as device buffers; kernels are enqueued on torch's current
stream.  There is no fallback: if the library is missing, loading raises.
"""
import ctypes
import importlib.util
import os
import re

import torch

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libburst.so")

BURST_BF16, BURST_F32 = 0, 1

EXPORTS = [
    "burst_state_init", "burst_local_fwd", "burst_finalize", "burst_merge_state",
    "burst_bwd_prepare", "burst_local_bwd", "burst_local_bwd_dq", "burst_local_bwd_dkv", "burst_event_create", "burst_event_record",
    "burst_event_elapsed_ms", "burst_event_destroy", "burst_strerror", "burst_version",
    "burst_materialized_workspace_bytes", "burst_local_fwd_materialized", "burst_workspace_bytes",
    "burst_materialized_bwd_workspace_bytes", "burst_local_bwd_materialized", "burst_set_kernel_family",
    "burst_kernel_family_for", "burst_local_bwd_static", "burst_probe_mfma", "burst_probe_atomic_dq",
    "burst_walk_fwd", "burst_walk_bwd", "burst_walk_workspace_bytes", "burst_walk_dkv_form",
    "burst_rotate", "burst_norm_rotate", "burst_norm_rotate_bwd", "burst_norm_workspace_bytes", "burst_cache_append", "burst_cache_store", "burst_paged_fwd", "burst_paged_workspace_bytes", "burst_paged_tree_fwd",
    "burst_cache_plan", "burst_cache_keep",
]


class BurstParams(ctypes.Structure):
    _fields_ = [
        ("B", ctypes.c_int32), ("H", ctypes.c_int32), ("Nq", ctypes.c_int32), ("Nc", ctypes.c_int32),
        ("d", ctypes.c_int32), ("dtype", ctypes.c_int32), ("causal", ctypes.c_int32),
        ("scale", ctypes.c_float), ("q_off", ctypes.c_int64), ("k_off", ctypes.c_int64),
        ("window", ctypes.c_int64), ("block_mask", ctypes.c_void_p), ("block", ctypes.c_int32),
        ("kv_heads", ctypes.c_int32), ("block_mask_stride", ctypes.c_int64),
        ("q_strides", ctypes.c_int64 * 3), ("kv_strides", ctypes.c_int64 * 3),
    ]


class BurstChunk(ctypes.Structure):
    _fields_ = [
        ("K", ctypes.c_void_p), ("V", ctypes.c_void_p), ("dK", ctypes.c_void_p), ("dV", ctypes.c_void_p),
        ("block_mask", ctypes.c_void_p), ("block_mask_stride", ctypes.c_int64), ("k_off", ctypes.c_int64),
        ("kv_strides", ctypes.c_int64 * 3), ("Nc", ctypes.c_int32), ("reserved", ctypes.c_int32),
    ]


class BurstRotary(ctypes.Structure):
    _fields_ = [("turns", ctypes.c_void_p), ("dims", ctypes.c_int32), ("interleaved", ctypes.c_int32),
                ("amplitude", ctypes.c_float), ("inverse", ctypes.c_int32)]


class BurstRows(ctypes.Structure):
    _fields_ = [("x", ctypes.c_void_p), ("y", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("positions_stride", ctypes.c_int64), ("offset", ctypes.c_int64),
                ("x_strides", ctypes.c_int64 * 3), ("y_strides", ctypes.c_int64 * 3),
                ("B", ctypes.c_int32), ("heads", ctypes.c_int32), ("rows", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class BurstNormRows(ctypes.Structure):
    _fields_ = [("rows", BurstRows), ("from_", ctypes.c_void_p), ("from_strides", ctypes.c_int64 * 3), ("weight", ctypes.c_int32),
                ("reserved", ctypes.c_int32)]


class BurstNormWeight(ctypes.Structure):
    _fields_ = [("w", ctypes.c_void_p), ("dw", ctypes.c_void_p), ("f32", ctypes.c_int32), ("reserved", ctypes.c_int32)]


class BurstStore(ctypes.Structure):
    _fields_ = [("q_weight", ctypes.c_void_p), ("k_weight", ctypes.c_void_p), ("q_weight_f32", ctypes.c_int32), ("k_weight_f32", ctypes.c_int32),
                ("eps", ctypes.c_float), ("reserved", ctypes.c_int32), ("slots", ctypes.c_void_p), ("positions", ctypes.c_void_p),
                ("offsets", ctypes.c_void_p)]


class BurstPlan(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("sequences", "rows", "pages", "page", "width", "words", "most", "window")] + [
        ("added", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
        ("free_pages", ctypes.c_void_p), ("free_count", ctypes.c_void_p), ("parents", ctypes.c_void_p), ("parents_stride", ctypes.c_int64),
        ("starts", ctypes.c_void_p), ("totals", ctypes.c_void_p), ("slots", ctypes.c_void_p), ("positions", ctypes.c_void_p), ("tree", ctypes.c_void_p)]


class BurstPagedParams(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in ("sequences", "rows", "H", "kv_heads", "d", "dtype", "pages", "page", "width",
                                              "max_new", "causal", "out_f32")] + [
        ("scale", ctypes.c_float), ("full_p", ctypes.c_int32), ("window", ctypes.c_int64),
        ("starts", ctypes.c_void_p), ("lengths", ctypes.c_void_p), ("table", ctypes.c_void_p), ("table_stride", ctypes.c_int64),
        ("page_strides", ctypes.c_int64 * 3), ("q_strides", ctypes.c_int64 * 2), ("kv_strides", ctypes.c_int64 * 2),
        ("o_strides", ctypes.c_int64 * 2)]


class BurstError(RuntimeError):
    def __init__(self, code, where):
        self.code = code
        super().__init__(f"{where}: {strerror(code)} (status {code})")


def from_native(e):
    """The exception of a failed library call inside the torch module as a BurstError (others as they are)."""
    m = re.match(r"(burst_\w+): .* \(status (-\d+)\)", str(e))
    return BurstError(int(m.group(2)), m.group(1)) if m else e


_lib, _torch_module, _walk_module = None, None, None
TORCH_LIB_PATH = os.path.join(_HERE, "_burst_torch.so")


def load_torch_module():
    """Loads the torch module of the differentiable call (once).  Raises if it has not been built."""
    global _torch_module
    if _torch_module is None:
        if not os.path.exists(TORCH_LIB_PATH):
            raise FileNotFoundError(
                f"{TORCH_LIB_PATH} not found: build it first (python -c 'import __graft_entry__ as g; g.build()')")
        load()
        spec = importlib.util.spec_from_file_location("_burst_torch", TORCH_LIB_PATH)
        module = importlib.util.module_from_spec(spec)
        spec.loader.exec_module(module)
        _torch_module = module
    return _torch_module


def walk_module():
    """The torch module for RingWalk's native calls, or None where it is not built or does not load (looked for once): a walk
    marshalled here needs libburst.so alone."""
    global _walk_module
    if _walk_module is None:
        try:
            _walk_module = load_torch_module()
        except (ImportError, OSError):
            _walk_module = False
    return _walk_module or None


def load():
    """Loads the shared library (once).  Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise FileNotFoundError(
            f"{LIB_PATH} not found: build it first (python -c 'import __graft_entry__ as g; g.build()')")
    lib = ctypes.CDLL(LIB_PATH)
    vp, fp, pp = ctypes.c_void_p, ctypes.c_void_p, ctypes.POINTER(BurstParams)
    lib.burst_state_init.argtypes = [fp, fp, fp, pp, vp]
    lib.burst_local_fwd.argtypes = [vp, vp, vp, fp, fp, fp, pp, vp]
    lib.burst_finalize.argtypes = [fp, fp, fp, vp, fp, pp, vp]
    lib.burst_materialized_workspace_bytes.argtypes = [pp]
    lib.burst_materialized_workspace_bytes.restype = ctypes.c_size_t
    lib.burst_materialized_bwd_workspace_bytes.argtypes = [pp]
    lib.burst_materialized_bwd_workspace_bytes.restype = ctypes.c_size_t
    lib.burst_workspace_bytes.argtypes = [pp]
    lib.burst_workspace_bytes.restype = ctypes.c_size_t
    lib.burst_local_fwd_materialized.argtypes = [vp, vp, vp, fp, fp, fp, vp, ctypes.c_size_t, pp, vp]
    lib.burst_local_fwd_materialized.restype = ctypes.c_int
    lib.burst_local_bwd_materialized.argtypes = [vp, vp, vp, vp, fp, fp, fp, fp, fp, ctypes.c_int, ctypes.c_int,
                                                 vp, ctypes.c_size_t, pp, vp]
    lib.burst_local_bwd_materialized.restype = ctypes.c_int
    lib.burst_merge_state.argtypes = [fp, fp, fp, fp, fp, fp, pp, vp]
    lib.burst_bwd_prepare.argtypes = [vp, vp, fp, pp, vp]
    lib.burst_local_bwd.argtypes = [vp, vp, vp, vp, vp, fp, fp, fp, fp, fp, ctypes.c_int, ctypes.c_int, pp, vp]
    lib.burst_local_bwd_static.argtypes = [vp, vp, vp, vp, vp, fp, fp, fp, fp, ctypes.c_int, ctypes.c_int, pp, vp]
    lib.burst_local_bwd_static.restype = ctypes.c_int
    lib.burst_local_bwd_dq.argtypes = [vp, vp, vp, vp, fp, fp, fp, ctypes.c_int, pp, vp]
    lib.burst_local_bwd_dkv.argtypes = [vp, vp, vp, vp, fp, fp, fp, fp, ctypes.c_int, pp, vp]
    for name in ("burst_local_bwd_dq", "burst_local_bwd_dkv", "burst_state_init", "burst_local_fwd", "burst_finalize", "burst_merge_state",
                 "burst_bwd_prepare", "burst_local_bwd", "burst_event_record", "burst_version"):
        getattr(lib, name).restype = ctypes.c_int
    cp, sz, ci = ctypes.POINTER(BurstChunk), ctypes.c_size_t, ctypes.c_int
    lib.burst_walk_workspace_bytes.argtypes = [cp, ci, pp, ci]
    lib.burst_walk_workspace_bytes.restype = sz
    lib.burst_walk_dkv_form.argtypes = [cp, ci, pp, ci]
    lib.burst_walk_dkv_form.restype = ci
    lib.burst_walk_fwd.argtypes = [vp, cp, ci, fp, fp, fp, vp, fp, vp, sz, pp, vp]
    lib.burst_walk_fwd.restype = ctypes.c_int
    lib.burst_walk_bwd.argtypes = [vp, cp, ci, vp, vp, fp, fp, vp, ci, ci, ci, vp, sz, pp, vp]
    lib.burst_walk_bwd.restype = ctypes.c_int
    rp, gp = ctypes.POINTER(BurstRotary), ctypes.POINTER(BurstPagedParams)
    lib.burst_rotate.argtypes = [ctypes.POINTER(BurstRows), ci, rp, ci, ci, vp]
    lib.burst_cache_append.argtypes = [vp, vp, vp, vp, vp, vp, vp, rp, gp, vp]
    lib.burst_paged_fwd.argtypes = [vp, vp, vp, vp, fp, vp, sz, gp, vp]
    np_, wp = ctypes.POINTER(BurstNormRows), ctypes.POINTER(BurstNormWeight)
    lib.burst_norm_rotate.argtypes = [np_, ci, wp, ci, ctypes.c_float, rp, ci, ci, vp]
    lib.burst_norm_rotate_bwd.argtypes = [np_, ci, wp, ci, ctypes.c_float, rp, ci, ci, vp, sz, vp]
    lib.burst_norm_workspace_bytes.argtypes = [np_, ci, wp, ci, ctypes.c_float, rp, ci, ci]
    lib.burst_norm_workspace_bytes.restype = sz
    lib.burst_cache_store.argtypes = [vp, vp, vp, vp, vp, vp, ctypes.POINTER(BurstStore), rp, gp, vp]
    lib.burst_paged_tree_fwd.argtypes = [vp, vp, vp, vp, fp, vp, ci, ctypes.c_int64, vp, sz, gp, vp]
    lib.burst_cache_plan.argtypes = [ctypes.POINTER(BurstPlan), vp]
    lib.burst_cache_keep.argtypes = [ctypes.POINTER(vp), ci, vp, ctypes.c_int64, ci, vp, vp, gp, vp]
    for name in ("burst_cache_plan", "burst_cache_keep", "burst_paged_tree_fwd", "burst_rotate", "burst_norm_rotate", "burst_norm_rotate_bwd", "burst_cache_append", "burst_cache_store", "burst_paged_fwd"):
        getattr(lib, name).restype = ci
    lib.burst_paged_workspace_bytes.argtypes = [gp]
    lib.burst_paged_workspace_bytes.restype = sz
    lib.burst_event_create.argtypes = []
    lib.burst_event_create.restype = vp
    lib.burst_event_record.argtypes = [vp, vp]
    lib.burst_event_elapsed_ms.argtypes = [vp, vp, ctypes.POINTER(ctypes.c_float)]
    lib.burst_event_elapsed_ms.restype = ctypes.c_int
    lib.burst_event_destroy.argtypes = [vp]
    lib.burst_event_destroy.restype = None
    lib.burst_strerror.argtypes = [ctypes.c_int]
    lib.burst_strerror.restype = ctypes.c_char_p
    _lib = lib
    return lib


def strerror(code):
    return load().burst_strerror(int(code)).decode()


def version():
    return load().burst_version()


def strides_of(t):
    """(batch, head, row) element strides of a [B, H, rows, d] tensor whose last dimension is
    contiguous, for params(); None if the tensor is contiguous.  Dimensions of size 1 (whose
    stride addresses nothing) are given the row length."""
    if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
        raise ValueError("a [B, H, rows, d] tensor with a contiguous last dimension expected")
    if t.is_contiguous():
        return None
    return tuple(int(t.stride(i)) if t.shape[i] > 1 else int(t.shape[3]) for i in range(3))


def _mask(block_mask, block, B, H, Nq, Nc):
    """(address, bytes between heads' matrices) of a chunk's block flags."""
    if block_mask.dtype != torch.uint8 or not block_mask.is_cuda or not block_mask.is_contiguous():
        raise ValueError("block_mask: contiguous uint8 device tensor expected")
    if block <= 0:
        raise ValueError("block_mask needs block > 0")
    one = (-(-Nq // block), -(-Nc // block))
    if tuple(block_mask.shape) == (B, H) + one:
        return block_mask.data_ptr(), one[0] * one[1]
    if tuple(block_mask.shape) != one:
        raise ValueError("block_mask: shape must be [ceil(Nq/block), ceil(Nc/block)], alone or after [B, H]")
    return block_mask.data_ptr(), 0


def params(B, H, Nq, Nc, d, dtype, scale, causal=False, q_off=0, k_off=0, window=0, block_mask=None, block=0,
           kv_heads=0, q_strides=None, kv_strides=None):
    """block_mask: a contiguous uint8 device tensor [ceil(Nq/block), ceil(Nc/block)] shared by all
    heads, or [B, H, ceil(Nq/block), ceil(Nc/block)] with one matrix per (batch, query head) (or
    None); the caller keeps it alive and unchanged until the kernels that use these parameters
    have run.  q_strides / kv_strides: (batch, head, row) element strides of Q, dO, O and of
    K, V (see strides_of); None = contiguous."""
    code = {torch.bfloat16: BURST_BF16, torch.float32: BURST_F32, "bf16": BURST_BF16, "f32": BURST_F32}.get(dtype, dtype)
    ptr, stride = (None, 0) if block_mask is None else _mask(block_mask, block, B, H, Nq, Nc)
    return BurstParams(B, H, Nq, Nc, d, code, 1 if causal else 0, scale, q_off, k_off, window, ptr,
                       block if block_mask is not None else 0, kv_heads, stride,
                       (ctypes.c_int64 * 3)(*(q_strides or (0, 0, 0))), (ctypes.c_int64 * 3)(*(kv_strides or (0, 0, 0))))


def _ptr(t):
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    if not t.is_contiguous():
        raise ValueError("contiguous tensor expected")
    return ctypes.c_void_p(t.data_ptr())


def _strided(t, want):
    """Pointer of a storage-type tensor that must lie in memory as the parameter block says."""
    if t is None:
        return None
    if not t.is_cuda:
        raise ValueError("device tensor expected")
    want = tuple(want)
    if want == (0, 0, 0):
        if not t.is_contiguous():
            raise ValueError("contiguous tensor expected (or give its strides to params())")
    else:
        if t.dim() != 4 or (t.shape[3] > 1 and t.stride(3) != 1):
            raise ValueError("a [B, H, rows, d] tensor with a contiguous last dimension expected")
        if any(t.shape[i] > 1 and t.stride(i) != want[i] for i in range(3)):
            raise ValueError(f"tensor strides {tuple(t.stride())} differ from the parameter block's {want}")
    return ctypes.c_void_p(t.data_ptr())


def _q(t, p):
    return _strided(t, p.q_strides)


def _kv(t, p):
    return _strided(t, p.kv_strides)


def _f32(t):
    if t is not None and t.dtype != torch.float32:
        raise ValueError("float32 tensor expected")
    return _ptr(t)


def _stream():
    return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)


def _check(code, where):
    if code != 0:
        raise BurstError(code, where)


def burst_state_init(O_acc, m, l, p):
    _check(load().burst_state_init(_f32(O_acc), _f32(m), _f32(l), ctypes.byref(p), _stream()), "burst_state_init")


def burst_local_fwd(Q, K_chunk, V_chunk, O_acc, m, l, p):
    _check(load().burst_local_fwd(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _f32(O_acc), _f32(m), _f32(l),
                                  ctypes.byref(p), _stream()), "burst_local_fwd")


def burst_set_kernel_family(family):
    """0 = automatic, 1 = hand-scheduled d = 128 kernels only, 2 = plainly written ones (see burst.h)."""
    lib = load()
    lib.burst_set_kernel_family.argtypes = [ctypes.c_int]
    lib.burst_set_kernel_family.restype = ctypes.c_int
    _check(lib.burst_set_kernel_family(int(family)), "burst_set_kernel_family")


def burst_kernel_family_for(p):
    lib = load()
    lib.burst_kernel_family_for.argtypes = [ctypes.POINTER(BurstParams)]
    lib.burst_kernel_family_for.restype = ctypes.c_int
    return int(lib.burst_kernel_family_for(ctypes.byref(p)))


def burst_probe_mfma(a_from_lds, wavefronts_per_simd, operands, sink, iters):
    """operands: >= 64 KiB of bf16 on the device; sink: >= 256 * 512 float32 (see burst.h)."""
    lib = load()
    lib.burst_probe_mfma.argtypes = [ctypes.c_int, ctypes.c_int, ctypes.c_void_p, ctypes.c_void_p, ctypes.c_int,
                                     ctypes.c_void_p]
    lib.burst_probe_mfma.restype = ctypes.c_int
    if operands.numel() * operands.element_size() < 65536 or sink.numel() < 256 * 512:
        raise ValueError("burst_probe_mfma: operands >= 64 KiB and sink >= 131072 floats expected")
    _check(lib.burst_probe_mfma(int(a_from_lds), int(wavefronts_per_simd), _ptr(operands), _f32(sink), int(iters),
                                _stream()), "burst_probe_mfma")


def burst_probe_atomic_dq(dQ, heads, Nq, key_blocks, mode):
    """mode: 1 = fp32 atomic adds, 0 = plain stores, 2 = plain load-add-store (see burst.h)."""
    lib = load()
    lib.burst_probe_atomic_dq.argtypes = [ctypes.c_void_p, ctypes.c_int, ctypes.c_int, ctypes.c_int, ctypes.c_int,
                                          ctypes.c_void_p]
    lib.burst_probe_atomic_dq.restype = ctypes.c_int
    if dQ.numel() < heads * Nq * 128:
        raise ValueError("burst_probe_atomic_dq: dQ too small")
    _check(lib.burst_probe_atomic_dq(_f32(dQ), int(heads), int(Nq), int(key_blocks), int(mode), _stream()),
           "burst_probe_atomic_dq")


def burst_workspace_bytes(p):
    return int(load().burst_workspace_bytes(ctypes.byref(p)))


def burst_materialized_workspace_bytes(p):
    return int(load().burst_materialized_workspace_bytes(ctypes.byref(p)))


def burst_local_fwd_materialized(Q, K_chunk, V_chunk, O_acc, m, l, workspace, p):
    """workspace: a contiguous uint8 device tensor (see burst_materialized_workspace_bytes)."""
    _check(load().burst_local_fwd_materialized(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _f32(O_acc), _f32(m), _f32(l),
                                               _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                               ctypes.byref(p), _stream()), "burst_local_fwd_materialized")


def burst_materialized_bwd_workspace_bytes(p):
    return int(load().burst_materialized_bwd_workspace_bytes(ctypes.byref(p)))


def burst_local_bwd_materialized(Q, K_chunk, V_chunk, dO, lse, D, dQ, dK_chunk, dV_chunk, workspace, p,
                                 accumulate_dq=True, accumulate_dkv=False):
    """workspace: a contiguous uint8 device tensor (see burst_materialized_bwd_workspace_bytes)."""
    _check(load().burst_local_bwd_materialized(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _q(dO, p), _f32(lse), _f32(D),
                                               _f32(dQ), _f32(dK_chunk), _f32(dV_chunk),
                                               1 if accumulate_dq else 0, 1 if accumulate_dkv else 0,
                                               _ptr(workspace), ctypes.c_size_t(workspace.numel() * workspace.element_size()),
                                               ctypes.byref(p), _stream()), "burst_local_bwd_materialized")


def burst_finalize(O_acc, m, l, O_out, lse, p):
    _check(load().burst_finalize(_f32(O_acc), _f32(m), _f32(l), _q(O_out, p), _f32(lse),
                                 ctypes.byref(p), _stream()), "burst_finalize")


def burst_merge_state(O_a, m_a, l_a, O_b, m_b, l_b, p):
    _check(load().burst_merge_state(_f32(O_a), _f32(m_a), _f32(l_a), _f32(O_b), _f32(m_b), _f32(l_b),
                                    ctypes.byref(p), _stream()), "burst_merge_state")


def burst_bwd_prepare(O, dO, D, p):
    _check(load().burst_bwd_prepare(_q(O, p), _q(dO, p), _f32(D), ctypes.byref(p), _stream()), "burst_bwd_prepare")


def burst_local_bwd(Q, K_chunk, V_chunk, O, dO, lse, D, dQ, dK_chunk, dV_chunk, p,
                    accumulate_dq=True, accumulate_dkv=False):
    _check(load().burst_local_bwd(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _q(O, p), _q(dO, p), _f32(lse), _f32(D),
                                  _f32(dQ), _f32(dK_chunk), _f32(dV_chunk),
                                  1 if accumulate_dq else 0, 1 if accumulate_dkv else 0,
                                  ctypes.byref(p), _stream()), "burst_local_bwd")


BURST_STATIC_MAX_ROWS = 2 * 1024 * 1024


def burst_local_bwd_static(Q, K_chunk, V_chunk, O, dO, lse, dQ, dK_chunk, dV_chunk, p,
                           accumulate_dq=True, accumulate_dkv=False):
    """burst_local_bwd with D computed into the library's static device scratch: allocates nothing."""
    _check(load().burst_local_bwd_static(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _q(O, p), _q(dO, p), _f32(lse),
                                         _f32(dQ), _f32(dK_chunk), _f32(dV_chunk),
                                         1 if accumulate_dq else 0, 1 if accumulate_dkv else 0,
                                         ctypes.byref(p), _stream()), "burst_local_bwd_static")


def burst_local_bwd_dq(Q, K_chunk, V_chunk, dO, lse, D, dQ, p, accumulate_dq=True):
    _check(load().burst_local_bwd_dq(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _q(dO, p), _f32(lse), _f32(D),
                                     _f32(dQ), 1 if accumulate_dq else 0, ctypes.byref(p), _stream()),
           "burst_local_bwd_dq")


def burst_local_bwd_dkv(Q, K_chunk, V_chunk, dO, lse, D, dK_chunk, dV_chunk, p, accumulate_dkv=False):
    _check(load().burst_local_bwd_dkv(_q(Q, p), _kv(K_chunk, p), _kv(V_chunk, p), _q(dO, p), _f32(lse), _f32(D),
                                      _f32(dK_chunk), _f32(dV_chunk), 1 if accumulate_dkv else 0,
                                      ctypes.byref(p), _stream()), "burst_local_bwd_dkv")


def chunk_array(Ks, Vs, k_offs, masks, p, dKs=None, dVs=None, grad_dtype=None):
    """The chunks of a walk as the C array burst_walk_fwd / burst_walk_bwd take.  `p`: the walk's parameter
    block (its `block` is the edge of the masks' blocks).  grad_dtype: the type of dQ, which dKs and dVs must have."""
    arr = (BurstChunk * len(Ks))()
    dtype = torch.bfloat16 if p.dtype == BURST_BF16 else torch.float32
    for j in range(len(Ks)):                         # (by index: a list of values that is too short is an IndexError)
        K, V, c = Ks[j], Vs[j], arr[j]
        if not K.is_cuda or not V.is_cuda:
            raise ValueError("device tensor expected")
        if K.dtype != dtype or V.dtype != dtype or K.shape != V.shape or \
                tuple(K.shape) != (p.B, p.kv_heads or p.H, K.shape[2], p.d):
            raise ValueError("K, V: [B, kv_heads, Nc, d] of the type of Q expected")
        if not (K.is_contiguous() and V.is_contiguous()):
            s = strides_of(K) or (0, 0, 0)
            _strided(V, s)
            c.kv_strides[:] = s
        c.K, c.V, c.k_off, c.Nc = K.data_ptr(), V.data_ptr(), k_offs[j], K.shape[2]
        if masks is not None and masks[j] is not None:
            c.block_mask, c.block_mask_stride = _mask(masks[j], p.block, p.B, p.H, p.Nq, c.Nc)
        if dKs is not None:
            dK, dV = dKs[j], dVs[j]
            if dK.dtype != grad_dtype or dV.dtype != grad_dtype:
                raise ValueError("dK, dV: the type of dQ expected")
            if dK.numel() < K.numel() or dV.numel() < V.numel():
                raise ValueError("dK, dV: the sizes of K and V expected")
            c.dK, c.dV = _ptr(dK).value, _ptr(dV).value
    return arr


BURST_WALK_HALF_GRADS, BURST_WALK_NO_STATE, BURST_WALK_FORWARD = 1, 2, 4


def burst_walk_workspace_bytes(chunks, p, flags=0):
    return int(load().burst_walk_workspace_bytes(chunks, len(chunks), ctypes.byref(p), int(flags)))


def burst_walk_dkv_form(chunks, p, with_workspace=True):
    """How the backward walk's (first) dK/dV launch is laid out: 0 a workgroup per block of keys, 1 walks cut into parts,
    2 one workgroup per CU that takes several blocks in turn.  For fp32 gradients (see burst.h)."""
    form = load().burst_walk_dkv_form(chunks, len(chunks), ctypes.byref(p), 1 if with_workspace else 0)
    if form < 0:
        _check(form, "burst_walk_dkv_form")
    return form


def _bytes(ws):
    return ctypes.c_size_t(0 if ws is None else ws.numel() * ws.element_size())


def burst_walk_fwd(Q, chunks, O_acc, m, l, O_out, lse, p, workspace=None):
    """chunks: see chunk_array.  workspace: None or a contiguous device tensor.  O_acc, m, l: None = not kept."""
    _check(load().burst_walk_fwd(_q(Q, p), chunks, len(chunks), _f32(O_acc), _f32(m), _f32(l), _q(O_out, p), _f32(lse),
                                 _ptr(workspace), _bytes(workspace), ctypes.byref(p), _stream()), "burst_walk_fwd")


def burst_walk_bwd(Q, chunks, O, dO, lse, D, dQ, p, accumulate_dq=True, accumulate_dkv=False, workspace=None):
    """O given: D = rowsum(dO o O) is computed first and written; O = None: D is read.  dQ and the chunks'
    dK, dV: all fp32, or all of Q's type (then nothing accumulates)."""
    half = dQ.dtype != torch.float32
    if half and dQ.dtype != Q.dtype:
        raise ValueError("gradients: float32 or the type of Q expected")
    _check(load().burst_walk_bwd(_q(Q, p), chunks, len(chunks), _q(O, p), _q(dO, p), _f32(lse), _f32(D), _ptr(dQ),
                                 1 if accumulate_dq else 0, 1 if accumulate_dkv else 0, 1 if half else 0,
                                 _ptr(workspace), _bytes(workspace), ctypes.byref(p), _stream()), "burst_walk_bwd")


def rotary(turns, interleaved=False, amplitude=1.0, inverse=False):
    """turns: a contiguous float64 device tensor with an entry for every pair of columns (see burst.h)."""
    if turns.dtype != torch.float64:
        raise ValueError("turns: float64 tensor expected")
    r = BurstRotary(_ptr(turns), 2 * turns.numel(), 1 if interleaved else 0, amplitude, 1 if inverse else 0)
    r.holds = turns                                           # (the block has its address alone)
    return r


def burst_rotate(xs, ys, r, offsets=None, positions=None):
    """xs, ys: lists of [B, heads, rows, d] tensors with a contiguous last dimension, of one type and d; offsets: the position of row 0
    of each; positions: None, or for each None or an int64 device tensor [B, rows] with contiguous rows, to which its offset is added."""
    if len(ys) != len(xs) or any(more is not None and len(more) != len(xs) for more in (offsets, positions)):
        raise ValueError("as many ys, offsets and positions as xs expected")
    offsets, positions = offsets or [0] * len(xs), positions or [None] * len(xs)
    for x, y, at in zip(xs, ys, positions):
        if x.dtype not in (torch.bfloat16, torch.float32) or x.dtype != xs[0].dtype or x.dim() != 4 or x.shape[3] != xs[0].shape[3]:
            raise ValueError("[B, heads, rows, d] tensors of bfloat16 or float32, of one type and d, expected")
        if at is not None and (at.dtype != torch.int64 or tuple(at.shape) != (x.shape[0], x.shape[2]) or (at.shape[1] > 1 and at.stride(1) != 1)):
            raise ValueError("positions: int64 device tensor [B, rows] with contiguous rows expected")
        if x.shape != y.shape or x.dtype != y.dtype:
            raise ValueError("x, y: device tensors of the same sizes and type expected")
        if not any(strides_of(x) or (1,)) or any(n > 1 and t == 0 for n, t in zip(y.shape, y.stride())):
            # (strides of 0 throughout, as of one row that stands for all, mean dense ones in the block)
            raise ValueError("x: not one row for all, y: a place for every row expected")
    items = (BurstRows * len(xs))()
    for x, y, at, offset, c in zip(xs, ys, positions, offsets, items):
        for t, what in ((x, "x"), (y, "y"), (at, "positions")):
            if t is not None:
                _here(t, what)
        c.x_strides[:], c.y_strides[:] = strides_of(x) or (0, 0, 0), strides_of(y) or (0, 0, 0)
        c.x, c.y, c.B, c.heads, c.rows, c.offset = x.data_ptr(), y.data_ptr(), x.shape[0], x.shape[1], x.shape[2], offset
        if at is not None:
            c.positions, c.positions_stride = at.data_ptr(), at.stride(0)
    dtype = BURST_BF16 if not len(xs) or xs[0].dtype == torch.bfloat16 else BURST_F32
    _check(load().burst_rotate(items, len(xs), ctypes.byref(r), xs[0].shape[3] if len(xs) else 2, dtype, _stream()), "burst_rotate")


def _norm_call(tensors, weights, r):
    """The C arrays of a call that normalises rows.  tensors: (x, y, from or None, place of its weight or -1, offset, positions or None) for each; weights:
    (w, dw or None) for each."""
    items, ws = (BurstNormRows * len(tensors))(), (BurstNormWeight * len(weights))()
    like = tensors[0][0] if tensors else None
    if like is not None and (like.dtype not in _TYPES.values() or like.dim() != 4):
        raise ValueError("[B, heads, rows, d] tensors of bfloat16 or float32 expected")
    for c, (x, y, frm, weight, offset, at) in zip(items, tensors):
        for t, what in ((x, "x"), (y, "y"), (frm, "from")):
            if t is None:
                continue
            if t.shape != x.shape or t.dtype != like.dtype or t.dim() != 4 or t.shape[3] != like.shape[3]:
                raise ValueError(f"{what}: a tensor [B, heads, rows, d] of the sizes of x, of one type and d, expected")
            if not any(strides_of(t) or (1,)) or (t is y and any(n > 1 and s == 0 for n, s in zip(t.shape, t.stride()))):
                raise ValueError(f"{what}: not one row for all expected")   # (strides of 0 throughout mean dense ones in the block)
            _here(t, what)
        if at is not None:
            if at.dtype != torch.int64 or tuple(at.shape) != (x.shape[0], x.shape[2]) or (at.shape[1] > 1 and at.stride(1) != 1):
                raise ValueError("positions: int64 device tensor [B, rows] with contiguous rows expected")
            _here(at, "positions")
            c.rows.positions, c.rows.positions_stride = at.data_ptr(), at.stride(0)
        c.rows.x, c.rows.B, c.rows.heads, c.rows.rows, c.rows.offset = x.data_ptr(), x.shape[0], x.shape[1], x.shape[2], offset
        c.rows.x_strides[:] = strides_of(x) or (0, 0, 0)
        if y is not None:
            c.rows.y, c.rows.y_strides[:] = y.data_ptr(), strides_of(y) or (0, 0, 0)
        if frm is not None:
            c.from_, c.from_strides[:] = frm.data_ptr(), strides_of(frm) or (0, 0, 0)
        c.weight = weight
    for c, (w, dw) in zip(ws, weights):
        for t, what in ((w, "w"), (dw, "dw")):
            if t is None:
                continue
            if t.dtype != w.dtype or (like is not None and (t.dtype not in (like.dtype, torch.float32) or t.numel() != like.shape[3])) or not t.is_contiguous():
                raise ValueError(f"{what}: contiguous [d] of the tensors' type or float32 expected")
            _here(t, what)
        c.w, c.dw, c.f32 = w.data_ptr(), None if dw is None else dw.data_ptr(), 1 if w.dtype == torch.float32 else 0
    dtype = BURST_BF16 if like is None or like.dtype == torch.bfloat16 else BURST_F32
    return items, len(tensors), ws, len(weights), None if r is None else ctypes.byref(r), like.shape[3] if like is not None else 2, dtype


def burst_norm_rotate(tensors, weights, eps, r):
    """tensors: (x, y, None, place of its weight or -1, offset, positions or None) for each; weights: (w, None) for each; r: see rotary, or None."""
    items, n, ws, k, rp, d, dtype = _norm_call(tensors, weights, r)
    _check(load().burst_norm_rotate(items, n, ws, k, eps, rp, d, dtype, _stream()), "burst_norm_rotate")


def burst_norm_workspace_bytes(tensors, weights, eps, r):
    items, n, ws, k, rp, d, dtype = _norm_call(tensors, weights, r)
    return int(load().burst_norm_workspace_bytes(items, n, ws, k, eps, rp, d, dtype))


def burst_norm_rotate_bwd(tensors, weights, eps, r, workspace=None):
    """tensors: (gradient of the result, gradient of x or None, x, place of its weight or -1, offset, positions or None) for each; weights: (w, dw or
    None) for each."""
    if any(t[2] is None for t in tensors):
        raise ValueError("from: what the forward call read expected")
    items, n, ws, k, rp, d, dtype = _norm_call(tensors, weights, r)
    _check(load().burst_norm_rotate_bwd(items, n, ws, k, eps, rp, d, dtype, _ptr(workspace), _bytes(workspace), _stream()), "burst_norm_rotate_bwd")


def _rows_lie(t):
    """Whether the rows of a matrix are contiguous, one behind the other (those of an empty one may have any strides)."""
    return t.numel() == 0 or ((t.shape[1] <= 1 or t.stride(1) == 1) and (t.shape[0] <= 1 or t.stride(0) >= t.shape[1]))


def paged_params(q_rows, H, kv_heads, d, dtype, k_pages, table, lengths, starts, scale=1.0, causal=True, window=0, max_new=0, out_f32=False, full_p=False):
    """k_pages: [pages, kv_heads, page, d] (its strides go into the block; V_pages lies likewise); table [sequences, width], lengths
    [sequences], starts [sequences + 1]: int32 device tensors.  Token tensors are dense unless their strides are set in the block."""
    code = {torch.bfloat16: BURST_BF16, torch.float32: BURST_F32, "bf16": BURST_BF16, "f32": BURST_F32}.get(dtype, dtype)
    if any(t.dtype != torch.int32 for t in (table, lengths, starts)) or table.dim() != 2 or lengths.shape != table.shape[:1] or \
            starts.shape != (table.shape[0] + 1,):
        raise ValueError("table [sequences, width], lengths [sequences], starts [sequences + 1]: int32 tensors expected")
    if not lengths.is_contiguous() or not starts.is_contiguous() or not _rows_lie(table):
        raise ValueError("lengths, starts and the table's rows: contiguous expected")
    if k_pages.dim() != 4 or tuple(k_pages.shape[1::2]) != (kv_heads, d) or (d > 1 and k_pages.stride(3) != 1):
        raise ValueError("k_pages: [pages, kv_heads, page, d] with a contiguous last dimension expected")
    if any(k_pages.shape[i] > 1 and k_pages.stride(i) < d for i in range(3)):   # (strides of 0, as of an expanded tensor, mean dense ones)
        raise ValueError("pages: rows that lie in memory one after the other expected")
    p = BurstPagedParams(sequences=lengths.shape[0], rows=q_rows, H=H, kv_heads=kv_heads, d=d, dtype=code, pages=k_pages.shape[0],
                         page=k_pages.shape[2], width=table.shape[1], max_new=max_new, causal=1 if causal else 0,
                         out_f32=1 if out_f32 else 0, scale=scale, full_p=1 if full_p else 0, window=window, starts=starts.data_ptr(), lengths=lengths.data_ptr(),
                         table=table.data_ptr(), table_stride=table.stride(0) if table.shape[0] > 1 else 0)
    p.page_strides[:] = strides_of(k_pages) or (0, 0, 0)
    p.holds = (starts, lengths, table)
    return p


def _here(t, what):
    """The device that the library launches on is the current one: a tensor of another device would be read across devices."""
    if not t.is_cuda:
        raise ValueError(f"{what}: device tensor expected")
    if t.device.index != torch.cuda.current_device():
        raise ValueError(f"{what}: tensor on the current device expected")


_TYPES = {BURST_BF16: torch.bfloat16, BURST_F32: torch.float32}


def _lying(t, shape, dtype, want, what):
    """Pointer of a tensor that must have these sizes (the first one at least), this type and these strides of all dimensions but the last
    (all 0: dense)."""
    if t.dtype != dtype or t.dim() != len(shape) or t.shape[0] < shape[0] or tuple(t.shape[1:]) != tuple(shape[1:]):
        raise ValueError(f"{what}: {dtype} tensor {list(shape)} expected")
    want = tuple(want)
    if any(want):
        lies = (shape[-1] <= 1 or t.stride(-1) == 1) and all(n <= 1 or t.stride(i) == want[i] for i, n in enumerate(shape[:-1]))
    else:
        lies = t.is_contiguous()
    if not lies:
        raise ValueError(f"{what}: strides as the parameter block says expected")
    _here(t, what)
    return ctypes.c_void_p(t.data_ptr())


def _pages(t, p, what):
    return _lying(t, (p.pages, p.kv_heads, p.page, p.d), _TYPES.get(p.dtype), p.page_strides, what)


def _tokens(t, heads, strides, p, what, dtype=None):
    return _lying(t, (p.rows, heads, p.d), dtype or _TYPES.get(p.dtype), strides, what)


def _offsets(t, p):
    if t is not None and (t.dtype != torch.int64 or tuple(t.shape) != (p.sequences,)):
        raise ValueError("offsets: int64 device tensor [sequences] expected")
    return _ptr(t)


def burst_cache_append(K, V, k_pages, v_pages, Q, Q_out, offsets, r, p):
    """Q, Q_out, offsets, r: None where there are none."""
    k, v = _tokens(K, p.kv_heads, p.kv_strides, p, "K"), _tokens(V, p.kv_heads, p.kv_strides, p, "V")
    q = None if Q is None else _tokens(Q, p.H, p.q_strides, p, "Q")
    q_out = None if Q_out is None else _tokens(Q_out, p.H, p.o_strides, p, "Q_out")
    _check(load().burst_cache_append(k, v, _pages(k_pages, p, "k_pages"), _pages(v_pages, p, "v_pages"), q, q_out, _offsets(offsets, p),
                                     None if r is None else ctypes.byref(r), ctypes.byref(p), _stream()), "burst_cache_append")


def store(p, q_weight=None, k_weight=None, eps=1e-6, slots=None, positions=None, offsets=None):
    """What burst_cache_store is told beside the parameter block: weights [d] of its type or float32, slots and positions int64 [rows]."""
    s = BurstStore(eps=eps)
    for name, w in (("q_weight", q_weight), ("k_weight", k_weight)):
        if w is None:
            continue
        if w.dtype not in (_TYPES.get(p.dtype), torch.float32) or tuple(w.shape) != (p.d,) or not w.is_contiguous():
            raise ValueError(f"{name}: contiguous [d] of the block's type or float32 expected")
        _here(w, name)
        setattr(s, name, w.data_ptr())
        setattr(s, name + "_f32", 1 if w.dtype == torch.float32 else 0)
    for name, t, n in (("slots", slots, p.rows), ("positions", positions, p.rows), ("offsets", offsets, p.sequences)):
        if t is None:
            continue
        if t.dtype != torch.int64 or tuple(t.shape) != (n,) or not t.is_contiguous():
            raise ValueError(f"{name}: contiguous int64 device tensor [{n}] expected")
        _here(t, name)
        setattr(s, name, t.data_ptr())
    s.holds = (q_weight, k_weight, slots, positions, offsets)
    return s


def burst_cache_store(K, V, k_pages, v_pages, Q, Q_out, how, r, p):
    """how: see store.  Q, Q_out, r: None where there are none."""
    k, v = _tokens(K, p.kv_heads, p.kv_strides, p, "K"), _tokens(V, p.kv_heads, p.kv_strides, p, "V")
    q = None if Q is None else _tokens(Q, p.H, p.q_strides, p, "Q")
    q_out = None if Q_out is None else _tokens(Q_out, p.H, p.o_strides, p, "Q_out")
    _check(load().burst_cache_store(k, v, _pages(k_pages, p, "k_pages"), _pages(v_pages, p, "v_pages"), q, q_out, ctypes.byref(how),
                                    None if r is None else ctypes.byref(r), ctypes.byref(p), _stream()), "burst_cache_store")


def burst_paged_workspace_bytes(p):
    return int(load().burst_paged_workspace_bytes(ctypes.byref(p)))


def burst_paged_fwd(Q, k_pages, v_pages, O, lse, p, workspace=None):
    if lse.numel() < p.rows * p.H:
        raise ValueError("lse: [rows, H] expected")
    _check(load().burst_paged_fwd(_tokens(Q, p.H, p.q_strides, p, "Q"), _pages(k_pages, p, "k_pages"), _pages(v_pages, p, "v_pages"),
                                  _tokens(O, p.H, p.o_strides, p, "O", torch.float32 if p.out_f32 else None), _f32(lse),
                                  _ptr(workspace), _bytes(workspace), ctypes.byref(p), _stream()), "burst_paged_fwd")


def burst_paged_tree_fwd(Q, k_pages, v_pages, O, lse, tree, p, workspace=None):
    """tree: int64 device tensor [rows, words] with contiguous rows (see burst.h)."""
    if lse.numel() < p.rows * p.H:
        raise ValueError("lse: [rows, H] expected")
    if tree.dtype != torch.int64 or tree.dim() != 2 or tree.shape[0] != p.rows or not _rows_lie(tree):
        raise ValueError("tree: int64 [rows, words] with contiguous rows expected")
    _here(tree, "tree")
    _check(load().burst_paged_tree_fwd(_tokens(Q, p.H, p.q_strides, p, "Q"), _pages(k_pages, p, "k_pages"), _pages(v_pages, p, "v_pages"),
                                       _tokens(O, p.H, p.o_strides, p, "O", torch.float32 if p.out_f32 else None), _f32(lse),
                                       ctypes.c_void_p(tree.data_ptr()), tree.shape[1], tree.stride(0) if p.rows > 1 else 0, _ptr(workspace), _bytes(workspace),
                                       ctypes.byref(p), _stream()), "burst_paged_tree_fwd")


def burst_cache_plan(added, lengths, table, free_pages, free_count, page, starts, totals, slots, positions, parents=None, tree=None, window=0):
    """int32 device tensors added, lengths, totals [sequences], table [sequences, width], free_pages [pages], free_count [1], starts [sequences + 1], parents
    [sequences, most] or None; int64 ones slots, positions [rows], tree [rows, words] or None (see burst.h)."""
    S, rows = added.shape[0], slots.shape[0]
    shapes = dict(added=(added, (S,)), lengths=(lengths, (S,)), totals=(totals, (S,)), starts=(starts, (S + 1,)), free_count=(free_count, (1,)),
                  free_pages=(free_pages, (free_pages.numel(),)), table=(table, (S, table.shape[-1])), slots=(slots, (rows,)), positions=(positions, (rows,)))
    if (parents is None) != (tree is None):
        raise ValueError("parents and tree: both or none expected")
    if parents is not None:
        shapes.update(parents=(parents, (S, parents.shape[-1])), tree=(tree, (rows, tree.shape[-1])))
    for name, (t, shape) in shapes.items():
        if t.dtype != (torch.int64 if name in ("slots", "positions", "tree") else torch.int32) or tuple(t.shape) != shape:
            raise ValueError(f"{name}: {'int64' if name in ('slots', 'positions', 'tree') else 'int32'} tensor {list(shape)} expected")
        if not (_rows_lie(t) if name in ("table", "parents") else t.is_contiguous()):
            raise ValueError(f"{name}: contiguous expected")
        _here(t, name)
    p = BurstPlan(sequences=S, rows=rows, pages=free_pages.shape[0], page=page, width=table.shape[1], added=added.data_ptr(), lengths=lengths.data_ptr(),
                  table=table.data_ptr(), table_stride=table.stride(0) if S > 1 else 0, free_pages=free_pages.data_ptr(), free_count=free_count.data_ptr(),
                  starts=starts.data_ptr(), totals=totals.data_ptr(), slots=slots.data_ptr(), positions=positions.data_ptr())
    if parents is not None:
        # (an empty tensor has no address, and a block without one says that there are no trees; this one is not read)
        p.words, p.most, p.tree, p.parents = tree.shape[1], parents.shape[1], tree.data_ptr(), parents.data_ptr() or starts.data_ptr()
        p.parents_stride, p.window = parents.stride(0) if S > 1 else 0, window
    _check(load().burst_cache_plan(ctypes.byref(p), _stream()), "burst_cache_plan")


def burst_cache_keep(pools, kept, counts, lengths_out, p):
    """pools: all layers' k_pages and v_pages, which lie as the parameter block says; kept [sequences, most], counts, lengths_out [sequences]: int32 device
    tensors."""
    for t, shape, what in ((kept, (p.sequences, kept.shape[-1]), "kept"), (counts, (p.sequences,), "counts"), (lengths_out, (p.sequences,), "lengths_out")):
        if t.dtype != torch.int32 or tuple(t.shape) != shape or (t.dim() == 1 and not t.is_contiguous()):
            raise ValueError(f"{what}: int32 tensor {list(shape)} expected")
        _here(t, what)
    if not _rows_lie(kept):
        raise ValueError("kept: contiguous rows expected")
    at = (ctypes.c_void_p * len(pools))(*[_pages(t, p, "pools").value for t in pools])
    _check(load().burst_cache_keep(at, len(pools), ctypes.c_void_p(kept.data_ptr()), kept.stride(0) if p.sequences > 1 else 0, kept.shape[1],
                                   ctypes.c_void_p(counts.data_ptr()), ctypes.c_void_p(lengths_out.data_ptr()), ctypes.byref(p), _stream()), "burst_cache_keep")


class Event:
    """HIP event recorded on the stream the kernels are launched on."""

    def __init__(self):
        self.h = load().burst_event_create()
        if not self.h:
            raise RuntimeError("burst_event_create failed")

    def record(self):
        _check(load().burst_event_record(self.h, _stream()), "burst_event_record")

    def elapsed_ms_until(self, stop):
        ms = ctypes.c_float(0.0)
        _check(load().burst_event_elapsed_ms(self.h, stop.h, ctypes.byref(ms)), "burst_event_elapsed_ms")
        return ms.value

    def __del__(self):
        try:
            if self.h:
                load().burst_event_destroy(self.h)
                self.h = None
        except Exception:
            pass
