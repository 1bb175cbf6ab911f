"""Thin ctypes binding of libpc (argument marshalling only; every step of the path runs in the library).

Function names mirror the C ABI declared in include/pc.h.  Device buffers are torch tensors (or raw
integer addresses); torch is used for device memory and streams only.  There is no CPU fallback: if
libpc.so is missing, importing a function from here raises.
"""
from __future__ import annotations

import ctypes as C
import os

import numpy as np

HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(HERE, "libpc.so")

PC_OK = 0
STATUS_NAMES = ["PC_OK", "PC_ERR_ARG", "PC_ERR_CYCLE", "PC_ERR_NOT_ALTERNATING", "PC_ERR_NOT_BLOCK_SPARSE",
                "PC_ERR_TIE", "PC_ERR_TOO_LARGE", "PC_ERR_WORKSPACE", "PC_ERR_STATE", "PC_ERR_HIP"]


class PcError(RuntimeError):
    def __init__(self, status: int, message: str):
        self.status = status
        self.status_name = STATUS_NAMES[status] if 0 <= status < len(STATUS_NAMES) else str(status)
        super().__init__(f"{self.status_name}: {message}")


class pc_dag(C.Structure):
    _fields_ = [("K", C.c_int32), ("n_blocks", C.c_int32), ("root_block", C.c_int32),
                ("type", C.POINTER(C.c_uint8)), ("n_real", C.POINTER(C.c_int32)),
                ("child_ptr", C.POINTER(C.c_int64)), ("child", C.POINTER(C.c_int32)),
                ("param_blk", C.POINTER(C.c_int32)), ("n_param_blocks", C.c_int32),
                ("in_var", C.POINTER(C.c_int32)), ("in_table", C.POINTER(C.c_int32)),
                ("n_vars", C.c_int32), ("n_cats", C.c_int32), ("n_tables", C.c_int32),
                ("max_groups", C.c_int32), ("tol_permille", C.c_int32), ("product_scratch", C.c_int32)]


class pc_sizes(C.Structure):
    _fields_ = [("K", C.c_int32), ("n_blocks", C.c_int32), ("n_layers", C.c_int32),
                ("n_rows", C.c_int64), ("theta_len", C.c_int64), ("tables_len", C.c_int64),
                ("n_vars", C.c_int32), ("n_cats", C.c_int32), ("n_tables", C.c_int32)]


class pc_layer_desc(C.Structure):
    _fields_ = [("kind", C.c_int32), ("depth", C.c_int32), ("n_fwd_groups", C.c_int32), ("n_bwd_groups", C.c_int32)]


class pc_group_desc(C.Structure):
    _fields_ = [("n_rows", C.c_int32), ("width", C.c_int32),
                ("ids", C.c_void_p), ("nbr", C.c_void_p), ("par", C.c_void_p)]


class pc_ws_layout(C.Structure):
    _fields_ = [("stride", C.c_int64), ("l_offset", C.c_size_t), ("f_offset", C.c_size_t),
                ("n_offset", C.c_size_t), ("r_offset", C.c_size_t), ("total_bytes", C.c_size_t), ("l_rows", C.c_int64)]


class pc_profile(C.Structure):
    _fields_ = [("n_classes", C.c_int32), ("launches", C.c_int64 * 16), ("ms", C.c_double * 16),
                ("bf16_launches", C.c_int64 * 16)]


class pc_mixture(C.Structure):
    _fields_ = [("K", C.c_int32), ("n_blocks", C.c_int32), ("n_cats", C.c_int32), ("n_tables", C.c_int32),
                ("n_rows", C.c_int64), ("stride", C.c_int64), ("weights", C.c_void_p), ("rows", C.c_void_p), ("table", C.c_void_p)]


class pc_distill(C.Structure):
    _fields_ = [("rows", C.c_int64), ("n_cats", C.c_int32), ("top", C.c_int32),
                ("student", C.c_void_p), ("student_type", C.c_int32), ("student_ld", C.c_int64),
                ("ids", C.c_void_p), ("ids_ld", C.c_int64),
                ("teacher", C.c_void_p), ("teacher_type", C.c_int32), ("teacher_ld", C.c_int64),
                ("teacher_lse", C.c_void_p), ("temperature", C.c_float), ("normalised", C.c_int32)]


class pc_beam(C.Structure):
    _fields_ = [("groups", C.c_int32), ("beams", C.c_int32), ("n_cats", C.c_int32), ("n_out", C.c_int32),
                ("scores", C.c_void_p), ("scores_type", C.c_int32), ("scores_ld", C.c_int64), ("normalise", C.c_int32),
                ("running", C.c_void_p), ("done", C.c_void_p), ("done_token", C.c_int32)]


class pc_state(C.Structure):
    _fields_ = [("src", C.c_void_p), ("dst", C.c_void_p), ("row_bytes", C.c_int64), ("src_stride", C.c_int64), ("dst_stride", C.c_int64)]


EXPORTS = ["pc_compile", "pc_compile_host", "pc_destroy", "pc_last_error", "pc_get_sizes", "pc_get_layer",
           "pc_get_group", "pc_copy_group", "pc_get_kernel", "pc_workspace_layout", "pc_workspace_bytes", "pc_forward",
           "pc_forward_static", "pc_backward", "pc_em_step", "pc_profile_enable", "pc_profile_read", "pc_kernel_class_name",
           "pc_measure_copy", "pc_measure_mfma_f32", "pc_collapse", "pc_collapsed_dag", "pc_collapsed_theta",
           "pc_collapsed_block_map", "pc_collapsed_destroy", "pc_order_for_scratch", "pc_set_wait_limit",
           "pc_get_mixture", "pc_predict_workspace_bytes", "pc_predict", "pc_predict_backward_workspace_bytes", "pc_predict_backward",
           "pc_distill_workspace_bytes", "pc_distill_forward", "pc_distill_backward", "pc_beam_workspace_bytes",
           "pc_beam_select", "pc_beam_reorder"]

_lib = None


def lib():
    """Load libpc.so (built by paper_2406_00766_amd/build.py).  Raises if it is missing."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(f"{LIB_PATH} not built: run `python -m paper_2406_00766_amd.build` "
                                    "(or __graft_entry__.build())")
        L = C.CDLL(LIB_PATH)
        L.pc_last_error.restype = C.c_char_p
        L.pc_destroy.restype = None
        L.pc_destroy.argtypes = [C.c_void_p]
        L.pc_compile.argtypes = [C.POINTER(pc_dag), C.c_void_p, C.POINTER(C.c_void_p)]
        L.pc_compile_host.argtypes = [C.POINTER(pc_dag), C.POINTER(C.c_void_p)]
        L.pc_get_sizes.argtypes = [C.c_void_p, C.POINTER(pc_sizes)]
        L.pc_get_layer.argtypes = [C.c_void_p, C.c_int32, C.POINTER(pc_layer_desc)]
        L.pc_get_group.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.POINTER(pc_group_desc)]
        L.pc_copy_group.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p]
        L.pc_get_kernel.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.POINTER(C.c_char_p)]
        L.pc_workspace_layout.argtypes = [C.c_void_p, C.c_int32, C.POINTER(pc_ws_layout)]
        L.pc_workspace_bytes.argtypes = [C.c_void_p, C.c_int32, C.POINTER(C.c_size_t)]
        L.pc_forward.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                 C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p]
        L.pc_forward_static.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                        C.c_void_p, C.c_void_p]
        L.pc_backward.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int32,
                                  C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p]
        L.pc_em_step.argtypes = [C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                 C.c_float, C.c_float, C.c_void_p]
        L.pc_profile_enable.argtypes = [C.c_void_p, C.c_int32]
        L.pc_profile_read.argtypes = [C.c_void_p, C.POINTER(pc_profile)]
        L.pc_set_wait_limit.argtypes = [C.c_void_p, C.c_int32]
        L.pc_kernel_class_name.argtypes = [C.c_int32]
        L.pc_kernel_class_name.restype = C.c_char_p
        L.pc_measure_copy.argtypes = [C.c_void_p, C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.pc_measure_mfma_f32.argtypes = [C.c_void_p, C.c_size_t, C.c_int32, C.c_void_p, C.POINTER(C.c_double)]
        L.pc_collapse.argtypes = [C.POINTER(pc_dag), C.c_void_p, C.POINTER(C.c_void_p)]
        L.pc_order_for_scratch.argtypes = [C.POINTER(pc_dag), C.POINTER(C.c_void_p)]
        L.pc_collapsed_dag.argtypes = [C.c_void_p]
        L.pc_collapsed_dag.restype = C.POINTER(pc_dag)
        L.pc_collapsed_theta.argtypes = [C.c_void_p, C.POINTER(C.c_int64)]
        L.pc_collapsed_theta.restype = C.POINTER(C.c_float)
        L.pc_collapsed_block_map.argtypes = [C.c_void_p]
        L.pc_collapsed_block_map.restype = C.POINTER(C.c_int32)
        L.pc_collapsed_destroy.argtypes = [C.c_void_p]
        L.pc_collapsed_destroy.restype = None
        L.pc_get_mixture.argtypes = [C.c_void_p, C.c_int32, C.c_int32, C.c_void_p, C.c_size_t, C.POINTER(pc_mixture)]
        L.pc_predict_workspace_bytes.argtypes = [C.POINTER(pc_mixture), C.c_int32, C.POINTER(C.c_size_t)]
        L.pc_predict.argtypes = [C.POINTER(pc_mixture), C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_size_t, C.c_void_p]
        L.pc_predict_backward.argtypes = [C.POINTER(pc_mixture), C.c_void_p, C.c_int32, C.c_void_p, C.c_int64, C.c_void_p, C.c_int64,
                                          C.c_float, C.c_int32, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]
        L.pc_predict_backward_workspace_bytes.argtypes = [C.POINTER(pc_mixture), C.c_int32, C.POINTER(C.c_size_t)]
        L.pc_distill_workspace_bytes.argtypes = [C.POINTER(pc_distill), C.POINTER(C.c_size_t)]
        L.pc_distill_forward.argtypes = [C.POINTER(pc_distill), C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p]
        L.pc_distill_backward.argtypes = [C.POINTER(pc_distill), C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_int64, C.c_void_p]
        L.pc_beam_workspace_bytes.argtypes = [C.POINTER(pc_beam), C.POINTER(C.c_size_t)]
        L.pc_beam_select.argtypes = [C.POINTER(pc_beam), C.c_void_p, C.c_size_t, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p]
        L.pc_beam_reorder.argtypes = [C.POINTER(pc_state), C.c_int32, C.c_void_p, C.c_int32, C.c_int32, C.c_int32, C.c_void_p]
        _lib = L
    return _lib


def _check(status: int):
    if status != PC_OK:
        raise PcError(status, (lib().pc_last_error() or b"").decode())


def _ptr(t):
    """Device address of a torch tensor / raw int / None."""
    if t is None:
        return None
    if isinstance(t, int):
        return t
    return t.data_ptr()


def _stream(stream):
    if stream is None:
        import torch
        return torch.cuda.current_stream().cuda_stream
    if isinstance(stream, int):
        return stream
    return stream.cuda_stream


def make_dag(w):
    """Marshal a workload-like object (see workloads.Workload) into a pc_dag; returns (dag, keepalive)."""
    arrs = dict(
        type=np.ascontiguousarray(w.type, dtype=np.uint8), n_real=np.ascontiguousarray(w.n_real, dtype=np.int32),
        child_ptr=np.ascontiguousarray(w.child_ptr, dtype=np.int64), child=np.ascontiguousarray(w.child, dtype=np.int32),
        param_blk=np.ascontiguousarray(w.param_blk, dtype=np.int32), in_var=np.ascontiguousarray(w.in_var, dtype=np.int32),
        in_table=np.ascontiguousarray(w.in_table, dtype=np.int32))
    d = pc_dag()
    d.K, d.n_blocks, d.root_block = int(w.K), int(w.n_blocks), int(w.root_block)
    d.type = arrs["type"].ctypes.data_as(C.POINTER(C.c_uint8))
    d.n_real = arrs["n_real"].ctypes.data_as(C.POINTER(C.c_int32))
    d.child_ptr = arrs["child_ptr"].ctypes.data_as(C.POINTER(C.c_int64))
    d.child = arrs["child"].ctypes.data_as(C.POINTER(C.c_int32))
    d.param_blk = arrs["param_blk"].ctypes.data_as(C.POINTER(C.c_int32))
    d.n_param_blocks = int(w.n_param_blocks)
    d.in_var = arrs["in_var"].ctypes.data_as(C.POINTER(C.c_int32))
    d.in_table = arrs["in_table"].ctypes.data_as(C.POINTER(C.c_int32))
    d.n_vars, d.n_cats, d.n_tables = int(w.n_vars), int(w.n_cats), int(w.n_tables)
    d.max_groups, d.tol_permille = int(w.max_groups), int(w.tol_permille)
    d.product_scratch = int(getattr(w, "product_scratch", 0))
    return d, arrs


def pc_compile(w, stream=None, host_only: bool = False) -> int:
    """Returns the opaque circuit handle (an integer address)."""
    d, keep = make_dag(w)
    out = C.c_void_p()
    if host_only:
        _check(lib().pc_compile_host(C.byref(d), C.byref(out)))
    else:
        _check(lib().pc_compile(C.byref(d), _stream(stream), C.byref(out)))
    del keep
    return out.value


def pc_collapse(w):
    """Footnote to Def. 2: the alternating form of a DAG with consecutive sum / sum or product / product blocks.
    Returns a copy of the workload-like object `w` with the rewritten DAG arrays, `theta` and `block_map`."""
    return _rewritten(w, collapse=True)


def pc_order_for_scratch(w):
    """Sec. 5, product-scratch mode: a copy of `w` with its blocks renumbered (input and sum blocks first, product
    blocks grouped by the sum layer that reads them, copied where sum layers of several depths read them),
    `product_scratch` set and `block_map` (old id -> new id)."""
    return _rewritten(w, collapse=False)


def _rewritten(w, collapse: bool):
    import copy
    d, keep = make_dag(w)
    theta = np.ascontiguousarray(w.theta, dtype=np.float32)
    out = C.c_void_p()
    if collapse:
        _check(lib().pc_collapse(C.byref(d), theta.ctypes.data, C.byref(out)))
    else:
        _check(lib().pc_order_for_scratch(C.byref(d), C.byref(out)))
    try:
        nd = lib().pc_collapsed_dag(out).contents
        n, ne = int(nd.n_blocks), int(nd.child_ptr[nd.n_blocks])
        r = copy.copy(w)
        r.n_blocks, r.root_block, r.n_param_blocks = n, int(nd.root_block), int(nd.n_param_blocks)
        r.type = np.ctypeslib.as_array(nd.type, (n,)).copy()
        r.n_real = np.ctypeslib.as_array(nd.n_real, (n,)).copy()
        r.child_ptr = np.ctypeslib.as_array(nd.child_ptr, (n + 1,)).copy()
        r.child = np.ctypeslib.as_array(nd.child, (max(ne, 1),))[:ne].copy()
        r.param_blk = np.ctypeslib.as_array(nd.param_blk, (max(ne, 1),))[:ne].copy()
        r.in_var = np.ctypeslib.as_array(nd.in_var, (n,)).copy()
        r.in_table = np.ctypeslib.as_array(nd.in_table, (n,)).copy()
        if collapse:
            ln = C.c_int64()
            tp = lib().pc_collapsed_theta(out, C.byref(ln))
            r.theta = np.ctypeslib.as_array(tp, (int(ln.value),)).copy().reshape(-1, w.K, w.K)
        else:
            r.product_scratch = 1
        r.block_map = np.ctypeslib.as_array(lib().pc_collapsed_block_map(out), (int(w.n_blocks),)).copy()
    finally:
        lib().pc_collapsed_destroy(out)
    del keep
    return r


def pc_destroy(handle: int):
    lib().pc_destroy(handle)


def pc_get_sizes(handle: int) -> pc_sizes:
    s = pc_sizes()
    _check(lib().pc_get_sizes(handle, C.byref(s)))
    return s


def pc_get_layer(handle: int, layer: int) -> pc_layer_desc:
    d = pc_layer_desc()
    _check(lib().pc_get_layer(handle, layer, C.byref(d)))
    return d


def pc_get_group(handle: int, layer: int, direction: int, group: int) -> pc_group_desc:
    g = pc_group_desc()
    _check(lib().pc_get_group(handle, layer, direction, group, C.byref(g)))
    return g


def pc_copy_group(handle: int, layer: int, direction: int, group: int):
    """(ids [R], nbr [R, W], par [R, W]) as int32 numpy arrays."""
    g = pc_get_group(handle, layer, direction, group)
    ids = np.empty(g.n_rows, dtype=np.int32)
    nbr = np.empty((g.n_rows, g.width), dtype=np.int32)
    par = np.empty((g.n_rows, g.width), dtype=np.int32)
    _check(lib().pc_copy_group(handle, layer, direction, group, ids.ctypes.data, nbr.ctypes.data, par.ctypes.data))
    return ids, nbr, par


def pc_get_kernel(handle: int, layer: int, direction: int, B: int) -> str:
    """The kernel that serves a layer at batch size B (direction 0 forward, 1 backward)."""
    name = C.c_char_p()
    _check(lib().pc_get_kernel(handle, layer, direction, int(B), C.byref(name)))
    return name.value.decode()


def pc_workspace_layout(handle: int, B: int) -> pc_ws_layout:
    lay = pc_ws_layout()
    _check(lib().pc_workspace_layout(handle, B, C.byref(lay)))
    return lay


def pc_workspace_bytes(handle: int, B: int) -> int:
    n = C.c_size_t()
    _check(lib().pc_workspace_bytes(handle, B, C.byref(n)))
    return int(n.value)


def pc_forward(handle, theta, tables, x, mask, B, workspace, workspace_bytes, ll, stream=None):
    _check(lib().pc_forward(handle, _ptr(theta), _ptr(tables), _ptr(x), _ptr(mask), int(B), _ptr(workspace),
                            int(workspace_bytes), _ptr(ll), _stream(stream)))


PC_STATIC_SCRATCH_BYTES = 64 << 20


def pc_forward_static(handle, theta, tables, x, mask, B, ll, stream=None):
    _check(lib().pc_forward_static(handle, _ptr(theta), _ptr(tables), _ptr(x), _ptr(mask), int(B), _ptr(ll),
                                   _stream(stream)))


def pc_backward(handle, theta, tables, x, mask, B, workspace, workspace_bytes, theta_flow, table_flow, stream=None):
    _check(lib().pc_backward(handle, _ptr(theta), _ptr(tables), _ptr(x), _ptr(mask), int(B), _ptr(workspace),
                             int(workspace_bytes), _ptr(theta_flow), _ptr(table_flow), _stream(stream)))


def pc_em_step(handle, theta, tables, theta_flow, table_flow, step, pseudocount, stream=None):
    _check(lib().pc_em_step(handle, _ptr(theta), _ptr(tables), _ptr(theta_flow), _ptr(table_flow),
                            float(step), float(pseudocount), _stream(stream)))


def pc_profile_enable(handle: int, on: bool):
    _check(lib().pc_profile_enable(handle, 1 if on else 0))


def pc_profile_read(handle: int, with_bf16: bool = False) -> dict:
    """{class name: (launches, total ms)} since pc_profile_enable; with_bf16 adds the launches that ran as bf16-split
    products as a third element."""
    p = pc_profile()
    _check(lib().pc_profile_read(handle, C.byref(p)))
    if with_bf16:
        return {lib().pc_kernel_class_name(i).decode(): (int(p.launches[i]), float(p.ms[i]), int(p.bf16_launches[i]))
                for i in range(p.n_classes)}
    return {lib().pc_kernel_class_name(i).decode(): (int(p.launches[i]), float(p.ms[i])) for i in range(p.n_classes)}


def pc_set_wait_limit(handle: int, polls: int):
    _check(lib().pc_set_wait_limit(handle, int(polls)))


def pc_measure_copy(src, dst, nbytes: int, reps: int = 5, stream=None) -> float:
    """GB/s (read + written) of a plain streaming copy between two device buffers."""
    out = C.c_double()
    _check(lib().pc_measure_copy(_ptr(src), _ptr(dst), int(nbytes), int(reps), _stream(stream), C.byref(out)))
    return float(out.value)


def pc_measure_mfma_f32(out_buf, out_bytes: int, reps: int = 5, stream=None) -> float:
    """TFLOP/s of a register-only fp32 MFMA loop; out_buf: device buffer of at least 2 MiB."""
    out = C.c_double()
    _check(lib().pc_measure_mfma_f32(_ptr(out_buf), int(out_bytes), int(reps), _stream(stream), C.byref(out)))
    return float(out.value)


# ---- token models over circuits: these take torch tensors, whose shapes, types and strides become the descriptors ----
# The kernels trust what is passed on from here, so everything is checked; a tensor that is plainly right passes _fits (calls of a few
# microseconds are common in decoding), any other goes through _tensor, which accepts strided rows and says what is wrong.
def _refuse(message: str):
    raise PcError(1, message)


def _fits(t, dtype, shape, index) -> bool:
    """A contiguous tensor on GPU `index` of this type and shape."""
    try:
        return t.dtype is dtype and t.shape == shape and t.get_device() == index and t.is_contiguous()
    except AttributeError:
        return False


def _tensor(name, t, dtype=None, shape=None, index=None, last=1):
    """Check one argument: a tensor on the GPU (on GPU `index`), of this type and shape (None: any length), its last `last` axes contiguous."""
    import torch
    if not isinstance(t, torch.Tensor):
        _refuse(f"{name} must be a tensor")
    if t.device.type != "cuda" or (index is not None and t.get_device() != index):
        _refuse(f"{name} must lie on {'a GPU' if index is None else f'GPU {index}'}, not on {t.device}")
    if dtype is not None and t.dtype != dtype:
        _refuse(f"{name} must be {dtype}, not {t.dtype}")
    if shape is not None and (t.dim() != len(shape) or any(n is not None and n != m for n, m in zip(shape, t.shape))):
        _refuse(f"{name} must have shape {shape}, not {tuple(t.shape)}")
    step = 1
    for n, st in list(zip(t.shape, t.stride()))[::-1][:last]:
        if n > 1 and st != step:
            _refuse(f"the last {last} axes of {name} must be contiguous")
        step *= n
    return t


def _matrix(t, dtype) -> bool:
    """A contiguous matrix of this type on a GPU."""
    import torch
    return isinstance(t, torch.Tensor) and t.is_cuda and t.dim() == 2 and t.dtype is dtype and t.is_contiguous()


def _ld(t):
    """Elements between the rows of a matrix (its length where there is but one row, whose stride means nothing)."""
    rows, n = t.shape
    if rows <= 1:
        return n
    ld = t.stride(0)
    if ld < n:
        _refuse("the rows of a matrix must not overlap")
    return ld


_types = {}


def _type(name, t):
    if not _types:
        import torch
        _types.update({torch.float32: 0, torch.bfloat16: 1, torch.float16: 2})     # PC_F32, PC_BF16, PC_F16
    code = _types.get(t.dtype)
    if code is None:
        _refuse(f"{name} must be float32, bfloat16 or float16, not {t.dtype}")
    return code


def _call(index, stream, function, *args):
    """function(*args, stream) with GPU `index` current; stream None: that GPU's current stream."""
    import torch
    if stream is None:
        stream = torch._C._cuda_getCurrentRawStream(index)
    elif not isinstance(stream, int):
        stream = stream.cuda_stream
    if torch.cuda.current_device() == index:
        _check(function(*args, stream))
    else:
        with torch.cuda.device(index):
            _check(function(*args, stream))


class mixture:
    """pc_mixture over tensors: weights float32 [n_rows, >= B], samples contiguous; block j is rows rows[j] .. + K and table
    table[j] (int32 tensors), or rows j * K .. and table j.  `n_tables` defaults to n_blocks."""

    def __init__(self, weights, K, n_cats, n_blocks, rows=None, table=None, n_tables=None):
        import torch
        if not _matrix(weights, torch.float32):
            _tensor("weights", weights, torch.float32, (None, None))
        self.index, self.columns = weights.get_device(), int(weights.shape[1])
        for name, t in (("rows", rows), ("table", table)):
            if t is not None:
                _tensor(name, t, torch.int32, (n_blocks,), self.index)
        self.keep = (weights, rows, table)
        self.struct = pc_mixture(int(K), int(n_blocks), int(n_cats), int(n_blocks if n_tables is None else n_tables), int(weights.shape[0]),
                                 _ld(weights), weights.data_ptr(), _ptr(rows), _ptr(table))


def pc_get_mixture(handle, var, B, workspace, workspace_bytes) -> mixture:
    """The input blocks of variable `var` with the node flows that pc_backward has left in the workspace (a tensor)."""
    m = mixture.__new__(mixture)
    m.struct = pc_mixture()
    _check(lib().pc_get_mixture(handle, int(var), int(B), _ptr(workspace), int(workspace_bytes), C.byref(m.struct)))
    m.index, m.columns, m.keep = workspace.get_device(), int(m.struct.stride), (workspace,)
    return m


def _floats(name, t, n, index):
    """A contiguous float32 tensor of n elements, of any shape."""
    import torch
    if not (isinstance(t, torch.Tensor) and _fits(t, torch.float32, t.shape, index)):
        _tensor(name, t, torch.float32, None, index, t.dim() if isinstance(t, torch.Tensor) else 1)
    if t.numel() != n:
        _refuse(f"{name} must hold {n} floats, not {t.numel()}")


def _rows(name, t, dtype, shape, index):
    if not _fits(t, dtype, shape, index):
        _tensor(name, t, dtype, shape, index)
    return t.data_ptr(), _ld(t)


def _bytes_of(function, struct, *args):
    n = C.c_size_t()
    _check(function(C.byref(struct), *args, C.byref(n)))
    return n.value


def _scratch(workspace, size, index, stream):
    """(address, bytes) of the caller's workspace, and what keeps it; None: `size` bytes are allocated on the call's stream, so that,
    freed, they serve that stream's later work only."""
    if workspace is not None or not size:
        return _workspace(workspace, index), workspace
    import torch
    if stream is None:
        t = torch.empty(size, dtype=torch.uint8, device=index)
    else:
        with torch.cuda.stream(torch.cuda.ExternalStream(stream, device=index) if isinstance(stream, int) else stream):
            t = torch.empty(size, dtype=torch.uint8, device=index)
    return (t.data_ptr(), size), t


def pc_predict_workspace_bytes(m: mixture, B) -> int:
    return int(_bytes_of(lib().pc_predict_workspace_bytes, m.struct, int(B)))


def pc_predict(m: mixture, tables, B, logp, stream=None, workspace=None):
    """logp float32 [B, n_cats] (rows may be strided) = log sum of weights * tables.  workspace: a uint8 tensor of
    pc_predict_workspace_bytes; None: one is allocated where the call needs it."""
    import torch
    s, B = m.struct, int(B)
    _floats("tables", tables, s.n_tables * s.n_cats * s.K, m.index)
    if B > m.columns:
        _refuse("weights have fewer than B columns")
    out = _rows("logp", logp, torch.float32, (B, s.n_cats), m.index)
    (ws, size), keep = _scratch(workspace, workspace is None and _bytes_of(lib().pc_predict_workspace_bytes, s, B), m.index, stream)
    _call(m.index, stream, lib().pc_predict, C.byref(s), tables.data_ptr(), B, *out, ws, size)


def pc_predict_backward_workspace_bytes(m: mixture, B) -> int:
    return int(_bytes_of(lib().pc_predict_backward_workspace_bytes, m.struct, int(B)))


def pc_predict_backward(m: mixture, tables, B, logp, dlogp, scale, table_flow, accumulate=True, stream=None, workspace=None):
    """Table flows for a gradient dlogp [B, n_cats] of an objective; added to table_flow, or stored.  workspace: a uint8 tensor of
    pc_predict_backward_workspace_bytes; None: one is allocated where the call needs it."""
    import torch
    s, B = m.struct, int(B)
    n = s.n_tables * s.n_cats * s.K
    _floats("tables", tables, n, m.index)
    _floats("table_flow", table_flow, n, m.index)
    if B > m.columns:
        _refuse("weights have fewer than B columns")
    shape = (B, s.n_cats)
    args = (*_rows("logp", logp, torch.float32, shape, m.index), *_rows("dlogp", dlogp, torch.float32, shape, m.index))
    (ws, size), keep = _scratch(workspace, workspace is None and _bytes_of(lib().pc_predict_backward_workspace_bytes, s, B), m.index, stream)
    _call(m.index, stream, lib().pc_predict_backward, C.byref(s), tables.data_ptr(), B, *args, float(scale), 1 if accumulate else 0,
          table_flow.data_ptr(), ws, size)


class distill:
    """pc_distill over tensors: student [rows, n_cats], ids int32 [rows, top], teacher [rows, top], teacher_lse float32 [rows]."""

    def __init__(self, student, ids, teacher, temperature=1.0, teacher_lse=None, normalised=False):
        import torch
        if not (isinstance(student, torch.Tensor) and _matrix(student, student.dtype)):
            _tensor("student", student, None, (None, None))
        self.index = index = student.get_device()
        self.student, self.keep = student, (ids, teacher, teacher_lse)
        self.rows, n_cats = student.shape
        if not (isinstance(ids, torch.Tensor) and ids.dim() == 2 and _fits(ids, torch.int32, (self.rows, ids.shape[1]), index)):
            _tensor("ids", ids, torch.int32, (self.rows, None), index)
        if not (isinstance(teacher, torch.Tensor) and _fits(teacher, teacher.dtype, ids.shape, index)):
            _tensor("teacher", teacher, None, tuple(ids.shape), index)
        if teacher_lse is not None:
            _tensor("teacher_lse", teacher_lse, torch.float32, (self.rows,), index)
        self.struct = pc_distill(self.rows, n_cats, ids.shape[1], student.data_ptr(), _type("student", student), _ld(student), ids.data_ptr(),
                                 _ld(ids), teacher.data_ptr(), _type("teacher", teacher), _ld(teacher), _ptr(teacher_lse),
                                 temperature, 1 if normalised else 0)


def pc_distill_workspace_bytes(d: distill) -> int:
    n = C.c_size_t()
    _check(lib().pc_distill_workspace_bytes(C.byref(d.struct), C.byref(n)))
    return int(n.value)


def _workspace(t, index):
    import torch
    if t is None:
        return None, 0
    if not (isinstance(t, torch.Tensor) and _fits(t, torch.uint8, (t.numel(),), index)):
        _tensor("workspace", t, torch.uint8, (None,), index)
    return t.data_ptr(), t.numel()


def _array(name, t, dtype, shape, index):
    if not _fits(t, dtype, shape, index):
        _tensor(name, t, dtype, shape, index, len(shape))
    return t.data_ptr()


def pc_distill_forward(d: distill, workspace, loss, stats, stream=None):
    """loss float32 [rows], stats float32 [rows, 2].  workspace: None (none is needed)."""
    import torch
    _call(d.index, stream, lib().pc_distill_forward, C.byref(d.struct), *_workspace(workspace, d.index),
          _array("loss", loss, torch.float32, (d.rows,), d.index), _array("stats", stats, torch.float32, (d.rows, 2), d.index))


def pc_distill_backward(d: distill, stats, dloss, scale, dstudent, stream=None):
    """dstudent [rows, n_cats] of the student's type = scale * dloss (float32 [rows] or None) * gradient; it may be the student itself."""
    import torch
    _call(d.index, stream, lib().pc_distill_backward, C.byref(d.struct), _array("stats", stats, torch.float32, (d.rows, 2), d.index),
          None if dloss is None else _array("dloss", dloss, torch.float32, (d.rows,), d.index), float(scale),
          *_rows("dstudent", dstudent, d.student.dtype, d.student.shape, d.index))


class beam:
    """pc_beam over tensors: scores [groups * beams, n_cats], running float32 [groups, beams], done uint8 [groups, beams]."""

    def __init__(self, scores, running, n_out, done=None, done_token=0, normalise=False):
        import torch
        if not (isinstance(scores, torch.Tensor) and _matrix(scores, scores.dtype)):
            _tensor("scores", scores, None, (None, None))
        self.index = index = scores.get_device()
        if not (isinstance(running, torch.Tensor) and running.dim() == 2 and _fits(running, torch.float32, running.shape, index)):
            _tensor("running", running, torch.float32, (None, None), index, 2)
        groups, beams = running.shape
        rows, n_cats = scores.shape
        if rows != groups * beams:
            _refuse("scores must have a row for each running score")
        if done is not None:
            _array("done", done, torch.uint8, (groups, beams), index)
        self.keep = (scores, running, done)
        self.shape = (groups, int(n_out))
        self.struct = pc_beam(groups, beams, n_cats, self.shape[1], scores.data_ptr(), _type("scores", scores), _ld(scores),
                              1 if normalise else 0, running.data_ptr(), _ptr(done), int(done_token))


def pc_beam_workspace_bytes(a: beam) -> int:
    n = C.c_size_t()
    _check(lib().pc_beam_workspace_bytes(C.byref(a.struct), C.byref(n)))
    return int(n.value)


def pc_beam_select(a: beam, workspace, out_scores, parents, tokens, stream=None):
    """The n_out best of each group: out_scores float32, parents int32 and tokens int32, all [groups, n_out]."""
    import torch
    shape, index = a.shape, a.index
    _call(index, stream, lib().pc_beam_select, C.byref(a.struct), *_workspace(workspace, index), _array("out_scores", out_scores, torch.float32, shape, index),
          _array("parents", parents, torch.int32, shape, index), _array("tokens", tokens, torch.int32, shape, index))


def pc_beam_reorder(states, parents, beams, stream=None):
    """For each (src, dst) of `states`: row g * n_out + i of dst = row g * beams + parents[g, i] of src.  Rows are the leading axis;
    a row's elements are contiguous, rows may be strided."""
    import torch
    if not _matrix(parents, torch.int32):
        _tensor("parents", parents, torch.int32, (None, None), None, 2)
    groups, n_out = parents.shape
    beams, index = int(beams), parents.get_device()
    if not 1 <= len(states) <= 16:
        _refuse("1 .. 16 states")
    array = (pc_state * len(states))()
    for s, (src, dst) in zip(array, states):
        for name, t, rows in (("src", src, groups * beams), ("dst", dst, groups * n_out)):
            if not (isinstance(t, torch.Tensor) and t.get_device() == index and t.is_contiguous()):
                _tensor(name, t, None, None, index, max(1, t.dim() - 1) if isinstance(t, torch.Tensor) else 1)
            if t.dim() < 1 or t.shape[0] != rows:
                _refuse(f"{name} must have {rows} rows")
        shape = src.shape[1:]
        if src.dtype != dst.dtype or shape != dst.shape[1:]:
            _refuse("src and dst must have rows of one shape and type")
        e = src.element_size()
        n = shape.numel() * e
        s.src, s.dst, s.row_bytes = src.data_ptr(), dst.data_ptr(), n
        s.src_stride = src.stride(0) * e if src.shape[0] > 1 else n
        s.dst_stride = dst.stride(0) * e if dst.shape[0] > 1 else n
    _call(index, stream, lib().pc_beam_reorder, array, len(states), parents.data_ptr(), groups, beams, n_out)


def compiled_tables(handle: int) -> list[dict]:
    """All layers with their groups copied to host: [{kind, depth, fwd: [(ids, nbr, par)], bwd: [...]}]."""
    out = []
    for li in range(pc_get_sizes(handle).n_layers):
        d = pc_get_layer(handle, li)
        out.append({"kind": d.kind, "depth": d.depth,
                    "fwd": [pc_copy_group(handle, li, 0, g) for g in range(d.n_fwd_groups)],
                    "bwd": [pc_copy_group(handle, li, 1, g) for g in range(d.n_bwd_groups)]})
    return out


class Circuit:
    """Convenience owner of a handle plus device copies of one workload's arrays (tests / benchmark)."""

    def __init__(self, w, device="cuda:0"):
        import torch
        self.torch = torch
        self.device = torch.device(device)
        torch.cuda.set_device(self.device)
        self.handle = pc_compile(w)
        self.sizes = pc_get_sizes(self.handle)
        self.K = w.K
        self.theta = torch.from_numpy(np.ascontiguousarray(w.theta, dtype=np.float32).reshape(-1)).to(self.device)
        self.tables = torch.from_numpy(np.ascontiguousarray(w.tables, dtype=np.float32).reshape(-1)).to(self.device)
        assert self.theta.numel() == self.sizes.theta_len and self.tables.numel() == self.sizes.tables_len
        self.theta_flow = torch.zeros_like(self.theta)
        self.table_flow = torch.zeros_like(self.tables)
        self._ws = None
        self._ws_B = 0
        self.x = self.mask = self.ll = None
        self.B = 0

    def close(self):
        if self.handle:
            pc_destroy(self.handle)
            self.handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def set_batch(self, x, mask=None):
        torch = self.torch
        self.x = torch.from_numpy(np.ascontiguousarray(x, dtype=np.int32)).to(self.device)
        self.mask = None if mask is None else torch.from_numpy(np.ascontiguousarray(mask, dtype=np.uint8)).to(self.device)
        self.B = int(x.shape[0])
        need = pc_workspace_bytes(self.handle, self.B)
        if self._ws is None or self._ws.numel() < need:
            self._ws = torch.empty(need, dtype=torch.uint8, device=self.device)
        self.ll = torch.empty(self.B, dtype=torch.float32, device=self.device)

    def forward(self):
        pc_forward(self.handle, self.theta, self.tables, self.x, self.mask, self.B, self._ws, self._ws.numel(), self.ll)
        return self.ll

    def backward(self, theta_flow=True, table_flow=True):
        pc_backward(self.handle, self.theta, self.tables, self.x, self.mask, self.B, self._ws, self._ws.numel(),
                    self.theta_flow if theta_flow else None, self.table_flow if table_flow else None)

    def em_step(self, step=1.0, pseudocount=0.0):
        pc_em_step(self.handle, self.theta, self.tables, self.theta_flow, self.table_flow, step, pseudocount)

    def predict(self, var, logp=None):
        """log p(x_var = c | the batch's evidence) [B, n_cats], after backward() on a batch in which `var` is marginalised."""
        m = pc_get_mixture(self.handle, var, self.B, self._ws, self._ws.numel())
        if logp is None:
            logp = self.torch.empty((self.B, self.sizes.n_cats), dtype=self.torch.float32, device=self.device)
        pc_predict(m, self.tables, self.B, logp)
        return logp

    def predict_backward(self, var, logp, dlogp, scale=1.0):
        """Adds the table flows of a gradient with respect to predict(var) to table_flow."""
        m = pc_get_mixture(self.handle, var, self.B, self._ws, self._ws.numel())
        pc_predict_backward(m, self.tables, self.B, logp, dlogp, scale, self.table_flow)

    def node_buffers(self):
        """(l, F, R) float32 views of the workspace: l, F are [n_rows, stride] (row = compiled node offset),
        R is [n_blocks + 1, stride]; the log-probability of row n is R[n // K] + l[n]."""
        lay = pc_workspace_layout(self.handle, self.B)
        n = self.sizes.n_rows * lay.stride
        nb = (self.sizes.n_blocks + 1) * lay.stride
        f32 = self.torch.float32
        l = self._ws[lay.l_offset:lay.l_offset + 4 * lay.l_rows * lay.stride].view(f32).view(lay.l_rows, lay.stride)
        F = self._ws[lay.f_offset:lay.f_offset + 4 * lay.l_rows * lay.stride].view(f32).view(lay.l_rows, lay.stride)
        R = self._ws[lay.r_offset:lay.r_offset + 4 * nb].view(f32).view(self.sizes.n_blocks + 1, lay.stride)
        return l, F, R
