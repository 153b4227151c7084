"""Thin binding over the CUDA C-ABI library (``include/randes.h``).

Argument marshalling only: every step of the path runs in the library's
kernels.  PyTorch supplies device memory and the stream.  There is no CPU
fallback: if the compiled library is missing, loading raises.

Two levels:

* module functions ``randes_plan``, ``randes_compress``, ``randes_add_model``,
  ``randes_remove_model``, ``randes_retrieve`` ... with the C names, taking
  ctypes pointer arrays / raw addresses;
* ``Plan``: the same calls on lists of torch CUDA tensors.
"""
from __future__ import annotations

import ctypes
import functools
import math
import os
from typing import Any, List, NamedTuple, Optional, Sequence

F32 = 0
BF16 = 1
SHUFFLE = 1
FLIP = 2
SHIFT = 4
GAUSS = 1 << 16   # RANDES_GAUSS: Gaussian-like diagonal context (the paper's "RD" ablation) instead of the +-1 one


def SKIP(k: int) -> int:
    """Group flag bits of RANDES_SKIP(k): only every k-th member of the group takes part."""
    return (int(k) & 0xFF) << 8

OK = 0
INVALID_ARGUMENT = -1
SHAPE_MISMATCH = -2
UNKNOWN_TASK = -3
DUPLICATE_TASK = -4
WORKSPACE_TOO_SMALL = -5
UNSUPPORTED_DTYPE = -6
MISALIGNED = -7
CAPACITY = -8
CUDA_ERROR = -9
OUT_OF_MEMORY = -10

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "librandes.so")
_lib = None


class RandesError(RuntimeError):
    def __init__(self, code: int, message: str):
        super().__init__("randes error %d: %s" % (code, message))
        self.code = code


class Layer(ctypes.Structure):
    _fields_ = [("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32), ("group", ctypes.c_uint32)]


class Group(ctypes.Structure):
    _fields_ = [("flags", ctypes.c_uint32)]


class Matrix(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("rows", ctypes.c_uint32), ("cols", ctypes.c_uint32), ("stride", ctypes.c_uint64)]


def lib():
    """The loaded shared library; raises if it has not been built."""
    global _lib
    if _lib is None:
        if not os.path.exists(LIB_PATH):
            raise RuntimeError(
                "%s is missing: build it with `python -m paper_2505_11204_b200.build` "
                "(there is no CPU fallback)" % LIB_PATH)
        L = ctypes.CDLL(LIB_PATH)
        vp, u32, u64, sz = ctypes.c_void_p, ctypes.c_uint32, ctypes.c_uint64, ctypes.c_size_t
        L.randes_plan_workspace_bytes.argtypes = [vp, u32, u32]
        L.randes_plan_workspace_bytes.restype = sz
        L.randes_plan_workspace_bytes_groups.argtypes = [vp, u32, vp, u32, u32]
        L.randes_plan_workspace_bytes_groups.restype = sz
        L.randes_plan.argtypes = [vp, u32, vp, u32, ctypes.c_int, ctypes.c_int, vp, vp, u32, u32, vp, sz, vp,
                                  ctypes.POINTER(vp)]
        L.randes_plan.restype = ctypes.c_int
        L.randes_plan_destroy.argtypes = [vp]
        L.randes_plan_destroy.restype = None
        L.randes_plan_validate.argtypes = [vp]
        L.randes_plan_validate.restype = ctypes.c_int
        L.randes_debug_violation.argtypes = [ctypes.POINTER(ctypes.c_uint64), ctypes.POINTER(ctypes.c_int)]
        L.randes_debug_violation.restype = ctypes.c_int
        L.randes_superposition_bytes.argtypes = [vp]
        L.randes_superposition_bytes.restype = sz
        L.randes_layer_offset.argtypes = [vp, u32]
        L.randes_layer_offset.restype = sz
        L.randes_num_layers.argtypes = [vp]
        L.randes_num_layers.restype = u32
        L.randes_num_tasks.argtypes = [vp]
        L.randes_num_tasks.restype = u32
        L.randes_task_list.argtypes = [vp, vp, vp]
        L.randes_task_list.restype = ctypes.c_int
        L.randes_task_tables.argtypes = [vp, u32, vp, vp]
        L.randes_task_tables.restype = ctypes.c_int
        L.randes_compress.argtypes = [vp, vp, vp, vp, vp]
        L.randes_compress.restype = ctypes.c_int
        L.randes_add_model.argtypes = [vp, u32, u64, vp, vp, vp, vp]
        L.randes_add_model.restype = ctypes.c_int
        L.randes_add_models.argtypes = [vp, vp, vp, u32, vp, vp, vp, vp]
        L.randes_add_models.restype = ctypes.c_int
        L.randes_remove_model.argtypes = [vp, u32, vp, vp, vp, vp]
        L.randes_remove_model.restype = ctypes.c_int
        L.randes_retrieve.argtypes = [vp, u32, ctypes.c_float, ctypes.c_int, vp, vp, vp, vp]
        L.randes_retrieve.restype = ctypes.c_int
        L.randes_plan_serialize.argtypes = [vp, vp, sz]
        L.randes_plan_serialize.restype = sz
        L.randes_plan_deserialize.argtypes = [vp, sz, u32, vp, sz, vp, ctypes.POINTER(vp)]
        L.randes_plan_deserialize.restype = ctypes.c_int
        L.randes_plan_workspace_needed.argtypes = [vp]
        L.randes_plan_workspace_needed.restype = sz
        L.randes_delta_gram_scratch_bytes.argtypes = [vp]
        L.randes_delta_gram_scratch_bytes.restype = sz
        L.randes_delta_gram.argtypes = [vp, vp, vp, vp, vp, sz, vp]
        L.randes_delta_gram.restype = ctypes.c_int
        L.randes_interference_norm.argtypes = [vp, u32, u32, ctypes.c_double, ctypes.POINTER(ctypes.c_double)]
        L.randes_interference_norm.restype = ctypes.c_int
        L.randes_pairwise_cosines.argtypes = [vp, u32, ctypes.c_int32, vp, ctypes.POINTER(ctypes.c_double)]
        L.randes_pairwise_cosines.restype = ctypes.c_int
        L.randes_retrieve_batch.argtypes = [vp, vp, u32, ctypes.c_float, ctypes.c_int, vp, vp, vp, vp]
        L.randes_retrieve_batch.restype = ctypes.c_int
        L.randes_retrieve_static.argtypes = [vp, u32, ctypes.c_float, ctypes.c_int, vp, vp, vp, vp]
        L.randes_retrieve_static.restype = ctypes.c_int
        L.randes_linear.argtypes = [vp, u32, ctypes.c_float, u32, vp, u32, vp, vp, vp, ctypes.c_int, vp]
        L.randes_linear.restype = ctypes.c_int
        L.randes_linear_gated.argtypes = [vp, u32, ctypes.c_float, u32, vp, u32, vp, vp, vp, ctypes.c_int, vp, u64, vp]
        L.randes_linear_gated.restype = ctypes.c_int
        L.randes_linear_giveups.argtypes = [ctypes.POINTER(ctypes.c_uint)]
        L.randes_linear_giveups.restype = ctypes.c_int
        f32, dt = ctypes.c_float, ctypes.c_int
        L.randes_packed_bytes.argtypes = [u32, u32, u32]
        L.randes_packed_bytes.restype = sz
        L.randes_pack.argtypes = [vp, u32, dt, u32, vp, vp]
        L.randes_pack.restype = ctypes.c_int
        L.randes_unpack.argtypes = [vp, u32, u32, vp, dt, vp]
        L.randes_unpack.restype = ctypes.c_int
        L.randes_retrieve_packed.argtypes = [vp, u32, f32, vp, u32, vp, vp, u32, vp, vp]
        L.randes_retrieve_packed.restype = ctypes.c_int
        L.randes_packed_linear_workspace.argtypes = [u32, u32, dt, u32, ctypes.c_int]
        L.randes_packed_linear_workspace.restype = sz
        L.randes_packed_linear.argtypes = [vp, u32, u32, u32, vp, dt, u64, u32, vp, dt, u64, vp, sz, vp]
        L.randes_packed_linear.restype = ctypes.c_int
        L.randes_packed_linear_tasks.argtypes = [vp, f32, u32, u32, vp, u32, vp, dt, u64, vp, vp, vp, dt, u64, vp, sz, vp]
        L.randes_packed_linear_tasks.restype = ctypes.c_int
        L.randes_token_scores.argtypes = [vp, dt, u32, u32, u64, vp, f32, u32, vp, vp, vp, vp, vp, vp]
        L.randes_token_scores.restype = ctypes.c_int
        L.randes_token_scores_backward.argtypes = [vp, dt, u32, u32, u64, vp, f32, vp, vp, vp, vp, vp, u64, vp]
        L.randes_token_scores_backward.restype = ctypes.c_int
        L.randes_launch_count.argtypes = []
        L.randes_launch_count.restype = u64
        L.randes_last_error.argtypes = []
        L.randes_last_error.restype = ctypes.c_char_p
        _lib = L
    return _lib


EXPORTS = [
    "randes_plan_workspace_bytes", "randes_plan_workspace_bytes_groups", "randes_plan", "randes_plan_destroy", "randes_plan_validate", "randes_debug_violation", "randes_superposition_bytes",
    "randes_layer_offset", "randes_num_layers", "randes_num_tasks", "randes_task_list",
    "randes_task_tables", "randes_plan_serialize", "randes_plan_workspace_needed", "randes_plan_deserialize", "randes_compress", "randes_add_model", "randes_add_models", "randes_remove_model",
    "randes_retrieve", "randes_delta_gram_scratch_bytes", "randes_delta_gram", "randes_interference_norm", "randes_pairwise_cosines", "randes_retrieve_batch", "randes_retrieve_static", "randes_linear", "randes_linear_gated", "randes_linear_giveups", "randes_launch_count", "randes_last_error",
    "randes_packed_bytes", "randes_pack", "randes_unpack", "randes_retrieve_packed", "randes_packed_linear_workspace", "randes_packed_linear", "randes_packed_linear_tasks",
    "randes_token_scores", "randes_token_scores_backward",
]


def randes_last_error() -> str:
    return lib().randes_last_error().decode()


def _check(rc: int) -> None:
    if rc != OK:
        raise RandesError(rc, randes_last_error())


def _addr(x) -> Optional[int]:
    if x is None:
        return None
    if isinstance(x, int):
        return x
    if isinstance(x, ctypes.Array):
        return ctypes.addressof(x)
    return int(x.data_ptr())  # torch tensor


# ---- C-named entry points (raw addresses / ctypes arrays) ----------------------------------
def randes_plan_workspace_bytes(layers, n_layers: int, max_tasks: int) -> int:
    return int(lib().randes_plan_workspace_bytes(_addr(layers), n_layers, max_tasks))


def randes_plan_workspace_bytes_groups(layers, n_layers: int, groups, n_groups: int, max_tasks: int) -> int:
    """Workspace bytes of a plan with these groups (larger than the plain figure only with a RANDES_GAUSS group)."""
    return int(lib().randes_plan_workspace_bytes_groups(_addr(layers), n_layers, _addr(groups), n_groups, max_tasks))


def randes_plan(layers, n_layers, groups, n_groups, storage_dtype, m_dtype, task_ids, seeds, n_tasks, max_tasks,
                dev_workspace, dev_workspace_bytes, stream) -> int:
    """Returns the plan handle (an address); raises RandesError on failure."""
    out = ctypes.c_void_p()
    _check(lib().randes_plan(_addr(layers), n_layers, _addr(groups), n_groups, storage_dtype, m_dtype,
                             _addr(task_ids), _addr(seeds), n_tasks, max_tasks, _addr(dev_workspace),
                             dev_workspace_bytes, stream, ctypes.byref(out)))
    return out.value


def randes_plan_serialize(plan) -> bytes:
    """The plan's shapes, flags, element types and (id, seed) pairs as a self-contained blob."""
    n = int(lib().randes_plan_serialize(plan, None, 0))
    if n == 0:
        raise RandesError(INVALID_ARGUMENT, randes_last_error())
    buf = ctypes.create_string_buffer(n)
    if int(lib().randes_plan_serialize(plan, ctypes.addressof(buf), n)) != n:
        raise RandesError(INVALID_ARGUMENT, randes_last_error())
    return buf.raw


def randes_plan_workspace_needed(plan) -> int:
    """Workspace bytes a plan equal to this one needs (also answered by a host-only plan)."""
    return int(lib().randes_plan_workspace_needed(plan))


def randes_plan_deserialize(blob: bytes, max_tasks: int = 0, dev_workspace=None, dev_workspace_bytes: int = 0, stream=None) -> int:
    """A plan handle rebuilt from randes_plan_serialize's blob (host-only without a workspace)."""
    out = ctypes.c_void_p()
    buf = ctypes.create_string_buffer(blob, len(blob))
    _check(lib().randes_plan_deserialize(ctypes.addressof(buf), len(blob), max_tasks, _addr(dev_workspace), dev_workspace_bytes,
                                         stream, ctypes.byref(out)))
    return out.value


def randes_plan_destroy(plan) -> None:
    lib().randes_plan_destroy(plan)


def randes_plan_validate(plan) -> None:
    """Host-side self-check of a plan's tables; raises RandesError naming the first violation."""
    _check(lib().randes_plan_validate(plan))


def randes_debug_violation():
    """(word, checked_build): the first bounds violation recorded by a checked build's kernels (0 = none)."""
    word, flag = ctypes.c_uint64(0), ctypes.c_int(0)
    _check(lib().randes_debug_violation(ctypes.byref(word), ctypes.byref(flag)))
    return int(word.value), bool(flag.value)


def randes_superposition_bytes(plan) -> int:
    return int(lib().randes_superposition_bytes(plan))


def randes_layer_offset(plan, layer: int) -> int:
    return int(lib().randes_layer_offset(plan, layer))


def randes_num_layers(plan) -> int:
    return int(lib().randes_num_layers(plan))


def randes_num_tasks(plan) -> int:
    return int(lib().randes_num_tasks(plan))


def randes_compress(plan, base, tasks, M, stream) -> None:
    _check(lib().randes_compress(plan, _addr(base), _addr(tasks), _addr(M), stream))


def randes_add_model(plan, task_id, seed, base, task, M, stream) -> None:
    _check(lib().randes_add_model(plan, task_id, seed, _addr(base), _addr(task), _addr(M), stream))


def randes_add_models(plan, task_ids, seeds, base, tasks, M, stream) -> None:
    """Several models added in one pass over M; ``tasks`` holds n_tasks * n_layers pointers, task-major."""
    n = len(task_ids)
    ids = (ctypes.c_uint32 * max(n, 1))(*[int(t) for t in task_ids])
    sds = (ctypes.c_uint64 * max(n, 1))(*[int(t) for t in seeds])
    _check(lib().randes_add_models(plan, ctypes.addressof(ids), ctypes.addressof(sds), n, _addr(base), _addr(tasks), _addr(M), stream))


def randes_remove_model(plan, task_id, base, task, M, stream) -> None:
    _check(lib().randes_remove_model(plan, task_id, _addr(base), _addr(task), _addr(M), stream))


def randes_retrieve(plan, task_id, lam, out_dtype, base, M, out, stream) -> None:
    _check(lib().randes_retrieve(plan, task_id, lam, out_dtype, _addr(base), _addr(M), _addr(out), stream))


def randes_delta_gram_scratch_bytes(plan) -> int:
    return int(lib().randes_delta_gram_scratch_bytes(plan))


def randes_delta_gram(plan, base, tasks, gram, scratch, scratch_bytes, stream) -> None:
    _check(lib().randes_delta_gram(plan, _addr(base), _addr(tasks), _addr(gram), _addr(scratch), scratch_bytes, stream))


def randes_retrieve_batch(plan, task_ids, lam, out_dtype, base, M, out, stream) -> None:
    """Several tasks in one pass; ``out`` holds n_tasks * n_layers pointers, task-major."""
    ids = (ctypes.c_uint32 * len(task_ids))(*[int(t) for t in task_ids])
    _check(lib().randes_retrieve_batch(plan, ctypes.addressof(ids), len(task_ids), lam, out_dtype, _addr(base), _addr(M),
                                       _addr(out), stream))


def randes_retrieve_static(plan, task_id, lam, out_dtype, base, M, out, stream) -> None:
    """retrieve with the kernel's tables in the library's built-in device array (no workspace)."""
    _check(lib().randes_retrieve_static(plan, task_id, lam, out_dtype, _addr(base), _addr(M), _addr(out), stream))


def randes_linear(plan, task_id, lam, layer, x, n_tokens, base, M, y, stream, y_dtype: int = F32) -> None:
    """y = x What_t[layer]^T on the tensor cores, the retrieved weight never written to memory."""
    _check(lib().randes_linear(plan, task_id, lam, layer, _addr(x), n_tokens, _addr(base), _addr(M), _addr(y), y_dtype, stream))


def randes_linear_gated(plan, task_id, lam, layer, x, n_tokens, base, M, y, gate, wait_ns, stream, y_dtype: int = F32) -> None:
    """randes_linear whose thread blocks first wait (at most wait_ns nanoseconds; 0 = one second) for the device word
    ``gate`` to become non-zero; blocks whose wait runs out write nothing and count in randes_linear_giveups()."""
    _check(lib().randes_linear_gated(plan, task_id, lam, layer, _addr(x), n_tokens, _addr(base), _addr(M), _addr(y), y_dtype,
                                     _addr(gate), int(wait_ns), stream))


def randes_linear_giveups() -> int:
    """Thread blocks of randes_linear that gave up on a bounded wait (0 in a healthy run); synchronises."""
    n = ctypes.c_uint(0)
    _check(lib().randes_linear_giveups(ctypes.byref(n)))
    return int(n.value)


def randes_packed_bytes(rows: int, cols: int, group: int) -> int:
    """Bytes of a [rows, cols] matrix in four bits with scales for groups of `group` columns (0 on bad arguments)."""
    return int(lib().randes_packed_bytes(rows, cols, group))


def randes_pack(matrices, n: int, dtype: int, group: int, packed, stream) -> None:
    """Pack `n` matrices (a ctypes array of Matrix) into the buffers whose addresses `packed` holds."""
    _check(lib().randes_pack(_addr(matrices), n, dtype, group, _addr(packed), stream))


def randes_unpack(packed, n: int, group: int, matrices, out_dtype: int, stream) -> None:
    _check(lib().randes_unpack(_addr(packed), n, group, _addr(matrices), out_dtype, stream))


def randes_retrieve_packed(plan, task_id, lam, layers, n, base, M, group, packed, stream) -> None:
    """Pack the retrieved weight of the `n` named layers without storing it in its own type."""
    _check(lib().randes_retrieve_packed(plan, task_id, lam, _addr(layers), n, _addr(base), _addr(M), group, _addr(packed), stream))


def randes_packed_linear_workspace(rows: int, cols: int, x_dtype: int, n_tokens: int, with_tasks: bool) -> int:
    """Bytes of device workspace the two calls below need (0 for up to 8 tokens, unless they are fp32 and the matrix is large)."""
    return int(lib().randes_packed_linear_workspace(rows, cols, x_dtype, n_tokens, int(with_tasks)))


def randes_packed_linear(packed, rows, cols, group, x, x_dtype, x_stride, n_tokens, y, y_dtype, y_stride, stream, workspace=None,
                         workspace_bytes: int = 0) -> None:
    _check(lib().randes_packed_linear(_addr(packed), rows, cols, group, _addr(x), x_dtype, x_stride, n_tokens, _addr(y), y_dtype, y_stride,
                                      _addr(workspace), workspace_bytes, stream))


def randes_packed_linear_tasks(plan, lam, layer, group, task_ids, n_tokens, x, x_dtype, x_stride, packed_base, packed_m, y, y_dtype, y_stride,
                               stream, workspace=None, workspace_bytes: int = 0) -> None:
    _check(lib().randes_packed_linear_tasks(plan, lam, layer, group, _addr(task_ids), n_tokens, _addr(x), x_dtype, x_stride,
                                            _addr(packed_base), _addr(packed_m), _addr(y), y_dtype, y_stride, _addr(workspace), workspace_bytes,
                                            stream))


def randes_token_scores(logits, dtype, n_rows, vocab, stride, targets, scale, top_k, logprob, entropy, stats, top_ids, top_logprobs,
                        stream) -> None:
    _check(lib().randes_token_scores(_addr(logits), dtype, n_rows, vocab, stride, _addr(targets), scale, top_k, _addr(logprob),
                                     _addr(entropy), _addr(stats), _addr(top_ids), _addr(top_logprobs), stream))


def randes_token_scores_backward(logits, dtype, n_rows, vocab, stride, targets, scale, stats, entropy, g_logprob, g_entropy, grad, grad_stride,
                                 stream) -> None:
    _check(lib().randes_token_scores_backward(_addr(logits), dtype, n_rows, vocab, stride, _addr(targets), scale, _addr(stats),
                                              _addr(entropy), _addr(g_logprob), _addr(g_entropy), _addr(grad), grad_stride, stream))


def randes_launch_count() -> int:
    return int(lib().randes_launch_count())


def ptr_array(tensors: Sequence) -> ctypes.Array:
    """Host array of device addresses, one per tensor (nested lists are flattened)."""
    flat = []
    for t in tensors:
        if isinstance(t, (list, tuple)):
            flat.extend(t)
        else:
            flat.append(t)
    arr = (ctypes.c_void_p * max(len(flat), 1))()
    for i, t in enumerate(flat):
        arr[i] = None if t is None else (t if isinstance(t, int) else int(t.data_ptr()))
    return arr


def _as_ptrs(x):
    if x is None or isinstance(x, ctypes.Array):
        return x
    return ptr_array(x)


def _host_gram(gram):
    """An [n, n] Gram matrix (torch tensor, numpy array or nested lists) as a host array of doubles."""
    if hasattr(gram, "detach"):
        gram = gram.detach().cpu().tolist()
    elif hasattr(gram, "tolist"):
        gram = gram.tolist()
    n = len(gram)
    return (ctypes.c_double * max(n * n, 1))(*[float(v) for row in gram for v in row]), n


def randes_interference_norm(gram, t: int, lam: float) -> float:
    """|| lam * sum_{j != t} T_t^-1 T_j d_j || from the Gram matrix; computed by the library."""
    g, n = _host_gram(gram)
    out = ctypes.c_double(0.0)
    _check(lib().randes_interference_norm(ctypes.addressof(g), n, int(t), float(lam), ctypes.byref(out)))
    return float(out.value)


def randes_pairwise_cosines(gram, exclude: int = -1):
    """(cosines as n lists of n floats, mean over pairs j < l that leave `exclude` out); computed by the library."""
    g, n = _host_gram(gram)
    cos = (ctypes.c_double * max(n * n, 1))()
    mean = ctypes.c_double(0.0)
    _check(lib().randes_pairwise_cosines(ctypes.addressof(g), n, -1 if exclude is None else int(exclude), ctypes.addressof(cos),
                                         ctypes.byref(mean)))
    return [[float(cos[j * n + l]) for l in range(n)] for j in range(n)], float(mean.value)


# ---- weights in four bits and token scores on torch tensors ----------------------------------
def _refuse(message: str):
    raise RandesError(INVALID_ARGUMENT, message)


_torch = None      # the module, once a call on tensors has been made: importing this file does not need it


def _rows_of(t, what: str):
    """(element type, rows, columns, elements between rows) of a 2-D CUDA tensor whose rows may be strided; refuses anything
    the library would misread."""
    global _torch
    if _torch is None:
        import torch as _torch
    dtype = t.dtype
    if dtype is _torch.bfloat16:
        code = BF16
    elif dtype is _torch.float32:
        code = F32
    else:
        raise RandesError(UNSUPPORTED_DTYPE, "%s is %s: float32 or bfloat16 is wanted" % (what, dtype))
    if t.dim() != 2 or not t.is_cuda:
        _refuse("%s must be a 2-D CUDA tensor" % what)
    rows, cols = t.shape
    stride, step = t.stride()
    if step != 1 and cols > 1:
        _refuse("%s must have neighbouring columns (its last stride is %d)" % (what, step))
    if rows <= 1:
        stride = cols
    elif stride < cols:
        _refuse("the rows of %s overlap (row stride %d, %d columns)" % (what, stride, cols))
    return code, rows, cols, stride


def _call(device, function, *args) -> None:
    """function(*args, stream) with the tensors' device current (as torch's own operators run: the library launches on the
    current one) and its current stream; raises what the library reports."""
    global _torch
    if _torch is None:
        import torch as _torch
    c, index = _torch._C, device.index
    stream = c._cuda_getCurrentRawStream(index)
    if index == c._cuda_getDevice():
        rc = function(*args, stream)
    else:
        with _torch.cuda.device(device):
            rc = function(*args, stream)
    if rc:
        raise RandesError(rc, randes_last_error())


@functools.lru_cache(maxsize=4096)
def _packed_size(rows: int, cols: int, group: int) -> int:
    if group not in (32, 64, 128):
        _refuse("group = %r is not 32, 64 or 128" % (group,))
    nbytes = randes_packed_bytes(rows, cols, group)
    if nbytes == 0 and rows * cols != 0:
        _refuse("a matrix of [%d, %d] cannot be packed" % (rows, cols))
    return nbytes


_MatrixOne, _PtrOne = Matrix * 1, ctypes.c_void_p * 1


class PackedMatrix:
    """A [rows, cols] weight in four bits with a scale per group of columns (see include/randes.h): one device buffer."""

    __slots__ = ("rows", "cols", "group", "data", "address", "device")

    def __init__(self, rows: int, cols: int, group: int, data):
        """Around a buffer that holds such a matrix: `data` of a PackedMatrix of the same shape and group, or a copy of it."""
        need, have = _packed_size(rows, cols, group), data.numel() * data.element_size()
        if not data.is_cuda or not data.is_contiguous() or have < need:
            _refuse("a packed [%d, %d] matrix in groups of %d columns is a contiguous CUDA tensor of %d bytes, not one of %d on %s"
                    % (rows, cols, group, need, have, data.device))
        if data.data_ptr() % 16:
            raise RandesError(MISALIGNED, "the buffer of a packed matrix starts on a 16-byte boundary")
        self._hold(rows, cols, group, data)

    def _hold(self, rows: int, cols: int, group: int, data):
        self.rows, self.cols, self.group, self.data = rows, cols, group, data
        self.address, self.device = data.data_ptr(), data.device

    @property
    def nbytes(self) -> int:
        return self.data.numel() * self.data.element_size()

    def unpack(self, out_dtype: int = F32, out=None):
        """The [rows, cols] values that the four bits stand for."""
        import torch

        rows, cols = self.rows, self.cols
        if out is None:
            out = torch.empty(rows, cols, dtype=torch.bfloat16 if out_dtype == BF16 else torch.float32, device=self.device)
            stride = cols
        else:
            out_dtype, r, c, stride = _rows_of(out, "out")
            if (r, c) != (rows, cols) or out.device != self.device:
                _refuse("out is [%d, %d] on %s, the matrix [%d, %d] on %s" % (r, c, out.device, rows, cols, self.device))
        _call(self.device, lib().randes_unpack, _PtrOne(self.address), 1, self.group, _MatrixOne((out.data_ptr(), rows, cols, stride)), out_dtype)
        return out


def _new_packed(rows: int, cols: int, group: int, device) -> PackedMatrix:
    import torch

    p = PackedMatrix.__new__(PackedMatrix)      # (the size is right)
    p._hold(rows, cols, group, torch.empty(_packed_size(rows, cols, group), dtype=torch.uint8, device=device))
    return p


def pack(weights, group: int = 64):
    """Four-bit form of a weight, or of a list of weights of one type (2-D CUDA tensors, fp32 or bf16; rows may be strided)."""
    if not isinstance(weights, (list, tuple)):
        dtype, rows, cols, stride = _rows_of(weights, "the weight")
        p = _new_packed(rows, cols, group, weights.device)
        _call(p.device, lib().randes_pack, _MatrixOne((weights.data_ptr(), rows, cols, stride)), 1, dtype, group, _PtrOne(p.address))
        return p
    if not weights:
        return []
    device, n = weights[0].device, len(weights)
    shapes = [_rows_of(w, "a weight") for w in weights]
    if len({s[0] for s in shapes}) != 1 or any(w.device != device for w in weights):
        _refuse("the weights of one call have one type and one device")
    made = [_new_packed(r, c, group, device) for _, r, c, _ in shapes]
    mats = (Matrix * n)(*[(w.data_ptr(), r, c, s) for w, (_, r, c, s) in zip(weights, shapes)])
    _call(device, lib().randes_pack, mats, n, shapes[0][0], group, (ctypes.c_void_p * n)(*[p.address for p in made]))
    return made


def _linear_tensors(x, w: PackedMatrix, y, y_dtype: int):
    """(n_tokens, x's type and row stride, y, y's type and row stride) of a product of x [n_tokens, cols] with a [rows, cols] weight."""
    rows, cols = w.rows, w.cols
    x_dtype, n, c, x_stride = _rows_of(x, "x")
    if c != cols:
        _refuse("x has %d columns, the weight %d" % (c, cols))
    device = w.device
    if x.device != device:
        _refuse("x is on %s, the weight on %s" % (x.device, device))
    if y is None:
        return n, x_dtype, x_stride, _torch.empty(n, rows, dtype=_torch.bfloat16 if y_dtype == BF16 else _torch.float32, device=device), y_dtype, rows
    y_dtype, yn, yr, y_stride = _rows_of(y, "y")
    if (yn, yr) != (n, rows) or y.device != device:
        _refuse("y is [%d, %d] on %s, [%d, %d] on %s is wanted" % (yn, yr, y.device, n, rows, device))
    return n, x_dtype, x_stride, y, y_dtype, y_stride


_linear_workspace_bytes = functools.lru_cache(maxsize=4096)(randes_packed_linear_workspace)


def _linear_workspace(device, rows: int, cols: int, x_dtype: int, n: int, with_tasks: bool):
    """(tensor or None, its address, its bytes): what a product of many tokens lays its activations out in."""
    nbytes = _linear_workspace_bytes(rows, cols, x_dtype, n, with_tasks)
    if nbytes == 0:
        return None, None, 0
    t = _torch.empty(nbytes, dtype=_torch.uint8, device=device)
    return t, t.data_ptr(), nbytes


def packed_linear(x, w: PackedMatrix, y=None, y_dtype: int = F32):
    """x: [n_tokens, cols] fp32 or bf16 CUDA tensor (rows may be strided); returns y = x W^T [n_tokens, rows]."""
    rows, cols = w.rows, w.cols
    n, x_dtype, x_stride, y, y_dtype, y_stride = _linear_tensors(x, w, y, y_dtype)
    workspace, ws_at, ws_bytes = _linear_workspace(w.device, rows, cols, x_dtype, n, False)
    _call(w.device, lib().randes_packed_linear, w.address, rows, cols, w.group, x.data_ptr(), x_dtype, x_stride, n, y.data_ptr(), y_dtype,
          y_stride, ws_at, ws_bytes)
    return y


class TokenScores(NamedTuple):
    """What token_scores returns. ``stats`` [4, n] is what the backward call needs: rows logprob, entropy, greatest logit, log
    of the sum of exponentials relative to it (of scale * logits). ``logprob`` and ``entropy`` are views of its first two rows:
    clone them before changing them in place, an entropy that has changed changes the entropy's gradient."""

    logprob: Any
    entropy: Any
    stats: Any
    top_ids: Any
    top_logprobs: Any


def _target_address(targets, n: int, device):
    if targets is None:
        return None
    if targets.dtype is not _torch.int64 or targets.shape != (n,) or not targets.is_contiguous() or targets.device != device:
        _refuse("targets must be a contiguous int64 tensor [%d] on %s" % (n, device))
    return targets.data_ptr()


def token_scores(logits, targets=None, top_k: int = 0, scale: float = 1.0) -> TokenScores:
    """Log probability of `targets`, entropy, and the `top_k` best tokens of every row of logits * scale (see include/randes.h).

    logits: [n, vocab] fp32 or bf16 CUDA tensor (rows may be strided); targets: int64 [n], negative = not scored."""
    dtype, n, vocab, stride = _rows_of(logits, "logits")
    device = logits.device
    target = _target_address(targets, n, device)
    if not 0 <= top_k <= 64:
        _refuse("top_k = %d is not in 0 .. 64" % top_k)
    stats = _torch.empty(4, n, dtype=_torch.float32, device=device)
    at = stats.data_ptr()
    ids = tops = None
    if top_k:
        ids = _torch.empty(n, top_k, dtype=_torch.int64, device=device)
        tops = _torch.empty(n, top_k, dtype=_torch.float32, device=device)
    _call(device, lib().randes_token_scores, logits.data_ptr(), dtype, n, vocab, stride, target, scale, top_k, at if target is not None else None,
          at + 4 * n, at + 8 * n, ids.data_ptr() if top_k else None, tops.data_ptr() if top_k else None)
    return TokenScores(stats[0] if targets is not None else None, stats[1], stats, ids, tops)


def _row_gradient(g, what: str, n: int, device):
    if g is None:
        return None
    if g.dtype is not _torch.float32 or g.shape != (n,) or not g.is_contiguous() or g.device != device:
        _refuse("%s must be a contiguous float32 tensor [%d] on %s" % (what, n, device))
    return g.data_ptr()


def token_scores_backward(logits, targets, scores: TokenScores, g_logprob=None, g_entropy=None, scale: float = 1.0, out=None):
    """Gradient of sum(g_logprob * logprob + g_entropy * entropy) with respect to the logits; `out` may be the logits themselves.

    Reads ``scores.stats`` (of token_scores on the same logits and scale), the entropy in it only with ``g_entropy``."""
    dtype, n, vocab, stride = _rows_of(logits, "logits")
    device, stats = logits.device, scores.stats
    target = _target_address(targets, n, device)
    g_lp, g_h = _row_gradient(g_logprob, "g_logprob", n, device), _row_gradient(g_entropy, "g_entropy", n, device)
    if stats.dtype is not _torch.float32 or stats.shape != (4, n) or not stats.is_contiguous() or stats.device != device:
        _refuse("the scores are not those of %d rows on %s" % (n, device))
    if out is None:
        out, out_stride = _torch.empty(n, vocab, dtype=logits.dtype, device=device), vocab
    else:
        out_dtype, on, ov, out_stride = _rows_of(out, "out")
        if (out_dtype, on, ov) != (dtype, n, vocab) or out.device != device:
            _refuse("out must have the logits' shape, type and device")
    at = stats.data_ptr()
    _call(device, lib().randes_token_scores_backward, logits.data_ptr(), dtype, n, vocab, stride, target, scale, at + 8 * n, at + 4 * n, g_lp,
          g_h, out.data_ptr(), out_stride)
    return out


# ---- convenience object over torch tensors --------------------------------------------------
class Plan:
    """A plan plus the device workspace it lives in.

    ``rows, cols, group`` describe the layers, ``gflags`` the groups (see
    ``include/randes.h``).  Tensors passed to the methods are torch CUDA tensors
    of the storage dtype (float32 or bfloat16), one per layer.
    """

    def __init__(self, rows, cols, group, gflags, storage: int = F32, task_ids=(), seeds=(),
                 max_tasks: Optional[int] = None, device="cuda", host_only: bool = False, m_dtype: int = F32):
        n_layers, n_groups = len(rows), len(gflags)
        self._layers = (Layer * max(n_layers, 1))()
        for l in range(n_layers):
            self._layers[l] = Layer(int(rows[l]), int(cols[l]), int(group[l]))
        self._groups = (Group * max(n_groups, 1))()
        for g in range(n_groups):
            self._groups[g] = Group(int(gflags[g]))
        n_tasks = len(task_ids)
        if max_tasks is None:
            max_tasks = max(1, n_tasks + 8)
        ids = (ctypes.c_uint32 * max(n_tasks, 1))(*[int(t) for t in task_ids])
        sds = (ctypes.c_uint64 * max(n_tasks, 1))(*[int(s) for s in seeds])
        self.n_layers = n_layers
        self.rows, self.cols = [int(r) for r in rows], [int(c) for c in cols]
        self.storage = storage
        self.m_dtype = m_dtype
        self.handle = None
        self.workspace = None
        self.device = device
        ws_ptr, ws_bytes, stream = None, 0, None
        if not host_only:
            import torch

            ws_bytes = randes_plan_workspace_bytes_groups(self._layers, n_layers, self._groups, n_groups, max_tasks)
            if ws_bytes == 0:
                raise RandesError(INVALID_ARGUMENT, randes_last_error())
            self.workspace = torch.empty(ws_bytes, dtype=torch.uint8, device=device)
            ws_ptr = self.workspace.data_ptr()
            stream = self._stream()
        self.handle = randes_plan(self._layers, n_layers, self._groups, n_groups, storage, m_dtype, ids, sds, n_tasks,
                                  max_tasks, ws_ptr, ws_bytes, stream)
        self.m_bytes = randes_superposition_bytes(self.handle)
        self.offsets = [randes_layer_offset(self.handle, l) for l in range(n_layers)]

    @classmethod
    def from_workload(cls, w, **kw) -> "Plan":
        kw.setdefault("task_ids", w.task_ids)
        kw.setdefault("seeds", w.seeds)
        return cls(w.rows, w.cols, w.group, w.gflags, storage=w.storage, **kw)

    def _stream(self):
        import torch

        return torch.cuda.current_stream(self.device).cuda_stream

    def close(self) -> None:
        if self.handle is not None:
            randes_plan_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # -- queries
    @property
    def n_tasks(self) -> int:
        return randes_num_tasks(self.handle)

    def task_list(self):
        n = self.n_tasks
        ids = (ctypes.c_uint32 * max(n, 1))()
        sds = (ctypes.c_uint64 * max(n, 1))()
        _check(lib().randes_task_list(self.handle, ctypes.addressof(ids), ctypes.addressof(sds)))
        return [int(x) for x in ids[:n]], [int(x) for x in sds[:n]]

    def task_tables(self, task_id: int):
        src = (ctypes.c_uint32 * max(self.n_layers, 1))()
        pos = (ctypes.c_uint32 * max(self.n_layers, 1))()
        _check(lib().randes_task_tables(self.handle, task_id, ctypes.addressof(src), ctypes.addressof(pos)))
        return [int(x) for x in src[:self.n_layers]], [int(x) for x in pos[:self.n_layers]]

    # -- device buffers
    def new_superposition(self):
        import torch

        if self.m_dtype == BF16:
            return torch.empty(self.m_bytes // 2, dtype=torch.bfloat16, device=self.device)
        return torch.empty(self.m_bytes // 4, dtype=torch.float32, device=self.device)

    def slot(self, M, layer: int):
        """View of slot ``layer`` of the arena M as a [rows, cols] tensor."""
        o = self.offsets[layer] // (2 if self.m_dtype == BF16 else 4)
        n = self.rows[layer] * self.cols[layer]
        return M[o:o + n].view(self.rows[layer], self.cols[layer])

    def new_output(self, out_dtype: int = F32):
        import torch

        dt = torch.bfloat16 if out_dtype == BF16 else torch.float32
        return [torch.empty(r, c, dtype=dt, device=self.device) for r, c in zip(self.rows, self.cols)]

    # -- the path
    def compress(self, base, tasks, M=None):
        if M is None:
            M = self.new_superposition()
        randes_compress(self.handle, _as_ptrs(base), _as_ptrs(tasks), M, self._stream())
        return M

    def add_model(self, task_id: int, seed: int, base, task, M):
        randes_add_model(self.handle, task_id, seed, _as_ptrs(base), _as_ptrs(task), M, self._stream())
        return M

    def add_models(self, task_ids, seeds, base, tasks, M):
        randes_add_models(self.handle, task_ids, seeds, _as_ptrs(base), _as_ptrs(tasks), M, self._stream())
        return M

    def remove_model(self, task_id: int, base, task, M):
        randes_remove_model(self.handle, task_id, _as_ptrs(base), _as_ptrs(task), M, self._stream())
        return M

    def delta_gram(self, base, tasks):
        """Gram matrix of the transformed deltas as an [n, n] float64 CUDA tensor (see include/randes.h)."""
        import torch

        n = self.n_tasks
        gram = torch.empty(n, n, dtype=torch.float64, device=self.device)
        nbytes = randes_delta_gram_scratch_bytes(self.handle)
        scratch = torch.empty(nbytes // 8, dtype=torch.float64, device=self.device)
        randes_delta_gram(self.handle, _as_ptrs(base), _as_ptrs(tasks), gram, scratch, nbytes, self._stream())
        return gram

    def retrieve_batch(self, task_ids, lam: float, base, M, out=None, out_dtype: int = F32):
        """Rebuild several tasks in one launch; returns a list (per task) of lists of tensors."""
        out_lists = None
        if out is None:
            out = out_lists = [self.new_output(out_dtype) for _ in task_ids]
        elif not isinstance(out, ctypes.Array):
            out_lists = out
        randes_retrieve_batch(self.handle, task_ids, lam, out_dtype, _as_ptrs(base), M, _as_ptrs(out), self._stream())
        return out_lists

    def linear(self, task_id: int, lam: float, layer: int, x, base, M, y=None, y_dtype: int = F32):
        """x: [n_tokens, cols] bf16 CUDA tensor; returns y [n_tokens, rows], fp32 or bf16."""
        import torch

        if y is None:
            y = torch.empty((x.shape[0], self.rows[layer]), dtype=torch.bfloat16 if y_dtype == BF16 else torch.float32, device=x.device)
        else:
            y_dtype = BF16 if y.dtype == torch.bfloat16 else F32
        randes_linear(self.handle, task_id, lam, layer, x, int(x.shape[0]), _as_ptrs(base), M, y, self._stream(), y_dtype)
        return y

    def retrieve(self, task_id: int, lam: float, base, M, out=None, out_dtype: int = F32):
        out_list = None
        if out is None:
            out = out_list = self.new_output(out_dtype)
        elif not isinstance(out, ctypes.Array):
            out_list = out
        randes_retrieve(self.handle, task_id, lam, out_dtype, _as_ptrs(base), M, _as_ptrs(out), self._stream())
        return out_list

    # -- four-bit weights (see PackedMatrix)
    def _layer(self, layer) -> int:
        if not 0 <= int(layer) < self.n_layers:
            _refuse("layer %d out of range (n_layers = %d)" % (int(layer), self.n_layers))
        return int(layer)

    @staticmethod
    def _stored(t, what: str, dtype: int, shape, device, at_least: bool = False) -> int:
        """Address of a tensor that the library reads as so many dense elements of this type; refuses any other."""
        import torch

        if not hasattr(t, "data_ptr"):
            _refuse("%s is no tensor" % what)
        want = torch.bfloat16 if dtype == BF16 else torch.float32
        if t.dtype is not want:
            raise RandesError(UNSUPPORTED_DTYPE, "%s is %s: this plan keeps it in %s" % (what, t.dtype, want))
        if t.shape != shape:
            n, have = math.prod(shape), t.numel()
            if (have < n if at_least else have != n) or (t.dim() == 2 and not at_least):
                _refuse("%s is %s, %s is wanted" % (what, list(t.shape), list(shape)))
        if not t.is_contiguous() or (not t.is_cuda if device is None else t.device != device):
            _refuse("%s must be a contiguous tensor on %s" % (what, "a CUDA device" if device is None else device))
        return t.data_ptr()

    def _arena(self, M) -> int:
        """Address of M, after the checks that a tensor has to pass before the library reads it as this plan's superposition."""
        return self._stored(M, "M", self.m_dtype, (self.m_bytes // (2 if self.m_dtype == BF16 else 4),), None, at_least=True)

    def _weights(self, base, layers, device):
        """Host array of the weights' addresses; the named ones are checked. Addresses (a ctypes array, or numbers in the list)
        are taken at the caller's word, as the other methods take them."""
        have, top = len(base), max(layers, default=-1)
        if have <= top or (isinstance(base, ctypes.Array) and base._type_ is not ctypes.c_void_p):
            _refuse("base has %d weights, layer %d is named" % (have, top))
        if isinstance(base, ctypes.Array):
            return base
        out = (ctypes.c_void_p * max(self.n_layers, 1))()
        for l in layers:
            w = base[l]
            out[l] = w if isinstance(w, int) else self._stored(w, "base[%d]" % l, self.storage, (self.rows[l], self.cols[l]), device)
        return out

    def pack_superposition(self, M, group: int = 64, slots=None):
        """Four-bit form of the slots of M, a list by slot (None for slots not named)."""
        self._arena(M)
        slots = list(range(self.n_layers)) if slots is None else [self._layer(l) for l in slots]
        made = pack([self.slot(M, l) for l in slots], group)
        out = [None] * self.n_layers
        for l, p in zip(slots, made):
            out[l] = p
        return out

    def retrieve_packed(self, task_id: int, lam: float, base, M, group: int = 64, layers=None):
        """Four-bit form of one retrieved model, its own type never stored; a list, one entry per named layer (default: all).

        ``base`` is the list of all layers' weights, dense and in the plan's type; only the named ones are read."""
        m = self._arena(M)
        device = M.device
        layers = list(range(self.n_layers)) if layers is None else [self._layer(l) for l in layers]
        n = len(layers)
        weights = self._weights(base, layers, device)
        made = [_new_packed(self.rows[l], self.cols[l], group, device) for l in layers]
        _call(device, lib().randes_retrieve_packed, self.handle, task_id, lam, (ctypes.c_uint32 * max(n, 1))(*layers), n, weights, m, group,
              (ctypes.c_void_p * max(n, 1))(*[p.address for p in made]))
        return made

    def packed_linear(self, task_ids, lam: float, layer: int, x, packed_base: PackedMatrix, packed_m, y=None, y_dtype: int = F32):
        """One layer applied to a few tokens, token b with the retrieved weight of task_ids[b].

        ``packed_base`` is the layer's W_0, ``packed_m`` the slots of M by slot (pack_superposition), all packed with one
        group size; x: [n_tokens, cols] fp32 or bf16; returns y [n_tokens, rows]."""
        layer = self._layer(layer)
        if not isinstance(packed_base, PackedMatrix):
            _refuse("packed_base is no PackedMatrix")
        rows, cols, group, device = self.rows[layer], self.cols[layer], packed_base.group, packed_base.device
        if (packed_base.rows, packed_base.cols) != (rows, cols):
            _refuse("packed_base is [%d, %d], layer %d is [%d, %d]" % (packed_base.rows, packed_base.cols, layer, rows, cols))
        if len(packed_m) != self.n_layers:
            _refuse("packed_m has %d entries, the plan %d slots" % (len(packed_m), self.n_layers))
        slots = (ctypes.c_void_p * max(self.n_layers, 1))()
        try:
            for l, p in enumerate(packed_m):
                if p is None or (p.rows, p.cols) != (rows, cols):
                    continue      # not a slot this layer can lie in
                if p.group != group or p.device != device:
                    _refuse("slot %d has groups of %d columns on %s, the base of %d on %s" % (l, p.group, p.device, group, device))
                slots[l] = p.address
        except AttributeError:
            _refuse("packed_m holds something that is no PackedMatrix")
        n, x_dtype, x_stride, y, y_dtype, y_stride = _linear_tensors(x, packed_base, y, y_dtype)
        if len(task_ids) != n:
            _refuse("%d task ids for %d tokens" % (len(task_ids), n))
        if not (isinstance(task_ids, ctypes.Array) and task_ids._type_ is ctypes.c_uint32):
            task_ids = (ctypes.c_uint32 * max(n, 1))(*task_ids)
        workspace, ws_at, ws_bytes = _linear_workspace(device, rows, cols, x_dtype, n, True)
        _call(device, lib().randes_packed_linear_tasks, self.handle, lam, layer, group, task_ids, n, x.data_ptr(), x_dtype, x_stride,
              packed_base.address, slots, y.data_ptr(), y_dtype, y_stride, ws_at, ws_bytes)
        return y
