"""ctypes binding of libfira.so: argument marshalling only.

Every entry point of include/fira.h has a function of the same name on `lib()`;
`Fira` wraps a context and takes torch tensors for device memory.  Nothing here
computes: all arithmetic runs in the library's CUDA kernels.  If the shared
library is missing, `lib()` raises; there is no fallback.
"""
from __future__ import annotations

import ctypes as C
import importlib
import os
import sysconfig
import warnings
from array import array
from typing import Optional, Sequence, Tuple

import torch

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libfira.so")

FIRA_OK = 0
FIRA_F32, FIRA_BF16 = 0, 1
FLAG_ALPHA_LOWRANK_ONLY, FLAG_AUTO_REFRESH, FLAG_FORCE_SIMT = 1, 2, 4
FLAG_MATRIX_SCALING, FLAG_NO_SCALING, FLAG_NO_RESIDUAL = 8, 16, 32
FLAG_PSI_RMSPROP, FLAG_PSI_ADAGRAD = 64, 128
FLAG_ONLY_SCALING = 256
FLAG_ROW_PADDING_WRITABLE = 512

STATUS_NAMES = {0: "FIRA_OK", 1: "FIRA_ERR_INVALID_ARG", 2: "FIRA_ERR_WORKSPACE_TOO_SMALL",
                3: "FIRA_ERR_UNSUPPORTED", 4: "FIRA_ERR_CUDA", 5: "FIRA_ERR_DEVICE_TIMEOUT",
                6: "FIRA_ERR_NONFINITE"}


class Hparams(C.Structure):
    _fields_ = [("beta1", C.c_float), ("beta2", C.c_float), ("eps", C.c_float), ("lr", C.c_float),
                ("alpha", C.c_float), ("gamma", C.c_float), ("T", C.c_int32), ("flags", C.c_uint32)]


class MatrixDesc(C.Structure):
    _fields_ = [("m", C.c_int32), ("n", C.c_int32), ("r", C.c_int32), ("dtype", C.c_int32),
                ("ld", C.c_int64)]


class Diag(C.Structure):
    _fields_ = [("norm_scaled", C.c_float), ("lambda_", C.c_float), ("norm_prev", C.c_float),
                ("k_min", C.c_float), ("k_max", C.c_float), ("t", C.c_int64), ("engine", C.c_int32)]


class GradDesc(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int64), ("ld", C.c_int64), ("out_ld", C.c_int64),
                ("dtype", C.c_int32), ("out_dtype", C.c_int32)]


class FiraError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"{STATUS_NAMES.get(status, status)}: {message}")
        self.status = status


# name -> (restype, argtypes); mirrors include/fira.h one to one
SIGNATURES = {
    "fira_query_workspace": (C.c_int, [C.POINTER(Hparams), C.POINTER(MatrixDesc), C.c_int32,
                                       C.POINTER(C.c_size_t), C.POINTER(C.c_size_t)]),
    "fira_init": (C.c_int, [C.POINTER(C.c_void_p), C.POINTER(Hparams), C.POINTER(MatrixDesc), C.c_int32,
                            C.c_void_p, C.c_size_t, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fira_step": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_float]),
    "fira_step_host": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.c_float,
                                 C.c_void_p, C.c_size_t]),
    "fira_staging_bytes": (C.c_size_t, [C.c_void_p]),
    "fira_refresh_projection": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_int32),
                                          C.c_int32, C.c_uint64, C.c_int32]),
    "fira_refresh_projection_f32": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_int32),
                                              C.c_int32, C.c_uint64, C.c_int32, C.POINTER(C.c_void_p)]),
    "fira_refresh_side_work_bytes": (C.c_size_t, [C.c_void_p]),
    "fira_refresh_projection_side": (C.c_int, [C.c_void_p, C.POINTER(C.c_void_p), C.POINTER(C.c_int32), C.c_int32,
                                               C.c_uint64, C.c_int32, C.POINTER(C.c_void_p), C.c_void_p,
                                               C.c_size_t, C.c_void_p]),
    "fira_set_projection": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p]),
    "fira_get_projection": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p]),
    "fira_get_state": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.POINTER(C.c_float),
                                 C.POINTER(C.c_int64)]),
    "fira_set_state": (C.c_int, [C.c_void_p, C.c_int32, C.c_void_p, C.c_void_p, C.c_float, C.c_int64]),
    "fira_state_elements": (C.c_int64, [C.c_void_p, C.c_int32]),
    "fira_get_diagnostics": (C.c_int, [C.c_void_p, C.c_int32, C.POINTER(Diag)]),
    "fira_poll": (C.c_int, [C.c_void_p]),
    "fira_selftest_bounded_wait": (C.c_int, [C.c_void_p, C.c_int32]),
    "fira_last_step_launches": (C.c_int32, [C.c_void_p]),
    "fira_enable_phase_timing": (C.c_int, [C.c_void_p, C.c_int32]),
    "fira_get_phase_times": (C.c_int, [C.c_void_p, C.POINTER(C.c_int32), C.POINTER(C.c_float),
                                       C.POINTER(C.c_int32)]),
    "fira_phase_name": (C.c_char_p, [C.c_void_p, C.c_int32]),
    "fira_step_single_noalloc": (C.c_int, [C.POINTER(Hparams), C.POINTER(MatrixDesc), C.c_void_p,
                                           C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p,
                                           C.c_void_p, C.c_float, C.c_void_p]),
    "fira_noalloc_max_scratch_bytes": (C.c_size_t, []),
    "fira_noalloc_poll": (C.c_int, [C.c_void_p]),
    "fira_adam_dense": (C.c_int, [C.POINTER(Hparams), C.c_int32, C.POINTER(C.c_void_p), C.POINTER(C.c_void_p),
                                  C.POINTER(C.c_void_p), C.POINTER(C.c_void_p), C.POINTER(C.c_int64), C.c_int,
                                  C.c_int64, C.c_float, C.c_void_p]),
    "fira_grad_work_bytes": (C.c_size_t, [C.c_int32]),
    # (host arrays as bytes objects, or by address: GradDesc and device pointers)
    "fira_grad_norm": (C.c_int, [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fira_clip_grads": (C.c_int, [C.c_int32, C.c_void_p, C.c_void_p, C.c_void_p, C.c_float, C.c_void_p, C.c_void_p,
                                  C.c_void_p, C.c_size_t, C.c_void_p]),
    "fira_embedding": (C.c_int, [C.c_void_p, C.c_int64, C.c_int64, C.c_int64, C.c_int, C.c_void_p, C.c_int32, C.c_int64,
                                 C.c_float, C.c_void_p, C.c_int64, C.c_void_p]),
    "fira_embedding_grad_work_bytes": (C.c_size_t, [C.c_int64, C.c_int64, C.c_int64, C.c_int]),
    "fira_embedding_grad": (C.c_int, [C.c_void_p, C.c_int32, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.c_int64, C.c_int64,
                                      C.c_float, C.c_void_p, C.c_int64, C.c_int, C.c_int32, C.c_void_p, C.c_size_t,
                                      C.c_void_p]),
    "fira_layer_norm": (C.c_int, [C.c_void_p, C.c_int64, C.c_int, C.c_int64, C.c_int64, C.c_void_p, C.c_void_p, C.c_int,
                                  C.c_float, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p, C.c_void_p]),
    "fira_layer_norm_grad_work_bytes": (C.c_size_t, [C.c_int64, C.c_int64, C.c_int]),
    "fira_layer_norm_grad": (C.c_int, [C.c_void_p, C.c_int64, C.c_void_p, C.c_int64, C.c_int, C.c_int64, C.c_int64, C.c_void_p,
                                       C.c_int, C.c_void_p, C.c_void_p, C.c_void_p, C.c_int64, C.c_void_p, C.c_void_p,
                                       C.c_int, C.c_int32, C.c_void_p, C.c_size_t, C.c_void_p]),
    "fira_status_string": (C.c_char_p, [C.c_int]),
    "fira_last_error": (C.c_char_p, []),
    "fira_destroy": (None, [C.c_void_p]),
}

_LIB = None


def lib() -> C.CDLL:
    """Loads libfira.so (once).  Raises if it has not been built."""
    global _LIB
    if _LIB is None:
        if not os.path.exists(LIB_PATH):
            raise FileNotFoundError(
                f"{LIB_PATH} not found: build it with `python -m paper_2410_01623_b200.build`")
        handle = C.CDLL(LIB_PATH)
        for name, (res, args) in SIGNATURES.items():
            fn = getattr(handle, name)
            fn.restype = res
            fn.argtypes = args
        _LIB = handle
    return _LIB


def check(status: int) -> None:
    if status != FIRA_OK:
        raise FiraError(status, lib().fira_last_error().decode())


def ptr_array(tensors: Sequence[Optional[torch.Tensor]]):
    arr = (C.c_void_p * len(tensors))()
    for i, t in enumerate(tensors):
        arr[i] = None if t is None else t.data_ptr()
    return arr


def make_hparams(lr=1e-2, beta1=0.9, beta2=0.999, eps=1e-8, alpha=0.25, gamma=1.01, T=0,
                 flags=0) -> Hparams:
    return Hparams(beta1, beta2, eps, lr, alpha, gamma, T, flags)


def adam_dense(hp: Hparams, Ws: Sequence[torch.Tensor], Gs: Sequence[torch.Tensor], Ms: Sequence[torch.Tensor],
               Vs: Sequence[torch.Tensor], t: int, lr: Optional[float] = None) -> None:
    """fira_adam_dense: one plain Adam step (Eq. 1-4) of a list of unprojected tensors, in place.
    Argument marshalling only."""
    n = len(Ws)
    assert n == len(Gs) == len(Ms) == len(Vs) and n > 0
    dt = Ws[0].dtype
    for w, g, m, v in zip(Ws, Gs, Ms, Vs):
        assert w.is_cuda and w.is_contiguous() and g.is_contiguous() and m.is_contiguous() and v.is_contiguous()
        assert w.dtype == g.dtype == dt and m.dtype == v.dtype == torch.float32
        assert w.numel() == g.numel() == m.numel() == v.numel()
    numel = (C.c_int64 * n)(*[w.numel() for w in Ws])
    stream = torch.cuda.current_stream(Ws[0].device).cuda_stream
    with torch.cuda.device(Ws[0].device):
        check(lib().fira_adam_dense(C.byref(hp), n, ptr_array(Ws), ptr_array(Gs), ptr_array(Ms), ptr_array(Vs),
                                    numel, 1 if dt == torch.bfloat16 else 0, int(t),
                                    -1.0 if lr is None else float(lr), C.c_void_p(stream)))


_CODES = {torch.float32: FIRA_F32, torch.bfloat16: FIRA_BF16}
_TOKEN_BITS = {torch.int32: 32, torch.int64: 64}
_T = torch.Tensor

# The stream's address by itself (0.1 us instead of 3, where a small call takes 10 in all).
_raw_stream = getattr(torch._C, "_cuda_getCurrentRawStream", None) or (
    lambda index: torch.cuda.current_stream(index).cuda_stream)


def _refuse(what: str):
    raise ValueError(what)


def _not_recorded(name: str) -> None:
    warnings.warn(f"{name} is not recorded for autograd: no gradient reaches its inputs by backward(), call {name}_grad (under "
                  "torch.no_grad() this is not said)", stacklevel=3)


def _code(t: torch.Tensor, what: str) -> int:
    code = _CODES.get(t.dtype)
    return _refuse(f"{what}: float32 or bfloat16, not {t.dtype}") if code is None else code


def _device_of(first: torch.Tensor, *others: Optional[torch.Tensor]) -> int:
    """The index of the CUDA device that all of a call's tensors lie on."""
    index = first.get_device()
    if index < 0:
        raise ValueError(f"the Fira library runs on a CUDA device only, not on {first.device}")
    for t in others:
        if t is not None and t.get_device() != index:
            raise ValueError(f"tensors on {t.device} and on {first.device}")
    return index


def _check_work(work: Optional[torch.Tensor]) -> None:
    """A workspace is as large as its elements say: an expanded tensor is not."""
    if work is not None and not work.is_contiguous():
        raise ValueError(f"work: a contiguous tensor is needed, not strides {tuple(work.stride())} of shape {tuple(work.shape)}")


def _pitch_of(t: torch.Tensor) -> Optional[int]:
    """Elements from row to row of a tensor whose last dimension is a row (0: contiguous); None if that is not one number."""
    if t.is_contiguous():
        return 0
    *counts, width = t.shape
    *steps, step = t.stride()
    if width != 1 and step != 1:
        return None
    pitch, rows = None, 1
    for n, s in zip(reversed(counts), reversed(steps)):
        if n == 1:
            continue
        if pitch is None:
            pitch = s
        elif s != pitch * rows:
            return None
        rows *= n
    if pitch is None:
        return 0
    return pitch if pitch >= width else None


def _pitch(t: torch.Tensor, what: str) -> int:
    """_pitch_of, where there has to be one."""
    pitch = _pitch_of(t)
    if pitch is None:
        raise ValueError(f"{what}: strides {tuple(t.stride())} of shape {tuple(t.shape)}: rows of one pitch are needed")
    return pitch


def _rows_or_copy(t: torch.Tensor) -> torch.Tensor:
    """t, or its rows one behind another where they have no one pitch."""
    return t if _pitch_of(t) is not None else t.contiguous()


def _norm_rows(x: torch.Tensor) -> Tuple[torch.Tensor, int]:
    """x as layer norm reads it, and its pitch: rows of more than two dimensions that have no one pitch (a slice of a batch) are
    copied."""
    if x.dim() > 2 and x.stride(-1) == 1:
        x = _rows_or_copy(x)
    return x, _pitch(x, "x")


def _rows(t: torch.Tensor, flip: bool):
    """(rows, cols, ld) of a 2-D tensor, or of its transpose, as a row-major matrix; None if it is none."""
    if t.dim() != 2:
        return None
    (m, n), (a, b) = (t.shape, t.stride()) if not flip else (t.shape[::-1], t.stride()[::-1])
    if (n > 1 and b != 1) or (m > 1 and a < n):
        return None
    return m, n, (a if m > 1 else n)


def _grad_words(i: int, g: torch.Tensor, o: torch.Tensor):
    """rows, cols, ld, out_ld of one gradient and the tensor that it is scaled into."""
    if g.shape != o.shape:
        raise ValueError(f"gradient {i}: its shape is {tuple(g.shape)}, its output's {tuple(o.shape)}")
    if g.is_contiguous() and o.is_contiguous():
        return 1, g.numel(), 0, 0
    for flip in (False, True):                 # a matrix and its transpose have the same elements, in another order
        a, b = _rows(g, flip), _rows(o, flip)
        if a is not None and b is not None:
            return (*a, b[2])
    raise ValueError(f"gradient {i}: strides {tuple(g.stride())} and, of its output, {tuple(o.stride())} of shape "
                     f"{tuple(g.shape)}: not both row-major, or both transposed, matrices")


def _grad_codes(tensors: Sequence[torch.Tensor]):
    """The type codes of a list: a number where all are of one type, else an array."""
    types = {t.dtype for t in tensors}
    if not types <= _CODES.keys():
        raise ValueError(f"gradients and their outputs are float32 or bfloat16, not {types}")
    return _CODES[types.pop()] if len(types) == 1 else array("i", [_CODES[t.dtype] for t in tensors])


_LISTS_PATH = os.path.join(_PKG, "_native_lists" + sysconfig.get_config_var("EXT_SUFFIX"))


def _native_grad_list(Gs, out):
    """Lists of tensors read natively (csrc/grad_list.cpp): speed alone.  The module may be built after this one is imported, so
    it is looked for until it is there; one that is made for other descriptors or another torch is not used."""
    global _native_grad_list
    if not os.path.exists(_LISTS_PATH):
        return None
    importlib.invalidate_caches()
    try:
        module = importlib.import_module("._native_lists", __package__)
        fits = (module.torch_version, module.desc_bytes) == (torch.__version__, C.sizeof(GradDesc))
    except (ImportError, AttributeError, TypeError):     # (TypeError: this file on its own, in no package)
        fits = False
    _native_grad_list = module.grad_list if fits else lambda Gs, out: None
    return _native_grad_list(Gs, out)


def _grad_list(Gs: Sequence[torch.Tensor], out: Optional[Sequence[torch.Tensor]]):
    """The device's index and what goes to the library: descriptors, addresses, the outputs' addresses.  Contiguous
    tensors are read natively; the others' lists go through map() and arrays."""
    native = _native_grad_list(Gs, out)
    if native is not None:
        return native
    n = len(Gs)
    if n == 0:
        raise ValueError("an empty list of gradients")
    codes = _grad_codes(Gs)
    out_codes = codes if out is None else _grad_codes(out)
    devices = set(map(_T.get_device, Gs))
    if out is not None:
        devices.update(map(_T.get_device, out))
    if len(devices) > 1:
        raise ValueError("the gradients and their outputs lie on different devices")
    words = array("q", bytes(40 * n))
    if all(map(_T.is_contiguous, Gs)) and (out is None or (all(map(_T.is_contiguous, out)) and
                                                           [g.shape for g in Gs] == [o.shape for o in out])):
        words[0::5] = array("q", (1,)) * n
        words[1::5] = array("q", map(_T.numel, Gs))
    else:
        flat = [w for i, (g, o) in enumerate(zip(Gs, Gs if out is None else out)) for w in _grad_words(i, g, o)]
        for k in range(4):
            words[k::5] = array("q", flat[k::4])
    if type(codes) is int and type(out_codes) is int:
        words[4::5] = array("q", (codes | out_codes << 32,)) * n
    else:
        both = array("i", bytes(8 * n))
        both[0::2] = array("i", (codes,)) * n if type(codes) is int else codes
        both[1::2] = array("i", (out_codes,)) * n if type(out_codes) is int else out_codes
        words[4::5] = array("q", both.tobytes())
    index = devices.pop()
    if index < 0:
        raise ValueError(f"the Fira library runs on a CUDA device only, not on {Gs[0].device}")
    return (index, words.tobytes(), array("Q", map(_T.data_ptr, Gs)).tobytes(),
            None if out is None else array("Q", map(_T.data_ptr, out)).tobytes())


def grad_work_bytes(count: int) -> int:
    return lib().fira_grad_work_bytes(count)


def grad_norm(Gs: Sequence[torch.Tensor], work: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fira_grad_norm: the norm over all elements of a list of gradients (float32 and bfloat16 may be mixed), as a
    float32 tensor of one element on the device; nothing waits for it.  work: a byte tensor of at least
    grad_work_bytes(len(Gs)) bytes; by default torch's allocator lends one for the call."""
    _check_work(work)
    index, words, at, _ = _grad_list(Gs, None)
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return grad_norm(Gs, work)
    L, n = lib(), len(Gs)
    norm = Gs[0].new_empty((), dtype=torch.float32)
    if work is None:                           # (float32 by norm's type: the shortest way)
        work = norm.new_empty(L.fira_grad_work_bytes(n) // 4)
    elif work.get_device() != index:
        raise ValueError(f"work is on {work.device}, the gradients on {norm.device}")
    status = L.fira_grad_norm(n, words, at, norm.data_ptr(), work.data_ptr(), work.nbytes, _raw_stream(index))
    if status:
        check(status)
    return norm


def clip_grads(Gs: Sequence[torch.Tensor], max_norm: float, out: Optional[Sequence[torch.Tensor]] = None,
               work: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """fira_clip_grads: scales a list of gradients so that their global norm is at most max_norm, in place or into `out`
    (tensors of the same shapes, float32 or bfloat16 each, which overlap no gradient but their own, and that from its first
    element on), and returns the norm before it and the factor, as float32 tensors of one element on the device.  work: as
    for grad_norm."""
    if out is not None and len(out) != len(Gs):
        raise ValueError(f"{len(out)} outputs for {len(Gs)} gradients")
    _check_work(work)
    index, words, at, out_at = _grad_list(Gs, out)
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return clip_grads(Gs, max_norm, out, work)
    L, n = lib(), len(Gs)
    norm = Gs[0].new_empty((), dtype=torch.float32)
    if work is None:                           # (float32 by norm's type: the shortest way)
        work = norm.new_empty(L.fira_grad_work_bytes(n) // 4)
    elif work.get_device() != index:
        raise ValueError(f"work is on {work.device}, the gradients on {norm.device}")
    scale = torch.empty_like(norm)
    status = L.fira_clip_grads(n, words, at, out_at, max_norm, norm.data_ptr(), scale.data_ptr(), work.data_ptr(),
                               work.nbytes, _raw_stream(index))
    if status:
        check(status)
    return norm, scale


def embedding(table: torch.Tensor, tokens: torch.Tensor, scale: float = 1.0,
              out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fira_embedding: scale * table[tokens] (shape of tokens + (hidden,)); zeros where a token is not in 0 .. vocab-1.
    out must not overlap the table.  Not recorded for autograd: the gradient is embedding_grad's."""
    if table.requires_grad and torch.is_grad_enabled():
        _not_recorded("embedding")
    code = _code(table, "table")
    bits = _TOKEN_BITS.get(tokens.dtype) or _refuse(f"tokens are int32 or int64, not {tokens.dtype}")
    if table.ndim != 2 or table.numel() == 0:
        raise ValueError(f"the table is a matrix, not {tuple(table.shape)}")
    vocab, hidden = table.shape
    ld = 0 if table.is_contiguous() else _pitch(table, "table")
    index = _device_of(table, tokens, out)
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return embedding(table, tokens, scale, out)
    if not tokens.is_contiguous():
        tokens = tokens.contiguous()
    if out is None:
        out, ld_out = table.new_empty((*tokens.shape, hidden)), 0
    elif out.shape != (*tokens.shape, hidden) or out.dtype != table.dtype:
        raise ValueError(f"out: {(*tokens.shape, hidden)} of {table.dtype} is needed, not {tuple(out.shape)} of {out.dtype}")
    else:
        ld_out = _pitch(out, "out")
    status = lib().fira_embedding(table.data_ptr(), vocab, hidden, ld, code, tokens.data_ptr(), bits, tokens.numel(), scale,
                                  out.data_ptr(), ld_out, _raw_stream(index))
    if status:
        check(status)
    return out


def embedding_grad(tokens: torch.Tensor, dY: torch.Tensor, vocab: int, scale: float = 1.0,
                   out: Optional[torch.Tensor] = None, accumulate: bool = False,
                   work: Optional[torch.Tensor] = None) -> torch.Tensor:
    """fira_embedding_grad: the gradient (vocab, hidden) of the table from that of scale * table[tokens].  out: float32 or
    bfloat16, by default a new tensor of dY's type, and no part of dY; accumulate: added to what is in it.  work: a byte tensor of at least
    lib().fira_embedding_grad_work_bytes() bytes; by default torch's allocator lends one for the call."""
    code = _code(dY, "dY")
    bits = _TOKEN_BITS.get(tokens.dtype) or _refuse(f"tokens are int32 or int64, not {tokens.dtype}")
    if dY.dim() == 0 or dY.shape[:-1] != tokens.shape or dY.shape[-1] == 0 or vocab <= 0:
        raise ValueError(f"dY {tuple(dY.shape)} for tokens {tuple(tokens.shape)} of a vocabulary of {vocab}")
    if accumulate and out is None:
        raise ValueError("accumulate: out is needed")
    _check_work(work)
    hidden = dY.shape[-1]
    index = _device_of(dY, tokens, out, work)
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return embedding_grad(tokens, dY, vocab, scale, out, accumulate, work)
    L, count = lib(), tokens.numel()
    tokens, dY = tokens.contiguous(), _rows_or_copy(dY)
    if out is None:
        out = dY.new_empty((vocab, hidden))
    elif out.shape != (vocab, hidden):
        raise ValueError(f"out: {(vocab, hidden)} is needed, not {tuple(out.shape)}")
    if work is None:
        work = torch.empty(L.fira_embedding_grad_work_bytes(count, vocab, hidden, code), dtype=torch.uint8, device=dY.device)
    status = L.fira_embedding_grad(tokens.data_ptr(), bits, count, dY.data_ptr(), _pitch(dY, "dY"), code, vocab, hidden, scale,
                                   out.data_ptr(), _pitch(out, "out"), _code(out, "out"), 1 if accumulate else 0,
                                   work.data_ptr(), work.nbytes, _raw_stream(index))
    if status:
        check(status)
    return out


def _check_params(hidden: int, gain: torch.Tensor, bias: Optional[torch.Tensor], what: str) -> int:
    code = _code(gain, what)
    if (gain.ndim != 1 or gain.numel() != hidden or not gain.is_contiguous() or
            (bias is not None and (bias.ndim != 1 or bias.numel() != hidden or not bias.is_contiguous() or bias.dtype != gain.dtype))):
        raise ValueError(f"{what}: contiguous vectors of {hidden} elements of one type are needed, not {tuple(gain.shape)} of {gain.dtype}"
                         + ("" if bias is None else f" and {tuple(bias.shape)} of {bias.dtype}"))
    return code


def _check_stats(rows: int, mean: Optional[torch.Tensor], rstd: torch.Tensor, rms: bool) -> None:
    if (mean is None) != rms:
        raise ValueError("mean is None in the form without mean, and needed in the other")
    for t in (mean, rstd):
        if t is not None and (t.numel() != rows or t.dtype != torch.float32 or not t.is_contiguous()):
            raise ValueError(f"mean and rstd: {rows} contiguous float32 numbers are needed")


def _like(x: torch.Tensor, ld: int, out: Optional[torch.Tensor]):
    """A tensor for a result like x (whose rows are ld apart, 0: contiguous), given or new, and its pitch."""
    if out is None:
        return (x.new_empty(x.shape) if ld else torch.empty_like(x)), 0
    if out.shape != x.shape or out.dtype != x.dtype:
        raise ValueError(f"out: {tuple(x.shape)} of {x.dtype} is needed, not {tuple(out.shape)} of {out.dtype}")
    return out, _pitch(out, "out")


def _address(t: torch.Tensor):
    """A tensor's address; of an empty one, which has none, one that is not NULL and that nothing is read from."""
    return t.data_ptr() or 256


def layer_norm(x: torch.Tensor, gain: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               rms: bool = False, out: Optional[torch.Tensor] = None):
    """fira_layer_norm over the last dimension: (y, mean, rstd); rms: the form without mean and bias (mean is None).  mean
    and rstd are float32 of x's other dimensions, for layer_norm_grad.  x's rows have one pitch, or more than two dimensions (a
    slice of a batch: copied where its rows have no one pitch).  out: may be x itself, where that has one pitch, and overlaps
    it in no other way.  Not recorded for autograd: the gradients are layer_norm_grad's."""
    if (x.requires_grad or gain.requires_grad or (bias is not None and bias.requires_grad)) and torch.is_grad_enabled():
        _not_recorded("layer_norm")
    code = _code(x, "x")
    shape = x.shape
    hidden = shape[-1] if shape else 0
    if hidden == 0:
        raise ValueError(f"x has no rows: {tuple(shape)}")
    params = _check_params(hidden, gain, bias, "gain and bias")
    x, ld = (x, 0) if x.is_contiguous() else _norm_rows(x)
    index = _device_of(x, gain, bias, out)
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return layer_norm(x, gain, bias, eps, rms, out)
    out, ld_out = _like(x, ld, out)
    rstd = x.new_empty(shape[:-1], dtype=torch.float32)
    mean = None if rms else torch.empty_like(rstd)
    status = lib().fira_layer_norm(x.data_ptr(), ld, code, x.numel() // hidden, hidden, gain.data_ptr(),
                                   None if bias is None else bias.data_ptr(), params, eps, out.data_ptr(), ld_out,
                                   None if rms else _address(mean), _address(rstd), _raw_stream(index))
    if status:
        check(status)
    return out, mean, rstd


def layer_norm_grad(dY: torch.Tensor, x: torch.Tensor, gain: torch.Tensor, mean: Optional[torch.Tensor], rstd: torch.Tensor,
                    rms: bool = False, out: Optional[torch.Tensor] = None, dgain: Optional[torch.Tensor] = None,
                    dbias: Optional[torch.Tensor] = None, accumulate: bool = False, work: Optional[torch.Tensor] = None):
    """fira_layer_norm_grad: (dX, dgain, dbias) from the gradient of y and from what layer_norm returned; dbias is None in
    the form without mean.  out (dX): may be dY or x itself.  dgain, dbias: float32 or bfloat16, by default new tensors of
    the gain's type; accumulate: added to what is in them.  work: a byte tensor of at least
    lib().fira_layer_norm_grad_work_bytes() bytes; by default torch's allocator lends one for the call."""
    code = _code(x, "x")
    shape = x.shape
    hidden = shape[-1] if shape else 0
    if hidden == 0 or dY.shape != shape or dY.dtype != x.dtype:
        raise ValueError(f"dY {tuple(dY.shape)} of {dY.dtype} for x {tuple(shape)} of {x.dtype}")
    rows = x.numel() // hidden
    params = _check_params(hidden, gain, None, "gain")
    _check_stats(rows, mean, rstd, rms)
    if rms and dbias is not None:
        raise ValueError("the form without mean has no bias")
    if accumulate and (dgain is None or (dbias is None and not rms)):
        raise ValueError("accumulate: dgain and dbias are needed")
    _check_work(work)
    x, ld = (x, 0) if x.is_contiguous() else _norm_rows(x)
    index = _device_of(x, dY, gain, mean, rstd, out, dgain, dbias, work)
    if index != torch.cuda.current_device():
        with torch.cuda.device(index):
            return layer_norm_grad(dY, x, gain, mean, rstd, rms, out, dgain, dbias, accumulate, work)
    L = lib()
    # a result over dY keeps its place, whatever becomes of dY's rows
    (out, ld_out), dY = _like(x, ld, out), _rows_or_copy(dY)
    given = dgain is not None or dbias is not None
    if dgain is None:
        dgain = torch.empty_like(gain)
    if dbias is None and not rms:
        dbias = torch.empty_like(dgain)
    grads = _check_params(hidden, dgain, dbias, "dgain and dbias") if given else params
    if work is None:                           # (float32 by rstd's type: the shortest way)
        work = rstd.new_empty(-(-L.fira_layer_norm_grad_work_bytes(rows, hidden, code) // 4))
    status = L.fira_layer_norm_grad(dY.data_ptr(), 0 if dY.is_contiguous() else _pitch(dY, "dY"), x.data_ptr(), ld, code, rows,
                                    hidden, gain.data_ptr(), params, None if rms else _address(mean), rstd.data_ptr(),
                                    out.data_ptr(), ld_out, dgain.data_ptr(), None if rms else dbias.data_ptr(), grads,
                                    1 if accumulate else 0, work.data_ptr(), work.nbytes, _raw_stream(index))
    if status:
        check(status)
    return out, dgain, dbias


class Fira:
    """A library context over a list of weight matrices on one CUDA device.

    shapes: (m, n) per matrix; r: rank (int or one per matrix); dtype: torch.float32
    or torch.bfloat16 (storage of W, G and the projection).  The state and scratch
    buffers are torch byte tensors owned by this object."""

    GUARD_BYTE = 0xA5

    def __init__(self, shapes: Sequence[Tuple[int, int]], r, dtype: torch.dtype, hp: Hparams,
                 device="cuda", lds: Optional[Sequence[int]] = None, guard_bytes: int = 0):
        self.L = lib()
        self.device = torch.device(device)
        if self.device.type != "cuda":
            raise ValueError("the Fira library runs on a CUDA device only")
        self.shapes = [tuple(s) for s in shapes]
        self.count = len(self.shapes)
        self.ranks = [r] * self.count if isinstance(r, int) else list(r)
        self.dtype = dtype
        self.hp = hp
        code = FIRA_BF16 if dtype == torch.bfloat16 else FIRA_F32
        self.descs = (MatrixDesc * self.count)()
        for i, (m, n) in enumerate(self.shapes):
            self.descs[i] = MatrixDesc(m, n, self.ranks[i], code, 0 if lds is None else lds[i])
        sb, wb = C.c_size_t(), C.c_size_t()
        check(self.L.fira_query_workspace(C.byref(hp), self.descs, self.count, C.byref(sb), C.byref(wb)))
        self.state_bytes, self.scratch_bytes = sb.value, wb.value
        self.ctx = None
        # guard_bytes > 0 (a multiple of 256): both buffers get that many bytes of a fixed pattern on
        # either side, which guards_intact() checks: nothing the library launches may write there
        assert guard_bytes % 256 == 0
        self.guard_bytes = guard_bytes
        with torch.cuda.device(self.device):
            self.state = torch.full((sb.value + 2 * guard_bytes,), self.GUARD_BYTE, dtype=torch.uint8,
                                    device=self.device)
            self.scratch = torch.full((wb.value + 2 * guard_bytes,), self.GUARD_BYTE, dtype=torch.uint8,
                                      device=self.device)
            self.stream = torch.cuda.current_stream(self.device)
            ctx = C.c_void_p()
            check(self.L.fira_init(C.byref(ctx), C.byref(hp), self.descs, self.count,
                                   self.state.data_ptr() + guard_bytes, sb.value,
                                   self.scratch.data_ptr() + guard_bytes, wb.value,
                                   self.stream.cuda_stream))
        self.ctx = ctx

    def guards_intact(self) -> bool:
        g = self.guard_bytes
        if g == 0:
            return True
        torch.cuda.synchronize(self.device)
        return all(bool((buf[:g] == self.GUARD_BYTE).all()) and bool((buf[-g:] == self.GUARD_BYTE).all())
                   for buf in (self.state, self.scratch))

    def close(self):
        if getattr(self, "ctx", None):
            self.L.fira_destroy(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def _dl(self, idx):
        m, n = self.shapes[idx]
        return min(m, n), max(m, n)

    def step(self, Ws: Sequence[torch.Tensor], Gs: Sequence[torch.Tensor], lr: Optional[float] = None):
        assert len(Ws) == self.count and len(Gs) == self.count
        check(self.L.fira_step(self.ctx, ptr_array(Ws), ptr_array(Gs), -1.0 if lr is None else lr))

    def staging_bytes(self) -> int:
        return self.L.fira_staging_bytes(self.ctx)

    def step_host(self, Ws_host, Gs_host, staging: torch.Tensor, lr: Optional[float] = None):
        check(self.L.fira_step_host(self.ctx, ptr_array(Ws_host), ptr_array(Gs_host),
                                    -1.0 if lr is None else lr, staging.data_ptr(), staging.numel()))

    def refresh_projection(self, Gs: Sequence[Optional[torch.Tensor]],
                           which: Optional[Sequence[int]] = None, seed: int = 0, iters: int = -1,
                           basis_f32: Optional[Sequence[Optional[torch.Tensor]]] = None):
        """basis_f32: optional list (one entry per matrix, None to skip) of (d, r) float32 device
        tensors that receive the basis before it is rounded to the storage type."""
        w, nw = (None, 0) if which is None else ((C.c_int32 * len(which))(*which), len(which))
        if basis_f32 is None:
            check(self.L.fira_refresh_projection(self.ctx, ptr_array(Gs), w, nw, seed, iters))
        else:
            for i, b in enumerate(basis_f32):
                assert b is None or (b.dtype == torch.float32 and b.is_contiguous() and
                                     b.shape == (self._dl(i)[0], self.ranks[i]))
            check(self.L.fira_refresh_projection_f32(self.ctx, ptr_array(Gs), w, nw, seed, iters,
                                                     ptr_array(basis_f32)))

    def refresh_side_work_bytes(self) -> int:
        return self.L.fira_refresh_side_work_bytes(self.ctx)

    def refresh_projection_side(self, Gs: Sequence[Optional[torch.Tensor]], P_out: Sequence[Optional[torch.Tensor]],
                                work: torch.Tensor, stream: "torch.cuda.Stream",
                                which: Optional[Sequence[int]] = None, seed: int = 0, iters: int = -1):
        """The refresh on a side stream with its own work buffer; the bases go to P_out (one (d, r)
        tensor of the storage type per selected matrix) and the context is left as it is."""
        w, nw = (None, 0) if which is None else ((C.c_int32 * len(which))(*which), len(which))
        for i, p in enumerate(P_out):
            assert p is None or (p.dtype == self.dtype and p.is_contiguous() and
                                 p.shape == (self._dl(i)[0], self.ranks[i]))
        check(self.L.fira_refresh_projection_side(self.ctx, ptr_array(Gs), w, nw, seed, iters, ptr_array(P_out),
                                                  work.data_ptr(), work.numel() * work.element_size(),
                                                  stream.cuda_stream))

    def set_projection(self, idx: int, P: torch.Tensor):
        d, _ = self._dl(idx)
        assert P.shape == (d, self.ranks[idx]) and P.dtype == self.dtype and P.is_cuda
        P = P.contiguous()   # the copy below is ordered on the same stream as torch's allocator
        check(self.L.fira_set_projection(self.ctx, idx, P.data_ptr()))

    def get_projection(self, idx: int) -> torch.Tensor:
        d, _ = self._dl(idx)
        P = torch.empty(d, self.ranks[idx], dtype=self.dtype, device=self.device)
        check(self.L.fira_get_projection(self.ctx, idx, P.data_ptr()))
        return P

    def get_state(self, idx: int):
        """M, V as (l, r) float tensors (row i = column i of G for m <= n, row i of G
        otherwise), the remembered norm (None if unset) and the step count."""
        _, l = self._dl(idx)
        M = torch.empty(l, self.ranks[idx], dtype=torch.float32, device=self.device)
        V = torch.empty_like(M)
        pn, t = C.c_float(), C.c_int64()
        check(self.L.fira_get_state(self.ctx, idx, M.data_ptr(), V.data_ptr(), C.byref(pn), C.byref(t)))
        return M, V, (None if pn.value < 0 else pn.value), t.value

    def set_state(self, idx: int, M: torch.Tensor, V: torch.Tensor, prev_norm: Optional[float], t: int):
        _, l = self._dl(idx)
        assert M.shape == (l, self.ranks[idx]) and M.dtype == torch.float32 and M.is_contiguous()
        assert V.shape == M.shape and V.dtype == torch.float32 and V.is_contiguous()
        check(self.L.fira_set_state(self.ctx, idx, M.data_ptr(), V.data_ptr(),
                                    -1.0 if prev_norm is None else prev_norm, t))

    def state_elements(self, idx: int) -> int:
        return self.L.fira_state_elements(self.ctx, idx)

    def diagnostics(self, idx: int) -> dict:
        d = Diag()
        check(self.L.fira_get_diagnostics(self.ctx, idx, C.byref(d)))
        return dict(norm_scaled=d.norm_scaled, lam=d.lambda_, norm_prev=d.norm_prev, k_min=d.k_min,
                    k_max=d.k_max, t=d.t, engine=d.engine)

    def poll(self) -> int:
        return self.L.fira_poll(self.ctx)

    def selftest_bounded_wait(self, rounds: int = 1000):
        check(self.L.fira_selftest_bounded_wait(self.ctx, rounds))

    def last_step_launches(self) -> int:
        return self.L.fira_last_step_launches(self.ctx)

    def enable_phase_timing(self, enable: bool = True):
        check(self.L.fira_enable_phase_timing(self.ctx, 1 if enable else 0))

    def phase_times(self):
        """[(kernel name, mean ms per step)] over the steps recorded since enabling."""
        n, steps = C.c_int32(), C.c_int32()
        ms = (C.c_float * 16)()
        check(self.L.fira_get_phase_times(self.ctx, C.byref(n), ms, C.byref(steps)))
        return [(self.L.fira_phase_name(self.ctx, i).decode(), ms[i]) for i in range(n.value)], steps.value
