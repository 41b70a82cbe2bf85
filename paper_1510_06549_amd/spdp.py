"""ctypes binding of libspdp.so (the C ABI declared in include/spdp.h).

Argument marshalling only: every step of the sweep runs in the library's HIP
kernels.  Host buffers are numpy arrays (``where = 0``); device buffers are
torch tensors on the GPU (``where = 1``).  The library is required: importing
this module raises if ``libspdp.so`` has not been built.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os

import numpy as np

_HERE = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_HERE, "libspdp.so")

SPDP_OK = 0
SPDP_E_ARG = -1
SPDP_E_NOMEM = -2
SPDP_E_HIP = -3
SPDP_E_RANGE = -4
SPDP_E_STATE = -5
SPDP_MAX_K = 1024
SPDP_MAX_SOURCES = 8
SPDP_NKERNELS = 4
SPDP_F64, SPDP_F32, SPDP_F16, SPDP_BF16 = 0, 1, 2, 3
SPDP_BLOCK8 = 128
SPDP_MAX_TAKE = 256
KERNEL_CLASSES = ("sample", "rebuild", "base", "totals")

# Every entry point of include/spdp.h, in declaration order.
EXPORTS = (
    "spdp_create", "spdp_sweep", "spdp_counts", "spdp_totals", "spdp_loglik", "spdp_destroy",
    "spdp_get_assignments", "spdp_set_assignments", "spdp_debug_conditionals", "spdp_stats",
    "spdp_kernel_timing", "spdp_kernel_times", "spdp_info", "spdp_last_error",
    "spdp_estimates", "spdp_heldout", "spdp_hellinger", "spdp_align_topics",
    "spdp_create_assoc", "spdp_get_slots", "spdp_set_assignments_assoc", "spdp_max_sources",
    "spdp_sweep_async", "spdp_read_probe", "spdp_check", "spdp_debug_poke",
    "spdp_hellinger_noalloc", "spdp_debug_weight_rows",
    "spdp_pack8", "spdp_product8", "spdp_adjust", "spdp_words_work", "spdp_top", "spdp_draw",
    "spdp_predict_work", "spdp_predict",
)


class SpdpError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"spdp error {code}: {msg}")
        self.code = code


class _Corpus(C.Structure):
    _fields_ = [
        ("n_tokens", C.c_int64),
        ("n_docs", C.c_int32),
        ("vocab", C.c_int32),
        ("words", C.c_void_p),
        ("doc_offsets", C.c_void_p),
        ("init_seed", C.c_uint64),
        ("hip_stream", C.c_void_p),
    ]


class _Groups(C.Structure):
    _fields_ = [("n_groups", C.c_int32), ("doc_group", C.c_void_p)]


class _Assoc(C.Structure):
    _fields_ = [
        ("max_sources", C.c_int32),
        ("row_off", C.c_void_p),
        ("src", C.c_void_p),
        ("p", C.c_void_p),
    ]


class _Rows8(C.Structure):
    _fields_ = [("rows", C.c_int64), ("cols", C.c_int32), ("q", C.c_void_p), ("e", C.c_void_p)]


class _Rules(C.Structure):
    _fields_ = [
        ("rows", C.c_int64),
        ("n_words", C.c_int32),
        ("n_bias", C.c_int32),
        ("n_masks", C.c_int32),
        ("n_listed", C.c_int64),
        ("doc_off", C.c_void_p),
        ("words", C.c_void_p),
        ("penalties", C.c_void_p),
        ("bias", C.c_void_p),
        ("bias_of", C.c_void_p),
        ("mask", C.c_void_p),
        ("mask_of", C.c_void_p),
    ]


class _Answer(C.Structure):
    _fields_ = [
        ("scores", C.c_void_p),
        ("ld", C.c_int64),
        ("type", C.c_int32),
        ("k", C.c_int32),
        ("top_word", C.c_void_p),
        ("top_value", C.c_void_p),
        ("draws", C.c_int32),
        ("temperature", C.c_double),
        ("u", C.c_void_p),
        ("seed", C.c_uint64),
        ("step", C.c_uint32),
        ("draw_word", C.c_void_p),
        ("draw_logp", C.c_void_p),
    ]


def load_library() -> C.CDLL:
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is missing: build it with `python -c 'import __graft_entry__ as g; "
            f"g.build()'` (hipcc, gfx950) -- there is no fallback implementation")
    L = C.CDLL(LIB_PATH)
    vp, i32, i64, u32, u64, dbl = C.c_void_p, C.c_int32, C.c_int64, C.c_uint32, C.c_uint64, C.c_double
    cint = C.c_int
    L.spdp_create.argtypes = [vp, vp, i32, dbl, dbl, dbl, dbl, C.POINTER(vp)]
    L.spdp_create.restype = cint
    L.spdp_sweep.argtypes = [vp, u32, u64]
    L.spdp_sweep.restype = cint
    L.spdp_counts.argtypes = [vp, i32, i32, vp, vp, cint]
    L.spdp_counts.restype = cint
    L.spdp_totals.argtypes = [vp, vp, vp, vp, vp, cint]
    L.spdp_totals.restype = cint
    L.spdp_loglik.argtypes = [vp, C.POINTER(dbl)]
    L.spdp_loglik.restype = cint
    L.spdp_destroy.argtypes = [vp]
    L.spdp_destroy.restype = None
    L.spdp_get_assignments.argtypes = [vp, vp, vp, cint]
    L.spdp_get_assignments.restype = cint
    L.spdp_set_assignments.argtypes = [vp, vp, vp, cint]
    L.spdp_set_assignments.restype = cint
    L.spdp_debug_conditionals.argtypes = [vp, u32, u64, i64, i64, vp, vp, vp, cint]
    L.spdp_debug_conditionals.restype = cint
    L.spdp_stats.argtypes = [vp, C.POINTER(i64), C.POINTER(i64)]
    L.spdp_stats.restype = cint
    L.spdp_kernel_timing.argtypes = [vp, cint]
    L.spdp_kernel_timing.restype = cint
    L.spdp_kernel_times.argtypes = [vp, vp, vp]
    L.spdp_kernel_times.restype = cint
    L.spdp_info.argtypes = [vp, vp]
    L.spdp_info.restype = cint
    L.spdp_read_probe.argtypes = [vp, i64, cint, i64, cint, vp, vp]
    L.spdp_read_probe.restype = cint
    L.spdp_last_error.argtypes = []
    L.spdp_last_error.restype = C.c_char_p
    L.spdp_estimates.argtypes = [vp, i32, i32, vp, vp, vp, cint]
    L.spdp_estimates.restype = cint
    L.spdp_heldout.argtypes = [vp, vp, vp, i32, u64, vp, vp, cint]
    L.spdp_heldout.restype = cint
    L.spdp_hellinger.argtypes = [vp, vp, i32, vp, i32, i32, vp, cint]
    L.spdp_hellinger.restype = cint
    L.spdp_align_topics.argtypes = [vp, i32, i32, vp, vp]
    L.spdp_align_topics.restype = cint
    L.spdp_create_assoc.argtypes = [vp, vp, vp, i32, dbl, dbl, dbl, dbl, C.POINTER(vp)]
    L.spdp_create_assoc.restype = cint
    L.spdp_get_slots.argtypes = [vp, vp, cint]
    L.spdp_get_slots.restype = cint
    L.spdp_set_assignments_assoc.argtypes = [vp, vp, vp, vp, cint]
    L.spdp_set_assignments_assoc.restype = cint
    L.spdp_max_sources.argtypes = [vp, C.POINTER(i32)]
    L.spdp_max_sources.restype = cint
    L.spdp_sweep_async.argtypes = [vp, u32, u64, i32, i32]
    L.spdp_sweep_async.restype = cint
    L.spdp_hellinger_noalloc.argtypes = [vp, vp, i32, vp, i32, i32, vp]
    L.spdp_hellinger_noalloc.restype = cint
    L.spdp_check.argtypes = [vp, C.POINTER(i64)]
    L.spdp_check.restype = cint
    L.spdp_debug_poke.argtypes = [vp, i32, i32, i32, i32, i32]
    L.spdp_debug_poke.restype = cint
    L.spdp_debug_weight_rows.argtypes = [vp, i64, i64, vp, vp]
    L.spdp_debug_weight_rows.restype = cint
    L.spdp_pack8.argtypes = [vp, vp, i32, i64, vp]
    L.spdp_pack8.restype = cint
    L.spdp_product8.argtypes = [vp, vp, vp, i32, vp, i32, i64]
    L.spdp_product8.restype = cint
    L.spdp_adjust.argtypes = [vp, vp, i64, vp, i64, i32, vp]
    L.spdp_adjust.restype = cint
    L.spdp_words_work.argtypes = [i64, i32, i32, C.POINTER(i64)]
    L.spdp_words_work.restype = cint
    L.spdp_top.argtypes = [vp, vp, i64, i32, i64, i32, vp, i32, vp, vp, vp, i64]
    L.spdp_top.restype = cint
    L.spdp_draw.argtypes = [vp, vp, i64, i32, i64, i32, vp, dbl, i32, vp, u64, u32, vp, vp, vp,
                            i64]
    L.spdp_draw.restype = cint
    L.spdp_predict_work.argtypes = [i64, i32, i32, i32, C.POINTER(i64)]
    L.spdp_predict_work.restype = cint
    L.spdp_predict.argtypes = [vp, vp, vp, vp, vp, vp, i64]
    L.spdp_predict.restype = cint
    return L


_lib = None


def lib() -> C.CDLL:
    global _lib
    if _lib is None:
        _lib = load_library()
    return _lib


def spdp_last_error() -> str:
    return lib().spdp_last_error().decode()


def _check(rc: int):
    if rc != SPDP_OK:
        raise SpdpError(rc, spdp_last_error())


def _buf(x):
    """(pointer, where) of a numpy array (host) or a torch CUDA tensor (device)."""
    if x is None:
        return None, 0
    if isinstance(x, np.ndarray):
        assert x.flags.c_contiguous
        return x.ctypes.data, 0
    # torch tensor
    assert x.is_contiguous()
    return x.data_ptr(), (1 if x.is_cuda else 0)


def _where(*bufs) -> int:
    ws = {w for p, w in (_buf(b) for b in bufs) if p is not None}
    if len(ws) > 1:
        raise ValueError("mix of host and device buffers in one call")
    return ws.pop() if ws else 0


# ---------------------------------------------------------------------------
# Entry points (same names as the C ABI)
# ---------------------------------------------------------------------------
def spdp_create(words, doc_offsets, doc_group, n_groups, vocab, K, alpha, a, b, gamma,
                init_seed=0, hip_stream=None):
    words = np.ascontiguousarray(words, dtype=np.int32)
    doc_offsets = np.ascontiguousarray(doc_offsets, dtype=np.int64)
    doc_group = np.ascontiguousarray(doc_group, dtype=np.int32)
    corpus = _Corpus(int(words.shape[0]), int(doc_group.shape[0]), int(vocab), words.ctypes.data,
                     doc_offsets.ctypes.data, int(init_seed) & (2**64 - 1),
                     None if hip_stream is None else int(hip_stream))
    groups = _Groups(int(n_groups), doc_group.ctypes.data)
    h = C.c_void_p()
    _check(lib().spdp_create(C.byref(corpus), C.byref(groups), int(K), float(alpha), float(a),
                             float(b), float(gamma), C.byref(h)))
    return h


def spdp_create_assoc(words, doc_offsets, doc_group, n_groups, vocab, K, alpha, a, b, gamma,
                      row_off, src, p, max_sources=None, init_seed=0, hip_stream=None):
    """State of the model with word associations: row q = g V + w of P^g lists
    its sources src[row_off[q]:row_off[q+1]] with probabilities p (see
    include/spdp.h)."""
    words = np.ascontiguousarray(words, dtype=np.int32)
    doc_offsets = np.ascontiguousarray(doc_offsets, dtype=np.int64)
    doc_group = np.ascontiguousarray(doc_group, dtype=np.int32)
    row_off = np.ascontiguousarray(row_off, dtype=np.int64)
    src = np.ascontiguousarray(src, dtype=np.int32)
    p = np.ascontiguousarray(p, dtype=np.float64)
    if max_sources is None:
        max_sources = int(np.diff(row_off).max()) if row_off.size > 1 else 0
    corpus = _Corpus(int(words.shape[0]), int(doc_group.shape[0]), int(vocab), words.ctypes.data,
                     doc_offsets.ctypes.data, int(init_seed) & (2**64 - 1),
                     None if hip_stream is None else int(hip_stream))
    groups = _Groups(int(n_groups), doc_group.ctypes.data)
    assoc = _Assoc(int(max_sources), row_off.ctypes.data, src.ctypes.data, p.ctypes.data)
    h = C.c_void_p()
    _check(lib().spdp_create_assoc(C.byref(corpus), C.byref(groups), C.byref(assoc), int(K),
                                   float(alpha), float(a), float(b), float(gamma), C.byref(h)))
    return h


def spdp_get_slots(h, slot_out):
    _check(lib().spdp_get_slots(h, _buf(slot_out)[0], _where(slot_out)))


def spdp_set_assignments_assoc(h, z, r, slot):
    if isinstance(z, np.ndarray):
        z = np.ascontiguousarray(z, dtype=np.int32)
        r = np.ascontiguousarray(r, dtype=np.uint8)
        slot = np.ascontiguousarray(slot, dtype=np.uint8)
    where = _where(z, r, slot)
    _check(lib().spdp_set_assignments_assoc(h, _buf(z)[0], _buf(r)[0], _buf(slot)[0], where))


def spdp_max_sources(h) -> int:
    S = C.c_int32()
    _check(lib().spdp_max_sources(h, C.byref(S)))
    return int(S.value)


def spdp_sweep(h, sweep: int, seed: int):
    _check(lib().spdp_sweep(h, int(sweep) & 0xFFFFFFFF, int(seed) & (2**64 - 1)))


def spdp_sweep_async(h, sweep: int, seed: int, waves: int = 0, live_totals: bool = False):
    _check(lib().spdp_sweep_async(h, int(sweep) & 0xFFFFFFFF, int(seed) & (2**64 - 1),
                                  int(waves), 1 if live_totals else 0))


def spdp_counts(h, g_begin, g_end, n_out=None, t_out=None):
    where = _where(n_out, t_out)
    _check(lib().spdp_counts(h, int(g_begin), int(g_end), _buf(n_out)[0], _buf(t_out)[0], where))


def spdp_totals(h, N_gk=None, T_gk=None, B_wk=None, B_k=None):
    where = _where(N_gk, T_gk, B_wk, B_k)
    _check(lib().spdp_totals(h, _buf(N_gk)[0], _buf(T_gk)[0], _buf(B_wk)[0], _buf(B_k)[0], where))


def spdp_loglik(h) -> float:
    out = C.c_double()
    _check(lib().spdp_loglik(h, C.byref(out)))
    return float(out.value)


def spdp_destroy(h):
    if h:
        lib().spdp_destroy(h)


def spdp_get_assignments(h, z_out=None, r_out=None):
    where = _where(z_out, r_out)
    _check(lib().spdp_get_assignments(h, _buf(z_out)[0], _buf(r_out)[0], where))


def spdp_set_assignments(h, z, r):
    if isinstance(z, np.ndarray):
        z = np.ascontiguousarray(z, dtype=np.int32)
        r = np.ascontiguousarray(r, dtype=np.uint8)
    where = _where(z, r)
    _check(lib().spdp_set_assignments(h, _buf(z)[0], _buf(r)[0], where))


def spdp_debug_conditionals(h, sweep, seed, tok_begin, tok_end, w_out=None, u_out=None,
                            zr_out=None):
    where = _where(w_out, u_out, zr_out)
    _check(lib().spdp_debug_conditionals(h, int(sweep) & 0xFFFFFFFF, int(seed) & (2**64 - 1),
                                         int(tok_begin), int(tok_end), _buf(w_out)[0],
                                         _buf(u_out)[0], _buf(zr_out)[0], where))


def spdp_stats(h):
    c, r = C.c_int64(), C.c_int64()
    _check(lib().spdp_stats(h, C.byref(c), C.byref(r)))
    return int(c.value), int(r.value)


def spdp_kernel_timing(h, enable: bool):
    _check(lib().spdp_kernel_timing(h, 1 if enable else 0))


def spdp_kernel_times(h):
    ms = np.zeros(SPDP_NKERNELS, dtype=np.float64)
    n = np.zeros(SPDP_NKERNELS, dtype=np.int64)
    _check(lib().spdp_kernel_times(h, ms.ctypes.data, n.ctypes.data))
    return {k: (float(ms[i]), int(n[i])) for i, k in enumerate(KERNEL_CLASSES)}


def spdp_read_probe(buf_ptr: int, nbytes: int, row_bytes: int = 0, rows: int = 0,
                    waves: int = 4096, stream=None) -> float:
    """Milliseconds to read a device buffer: whole (row_bytes = 0) or rows of
    row_bytes at pseudo-random positions, one row at a time per wavefront."""
    ms = C.c_double(0.0)
    _check(lib().spdp_read_probe(C.c_void_p(buf_ptr), int(nbytes), int(row_bytes), int(rows),
                                 int(waves), None if stream is None else C.c_void_p(int(stream)),
                                 C.byref(ms)))
    return ms.value


def spdp_hellinger_noalloc(h, p, q, out):
    """Device tensors p [V, kp], q [V, kq], out [kp, kq] (float64); enqueues
    only, on the state's stream."""
    V, kp = p.shape
    kq = q.shape[1]
    assert q.shape[0] == V and tuple(out.shape) == (kp, kq)
    for x in (p, q, out):
        assert x.is_cuda and x.dtype.is_floating_point and x.element_size() == 8
        assert x.is_contiguous()
    _check(lib().spdp_hellinger_noalloc(h, p.data_ptr(), kp, q.data_ptr(), kq, V,
                                        out.data_ptr()))


def spdp_check(h):
    """Number of failing cells, tokens and totals; raises SpdpError
    (SPDP_E_STATE) if there is any."""
    bad = C.c_int64(0)
    rc = lib().spdp_check(h, C.byref(bad))
    if rc == SPDP_E_STATE:
        raise SpdpError(rc, spdp_last_error())
    _check(rc)
    return int(bad.value)


def spdp_debug_poke(h, g, w, k, dn, dt):
    _check(lib().spdp_debug_poke(h, int(g), int(w), int(k), int(dn), int(dt)))


def spdp_debug_weight_rows(h, row_begin, row_end, pw, rho):
    _check(lib().spdp_debug_weight_rows(h, int(row_begin), int(row_end), pw.ctypes.data,
                                        rho.ctypes.data))


def spdp_info(h) -> dict:
    out = np.zeros(8, dtype=np.int64)
    _check(lib().spdp_info(h, out.ctypes.data))
    keys = ("N", "D", "V", "G", "K", "Kp", "ncap", "device_bytes")
    return {k: int(v) for k, v in zip(keys, out)}


def spdp_estimates(h, g_begin, g_end, theta=None, phi0=None, phi=None):
    where = _where(theta, phi0, phi)
    _check(lib().spdp_estimates(h, int(g_begin), int(g_end), _buf(theta)[0], _buf(phi0)[0],
                                _buf(phi)[0], where))


def spdp_heldout(h, words, doc_offsets, doc_group, n_groups, vocab, n_sweeps, seed, z_out=None):
    """(perplexity, sum of log p) of held-out documents; see include/spdp.h."""
    words = np.ascontiguousarray(words, dtype=np.int32)
    doc_offsets = np.ascontiguousarray(doc_offsets, dtype=np.int64)
    doc_group = np.ascontiguousarray(doc_group, dtype=np.int32)
    corpus = _Corpus(int(words.shape[0]), int(doc_group.shape[0]), int(vocab), words.ctypes.data,
                     doc_offsets.ctypes.data, 0, None)
    groups = _Groups(int(n_groups), doc_group.ctypes.data)
    out = np.zeros(2, dtype=np.float64)
    where = _where(z_out)
    _check(lib().spdp_heldout(h, C.byref(corpus), C.byref(groups), int(n_sweeps),
                              int(seed) & (2**64 - 1), out.ctypes.data, _buf(z_out)[0], where))
    return float(out[0]), float(out[1])


def spdp_hellinger(h, p, q, out):
    """Hellinger distances out [kp, kq] between the columns of p [V, kp] (None:
    the state's phi0) and q [V, kq]; see include/spdp.h."""
    where = _where(p, q, out)
    V, kq = q.shape
    kp = out.shape[0]
    if out.shape != (kp, kq) or (p is not None and p.shape != (V, kp)):
        raise ValueError("p [V, kp], q [V, kq] and out [kp, kq] do not agree")
    _check(lib().spdp_hellinger(h, _buf(p)[0], int(kp), _buf(q)[0], int(kq), int(V),
                                _buf(out)[0], where))
    return out


def spdp_align_topics(dist):
    """(match [kp] int32, total) of the least-total matching of rows to columns."""
    dist = np.ascontiguousarray(dist, dtype=np.float64)
    kp, kq = dist.shape
    match = np.zeros(kp, dtype=np.int32)
    total = C.c_double()
    _check(lib().spdp_align_topics(dist.ctypes.data, int(kp), int(kq), match.ctypes.data,
                                   C.byref(total)))
    return match, float(total.value)


# ---------------------------------------------------------------------------
# Words of documents (device tensors; the calls only enqueue on the state's
# stream, so tensors have to be made and freed in that stream's order)
# ---------------------------------------------------------------------------
_TYPE_OF = {"torch.float64": SPDP_F64, "torch.float32": SPDP_F32, "torch.float16": SPDP_F16,
            "torch.bfloat16": SPDP_BF16}
_TYPES = {}  # torch dtype -> SPDP_F64 ...


def _type(x):
    t = _TYPES.get(x.dtype)
    if t is None:
        t = _TYPE_OF.get(str(x.dtype))
        if t is None:
            raise ValueError(f"no such type here: {x.dtype}")
        _TYPES[x.dtype] = t
    return t


def _matrix(x, what):
    """(pointer, rows, columns, elements from one row to the next) of a device matrix whose
    rows are contiguous."""
    if x.dim() != 2 or not x.is_cuda:
        raise ValueError(f"{what}: a device matrix")
    rows, cols = x.shape
    ld, step = x.stride()
    if step != 1 and cols > 1:
        raise ValueError(f"{what}: elements of a row must be contiguous")
    if rows <= 1 and ld < cols:
        ld = cols  # (a single row's stride says nothing)
    return x.data_ptr(), rows, cols, ld


def _vector(x, shape, dtype, what):
    """Pointer of a contiguous device tensor of this shape and type (None: null)."""
    if x is None:
        return None
    if tuple(x.shape) != shape or str(x.dtype) != dtype or not x.is_cuda or \
            not x.is_contiguous():
        raise ValueError(f"{what}: a contiguous device tensor {shape} of {dtype}")
    return x.data_ptr()


class _Device:
    """Device memory from the library's own HIP runtime, with what these calls ask of a tensor:
    for calls on host arrays, in programs that may have no tensor library (or have one that
    would bring a second runtime, were it loaded now)."""

    _SIZES = {"float64": 8, "int64": 8, "float32": 4, "int32": 4, "float8_e4m3fn": 1, "uint8": 1}
    is_cuda = True

    def __init__(self, shape, dtype, host=None):
        self.shape, self.dtype, self.ptr = tuple(int(n) for n in shape), "torch." + dtype, None
        self.size = self._SIZES[dtype]
        if self.numel():
            p = C.c_void_p()
            self._hip("hipMalloc", C.byref(p), C.c_size_t(self.numel() * self.size))
            self.ptr = p
            if host is not None:
                host = np.ascontiguousarray(host, dtype)
                assert host.size == self.numel()
                self._hip("hipMemcpy", p, C.c_void_p(host.ctypes.data), C.c_size_t(host.nbytes),
                          C.c_int(1))

    @staticmethod
    def _hip(name, *args):
        rc = getattr(lib(), name)(*args)
        if rc:
            lib().hipGetLastError()  # (else it is the error of the next launch)
            raise SpdpError(SPDP_E_HIP, f"{name}: HIP error {rc}")

    @classmethod
    def current(cls):
        d = C.c_int()
        cls._hip("hipGetDevice", C.byref(d))
        return d.value

    @classmethod
    @contextlib.contextmanager
    def on(cls, device):
        """Memory and waits are of this device inside; the caller's is current again after."""
        before = cls.current()
        cls._hip("hipSetDevice", C.c_int(device))
        try:
            yield
        finally:
            cls._hip("hipSetDevice", C.c_int(before))

    @classmethod
    def wait(cls):
        cls._hip("hipDeviceSynchronize")

    def host(self):
        out = np.empty(self.shape, self.dtype[6:])
        if self.ptr:
            self._hip("hipMemcpy", C.c_void_p(out.ctypes.data), self.ptr, C.c_size_t(out.nbytes),
                      C.c_int(2))
        return out

    def __del__(self):
        try:
            if self.ptr:
                lib().hipFree(self.ptr)
                self.ptr = None
        except Exception:
            pass

    def data_ptr(self):
        return self.ptr.value if self.ptr else 0

    def numel(self):
        n = 1
        for m in self.shape:
            n *= m
        return n

    def element_size(self):
        return self.size

    def dim(self):
        return len(self.shape)

    def stride(self):
        return tuple(int(np.prod(self.shape[i + 1:], dtype=np.int64))
                     for i in range(len(self.shape)))

    def is_contiguous(self):
        return True


class Rows8:
    """Rows in 8 bits: q [rows, blocks * 128] (torch.float8_e4m3fn) and e [rows, blocks]
    (uint8, exponent + 127 of each block's scale); see include/spdp.h."""

    def __init__(self, q, e, cols):
        nb = -(-cols // SPDP_BLOCK8)
        rows = q.shape[0]
        self.q, self.e, self.rows, self.cols = q, e, rows, cols
        self.c = _Rows8(rows, cols,
                        _vector(q, (rows, nb * SPDP_BLOCK8), "torch.float8_e4m3fn", "q"),
                        _vector(e, (rows, nb), "torch.uint8", "e"))
        self.ref = C.addressof(self.c)

    @classmethod
    def empty(cls, rows, cols, device="cuda"):
        import torch

        nb = -(-cols // SPDP_BLOCK8)
        return cls(torch.empty((rows, nb * SPDP_BLOCK8), dtype=torch.float8_e4m3fn,
                               device=device),
                   torch.empty((rows, nb), dtype=torch.uint8, device=device), cols)


class Rules:
    """Rules on the scores of `rows` documents over n_words words (device tensors, all of
    them optional; kept by the object):

    doc_off [rows + 1] int64, words [n] int32, penalties [rows, 3] float32 (repeat, presence,
    frequency); bias [tables, n_words] float32, bias_of [rows] int32; mask [tables,
    ceil(n_words / 32)] int32 bits, mask_of [rows] int32.  See include/spdp.h."""

    def __init__(self, rows, n_words, doc_off=None, words=None, penalties=None, bias=None,
                 bias_of=None, mask=None, mask_of=None):
        i32, f32 = "torch.int32", "torch.float32"
        tables = [0 if t is None else t.shape[0] for t in (bias, mask)]
        if any(t is not None and n == 0 for t, n in zip((bias, mask), tables)):
            raise ValueError("a table without rows")
        listed = 0 if words is None else words.shape[0]
        self.kept = (doc_off, words, penalties, bias, bias_of, mask, mask_of)
        self.rows, self.n_words = rows, n_words
        self.c = _Rules(
            rows, n_words, tables[0], tables[1], listed,
            _vector(doc_off, (rows + 1,), "torch.int64", "doc_off"),
            _vector(words, (listed,), i32, "words"),
            _vector(penalties, (rows, 3), f32, "penalties"),
            _vector(bias, (tables[0], n_words), f32, "bias"),
            _vector(bias_of, (rows,), i32, "bias_of"),
            _vector(mask, (tables[1], -(-n_words // 32)), i32, "mask"),
            _vector(mask_of, (rows,), i32, "mask_of"))
        self.ref = C.addressof(self.c)


def spdp_pack8(h, x, out: Rows8):
    """Round rows x [rows, cols] (float64 or float32) to out; returns out."""
    p, rows, cols, ld = _matrix(x, "x")
    if (rows, cols) != (out.rows, out.cols):
        raise ValueError(f"x {rows} x {cols}, out {out.rows} x {out.cols}")
    _check(lib().spdp_pack8(h, p, _type(x), ld, out.ref))
    return out


def spdp_product8(h, a: Rows8, b: Rows8, out, log: bool = False):
    """out [a.rows, b.rows] = a b^T, or its logarithm; returns out."""
    p, rows, cols, ld = _matrix(out, "out")
    if (rows, cols) != (a.rows, b.rows):
        raise ValueError(f"out {rows} x {cols} for {a.rows} x {b.rows} products")
    _check(lib().spdp_product8(h, a.ref, b.ref, 1 if log else 0, p, _type(out), ld))
    return out


def spdp_adjust(h, x, rules: Rules, out):
    """Scores x under the rules into out (x itself, or another matrix); returns out."""
    p, rows, cols, ld = _matrix(x, "x")
    po, rows_o, cols_o, ldo = _matrix(out, "out")
    if x.dtype != out.dtype or (rows, cols) != (rows_o, cols_o) or \
            (rows, cols) != (rules.rows, rules.n_words):
        raise ValueError("x, out and the rules do not agree")
    _check(lib().spdp_adjust(h, p, ld, po, ldo, _type(x), rules.ref))
    return out


def spdp_words_work(rows: int, n_words: int, take: int = 0) -> int:
    """Bytes of workspace of spdp_top (take = k) and spdp_draw."""
    n = C.c_int64()
    _check(lib().spdp_words_work(int(rows), int(n_words), int(take), C.byref(n)))
    return n.value


def _work(work):
    if work is None:
        return None, 0
    if not work.is_cuda or not work.is_contiguous():
        raise ValueError("work: a contiguous device tensor")
    return work.data_ptr(), work.numel() * work.element_size()


def spdp_top(h, x, word, value, work, rules: Rules = None):
    """The best words of every row of x: word [rows, k] int32, value [rows, k] float32;
    returns both."""
    p, rows, cols, ld = _matrix(x, "x")
    k = word.shape[1]
    _check(lib().spdp_top(h, p, ld, _type(x), rows, cols, rules and rules.ref, k,
                          _vector(word, (rows, k), "torch.int32", "word"),
                          _vector(value, (rows, k), "torch.float32", "value"), *_work(work)))
    return word, value


def spdp_draw(h, x, word, logp, work, u=None, rules: Rules = None, temperature: float = 1.0,
              seed: int = 0, step: int = 0):
    """Words drawn from every row of x: word [rows, draws] int32, logp [rows, draws] float32,
    by the uniforms u [rows, draws] float64 or the seed's; returns both."""
    p, rows, cols, ld = _matrix(x, "x")
    n = word.shape[1]
    _check(lib().spdp_draw(h, p, ld, _type(x), rows, cols, rules and rules.ref,
                           temperature, n, _vector(u, (rows, n), "torch.float64", "u"),
                           int(seed) & (2**64 - 1), int(step) & 0xFFFFFFFF,
                           _vector(word, (rows, n), "torch.int32", "word"),
                           _vector(logp, (rows, n), "torch.float32", "logp"), *_work(work)))
    return word, logp


def spdp_predict_work(docs: int, n_words: int, dtype, k: int = 0) -> int:
    """Bytes of workspace for a good number of documents at a time."""
    n = C.c_int64()
    _check(lib().spdp_predict_work(int(docs), int(n_words), _TYPE_OF[str(dtype)], int(k),
                                   C.byref(n)))
    return n.value


def spdp_predict(h, docs: Rows8, words: Rows8, work, rules: Rules = None, scores=None,
                 dtype=None, top=None, drawn=None, temperature: float = 1.0, u=None,
                 seed: int = 0, step: int = 0):
    """Words for documents: any of scores [docs, words] (else they are held in `dtype` in the
    workspace), top = (word, value) [docs, k] and drawn = (word, logp) [docs, draws]."""
    D, V = docs.rows, words.rows
    a = _Answer(type=SPDP_F32, temperature=temperature, seed=int(seed) & (2**64 - 1),
                step=int(step) & 0xFFFFFFFF)
    if scores is not None:
        a.scores, rows, cols, a.ld = _matrix(scores, "scores")
        a.type = _type(scores)
        if (rows, cols) != (D, V):
            raise ValueError(f"scores {rows} x {cols} for {D} documents, {V} words")
    elif dtype is not None:
        a.type = _TYPE_OF[str(dtype)]
    if top is not None:
        a.k = top[0].shape[1]
        a.top_word = _vector(top[0], (D, a.k), "torch.int32", "word")
        a.top_value = _vector(top[1], (D, a.k), "torch.float32", "value")
    if drawn is not None:
        a.draws = drawn[0].shape[1]
        a.draw_word = _vector(drawn[0], (D, a.draws), "torch.int32", "word")
        a.draw_logp = _vector(drawn[1], (D, a.draws), "torch.float32", "logp")
        a.u = _vector(u, (D, a.draws), "torch.float64", "u")
    _check(lib().spdp_predict(h, docs.ref, words.ref, rules and rules.ref, C.byref(a),
                              *_work(work)))


# ---------------------------------------------------------------------------
# Convenience wrapper (host numpy in and out)
# ---------------------------------------------------------------------------
class Sampler:
    """Owns one library state; thin host-side helpers around the entry points."""

    def __init__(self, words, doc_offsets, doc_group, n_groups, vocab, K, alpha, a, b, gamma,
                 init_seed=0, hip_stream=None, assoc=None):
        """assoc: None (P = I) or (row_off, src, p) of the word associations."""
        if assoc is None:
            self.h = spdp_create(words, doc_offsets, doc_group, n_groups, vocab, K, alpha, a, b,
                                 gamma, init_seed, hip_stream)
        else:
            row_off, src, p = assoc
            self.h = spdp_create_assoc(words, doc_offsets, doc_group, n_groups, vocab, K, alpha,
                                       a, b, gamma, row_off, src, p, init_seed=init_seed,
                                       hip_stream=hip_stream)
        self.device = _Device.current()  # (the state's: it is made on the current one)
        self.info = spdp_info(self.h)
        self.N, self.G, self.V, self.K = (self.info["N"], self.info["G"], self.info["V"],
                                          self.info["K"])
        self.S = spdp_max_sources(self.h)

    def close(self):
        if self.h:
            spdp_destroy(self.h)
            self.h = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def sweep(self, sweep, seed):
        spdp_sweep(self.h, sweep, seed)

    def sweep_async(self, sweep, seed, waves=0, live_totals=False):
        """The thesis's asynchronous sweep (an ablation; see include/spdp.h)."""
        spdp_sweep_async(self.h, sweep, seed, waves, live_totals)

    def assignments(self):
        z = np.empty(self.N, dtype=np.int32)
        r = np.empty(self.N, dtype=np.uint8)
        spdp_get_assignments(self.h, z, r)
        return z, r

    def set_assignments(self, z, r, slot=None):
        if slot is None:
            spdp_set_assignments(self.h, z, r)
        else:
            spdp_set_assignments_assoc(self.h, z, r, slot)

    def slots(self):
        """Source slot of each token's table (word associations; 0 for r = 0)."""
        s = np.empty(self.N, dtype=np.uint8)
        spdp_get_slots(self.h, s)
        return s

    def counts(self, g_begin=0, g_end=None):
        """n, t as [g][k][w] int32 arrays."""
        g_end = self.G if g_end is None else g_end
        n = np.empty((g_end - g_begin, self.K, self.V), dtype=np.int32)
        t = np.empty_like(n)
        spdp_counts(self.h, g_begin, g_end, n, t)
        return n, t

    def totals(self):
        N = np.empty((self.G, self.K), dtype=np.int32)
        T = np.empty_like(N)
        B = np.empty((self.V, self.K), dtype=np.int32)
        Bk = np.empty(self.K, dtype=np.int32)
        spdp_totals(self.h, N, T, B, Bk)
        return N, T, B, Bk

    def loglik(self):
        return spdp_loglik(self.h)

    def check(self):
        return spdp_check(self.h)

    def poke(self, g, w, k, dn, dt):
        spdp_debug_poke(self.h, g, w, k, dn, dt)

    def weight_rows(self):
        """(pw, rho) [G V, K] of the weight rows, fp32."""
        pw, rho = (np.empty((self.G * self.V, self.K), dtype=np.float32) for _ in range(2))
        spdp_debug_weight_rows(self.h, 0, self.G * self.V, pw, rho)
        return pw, rho

    def conditionals(self, sweep, seed, tok_begin, tok_end):
        T = tok_end - tok_begin
        per_topic = 2 if self.S == 0 else self.S + 1
        w = np.zeros((T, per_topic * self.K), dtype=np.float32)
        u = np.zeros(T, dtype=np.float32)
        zr = np.zeros(T, dtype=np.int32)
        spdp_debug_conditionals(self.h, sweep, seed, tok_begin, tok_end, w, u, zr)
        return w, u, zr

    def sampled(self, sweep, seed, tok_begin=0, tok_end=None):
        """Packed 2z + r of the sampling step only (before update and repair)."""
        tok_end = self.N if tok_end is None else tok_end
        zr = np.zeros(tok_end - tok_begin, dtype=np.int32)
        spdp_debug_conditionals(self.h, sweep, seed, tok_begin, tok_end, None, None, zr)
        return zr

    def stats(self):
        return spdp_stats(self.h)

    def estimates(self, g_begin=0, g_end=None):
        """(theta [D, K], phi0 [V, K], phi [g, V, K]) in fp64."""
        g_end = self.G if g_end is None else g_end
        theta = np.empty((self.info["D"], self.K), dtype=np.float64)
        phi0 = np.empty((self.V, self.K), dtype=np.float64)
        phi = np.empty((g_end - g_begin, self.V, self.K), dtype=np.float64)
        spdp_estimates(self.h, g_begin, g_end, theta, phi0, phi)
        return theta, phi0, phi

    def hellinger(self, q, p=None):
        """Hellinger distances [kp, kq] between the columns of p [V, kp] (default:
        this state's phi0) and q [V, kq], fp64 host arrays."""
        q = np.ascontiguousarray(q, dtype=np.float64)
        if p is not None:
            p = np.ascontiguousarray(p, dtype=np.float64)
        kp = self.K if p is None else p.shape[1]
        out = np.empty((kp, q.shape[1]), dtype=np.float64)
        return spdp_hellinger(self.h, p, q, out)

    def heldout(self, words, doc_offsets, doc_group, n_sweeps, seed):
        """(perplexity, sum of log p, fold-in topics) of held-out documents."""
        z = np.empty(len(words), dtype=np.int32)
        ppl, ll = spdp_heldout(self.h, words, doc_offsets, doc_group, self.G, self.V, n_sweeps,
                               seed, z)
        return ppl, ll, z

    def predict(self, theta, phi, top=0, draws=0, seed=0, step=0, temperature=1.0,
                doc_words=None, penalties=(1.0, 0.0, 0.0), bias=None, allowed=None):
        """Words for documents from host estimates theta [D, K] and phi [V, K] (a group's, or
        phi0): (top words [D, top], their scores, drawn words [D, draws], their log
        probabilities).  Both are rounded to 8 bits with a scale for each 128 topics (spdp_pack8:
        a value is off by 2^-4 of itself at most, or 2^-10 of its scale), so that words whose scores
        are closer than that may change places; both are packed anew by every call, and a program
        that asks often keeps Rows8 of its own and calls spdp_predict.  doc_words: a list of word ids for every document, which `penalties`
        = (repeat, presence, frequency) make less likely; bias [V]: added to the scores;
        allowed [V]: truth values, the words to choose from."""
        theta, phi = np.asarray(theta, np.float64), np.asarray(phi, np.float64)
        if theta.ndim != 2 or phi.ndim != 2 or theta.shape[1] != phi.shape[1]:
            raise ValueError("theta [D, K] and phi [V, K]")
        if top < 0 or draws < 0:
            raise ValueError("top and draws: how many words of each document")
        D, V = len(theta), len(phi)
        with _Device.on(self.device):
            return self._predict(theta, phi, D, V, top, draws, seed, step, temperature, doc_words,
                                 penalties, bias, allowed)

    def _predict(self, theta, phi, D, V, top, draws, seed, step, temperature, doc_words, penalties,
                 bias, allowed):
        def put(x, dtype):
            x = np.asarray(x, dtype)
            return _Device(x.shape, dtype, x)

        rules = None
        if doc_words is not None or bias is not None or allowed is not None:
            r = {}
            if doc_words is not None:
                if len(doc_words) != D:
                    raise ValueError("doc_words: one list per document")
                r["doc_off"] = put(np.cumsum([0] + [len(w) for w in doc_words]), "int64")
                w = np.concatenate([np.asarray(w, np.int64) for w in doc_words] +
                                   [np.empty(0, np.int64)])
                # (words that are none of the vocabulary's are ignored, those too that 32 bits
                # would turn into some)
                r["words"] = put(np.where((w >= 0) & (w < V), w, -1), "int32")
                r["penalties"] = put(np.broadcast_to(np.asarray(penalties, np.float32), (D, 3)),
                                     "float32")
            if bias is not None:
                r["bias"] = put(np.reshape(bias, (1, V)), "float32")
            if allowed is not None:
                bits = np.zeros(-(-V // 32) * 32, np.uint8)
                bits[:V] = np.reshape(allowed, V).astype(bool)
                r["mask"] = put(np.packbits(bits, bitorder="little").view("<i4")[None], "int32")
            rules = Rules(D, V, **r)
        packed = []
        for x in (theta, phi):
            nb = -(-x.shape[1] // SPDP_BLOCK8)
            packed.append(Rows8(_Device((len(x), nb * SPDP_BLOCK8), "float8_e4m3fn"),
                                _Device((len(x), nb), "uint8"), x.shape[1]))
        given = [put(x, "float64") for x in (theta, phi)]
        outs = [(_Device((D, n), "int32"), _Device((D, n), "float32")) for n in (top, draws)]
        work = _Device((spdp_predict_work(D, V, "torch.float32", top),), "uint8")
        try:
            for x, to in zip(given, packed):
                spdp_pack8(self.h, x, to)
            spdp_predict(self.h, packed[0], packed[1], work, rules=rules,
                         top=outs[0] if top else None, drawn=outs[1] if draws else None,
                         temperature=temperature, seed=seed, step=step)
        finally:
            _Device.wait()  # (before the memory is given back)
        return tuple(x.host() for pair in outs for x in pair)
