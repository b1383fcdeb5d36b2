"""ctypes binding of libretopk.so (include/retopk.h).

Argument marshalling only: every step of the decode path runs in the gfx950
kernels of the library.  Tensor arguments are torch tensors on the GPU (any
object with ``data_ptr()``) or raw device addresses; streams are torch streams,
raw ``hipStream_t`` values, or None for torch's current stream.
"""
from __future__ import annotations

import ctypes as C
import os

from . import build as _build

RETOPK_F32, RETOPK_BF16 = 0, 1
RETOPK_PAGES_F32, RETOPK_PAGES_BF16, RETOPK_PAGES_Q4 = 0, 1, 2
ROPE_SCALINGS = {"none": 0, "linear": 1, "ntk": 2, "bands": 3, "ramp": 4}
Q4_GROUP = 64               # elements of a 4-bit row that share a scale and a middle
REUSE, FALLBACK, REFRESH, COLD = 0, 1, 2, 3
PATH_NAMES = {REUSE: "reuse", FALLBACK: "fallback", REFRESH: "refresh", COLD: "cold"}
STATUS = {0: "ok", -1: "invalid argument", -2: "unsupported shape", -3: "device out of memory",
          -4: "HIP runtime error", -5: "call out of order or handle broken",
          -6: "workspace larger than the fixed scratch"}

# Every symbol include/retopk.h declares.
EXPORTS = ("retopk_create", "retopk_destroy", "retopk_prefill_init", "retopk_decode_step",
           "exact_topk_attention", "exact_topk_attention_noalloc", "full_attention",
           "retopk_stream_read", "retopk_stats",
           "retopk_get_state",
           "retopk_set_state",
           "retopk_profile", "retopk_profile_read", "retopk_kernel_name",
           "retopk_status_string",
           "retopk_rope_init", "rotary_embed", "paged_append", "paged_gather",
           "paged_attention_workspace", "paged_attention")


class RetopkError(RuntimeError):
    def __init__(self, fn: str, code: int, detail: str = ""):
        super().__init__(f"{fn}: {STATUS.get(code, code)} ({code})" + (f": {detail}" if detail else ""))
        self.code = code


def _check_tensor(fn: str, name: str, x, numel: int, itemsize: int):
    """A torch tensor argument must be on the GPU, contiguous, of the element size
    the call expects and at least as large as the layout the call indexes; the
    call is refused (RETOPK_ERR_ARG) before reaching the library otherwise.  Raw
    addresses (ints) and None pass unchecked."""
    if x is None or isinstance(x, int) or not hasattr(x, "is_cuda"):
        return
    if not x.is_cuda:
        raise RetopkError(fn, -1, f"{name} is not a GPU tensor")
    if not x.is_contiguous():
        raise RetopkError(fn, -1, f"{name} is not contiguous")
    if x.element_size() != itemsize:
        raise RetopkError(fn, -1, f"{name} has {x.element_size()}-byte elements, {itemsize} expected")
    if x.numel() < numel:
        raise RetopkError(fn, -1, f"{name} has {x.numel()} elements, {numel} expected")


class retopk_config(C.Structure):
    _fields_ = [("batch", C.c_int32), ("n_q_heads", C.c_int32), ("n_kv_heads", C.c_int32),
                ("head_dim", C.c_int32), ("max_len", C.c_int64), ("k", C.c_int32),
                ("cache_cap", C.c_int32), ("r", C.c_int32), ("window", C.c_int32),
                ("tau", C.c_float), ("refresh", C.c_int32), ("dtype", C.c_int32),
                ("retrieval", C.c_int32)]


class retopk_stats_t(C.Structure):
    _fields_ = [(n, C.c_uint64) for n in ("steps", "head_steps", "reuse", "fallback", "refresh",
                                          "cold", "kv_group_scans", "cand_sum", "cand_max")]


class retopk_debug(C.Structure):
    _fields_ = [("path", C.c_void_p), ("rho_max", C.c_void_p), ("retrieved", C.c_void_p),
                ("n_cand", C.c_void_p), ("cand", C.c_void_p)]


class retopk_pages(C.Structure):
    _fields_ = [("format", C.c_int32), ("n_kv_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32), ("n_pages", C.c_int32), ("n_seqs", C.c_int32),
                ("table_width", C.c_int32), ("k", C.c_void_p), ("v", C.c_void_p),
                ("k_par", C.c_void_p), ("v_par", C.c_void_p), ("table", C.c_void_p)]


class retopk_rows(C.Structure):
    _fields_ = [("p", C.c_void_p), ("token_stride", C.c_int64), ("head_stride", C.c_int64)]


class retopk_rope(C.Structure):
    _fields_ = [("rot_dim", C.c_int32), ("interleaved", C.c_int32), ("factor", C.c_double),
                ("freq", C.c_double * 64)]


class retopk_rope_scaling(C.Structure):
    _fields_ = [("kind", C.c_int32), ("factor", C.c_double), ("original_len", C.c_double),
                ("low", C.c_double), ("high", C.c_double)]


_LIB = None


def load(path: str | None = None):
    """Load the built library.  Raises if it has not been built: there is no
    fallback implementation.  The environment variable RETOPK_LIB names another
    build of it (the host-sanitizer test)."""
    global _LIB
    if _LIB is not None and path is None:
        return _LIB
    default = path is None
    path = path or os.environ.get("RETOPK_LIB") or _build.LIB
    if not os.path.exists(path):
        raise RuntimeError(f"{path} is missing: build it with __graft_entry__.build() "
                           "(hipcc --offload-arch=gfx950)")
    lib = C.CDLL(path)
    P, I32, I64 = C.c_void_p, C.c_int32, C.c_int64
    sig = {
        "retopk_create": ([C.POINTER(retopk_config), C.POINTER(P)], C.c_int),
        "retopk_destroy": ([P], C.c_int),
        "retopk_prefill_init": ([P, P, I32, P, P, I64, P], C.c_int),
        "retopk_decode_step": ([P, P, P, P, I64, P, P, C.POINTER(retopk_debug), P], C.c_int),
        "exact_topk_attention": ([P, P, P, P, I64, P, P, P], C.c_int),
        "exact_topk_attention_noalloc": ([C.POINTER(retopk_config), P, P, P, I64, P, P, P],
                                         C.c_int),
        "full_attention": ([P, P, P, P, I64, P, P], C.c_int),
        "retopk_stream_read": ([P, I64, P, P], C.c_int),
        "retopk_stats": ([P, C.POINTER(retopk_stats_t)], C.c_int),
        "retopk_get_state": ([P, P, P, P, C.POINTER(I64), C.POINTER(I64)], C.c_int),
        "retopk_set_state": ([P, P, P, P, I64, I64], C.c_int),
        "retopk_profile": ([P, I32], C.c_int),
        "retopk_profile_read": ([P, I32, P, P], C.c_int),
        "retopk_kernel_name": ([I32], C.c_char_p),
        "retopk_status_string": ([C.c_int], C.c_char_p),
        "retopk_rope_init": ([C.POINTER(retopk_rope), I32, I32, C.c_double,
                              C.POINTER(retopk_rope_scaling)], C.c_int),
        "rotary_embed": ([C.POINTER(retopk_rope), I32, I32, I32, I64, P, retopk_rows,
                          retopk_rows, I32, P], C.c_int),
        "paged_append": ([C.POINTER(retopk_pages), C.POINTER(retopk_rope), I32, I64, P, P,
                          retopk_rows, retopk_rows, I32, retopk_rows, retopk_rows, P], C.c_int),
        "paged_gather": ([C.POINTER(retopk_pages), I32, I64, P, P, retopk_rows, retopk_rows, P],
                         C.c_int),
        "paged_attention_workspace": ([C.POINTER(retopk_pages), I64, I32, I64, I64], I64),
        "paged_attention": ([C.POINTER(retopk_pages), I32, I64, I32, P, P, retopk_rows, I64, I64,
                             P, P, P, I64, P], C.c_int),
    }
    for name, (args, res) in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = res
    if default:
        _LIB = lib
    return lib


def _addr(x):
    if x is None:
        return None
    if isinstance(x, int):
        return x
    return x.data_ptr()


_CURRENT_STREAM = None


def _current_stream():
    """torch's current stream of the current device, by the call torch's own generated code
    makes where there is one: torch.cuda.current_stream() builds an object, 3 us a call."""
    global _CURRENT_STREAM
    import torch
    if _CURRENT_STREAM is None:
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        _CURRENT_STREAM = (lambda d: torch.cuda.current_stream(d).cuda_stream) if raw is None else raw
    return _CURRENT_STREAM(torch.cuda.current_device())


def _stream(s):
    if s is None:
        return _current_stream()
    if isinstance(s, int):
        return s
    return s.cuda_stream


def _check(fn: str, rc: int):
    if rc != 0:
        raise RetopkError(fn, rc)


def make_config(batch, n_q_heads, n_kv_heads, head_dim, max_len, k, cache_cap, r, window, tau,
                refresh, dtype, retrieval=0) -> retopk_config:
    dt = {"f32": RETOPK_F32, "bf16": RETOPK_BF16}.get(dtype, dtype)
    return retopk_config(batch, n_q_heads, n_kv_heads, head_dim, max_len, k, cache_cap, r,
                         window, tau, refresh, dt, retrieval)


# ---------------------------------------------------------------------------
# Functions with the C names
# ---------------------------------------------------------------------------

def retopk_create(cfg: retopk_config) -> int:
    h = C.c_void_p()
    _check("retopk_create", load().retopk_create(C.byref(cfg), C.byref(h)))
    return h.value


def retopk_destroy(h: int) -> None:
    _check("retopk_destroy", load().retopk_destroy(h))


def retopk_prefill_init(h, q_tail, n, k, v, prefill_len, stream=None) -> None:
    _check("retopk_prefill_init", load().retopk_prefill_init(
        h, _addr(q_tail), n, _addr(k), _addr(v), prefill_len, _stream(stream)))


def retopk_decode_step(h, q, k, v, length, out, sel=None, dbg: dict | None = None,
                       stream=None) -> None:
    d = None
    if dbg is not None:
        d = retopk_debug(_addr(dbg.get("path")), _addr(dbg.get("rho_max")),
                         _addr(dbg.get("retrieved")), _addr(dbg.get("n_cand")),
                         _addr(dbg.get("cand")))
    _check("retopk_decode_step", load().retopk_decode_step(
        h, _addr(q), _addr(k), _addr(v), length, _addr(out), _addr(sel),
        C.byref(d) if d is not None else None, _stream(stream)))


def exact_topk_attention(h, q, k, v, length, out, sel=None, stream=None) -> None:
    _check("exact_topk_attention", load().exact_topk_attention(
        h, _addr(q), _addr(k), _addr(v), length, _addr(out), _addr(sel), _stream(stream)))


def exact_topk_attention_noalloc(cfg: retopk_config, q, k, v, length, out, sel=None,
                                 stream=None) -> None:
    """exact_topk_attention without a handle, on the library's fixed scratch."""
    _check_io("exact_topk_attention_noalloc", _cfg_dict(cfg), q=q, k=k, v=v, out=out, sel=sel)
    _check("exact_topk_attention_noalloc", load().exact_topk_attention_noalloc(
        C.byref(cfg), _addr(q), _addr(k), _addr(v), length, _addr(out), _addr(sel),
        _stream(stream)))


def full_attention(h, q, k, v, length, out, stream=None) -> None:
    _check("full_attention", load().full_attention(
        h, _addr(q), _addr(k), _addr(v), length, _addr(out), _stream(stream)))


def retopk_stream_read(src, nbytes: int, sink, stream=None) -> None:
    """Read nbytes at src once (the streaming-read ceiling; a measurement aid)."""
    _check("retopk_stream_read", load().retopk_stream_read(_addr(src), nbytes, _addr(sink),
                                                            _stream(stream)))


def retopk_stats(h) -> dict:
    st = retopk_stats_t()
    _check("retopk_stats", load().retopk_stats(h, C.byref(st)))
    return {n: int(getattr(st, n)) for n, _ in retopk_stats_t._fields_}


def retopk_get_state(h, qbar=None, supp=None, cnt=None):
    """Fills numpy arrays (host) and returns (n_inserted, t_dec)."""
    n_ins, t_dec = C.c_int64(), C.c_int64()
    P = lambda a: None if a is None else a.ctypes.data  # noqa: E731
    _check("retopk_get_state", load().retopk_get_state(h, P(qbar), P(supp), P(cnt),
                                                       C.byref(n_ins), C.byref(t_dec)))
    return n_ins.value, t_dec.value


def retopk_set_state(h, qbar, supp, cnt, n_inserted: int, t_dec: int) -> None:
    import numpy as np
    qbar = np.ascontiguousarray(qbar, np.float32)
    supp = np.ascontiguousarray(supp, np.int32)
    cnt = np.ascontiguousarray(cnt, np.int32)
    _check("retopk_set_state", load().retopk_set_state(
        h, qbar.ctypes.data, supp.ctypes.data, cnt.ctypes.data, n_inserted, t_dec))


def retopk_profile(h, enable: bool) -> None:
    _check("retopk_profile", load().retopk_profile(h, 1 if enable else 0))


def retopk_kernel_name(kid: int) -> str | None:
    r = load().retopk_kernel_name(kid)
    return r.decode() if r is not None else None


def retopk_profile_read(h) -> dict:
    """{kernel name: (launches, total ms)} over the recording window."""
    n = 0
    while retopk_kernel_name(n) is not None:
        n += 1
    launches = (C.c_uint64 * n)()
    ms = (C.c_double * n)()
    _check("retopk_profile_read", load().retopk_profile_read(h, n, launches, ms))
    return {retopk_kernel_name(i): (int(launches[i]), float(ms[i])) for i in range(n)}


def retopk_status_string(code: int) -> str:
    return load().retopk_status_string(code).decode()


def _cfg_dict(cfg: retopk_config) -> dict:
    return {n: getattr(cfg, n) for n, _ in retopk_config._fields_}


def _check_io(fn: str, c: dict, q=None, k=None, v=None, out=None, sel=None, q_tail=None,
              n_tail: int = 0):
    """Layout checks of the tensor arguments against the configuration c (see
    include/retopk.h: q [B, Hq, d], k and v [B, Hkv, max_len, d], out [B, Hq, d]
    float32, sel [B, Hq, K] int32, q_tail [B, Hq, n, d])."""
    dt = c["dtype"]
    es = 2 if dt in ("bf16", RETOPK_BF16) else 4
    bhq = c["batch"] * c["n_q_heads"]
    d = c["head_dim"]
    _check_tensor(fn, "q", q, bhq * d, es)
    kv = c["batch"] * c["n_kv_heads"] * c["max_len"] * d
    _check_tensor(fn, "k", k, kv, es)
    _check_tensor(fn, "v", v, kv, es)
    _check_tensor(fn, "out", out, bhq * d, 4)
    _check_tensor(fn, "sel", sel, bhq * c["k"], 4)
    _check_tensor(fn, "q_tail", q_tail, bhq * n_tail * d, es)


# ---------------------------------------------------------------------------
# Rotary positions and the paged cache
# ---------------------------------------------------------------------------

def make_rope(rot_dim, theta=10000.0, interleaved=False, scaling="none", factor=1.0,
              original_len=0, low=0.0, high=0.0) -> retopk_rope:
    """Frequencies of a rotation (retopk_rope_init).  scaling: "none", "linear", "ntk",
    "bands" or "ramp"; the last two take original_len and the turns low < high."""
    if scaling not in ROPE_SCALINGS:
        raise RetopkError("retopk_rope_init", -1, f"scaling {scaling!r}")
    r = retopk_rope()
    sc = retopk_rope_scaling(ROPE_SCALINGS[scaling], factor, original_len, low, high)
    _check("retopk_rope_init", load().retopk_rope_init(C.byref(r), rot_dim, int(interleaved),
                                                       theta, C.byref(sc)))
    return r


_NO_ROWS = retopk_rows(None, 0, 0)
_DTYPE_OF = {}              # torch dtype: retopk_dtype


def _dtype_of(fn: str, name: str, x) -> int:
    """float32 or bfloat16 (or the bits of one, int16)."""
    if not _DTYPE_OF:
        import torch
        _DTYPE_OF.update({torch.float32: RETOPK_F32, torch.bfloat16: RETOPK_BF16,
                          torch.int16: RETOPK_BF16})
    got = _DTYPE_OF.get(x.dtype)
    if got is None:
        raise RetopkError(fn, -1, f"{name} is {x.dtype}: float32 or bfloat16 expected")
    return got


def _rows(fn: str, name: str, x, shape, dtype, dev: int) -> retopk_rows:
    """A [tokens, heads, d] tensor of this shape and type on this device, whose last dimension
    is dense."""
    if x.shape != shape or x.dtype != dtype or x.get_device() != dev:
        raise RetopkError(fn, -1, f"{name} is {x.dtype} {list(x.shape)} on {x.device}: {dtype} "
                                  f"{list(shape)} on GPU {dev} expected")
    ts, hs, es = x.stride()
    if es != 1:
        raise RetopkError(fn, -1, f"{name}: its last dimension is not dense")
    # the stride of a dimension of one element is never used
    return retopk_rows(x.data_ptr(), 0 if shape[0] == 1 else ts, 0 if shape[1] == 1 else hs)


def _first(fn: str, name: str, x, heads=None, d=None):
    """Checks the tensor that the others of a call are to be like; its shape, type and device."""
    if x.dim() != 3 or not x.is_cuda:
        raise RetopkError(fn, -1, f"{name}: a [tokens, heads, d] GPU tensor expected")
    shape = x.shape
    if heads is not None and shape[1] != heads or d is not None and shape[2] != d:
        raise RetopkError(fn, -1, f"{name} has shape {list(shape)}, [tokens, {heads or 'heads'}, {d}] "
                                  "expected")
    return shape, x.dtype, x.get_device()


def _index(fn: str, name: str, x, n: int, dev: int):
    """A dense int32 GPU tensor of n elements."""
    if x.numel() != n or x.element_size() != 4 or x.is_floating_point() or \
            x.get_device() != dev or not x.is_contiguous():
        raise RetopkError(fn, -1, f"{name}: {n} dense int32 elements on GPU {dev} expected")
    return x.data_ptr()


def _launch(name: str, dev: int, stream, *args):
    """Calls a library function with the device of its tensors current."""
    import torch
    fn = getattr(_LIB or load(), name)
    if dev == torch.cuda.current_device():
        rc = fn(*args, _stream(stream))
    else:
        with torch.cuda.device(dev):
            rc = fn(*args, _stream(stream))
    if rc:
        _check(name, rc)


def rotary_embed(rope: retopk_rope, x, pos, out, inverse=False, stream=None) -> None:
    """out = x [tokens, heads, d] rotated to the int32 positions pos [tokens]; with inverse,
    the gradient of x for the gradient x of out.  out may be x."""
    fn = "rotary_embed"
    shape, dt, dev = _first(fn, "x", x)
    _launch(fn, dev, stream, C.byref(rope), _dtype_of(fn, "x", x), shape[2], shape[1], shape[0],
            _index(fn, "pos", pos, shape[0], dev), _rows(fn, "x", x, shape, dt, dev),
            _rows(fn, "out", out, shape, dt, dev), 1 if inverse else 0)


class PagedCache:
    """Pages of keys and values and the table that maps positions to them
    (include/retopk.h, retopk_pages).  k, v: [n_pages, Hkv, page_size, d] float32 or bfloat16,
    or [n_pages, Hkv, page_size, d / 2] uint8 with k_par, v_par [n_pages, Hkv, page_size, d / 64]
    int32 for 4-bit rows; table: [n_seqs, table_width] int32.  The tensors stay the
    caller's: pages are added by writing their ids into the table."""

    def __init__(self, k, v, table, k_par=None, v_par=None):
        fn = "retopk_pages"
        if k.dim() != 4 or table.dim() != 2:
            raise RetopkError(fn, -1, "k: 4 dimensions, table: 2 expected")
        self.q4 = k.element_size() == 1
        n, hkv, page, d = k.shape
        if self.q4:
            import torch
            if k.dtype != torch.uint8:
                raise RetopkError(fn, -1, f"k is {k.dtype}: float32, bfloat16 or uint8 expected")
            d *= 2
            if k_par is None or v_par is None:
                raise RetopkError(fn, -1, "4-bit pages need k_par and v_par")
        per = {"k": (k, k.shape), "v": (v, k.shape), "table": (table, table.shape)}
        if self.q4:
            per["k_par"] = (k_par, (n, hkv, page, d // Q4_GROUP))
            per["v_par"] = (v_par, (n, hkv, page, d // Q4_GROUP))
        for name, (x, shape) in per.items():
            if not x.is_cuda or x.device != k.device or not x.is_contiguous():
                raise RetopkError(fn, -1, f"{name}: a dense tensor on {k.device} expected")
            if tuple(x.shape) != tuple(shape):
                raise RetopkError(fn, -1, f"{name} has shape {tuple(x.shape)}, {tuple(shape)} expected")
        if v.dtype != k.dtype:
            raise RetopkError(fn, -1, f"v is {v.dtype}, {k.dtype} expected")
        for name in ("table", "k_par", "v_par"):
            if name in per and (per[name][0].element_size() != 4 or
                                per[name][0].is_floating_point()):
                raise RetopkError(fn, -1, f"{name}: int32 expected")
        fmt = RETOPK_PAGES_Q4 if self.q4 else {RETOPK_F32: RETOPK_PAGES_F32,
                                               RETOPK_BF16: RETOPK_PAGES_BF16}[_dtype_of(fn, "k", k)]
        self.tensors = (k, v, table, k_par, v_par)
        self.device, self.n_kv_heads, self.head_dim = k.device, hkv, d
        self.dev = k.get_device()
        self.c = retopk_pages(fmt, hkv, d, page, n, table.shape[0], table.shape[1], k.data_ptr(),
                              v.data_ptr(), k_par.data_ptr() if self.q4 else None,
                              v_par.data_ptr() if self.q4 else None, table.data_ptr())

    @staticmethod
    def allocate(fmt, n_pages, n_kv_heads, page_size, head_dim, n_seqs, table_width,
                 device="cuda") -> "PagedCache":
        """A cache of empty pages; fmt: "f32", "bf16" or "q4".  No sequence has a page yet
        (the table holds -1)."""
        import torch
        if fmt not in ("f32", "bf16", "q4"):
            raise RetopkError("retopk_pages", -1, f"format {fmt!r}: f32, bf16 or q4 expected")
        shape, dev = (n_pages, n_kv_heads, page_size), dict(device=device)
        table = torch.full((n_seqs, table_width), -1, dtype=torch.int32, **dev)
        if fmt == "q4":
            k, v = (torch.zeros((*shape, head_dim // 2), dtype=torch.uint8, **dev)
                    for _ in range(2))
            kp, vp = (torch.zeros((*shape, head_dim // Q4_GROUP), dtype=torch.int32, **dev)
                      for _ in range(2))
            return PagedCache(k, v, table, kp, vp)
        dt = {"f32": torch.float32, "bf16": torch.bfloat16}[fmt]
        k, v = (torch.zeros((*shape, head_dim), dtype=dt, **dev) for _ in range(2))
        return PagedCache(k, v, table)

    @property
    def table(self):
        return self.tensors[2]

    @property
    def k(self):
        return self.tensors[0]

    def workspace(self, n_tokens, n_q_heads, max_len, window=0):
        """A workspace for paged_attention calls of these sizes, None where it needs none."""
        import torch
        n = paged_attention_workspace(self, n_tokens, n_q_heads, max_len, window)
        return torch.empty(n, dtype=torch.uint8, device=self.device) if n else None


def paged_append(cache: PagedCache, seq, pos, k, v, rope: retopk_rope | None = None, q=None,
                 q_out=None, stream=None) -> None:
    """Rows t of k and v [tokens, Hkv, d] to positions pos[t] of sequences seq[t], k rotated on
    the way when rope is given; q [tokens, Hq, d], rotated, to q_out."""
    fn = "paged_append"
    shape, dt, dev = _first(fn, "k", k, cache.n_kv_heads, cache.head_dim)
    t = shape[0]
    if dev != cache.dev:
        raise RetopkError(fn, -1, f"k is on {k.device}, the cache on {cache.device}")
    hq, rq, ro = 0, _NO_ROWS, _NO_ROWS
    if q is not None:
        if q_out is None:
            raise RetopkError(fn, -1, "q without q_out")
        q_shape = _first(fn, "q", q, None, cache.head_dim)[0]
        if q_shape[0] != t:
            raise RetopkError(fn, -1, f"q has {q_shape[0]} tokens, k {t}")
        hq = q_shape[1]
        rq = _rows(fn, "q", q, q_shape, dt, dev)
        ro = _rows(fn, "q_out", q_out, q_shape, dt, dev)
    _launch(fn, dev, stream, C.byref(cache.c), C.byref(rope) if rope is not None else None,
            _dtype_of(fn, "k", k), t, _index(fn, "seq", seq, t, dev),
            _index(fn, "pos", pos, t, dev), _rows(fn, "k", k, shape, dt, dev),
            _rows(fn, "v", v, shape, dt, dev), hq, rq, ro)


def paged_gather(cache: PagedCache, seq, pos, k=None, v=None, stream=None) -> None:
    """Positions pos[t] of sequences seq[t] read into rows t of k and v [tokens, Hkv, d]."""
    fn = "paged_gather"
    first = k if k is not None else v
    if first is None:
        return
    shape, dt, dev = _first(fn, "k" if k is not None else "v", first, cache.n_kv_heads,
                            cache.head_dim)
    t = shape[0]
    if dev != cache.dev:
        raise RetopkError(fn, -1, f"k or v is on {first.device}, the cache on {cache.device}")
    rk = _rows(fn, "k", k, shape, dt, dev) if k is not None else _NO_ROWS
    rv = _rows(fn, "v", v, shape, dt, dev) if v is not None else _NO_ROWS
    _launch(fn, dev, stream, C.byref(cache.c), _dtype_of(fn, "k", first), t,
            _index(fn, "seq", seq, t, dev), _index(fn, "pos", pos, t, dev), rk, rv)


def paged_attention_workspace(cache: PagedCache, n_tokens, n_q_heads, max_len, window=0) -> int:
    """Bytes of workspace that paged_attention needs."""
    n = load().paged_attention_workspace(C.byref(cache.c), n_tokens, n_q_heads, max_len, window)
    if n < 0:
        _check("paged_attention_workspace", n)
    return n


def _workspace_on(cache: PagedCache, t, hq, max_len, window, stream):
    """A workspace of the call's own, whose memory the allocator ties to its stream."""
    import torch
    if stream is None:
        return cache.workspace(t, hq, max_len, window)
    if isinstance(stream, int):
        stream = torch.cuda.ExternalStream(stream, device=cache.device)
    with torch.cuda.stream(stream):
        return cache.workspace(t, hq, max_len, window)


def paged_attention(cache: PagedCache, seq, pos, q, out, max_len, window=0, lse=None,
                    workspace=None, stream=None) -> None:
    """Row t of q [tokens, Hq, d] attends the positions up to pos[t] of sequence seq[t]; out
    [tokens, Hq, d] and lse [tokens, Hq] are float32.  workspace: PagedCache.workspace of the
    same sizes (None: a new one; hold one for graphs, and one a graph)."""
    fn = "paged_attention"
    shape, dt, dev = _first(fn, "q", q, None, cache.head_dim)
    t, hq = shape[0], shape[1]
    if dev != cache.dev:
        raise RetopkError(fn, -1, f"q is on {q.device}, the cache on {cache.device}")
    for name, x, n in (("out", out, t * hq * cache.head_dim), ("lse", lse, t * hq)):
        if x is not None and (x.element_size() != 4 or not x.is_floating_point() or
                              x.numel() != n or x.get_device() != dev or not x.is_contiguous()):
            raise RetopkError(fn, -1, f"{name}: {n} dense float32 elements on {q.device} expected")
    if workspace is None:
        workspace = _workspace_on(cache, t, hq, max_len, window, stream)
    elif workspace.get_device() != dev or not workspace.is_contiguous():
        raise RetopkError(fn, -1, f"workspace: a dense tensor on {q.device} expected")
    _launch(fn, dev, stream, C.byref(cache.c), _dtype_of(fn, "q", q), t, hq,
            _index(fn, "seq", seq, t, dev), _index(fn, "pos", pos, t, dev),
            _rows(fn, "q", q, shape, dt, dev), max_len, window, out.data_ptr(),
            None if lse is None else lse.data_ptr(),
            None if workspace is None else workspace.data_ptr(),
            0 if workspace is None else workspace.numel() * workspace.element_size())


# ---------------------------------------------------------------------------
# Convenience wrapper
# ---------------------------------------------------------------------------

class Handle:
    """Owns one retopk handle.  Construct from keyword config fields."""

    def __init__(self, **cfg):
        self.cfg = dict(cfg)
        self.h = retopk_create(make_config(**cfg))

    def close(self):
        if self.h:
            retopk_destroy(self.h)
            self.h = None

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def prefill_init(self, q_tail, n, k, v, prefill_len, stream=None):
        _check_io("retopk_prefill_init", self.cfg, k=k, v=v, q_tail=q_tail, n_tail=n)
        retopk_prefill_init(self.h, q_tail, n, k, v, prefill_len, stream)

    def decode_step(self, q, k, v, length, out, sel=None, dbg=None, stream=None):
        _check_io("retopk_decode_step", self.cfg, q=q, k=k, v=v, out=out, sel=sel)
        retopk_decode_step(self.h, q, k, v, length, out, sel, dbg, stream)

    def exact(self, q, k, v, length, out, sel=None, stream=None):
        _check_io("exact_topk_attention", self.cfg, q=q, k=k, v=v, out=out, sel=sel)
        exact_topk_attention(self.h, q, k, v, length, out, sel, stream)

    def full(self, q, k, v, length, out, stream=None):
        _check_io("full_attention", self.cfg, q=q, k=k, v=v, out=out)
        full_attention(self.h, q, k, v, length, out, stream)

    def stats(self):
        return retopk_stats(self.h)

    def get_state(self):
        import numpy as np
        c = self.cfg
        bh = c["batch"] * c["n_q_heads"]
        qbar = np.zeros((bh, c["cache_cap"], c["head_dim"]), np.float32)
        supp = np.zeros((bh, c["cache_cap"], c["k"]), np.int32)
        cnt = np.zeros((bh, c["cache_cap"]), np.int32)
        n_ins, t_dec = retopk_get_state(self.h, qbar, supp, cnt)
        return dict(qbar=qbar, supp=supp, cnt=cnt, n_inserted=n_ins, t_dec=t_dec)

    def set_state(self, qbar, supp, cnt, n_inserted, t_dec):
        import numpy as np
        c = self.cfg
        bh = c["batch"] * c["n_q_heads"]
        want = {"qbar": (bh, c["cache_cap"], c["head_dim"]), "supp": (bh, c["cache_cap"], c["k"]),
                "cnt": (bh, c["cache_cap"])}
        for name, arr in (("qbar", qbar), ("supp", supp), ("cnt", cnt)):
            if tuple(np.shape(arr)) != want[name]:
                raise RetopkError("retopk_set_state", -1,
                                  f"{name} has shape {tuple(np.shape(arr))}, {want[name]} expected")
        retopk_set_state(self.h, qbar, supp, cnt, n_inserted, t_dec)

    def profile(self, enable=True):
        retopk_profile(self.h, enable)

    def profile_read(self):
        return retopk_profile_read(self.h)
