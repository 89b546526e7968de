"""Python binding of libjb, the sm_103a seeded-perturbation library.

Argument marshalling only: every element-wise step runs in the CUDA kernels
behind the C ABI of ``include/jb.h``; PyTorch supplies device memory and
streams. The functions keep the C names:

* ``jb_perturb``        PerturbParameters(theta, eps, s) (Algorithm 1, subroutine)
* ``jb_apply_updates``  the fused K-pair step update (Section 2; Algorithm 1)
* ``jb_apply_updates_from``  the same update read from the weight backup, with the
  restore of Algorithm 1 fused in
* ``jb_replay_updates``  several steps' updates in one pass (a late joiner's
  catch-up, Appendix B)
* ``jb_checksum``  the model hash of ChecksumMatch (Algorithm 1)
* ``jb_perturb_q4``  the perturbation of 4-bit weights (Section 3)
* ``jb_quantize_grad`` / ``jb_dequantize_grad``  the one-byte projected
  gradient (Section 3, Training Speed)

and, for scores that are not losses, what writing an answer with the perturbed model needs:

* ``jb_cache_reserve``, ``jb_cache_fork``, ``jb_cache_free``, ``jb_cache_compact``  the pages
  of a key-value cache (``PageTable``, ``KVCache``)
* ``jb_cache_write``  new keys and values to their places in the pages
* ``jb_attend``  attention of new tokens over the pages
* ``jb_sample``  the next token from its logits and a given random word

Their tensors are on one device, the current one. No gradients flow through any call here: results
of tensors that require them carry none.

There is no CPU fallback: if ``libjb.so`` is missing, loading it raises.
"""
from __future__ import annotations

import ctypes
import os
import threading
from typing import Iterable, List, Optional, Sequence

import numpy as np

from .build import LIB as _LIB_PATH

JB_OK = 0
JB_F32, JB_BF16 = 0, 1

# Memory layout of jb_seed (16 bytes); arrays of it are passed without copying.
SEED_DTYPE = np.dtype([("machine_id", "<u8"), ("step", "<u4"), ("sample_id", "<u4")])

FLAT_ALIGN = 8
ATTEND_ZEROS = 65536  # bytes of a workspace of jb_attend that are zero between calls


class JbError(RuntimeError):
    def __init__(self, status: int, message: str):
        super().__init__(f"libjb status {status}: {message}")
        self.status = status


class jb_segment(ctypes.Structure):
    _fields_ = [("ptr", ctypes.c_void_p), ("numel", ctypes.c_uint64),
                ("flat_offset", ctypes.c_uint64)]


class jb_q4_segment(ctypes.Structure):
    _fields_ = [("codes", ctypes.c_void_p), ("scale", ctypes.c_void_p), ("numel", ctypes.c_uint64),
                ("flat_offset", ctypes.c_uint64)]


class jb_pages(ctypes.Structure):
    _fields_ = [("table", ctypes.c_void_p), ("lens", ctypes.c_void_p), ("refs", ctypes.c_void_p),
                ("n_rows", ctypes.c_int32), ("row_pages", ctypes.c_int32),
                ("n_pages", ctypes.c_int32), ("page_tokens", ctypes.c_int32)]


class jb_kv(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("page_stride", ctypes.c_uint64),
                ("heads", ctypes.c_int32), ("head_dim", ctypes.c_int32), ("dtype", ctypes.c_int32),
                ("by_token", ctypes.c_int32)]


class jb_scores(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("window", ctypes.c_int32),
                ("slopes", ctypes.c_void_p)]


class jb_sampling(ctypes.Structure):
    _fields_ = [("temperature", ctypes.c_void_p), ("top_k", ctypes.c_void_p),
                ("top_p", ctypes.c_void_p), ("min_p", ctypes.c_void_p)]


class jb_seed(ctypes.Structure):
    _fields_ = [("machine_id", ctypes.c_uint64), ("step", ctypes.c_uint32),
                ("sample_id", ctypes.c_uint32)]


_lock = threading.Lock()
_lib: Optional[ctypes.CDLL] = None


def lib() -> ctypes.CDLL:
    """The loaded libjb.so. Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    with _lock:
        if _lib is None:
            if not os.path.exists(_LIB_PATH):
                raise RuntimeError(
                    f"libjb.so not found at {_LIB_PATH}; build it with "
                    "`python -m paper_2306_10015_gb300.build` (needs nvcc)")
            L = ctypes.CDLL(_LIB_PATH)
            vp, i32, u64, f32 = ctypes.c_void_p, ctypes.c_int, ctypes.c_uint64, ctypes.c_float
            L.jb_perturb.argtypes = [vp, i32, i32, jb_seed, f32, vp]
            L.jb_perturb_with_grid.argtypes = [vp, i32, i32, jb_seed, f32, i32, vp]
            L.jb_apply_updates.argtypes = [vp, i32, i32, vp, vp, i32, f32, f32, f32, vp]
            L.jb_apply_updates_with_grid.argtypes = [vp, i32, i32, vp, vp, i32, f32, f32, f32,
                                                     i32, vp]
            L.jb_apply_updates_from.argtypes = [vp, vp, i32, i32, vp, vp, i32, f32, f32, f32,
                                                i32, vp]
            L.jb_replay_updates.argtypes = [vp, i32, i32, vp, vp, vp, i32, vp, vp, f32, vp]
            L.jb_perturb_q4.argtypes = [vp, i32, jb_seed, f32, vp]
            L.jb_q4_levels.argtypes = [vp]
            L.jb_checksum.argtypes = [vp, i32, i32, vp, vp]
            L.jb_checksum_with_grid.argtypes = [vp, i32, i32, vp, i32, vp]
            L.jb_quantize_grad.argtypes = [ctypes.c_double, f32, ctypes.POINTER(ctypes.c_int8)]
            L.jb_dequantize_grad.argtypes = [ctypes.c_int8, f32, ctypes.POINTER(ctypes.c_float)]
            L.jb_max_seeds_per_call.argtypes = []
            L.jb_status_string.argtypes = [i32]
            L.jb_status_string.restype = ctypes.c_char_p
            L.jb_cache_reserve.argtypes = [vp, vp, vp, i32, vp, vp]
            L.jb_cache_free.argtypes = [vp, vp, i32, vp]
            L.jb_cache_fork.argtypes = [vp, vp, i32, vp, vp, i32, vp, vp, u64, vp]
            L.jb_cache_compact.argtypes = [vp, vp, i32, vp, vp, u64, vp]
            L.jb_cache_write.argtypes = [vp, vp, vp, u64, u64, vp, u64, u64, vp, vp, i32, vp]
            L.jb_attend.argtypes = [vp, vp, vp, vp, u64, u64, i32, vp, vp, i32, vp, u64, u64, vp,
                                    u64, vp]
            L.jb_sample.argtypes = [vp, u64, i32, i32, i32, vp, vp, vp, vp, vp]
            L.jb_cache_workspace.argtypes = [vp, i32]
            L.jb_cache_workspace.restype = u64
            L.jb_attend_workspace.argtypes = [vp, i32]
            L.jb_attend_workspace.restype = u64
            L.jb_debug_philox.argtypes = [jb_seed, u64, u64, vp, vp]
            L.jb_debug_philox_fold.argtypes = [jb_seed, u64, u64, vp, vp]
            L.jb_debug_gaussian.argtypes = [jb_seed, u64, u64, vp, vp]
            L.jb_debug_box_muller.argtypes = [vp, u64, vp, vp]
            for f in ("jb_perturb", "jb_perturb_with_grid", "jb_apply_updates",
                      "jb_apply_updates_with_grid", "jb_apply_updates_from", "jb_replay_updates",
                      "jb_checksum", "jb_checksum_with_grid", "jb_perturb_q4", "jb_q4_levels",
                      "jb_cache_reserve", "jb_cache_free", "jb_cache_fork", "jb_cache_compact",
                      "jb_cache_write", "jb_attend", "jb_sample",
                      "jb_quantize_grad", "jb_dequantize_grad",
                      "jb_max_seeds_per_call", "jb_debug_philox", "jb_debug_philox_fold",
                      "jb_debug_gaussian",
                      "jb_debug_box_muller"):
                getattr(L, f).restype = i32
            _lib = L
    return _lib


def jb_status_string(status: int) -> str:
    return lib().jb_status_string(int(status)).decode()


def _check(rc: int) -> None:
    if rc != JB_OK:
        raise JbError(rc, jb_status_string(rc))


def _stream(stream, device=None) -> ctypes.c_void_p:
    """The stream's handle; of None the current one's, on the current device, which a caller that knows it gives."""
    if stream is None:
        import torch
        # the current stream's handle without a Stream object around it (0.1 us, not 3); the
        # function is not part of torch's public interface, so it may be missing
        raw = getattr(torch._C, "_cuda_getCurrentRawStream", None)
        if raw is not None and torch.cuda.is_initialized():
            return ctypes.c_void_p(raw(torch.cuda.current_device() if device is None else device))
        return ctypes.c_void_p(torch.cuda.current_stream().cuda_stream)
    if isinstance(stream, int):
        return ctypes.c_void_p(stream)
    return ctypes.c_void_p(stream.cuda_stream)


def _seed(s) -> jb_seed:
    if isinstance(s, jb_seed):
        return s
    if isinstance(s, np.void):
        return jb_seed(int(s["machine_id"]), int(s["step"]), int(s["sample_id"]))
    m, t, j = s
    return jb_seed(int(m), int(t), int(j))


def seeds_array(seeds) -> np.ndarray:
    """Seeds as a contiguous jb_seed array (machine_id, step, sample_id)."""
    if isinstance(seeds, np.ndarray) and seeds.dtype == SEED_DTYPE:
        return np.ascontiguousarray(seeds)
    out = np.zeros(len(seeds), dtype=SEED_DTYPE)
    for i, s in enumerate(seeds):
        out[i] = (int(s[0]), int(s[1]), int(s[2]))
    return out


# Host arrays go to the library as bytes objects (it copies them during the call): for the
# few kilobytes of a call that is cheaper than asking numpy for a pointer (1 us an array).
def _codes_array(q) -> np.ndarray:
    return np.ascontiguousarray(np.asarray(q, dtype=np.int8))


def _bytes(a: np.ndarray):
    return a.tobytes() if a.size else None


def default_flat_offsets(numels: Sequence[int], align: int = FLAT_ALIGN) -> List[int]:
    """flat_offset of tensor t = align_up(flat_offset of t-1 + numel of t-1, align)."""
    offs, cur = [], 0
    for n in numels:
        offs.append(cur)
        cur = (cur + int(n) + align - 1) // align * align
    return offs


class ParamTable:
    """Segment table (jb_segment array) over CUDA tensors of one dtype.

    Holds references to the tensors so their memory stays alive. Element i of
    tensor t has global index flat_offsets[t] + i; every replica must build the
    table with the same offsets.
    """

    def __init__(self, tensors: Iterable, flat_offsets: Optional[Sequence[int]] = None):
        import torch
        self.tensors = list(tensors)
        if not self.tensors:
            raise ValueError("empty parameter list")
        dt = self.tensors[0].dtype
        if dt == torch.float32:
            self.dtype = JB_F32
        elif dt == torch.bfloat16:
            self.dtype = JB_BF16
        else:
            raise TypeError(f"parameters must be float32 or bfloat16, got {dt}")
        for t in self.tensors:
            if t.dtype != dt or not t.is_cuda or not t.is_contiguous():
                raise ValueError("parameters must be contiguous CUDA tensors of one dtype")
        numels = [t.numel() for t in self.tensors]
        self.flat_offsets = (list(flat_offsets) if flat_offsets is not None
                             else default_flat_offsets(numels))
        if len(self.flat_offsets) != len(self.tensors):
            raise ValueError("one flat offset per tensor")
        n = len(self.tensors)
        self.segments = (jb_segment * n)()
        for i, (t, fo) in enumerate(zip(self.tensors, self.flat_offsets)):
            self.segments[i] = jb_segment(t.data_ptr(), t.numel(), int(fo))
        self.numel = sum(numels)
        self.n_segments = n

    @classmethod
    def from_module(cls, module, flat_offsets=None) -> "ParamTable":
        return cls([p.data for _, p in module.named_parameters()], flat_offsets)


def jb_perturb(table: ParamTable, seed, eps: float, stream=None, grid_ctas: int = 0) -> None:
    """theta <- theta + eps z(seed), in place on `stream` (asynchronous)."""
    L = lib()
    if grid_ctas:
        rc = L.jb_perturb_with_grid(table.segments, table.n_segments, table.dtype, _seed(seed),
                                    float(eps), int(grid_ctas), _stream(stream))
    else:
        rc = L.jb_perturb(table.segments, table.n_segments, table.dtype, _seed(seed), float(eps),
                          _stream(stream))
    _check(rc)


def jb_apply_updates(table: ParamTable, seeds, q, lr: float, denom: float, qscale: float,
                     stream=None, grid_ctas: int = 0) -> None:
    """theta <- theta - (lr / denom) sum_k deq(q_k) z(seed_k), one pass, in place."""
    s, qa = seeds_array(seeds), _codes_array(q)
    if qa.shape[0] != s.shape[0]:
        raise ValueError("one byte code per seed")
    K = s.shape[0]
    sp, qp = _bytes(s), _bytes(qa)
    L = lib()
    if grid_ctas:
        rc = L.jb_apply_updates_with_grid(table.segments, table.n_segments, table.dtype, sp, qp, K,
                                          float(lr), float(denom), float(qscale), int(grid_ctas),
                                          _stream(stream))
    else:
        rc = L.jb_apply_updates(table.segments, table.n_segments, table.dtype, sp, qp, K,
                                float(lr), float(denom), float(qscale), _stream(stream))
    _check(rc)


def jb_apply_updates_from(src: ParamTable, dst: ParamTable, seeds, q, lr: float, denom: float,
                          qscale: float, write_src: bool = False, stream=None) -> None:
    """dst <- src - (lr / denom) sum_k deq(q_k) z(seed_k) in one pass (restore fused)."""
    if src.n_segments != dst.n_segments or src.dtype != dst.dtype:
        raise ValueError("source and destination tables differ")
    s, qa = seeds_array(seeds), _codes_array(q)
    if qa.shape[0] != s.shape[0]:
        raise ValueError("one byte code per seed")
    _check(lib().jb_apply_updates_from(
        src.segments, dst.segments, src.n_segments, src.dtype, _bytes(s), _bytes(qa), s.shape[0],
        float(lr), float(denom), float(qscale), int(bool(write_src)), _stream(stream)))


def jb_replay_updates(table: ParamTable, steps, qscale: float, stream=None) -> None:
    """Apply several steps' updates in order, in place; steps = [(seeds, q, lr, denom), ...]."""
    seeds = [seeds_array(st[0]) for st in steps]
    codes = [np.asarray(st[1], dtype=np.int8, order="C") for st in steps]
    sizes = np.array([len(x) for x in seeds], dtype=np.int32)
    if any(len(c) != len(x) for c, x in zip(codes, seeds)):
        raise ValueError("one byte code per seed")
    # joined as bytes: what numpy's concatenation would refuse is refused here
    if {a.ndim for a in seeds + codes} != {1} and any(
            len({a.shape[1:] for a in arrays}) > 1 for arrays in (seeds, codes)):
        raise ValueError("the arrays of the steps differ in their dimensions")
    lr = np.array([float(st[2]) for st in steps], dtype=np.float32)
    denom = np.array([float(st[3]) for st in steps], dtype=np.float32)
    _check(lib().jb_replay_updates(table.segments, table.n_segments, table.dtype,
                                   b"".join(seeds) or None, b"".join(codes) or None, _bytes(sizes),
                                   len(steps), _bytes(lr), _bytes(denom), float(qscale),
                                   _stream(stream)))


class Q4Table:
    """jb_q4_segment array over 4-bit tensors: (codes uint8 CUDA tensor, scales float32 CUDA
    tensor, numel) triples; flat offsets default to the jb_segment rule."""

    def __init__(self, tensors, flat_offsets: Optional[Sequence[int]] = None):
        self.tensors = list(tensors)
        numels = [int(n) for _, _, n in self.tensors]
        self.flat_offsets = (list(flat_offsets) if flat_offsets is not None
                             else default_flat_offsets(numels))
        n = len(self.tensors)
        self.segments = (jb_q4_segment * n)()
        for i, ((codes, scale, numel), fo) in enumerate(zip(self.tensors, self.flat_offsets)):
            if codes.numel() < (numel + 1) // 2 or scale.numel() < (numel + 63) // 64:
                raise ValueError("codes or scales too short for numel")
            self.segments[i] = jb_q4_segment(codes.data_ptr(), scale.data_ptr(), int(numel), int(fo))
        self.n_segments = n


def jb_perturb_q4(table: "Q4Table", seed, eps: float, stream=None) -> None:
    """4-bit weights: dequantize, add eps z(seed), quantize again, in place."""
    _check(lib().jb_perturb_q4(table.segments, table.n_segments, _seed(seed), float(eps),
                               _stream(stream)))


def jb_q4_levels() -> np.ndarray:
    out = np.empty(16, dtype=np.float32)
    _check(lib().jb_q4_levels(out.ctypes.data))
    return out


def jb_checksum(table: ParamTable, out, stream=None, grid_ctas: int = 0) -> None:
    """out (CUDA int64 tensor, one element) <- the model checksum, on `stream`."""
    L = lib()
    if grid_ctas:
        rc = L.jb_checksum_with_grid(table.segments, table.n_segments, table.dtype, out.data_ptr(),
                                     int(grid_ctas), _stream(stream))
    else:
        rc = L.jb_checksum(table.segments, table.n_segments, table.dtype, out.data_ptr(),
                           _stream(stream))
    _check(rc)


# --- writing answers ------------------------------------------------------------

torch = None  # imported by the first call that needs it: the rest of the package works without


def _need_torch():
    global torch
    import torch as module
    torch = module


# The tensors of a call are on one device, and that is the current one: a kernel of another device would take their
# addresses for its own memory's. `device` is the number of the cache's or, of jb_sample, of the logits'.

def _list32(t, what: str, device: int):
    """A one-dimensional contiguous int32 tensor on the call's device: its address and length."""
    if torch is None:
        _need_torch()
    if t.dtype is not torch.int32 or t.get_device() != device or t.dim() != 1 or not t.is_contiguous():
        raise ValueError(f"{what} must be a contiguous one-dimensional int32 tensor on the call's CUDA device")
    return t.data_ptr(), t.numel()


def _two_lists(a, b, what: str, device: int):
    pa, n = _list32(a, what, device)
    pb, m = _list32(b, what, device)
    if n != m:
        raise ValueError(f"{what} must have the same length")
    return pa, pb, n


def _stream_on(device: int, stream) -> ctypes.c_void_p:
    if torch.cuda.current_device() != device:
        raise ValueError(f"the tensors are on CUDA device {device}, which is not the current device")
    return _stream(stream, device)


def _storage(dtype) -> int:
    if dtype is torch.bfloat16:
        return JB_BF16
    if dtype is torch.float32:
        return JB_F32
    raise TypeError(f"tensors must be float32 or bfloat16, got {dtype}")


class PageTable:
    """The rows of a cache and their pages (jb_pages): ``table`` [rows, row_pages], ``lens`` [rows]
    and ``refs`` [pages], int32 CUDA tensors that the jb_cache_* calls keep consistent. Holds
    references to them. ``PageTable.empty`` makes them."""

    def __init__(self, table, lens, refs, page_tokens: int):
        _need_torch()
        for t, dim in ((table, 2), (lens, 1), (refs, 1)):
            if t.dtype is not torch.int32 or not t.is_cuda or t.dim() != dim or not t.is_contiguous():
                raise ValueError("table [rows, row_pages], lens [rows] and refs [pages] must be contiguous int32 CUDA tensors")
        if lens.get_device() != table.get_device() or refs.get_device() != table.get_device():
            raise ValueError("table, lens and refs must be on one CUDA device")
        if lens.shape[0] != table.shape[0]:
            raise ValueError("one length per row of the table")
        if not 16 <= page_tokens <= 1024 or page_tokens % 16:
            raise ValueError("page_tokens must be a multiple of 16, at most 1024")
        self.table, self.lens, self.refs, self.page_tokens = table, lens, refs, int(page_tokens)
        self.device = table.get_device()
        self.struct = jb_pages(table.data_ptr(), lens.data_ptr(), refs.data_ptr(), table.shape[0],
                               table.shape[1], refs.shape[0], self.page_tokens)
        self.ref = ctypes.byref(self.struct)
        self._bytes = {}

    def workspace(self, n: int) -> int:
        """Device bytes that jb_cache_fork of n pairs works in, or jb_cache_compact (n = 0)."""
        nbytes = self._bytes.get(n)
        if nbytes is None:
            nbytes = self._bytes[n] = max(16, int(lib().jb_cache_workspace(self.ref, n)))
        return nbytes

    @classmethod
    def empty(cls, n_rows: int, row_pages: int, n_pages: int, page_tokens: int, device="cuda") -> "PageTable":
        _need_torch()
        return cls(torch.full((n_rows, row_pages), -1, dtype=torch.int32, device=device),
                   torch.zeros(n_rows, dtype=torch.int32, device=device),
                   torch.zeros(n_pages, dtype=torch.int32, device=device), page_tokens)


class _Workspaces:
    """Device bytes that calls work in: kept for each stream, and new for each call that a graph captures, since
    the graph may be replayed on another stream."""

    def __init__(self):
        self.kept = {}

    def get(self, key, nbytes: int, stream, handle, make):
        """Address and bytes of at least `nbytes`, made by make(nbytes), and what holds them."""
        if _new(stream, torch.cuda.is_current_stream_capturing):
            ws = make(nbytes)
            return ws.data_ptr(), nbytes, ws
        key = key, handle.value
        found = self.kept.get(key)
        if found is None or found[1] < nbytes:
            ws = make(nbytes)
            found = self.kept[key] = ws.data_ptr(), nbytes, ws
        return found


class KVCache:
    """Keys and values of a model's layers in pages: one tensor [pages, heads, page_tokens, head_dim]
    a layer in ``keys`` and ``values``, float32 or bfloat16, whose pages are contiguous with heads
    before tokens or (transposed view) tokens before heads. Holds references to the tensors."""

    def __init__(self, pages: PageTable, keys: Sequence, values: Sequence):
        self.pages, self.keys, self.values = pages, list(keys), list(values)
        if not self.keys or len(self.keys) != len(self.values):
            raise ValueError("one tensor of keys and one of values per layer")
        first = self.keys[0]
        self.dtype = _storage(first.dtype)
        if first.dim() != 4:
            raise ValueError("keys and values must be [pages, heads, page_tokens, head_dim]")
        n_pages, heads, tokens, d = first.shape
        if n_pages != pages.refs.shape[0] or tokens != pages.page_tokens:
            raise ValueError("the tensors' pages differ from the table's")
        inner = first.stride()[1:]
        if inner == (tokens * d, d, 1):
            by_token = 0
        elif inner == (d, heads * d, 1):
            by_token = 1
        else:
            raise ValueError("a page must be contiguous, by heads or by tokens")
        for t in self.keys + self.values:
            if t.shape != first.shape or t.dtype != first.dtype or t.stride() != first.stride() or not t.is_cuda:
                raise ValueError("keys and values must be CUDA tensors of one shape, type and layout")
            if t.get_device() != pages.device:
                raise ValueError("keys and values must be on the page table's device")
        n = len(self.keys)
        self.torch_dtype, self.heads, self.head_dim, self.n_layers, self.device = first.dtype, heads, d, n, pages.device
        self.layers = (jb_kv * n)()
        for i, (k, v) in enumerate(zip(self.keys, self.values)):
            self.layers[i] = jb_kv(k.data_ptr(), v.data_ptr(), first.stride(0), heads, d, self.dtype, by_token)
        self.layer_refs = [ctypes.byref(self.layers, i * ctypes.sizeof(jb_kv)) for i in range(n)]
        self._workspaces, self._attend_bytes = _Workspaces(), {}

    def new_workspace(self, q_heads: int, stream=None):
        """A workspace for jb_attend with so many query heads: a uint8 tensor, ready for use on the stream."""
        return self._zeroed(max(int(lib().jb_attend_workspace(self.layer_refs[0], q_heads)), ATTEND_ZEROS), stream)

    def _zeroed(self, nbytes, stream):
        ws = _new(stream, torch.empty, nbytes, dtype=torch.uint8, device=self.keys[0].device)
        _new(stream, ws[:ATTEND_ZEROS].zero_)
        return ws

    def _attend_workspace(self, q_heads: int, stream, handle):
        nbytes = self._attend_bytes.get(q_heads)
        if nbytes is None:
            nbytes = max(int(lib().jb_attend_workspace(self.layer_refs[0], q_heads)), ATTEND_ZEROS)
            self._attend_bytes[q_heads] = nbytes
        return self._workspaces.get("attend", nbytes, stream, handle, lambda size: self._zeroed(size, stream))

    def _pages_workspace(self, n: int, stream, handle):
        nbytes = self.pages.workspace(n)
        return self._workspaces.get("pages", nbytes, stream, handle,
                                    lambda size: _new(stream, torch.empty, size, dtype=torch.uint8, device=self.keys[0].device))


def _new(stream, make, *args, **kwargs):
    """make(...) on the call's stream: what the allocator hands out is ordered with that stream alone."""
    if stream is None:
        return make(*args, **kwargs)
    with torch.cuda.stream(torch.cuda.ExternalStream(stream) if isinstance(stream, int) else stream):
        return make(*args, **kwargs)


def _status_of(status, pages, stream):
    if status is None:
        return _new(stream, torch.empty, 1, dtype=torch.int32, device=pages.refs.device)
    if _list32(status, "status", pages.device)[1] != 1:
        raise ValueError("status must have one element")
    return status


def jb_cache_reserve(cache, rows, tokens, status=None, stream=None):
    """Room for tokens[i] more tokens in row rows[i]; returns the status tensor (0: done, > 0:
    that many pages too few, -1: bad list; then nothing is changed). `cache`: a KVCache or its
    PageTable."""
    pages = getattr(cache, "pages", cache)
    device = getattr(pages, "device", None)
    pr, pt, n = _two_lists(rows, tokens, "rows and tokens", device)
    status = _status_of(status, pages, stream)
    _check(lib().jb_cache_reserve(pages.ref, pr, pt, n, status.data_ptr(), _stream_on(device, stream)))
    return status


def jb_cache_free(cache, rows, stream=None) -> None:
    """The rows become empty; pages that no other row names are free."""
    pages = getattr(cache, "pages", cache)
    device = getattr(pages, "device", None)
    pr, n = _list32(rows, "rows", device)
    _check(lib().jb_cache_free(pages.ref, pr, n, _stream_on(device, stream)))


def jb_cache_fork(cache: KVCache, parents, children, status=None, stream=None):
    """Row children[i] becomes a copy of row parents[i] (all at once): full pages shared, the last
    one copied in every layer. Returns the status tensor as jb_cache_reserve does."""
    pages = cache.pages
    pp, pc, n = _two_lists(parents, children, "parents and children", cache.device)
    status = _status_of(status, pages, stream)
    handle = _stream_on(cache.device, stream)
    ws, nbytes, held = cache._pages_workspace(n, stream, handle)
    _check(lib().jb_cache_fork(pages.ref, cache.layers, cache.n_layers, pp, pc, n, status.data_ptr(), ws, nbytes, handle))
    return status


def jb_cache_compact(cache: KVCache, status=None, stream=None):
    """Moves the pages in use to the lowest ids; returns the status tensor: how many they are."""
    pages = cache.pages
    status = _status_of(status, pages, stream)
    handle = _stream_on(cache.device, stream)
    ws, nbytes, held = cache._pages_workspace(0, stream, handle)
    _check(lib().jb_cache_compact(pages.ref, cache.layers, cache.n_layers, status.data_ptr(), ws, nbytes, handle))
    return status


def _heads_of(t, heads: int, cache: KVCache, n: int, what: str):
    """Strides of a [n, heads, head_dim] CUDA tensor whose rows are contiguous."""
    if t.dtype is not cache.torch_dtype or t.get_device() != cache.device:
        raise ValueError(f"{what} must be tensors of the cache's type on its CUDA device")
    if t.dim() != 3 or t.shape != (n, heads, cache.head_dim):
        raise ValueError(f"{what} must be [{n}, {heads}, {cache.head_dim}], got {tuple(t.shape)}")
    a, b, c = t.stride()
    if c != 1 and cache.head_dim > 1:
        raise ValueError(f"{what} must be contiguous in their last dimension")
    return a, b


def jb_cache_write(cache: KVCache, layer: int, k, v, rows, pos, stream=None) -> None:
    """Keys and values k[i], v[i] ([n, heads, head_dim]) of a layer to position pos[i] of row rows[i]."""
    pr, pp, n = _two_lists(rows, pos, "rows and positions", cache.device)
    ka, kb = _heads_of(k, cache.heads, cache, n, "new keys")
    va, vb = _heads_of(v, cache.heads, cache, n, "new values")
    _check(lib().jb_cache_write(cache.pages.ref, cache.layer_refs[layer], k.data_ptr(), ka, kb, v.data_ptr(), va, vb,
                                pr, pp, n, _stream_on(cache.device, stream)))


def jb_attend(cache: KVCache, layer: int, q, rows, pos, out=None, scale: Optional[float] = None,
              softcap: float = 0.0, window: int = 0, slopes=None, workspace=None, stream=None):
    """Attention of queries q [n, q_heads, head_dim] over positions <= pos[i] of row rows[i];
    returns ``out``. Scores are scale q.k (default 1 / sqrt(head_dim)), capped by softcap tanh,
    biased by slopes[head] (t - pos), limited to the last `window` positions. The tokens of a prompt may be
    queries of one row, but each reads the row for itself: long prompts are slow. ``workspace``: by default
    one that the cache keeps for the stream; ``cache.new_workspace`` makes others, for instance one for
    all the calls that a CUDA graph captures (by default each gets its own there)."""
    pr, pp, n = _two_lists(rows, pos, "rows and positions", cache.device)
    heads = q.shape[1] if q.dim() == 3 else 0
    qa, qb = _heads_of(q, heads, cache, n, "queries")
    if out is None:
        out = _new(stream, torch.empty, (n, heads, cache.head_dim), dtype=q.dtype, device=q.device)
    oa, ob = _heads_of(out, heads, cache, n, "outputs")
    if slopes is not None and (slopes.dtype is not torch.float32 or slopes.get_device() != cache.device
                               or slopes.shape != (heads,) or not slopes.is_contiguous()):
        raise ValueError("slopes must be a contiguous float32 tensor on the cache's CUDA device, one per query head")
    handle = _stream_on(cache.device, stream)
    if workspace is None:
        ws, nbytes, held = cache._attend_workspace(heads, stream, handle)
    else:
        if workspace.get_device() != cache.device or not workspace.is_contiguous():
            raise ValueError("workspace must be a contiguous tensor on the cache's CUDA device")
        ws, nbytes = workspace.data_ptr(), workspace.numel() * workspace.element_size()
    scores = jb_scores(cache.head_dim ** -0.5 if scale is None else scale, softcap, window,
                       None if slopes is None else slopes.data_ptr())
    _check(lib().jb_attend(cache.pages.ref, cache.layer_refs[layer], ctypes.byref(scores), q.data_ptr(), qa, qb, heads,
                           pr, pp, n, out.data_ptr(), oa, ob, ws, nbytes, handle))
    return out


def _per_row(value, default, words, dtype, stream, device):
    """A setting of jb_sample as the address of its entries (None where it is the default) and the tensor
    that holds them, one for each of the words."""
    if type(value) is not torch.Tensor and not isinstance(value, torch.Tensor):
        if value == default:
            return None, None
        value = _new(stream, torch.full, words.shape, value, dtype=dtype, device=words.device)
    if value.dtype is not dtype or value.get_device() != device or value.shape != words.shape or not value.is_contiguous():
        raise ValueError(f"a setting per row must be a contiguous {dtype} tensor of one entry per word on the logits' CUDA device")
    return value.data_ptr(), value


def jb_sample(logits, words, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, tokens=None, logprobs=None,
              stream=None):
    """The next token of each row of logits [n, vocab] from its random word (int32 or uint32 bits),
    and its log-probability; returns (tokens int32, logprobs float32). Settings are numbers or one
    per row (float32, top_k int32 CUDA tensors)."""
    if torch is None:
        _need_torch()
    i32, f32 = torch.int32, torch.float32
    device = logits.get_device()
    if logits.dim() != 2 or device < 0:
        raise ValueError("logits must be a CUDA tensor [n, vocab]")
    n, vocab = logits.shape
    pitch, step = logits.stride()
    if step != 1 and vocab > 1:
        raise ValueError("logits must be contiguous in a row")
    if (words.dtype is not i32 and words.dtype is not torch.uint32) or words.get_device() != device or words.dim() != 1 \
            or words.numel() != n or not words.is_contiguous():
        raise ValueError("words must be a contiguous int32 or uint32 tensor on the logits' CUDA device, one per row")
    t, t_ = _per_row(temperature, 1.0, words, f32, stream, device)
    k, k_ = _per_row(top_k, 0, words, i32, stream, device)
    p, p_ = _per_row(top_p, 1.0, words, f32, stream, device)
    m, m_ = _per_row(min_p, 0.0, words, f32, stream, device)
    if tokens is None:
        tokens = _new(stream, torch.empty_like, words, dtype=i32)
    elif _list32(tokens, "tokens", device)[1] != n:
        raise ValueError("one token per row")
    if logprobs is None:
        logprobs = _new(stream, torch.empty_like, words, dtype=f32)
    elif logprobs.dtype is not f32 or logprobs.get_device() != device or logprobs.shape != words.shape or not logprobs.is_contiguous():
        raise ValueError("logprobs must be a contiguous float32 tensor on the logits' CUDA device, one per row")
    settings = jb_sampling(t, k, p, m)
    _check(lib().jb_sample(logits.data_ptr(), pitch, _storage(logits.dtype), n, vocab, ctypes.byref(settings),
                           words.data_ptr(), tokens.data_ptr(), logprobs.data_ptr(), _stream_on(device, stream)))
    return tokens, logprobs


def jb_quantize_grad(g: float, qscale: float = 1.0) -> int:
    out = ctypes.c_int8()
    _check(lib().jb_quantize_grad(float(g), float(qscale), ctypes.byref(out)))
    return int(out.value)


def jb_dequantize_grad(q: int, qscale: float = 1.0) -> float:
    out = ctypes.c_float()
    _check(lib().jb_dequantize_grad(int(q), float(qscale), ctypes.byref(out)))
    return float(out.value)


def jb_max_seeds_per_call() -> int:
    return int(lib().jb_max_seeds_per_call())


# --- test hooks ---------------------------------------------------------------

def jb_debug_philox(seed, first_block: int, n_blocks: int, out, stream=None) -> None:
    """out: CUDA int32/uint32 tensor of >= 4 n_blocks words, 16-byte aligned."""
    _check(lib().jb_debug_philox(_seed(seed), int(first_block), int(n_blocks), out.data_ptr(),
                                 _stream(stream)))


def jb_debug_philox_fold(seed, first_block: int, n_blocks: int, out, stream=None) -> None:
    """out: CUDA int32/uint32 tensor of >= 1 element; receives the XOR of all words."""
    _check(lib().jb_debug_philox_fold(_seed(seed), int(first_block), int(n_blocks),
                                      out.data_ptr(), _stream(stream)))


def jb_debug_gaussian(seed, first_elem: int, n: int, out, stream=None) -> None:
    """out: CUDA float32 tensor of >= n elements."""
    _check(lib().jb_debug_gaussian(_seed(seed), int(first_elem), int(n), out.data_ptr(),
                                   _stream(stream)))


def jb_debug_box_muller(words, n_pairs: int, out, stream=None) -> None:
    """words: CUDA int32 tensor of 2 n_pairs words; out: float32 tensor of 2 n_pairs."""
    _check(lib().jb_debug_box_muller(words.data_ptr(), int(n_pairs), out.data_ptr(),
                                     _stream(stream)))


__all__ = [
    "JB_OK", "JB_F32", "JB_BF16", "SEED_DTYPE", "JbError", "ParamTable", "jb_segment", "jb_seed",
    "lib", "seeds_array", "default_flat_offsets", "jb_perturb", "jb_apply_updates",
    "jb_apply_updates_from", "jb_replay_updates", "jb_checksum", "jb_perturb_q4", "jb_q4_levels",
    "Q4Table", "jb_q4_segment", "PageTable", "KVCache", "jb_pages", "jb_kv", "jb_scores", "jb_sampling",
    "jb_cache_reserve", "jb_cache_free", "jb_cache_fork", "jb_cache_compact", "jb_cache_write",
    "jb_attend", "jb_sample",
    "jb_quantize_grad", "jb_dequantize_grad", "jb_max_seeds_per_call", "jb_status_string",
    "jb_debug_philox", "jb_debug_gaussian", "jb_debug_box_muller",
]
