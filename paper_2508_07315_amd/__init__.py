"""ctcbeam - MI355X-native batched CTC beam search with n-gram LM fusion and
phrase boosting (the per-frame step of FlexCTC, arXiv 2508.07315, Algorithm 1).

This module is a thin ctypes binding over the C ABI declared in
``include/ctcbeam.h`` and implemented by ``libctcbeam.so`` (host builders in
``csrc/ctcbeam_host.cpp``, gfx950 kernels in ``csrc/ctcbeam_decode.inl`` and
``csrc/ctcbeam_greedy.inl``, compiled per vocabulary class by the
``csrc/*.hip`` units; the operators on rows of scores in
``csrc/ctcbeam_rows_host.cpp``, ``csrc/ctcbeam_process.inl``,
``csrc/ctcbeam_top.inl`` and ``csrc/ctcbeam_distill.inl``).  It only marshals arguments: every step of the search
runs in the HIP kernels.  PyTorch supplies device memory and streams; each
call runs with the inputs' device current, and tensors the binding allocates
are the launch stream's, and recorded on torch's current stream where that is
another one.
Outputs that the caller gives count as written in place for torch's autograd,
and may not require a gradient while torch records one.

If the shared library has not been built, importing the binding's entry
points raises; build it with ``python -m paper_2508_07315_amd.build_lib`` (or
``__graft_entry__.build()``).  There is no CPU fallback.
"""
from __future__ import annotations

import ctypes
import math
import os
from typing import Optional

import numpy as np

_PKG = os.path.dirname(os.path.abspath(__file__))
LIB_PATH = os.path.join(_PKG, "libctcbeam.so")
_lib = None
_torch = None         # the module, once the library is loaded

MAX_K = 128           # CTCBEAM_MAX_K (beams above 64 need V <= 1024)
MAX_V = 4096
MAX_ORDER = 8
MAX_LABELS = 1 << 18  # CTCBEAM_MAX_LABELS
MAX_TOP = 128         # CTCBEAM_MAX_TOP
MAX_ROWS = 1 << 21    # CTCBEAM_MAX_ROWS


class CtcbeamError(RuntimeError):
    def __init__(self, code: int, msg: str):
        super().__init__(f"ctcbeam error {code}: {msg}")
        self.code = code


def library_path() -> str:
    return LIB_PATH


def _load():
    global _lib, _torch
    if _lib is not None:
        return _lib
    if not os.path.exists(LIB_PATH):
        raise ImportError(
            f"{LIB_PATH} is not built; run `python -m paper_2508_07315_amd.build_lib` "
            "(the decoder has no CPU fallback)")
    # torch first: its HIP runtime and the system one share a SONAME, so the
    # first loaded serves the whole process; it must be the one that owns
    # torch's device memory and streams
    import torch
    _torch = torch
    lib = ctypes.CDLL(LIB_PATH)
    P = ctypes.c_void_p
    I = ctypes.c_int
    F = ctypes.c_float
    lib.ctcbeam_last_error.restype = ctypes.c_char_p
    lib.ctcbeam_last_error.argtypes = []
    for name in ("ctcbeam_lm_build", "ctcbeam_lm_build_host"):
        fn = getattr(lib, name)
        fn.restype = I
        fn.argtypes = [I, I, P, P, P, P, ctypes.POINTER(P)]
    for name in ("ctcbeam_lm_build_arpa", "ctcbeam_lm_build_arpa_host"):
        fn = getattr(lib, name)
        fn.restype = I
        fn.argtypes = [ctypes.c_char_p, I, ctypes.POINTER(P)]
    lib.ctcbeam_lm_free.restype = None
    lib.ctcbeam_lm_free.argtypes = [P]
    for name in ("ctcbeam_boost_build", "ctcbeam_boost_build_host"):
        fn = getattr(lib, name)
        fn.restype = I
        fn.argtypes = [I, I, P, P, ctypes.POINTER(P)]
    lib.ctcbeam_boost_free.restype = None
    lib.ctcbeam_boost_free.argtypes = [P]
    lib.ctcbeam_workspace_bytes.restype = ctypes.c_size_t
    lib.ctcbeam_workspace_bytes.argtypes = [I, I, I]
    dec = [P, P, I, I, I, I, F, F, F, P, P, P, ctypes.c_size_t, P, P, P, P]
    lib.ctcbeam_decode.restype = I
    lib.ctcbeam_decode.argtypes = dec
    lib.ctcbeam_decode_ex.restype = I
    lib.ctcbeam_decode_ex.argtypes = dec + [P]
    lib.ctcbeam_decode_nbest.restype = I
    lib.ctcbeam_decode_nbest.argtypes = dec + [P]
    lib.ctcbeam_greedy_decode.restype = I
    lib.ctcbeam_greedy_decode.argtypes = [P, P, I, I, I, F, F, F, P, P, P, ctypes.c_size_t, P, P, P, P, P]
    lib.ctcbeam_decode_noalloc.restype = I
    lib.ctcbeam_decode_noalloc.argtypes = [P, P, I, I, I, I, F, F, F, P, P, P, P, P, P, P]
    lib.ctcbeam_query_status.restype = I
    lib.ctcbeam_query_status.argtypes = [P, P, ctypes.POINTER(ctypes.c_uint32)]
    lib.ctcbeam_lm_tables.restype = I
    lib.ctcbeam_lm_tables.argtypes = [P, P]
    lib.ctcbeam_boost_tables.restype = I
    lib.ctcbeam_boost_tables.argtypes = [P, P]
    S, L = ctypes.c_size_t, ctypes.c_int64
    lib.ctcbeam_process_workspace_bytes.restype = S
    lib.ctcbeam_process_workspace_bytes.argtypes = [I, I, I]
    lib.ctcbeam_top_workspace_bytes.restype = S
    lib.ctcbeam_top_workspace_bytes.argtypes = [I, I, I, I]
    lib.ctcbeam_distill_workspace_bytes.restype = S
    lib.ctcbeam_distill_workspace_bytes.argtypes = [I, I, I]
    lib.ctcbeam_process_logits.restype = I
    lib.ctcbeam_process_logits.argtypes = [P, P, P, P, S, P]
    lib.ctcbeam_top_logits.restype = I
    lib.ctcbeam_top_logits.argtypes = [P, I, F, P, P, P, P, S, P]
    lib.ctcbeam_distill.restype = I
    lib.ctcbeam_distill.argtypes = [P, P, P, P, I, F, P, L, L, F, P, P, L, L, P, S, P]
    _lib = lib
    return lib


def _check(rc: int):
    if rc != 0:
        raise CtcbeamError(rc, _load().ctcbeam_last_error().decode())


def _size(n, name):
    """A size as the library's 32-bit int: ctypes would cut a larger one to
    its low bits, and the library would not see what it has to refuse."""
    n = int(n)
    if not -1 << 31 <= n < 1 << 31:
        raise CtcbeamError(2, f"{name} = {n} does not fit 32 bits")
    return n


class _Opts(ctypes.Structure):
    _fields_ = [("prune_theta", ctypes.c_float), ("stats", ctypes.c_void_p),
                ("flags", ctypes.c_int), ("reserved", ctypes.c_int * 3)]


FLAG_LOGSUMEXP = 1        # CTCBEAM_FLAG_LOGSUMEXP
FLAG_BOOST_ROLLBACK = 2   # CTCBEAM_FLAG_BOOST_ROLLBACK
FLAG_NO_ROW_CACHE = 4     # CTCBEAM_FLAG_NO_ROW_CACHE
FLAG_REPEAT_SCORE = 8     # CTCBEAM_FLAG_REPEAT_SCORE


def _opts(theta, stats, B, logsumexp, boost_rollback, row_cache=True, device=None,
          repeat_score=False):
    """ctcbeam_opts by reference, or None when every option is at its default."""
    import torch
    flags = (FLAG_LOGSUMEXP if logsumexp else 0) | (FLAG_BOOST_ROLLBACK if boost_rollback else 0) | \
        (0 if row_cache else FLAG_NO_ROW_CACHE) | (FLAG_REPEAT_SCORE if repeat_score else 0)
    if (theta is None or math.isinf(theta)) and stats is None and flags == 0:
        return None
    o = _Opts()
    o.prune_theta = float(theta if theta is not None else math.inf)
    o.stats = None if stats is None else _dptr(stats, torch.int64, "stats", (B, 8), device).value
    o.flags = flags
    return o


class _LmView(ctypes.Structure):
    _fields_ = [("order", ctypes.c_int), ("vocab_size", ctypes.c_int), ("nlev", ctypes.c_int),
                ("n_states", ctypes.c_int64), ("n_arcs", ctypes.c_int64),
                ("states", ctypes.c_void_p), ("arcs", ctypes.c_void_p),
                ("unigram", ctypes.c_void_p)]


class _BoostView(ctypes.Structure):
    _fields_ = [("vocab_size", ctypes.c_int), ("n_nodes", ctypes.c_int64),
                ("n_list", ctypes.c_int64), ("nodes", ctypes.c_void_p),
                ("list", ctypes.c_void_p), ("root_key", ctypes.c_void_p)]


class LM:
    """Owning wrapper of a ``ctcbeam_lm*`` handle."""

    def __init__(self, handle: int, vocab_size: int):
        self._h = ctypes.c_void_p(handle)
        self.vocab_size = vocab_size

    @property
    def handle(self):
        return self._h

    def close(self):
        if self._h and self._h.value:
            _load().ctcbeam_lm_free(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Boost:
    """Owning wrapper of a ``ctcbeam_boost*`` handle."""

    def __init__(self, handle: int, vocab_size: int):
        self._h = ctypes.c_void_p(handle)
        self.vocab_size = vocab_size

    @property
    def handle(self):
        return self._h

    def close(self):
        if self._h and self._h.value:
            _load().ctcbeam_boost_free(self._h)
            self._h = ctypes.c_void_p(None)

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


def _lm_args(arrays: dict):
    order = int(arrays["order"])
    ids = [np.ascontiguousarray(a, dtype=np.int32) for a in arrays["ids"]]
    pr = [np.ascontiguousarray(a, dtype=np.float32) for a in arrays["log10_prob"]]
    bo = [None if a is None else np.ascontiguousarray(a, dtype=np.float32)
          for a in arrays["log10_bow"]]
    counts = np.asarray([a.shape[0] for a in ids], dtype=np.int64)
    ptr = lambda a: None if a is None else a.ctypes.data_as(ctypes.c_void_p).value  # noqa: E731
    keep = (ids, pr, bo, counts)
    ids_p = (ctypes.c_void_p * order)(*[ptr(a) for a in ids])
    pr_p = (ctypes.c_void_p * order)(*[ptr(a) for a in pr])
    bo_p = (ctypes.c_void_p * order)(*[ptr(a) for a in bo])
    return order, counts.ctypes.data_as(ctypes.c_void_p), ids_p, pr_p, bo_p, keep


def ctcbeam_lm_build(arrays: dict, host_only: bool = False) -> LM:
    """Build an LM from ARPA-style arrays: dict(order, V, ids=[int32 [n_m, m]],
    log10_prob=[f32 [n_m]], log10_bow=[f32 [n_m] or None])."""
    lib = _load()
    order, counts, ids_p, pr_p, bo_p, keep = _lm_args(arrays)
    out = ctypes.c_void_p()
    fn = lib.ctcbeam_lm_build_host if host_only else lib.ctcbeam_lm_build
    _check(fn(order, _size(arrays["V"], "V"), counts, ids_p, pr_p, bo_p, ctypes.byref(out)))
    del keep
    return LM(out.value, int(arrays["V"]))


def ctcbeam_lm_build_host(arrays: dict) -> LM:
    return ctcbeam_lm_build(arrays, host_only=True)


def ctcbeam_lm_build_arpa(path: str, vocab_size: int, host_only: bool = False) -> LM:
    lib = _load()
    fn = lib.ctcbeam_lm_build_arpa_host if host_only else lib.ctcbeam_lm_build_arpa
    out = ctypes.c_void_p()
    _check(fn(path.encode(), _size(vocab_size, "vocab_size"), ctypes.byref(out)))
    return LM(out.value, int(vocab_size))


def ctcbeam_lm_build_arpa_host(path: str, vocab_size: int) -> LM:
    return ctcbeam_lm_build_arpa(path, vocab_size, host_only=True)


def ctcbeam_boost_build(vocab_size: int, offsets, tokens, host_only: bool = False) -> Boost:
    lib = _load()
    off = np.ascontiguousarray(offsets, dtype=np.int32)
    tok = np.ascontiguousarray(tokens, dtype=np.int32)
    if tok.size == 0:
        tok = np.zeros(1, dtype=np.int32)
    out = ctypes.c_void_p()
    fn = lib.ctcbeam_boost_build_host if host_only else lib.ctcbeam_boost_build
    _check(fn(_size(vocab_size, "vocab_size"), _size(off.shape[0] - 1, "phrases"), off.ctypes.data_as(ctypes.c_void_p),
              tok.ctypes.data_as(ctypes.c_void_p), ctypes.byref(out)))
    return Boost(out.value, int(vocab_size))


def ctcbeam_boost_build_host(vocab_size: int, offsets, tokens) -> Boost:
    return ctcbeam_boost_build(vocab_size, offsets, tokens, host_only=True)


def ctcbeam_lm_tables(lm: LM) -> dict:
    """Copies of the LM's host tables (see ``ctcbeam_lm_view``)."""
    v = _LmView()
    _check(_load().ctcbeam_lm_tables(lm.handle, ctypes.byref(v)))

    def arr(ptr, n, dt):
        if n == 0:
            return np.zeros(0, dtype=dt)
        return np.ctypeslib.as_array(ctypes.cast(ptr, ctypes.POINTER(
            ctypes.c_uint32 if dt == np.uint32 else ctypes.c_float)), shape=(n,)).copy()

    states = arr(v.states, v.n_states * v.nlev * 3, np.uint32).reshape(v.n_states, v.nlev, 3)
    arcs = arr(v.arcs, v.n_arcs * 3, np.uint32).reshape(v.n_arcs, 3)
    uni = arr(v.unigram, v.vocab_size + 1, np.float32)
    return dict(order=v.order, V=v.vocab_size, nlev=v.nlev, states=states, arcs=arcs, unigram=uni)


def ctcbeam_boost_tables(bt: Boost) -> dict:
    v = _BoostView()
    _check(_load().ctcbeam_boost_tables(bt.handle, ctypes.byref(v)))

    def arr(ptr, n):
        if n == 0:
            return np.zeros(0, dtype=np.uint32)
        return np.ctypeslib.as_array(ctypes.cast(ptr, ctypes.POINTER(ctypes.c_uint32)),
                                     shape=(n,)).copy()

    return dict(V=v.vocab_size, nodes=arr(v.nodes, v.n_nodes * 4).reshape(v.n_nodes, 4),
                list=arr(v.list, v.n_list * 2).reshape(v.n_list, 2),
                root_key=arr(v.root_key, v.vocab_size))


def ctcbeam_workspace_bytes(B: int, T: int, K: int) -> int:
    return int(_load().ctcbeam_workspace_bytes(_size(B, "B"), _size(T, "T"), _size(K, "K")))


def _dptr(t, dtype, name, shape=None, device=None):
    import torch
    if t is None:
        return None
    if not isinstance(t, torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if device is not None and t.device != device:
        raise ValueError(f"{name} is on {t.device}, the inputs on {device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    return ctypes.c_void_p(t.data_ptr())


def _shape(logprobs):
    if logprobs.dim() != 3:
        raise ValueError("logprobs must be [B, T, V+1]")
    B, T, W = (_size(n, name) for n, name in zip(logprobs.shape, ("B", "T", "V+1")))
    return B, T, W - 1, logprobs.device


def _stream_handle(stream, dev):
    """Raw hipStream_t of ``stream``: None (torch's current stream on dev), a
    torch.cuda.Stream, or a raw handle."""
    if stream is None:
        return _torch.cuda.current_stream(dev).cuda_stream
    if isinstance(stream, _torch.cuda.Stream):
        return stream.cuda_stream
    return int(stream)


def _empty(shape, dtype, dev, stream, owned):
    """A new tensor for a launch on ``stream``, in memory of that stream: what
    torch's current stream has freed may still be in use by work queued there,
    which the launch does not wait for."""
    if stream is None:
        t = _torch.empty(shape, dtype=dtype, device=dev)
    else:
        if not isinstance(stream, _torch.cuda.Stream):
            stream = _torch.cuda.ExternalStream(int(stream), device=dev)
        with _torch.cuda.stream(stream):
            t = _torch.empty(shape, dtype=dtype, device=dev)
    owned.append(t)
    return t


def _launch(call, dev, stream, owned, given):
    """Run ``call(raw_stream)`` (one C entry point, returning its code) with
    the inputs' device current.  Tensors the binding allocated (``owned``)
    are recorded on torch's current stream where that is not the launch stream,
    so the caching allocator does not hand their memory to other work before
    the caller's is done with it.  The caller's outputs (``given``) count as
    written in place, so that a backward pass that saved one before fails
    instead of reading what is there now."""
    with _torch.cuda.device(dev):
        raw = _stream_handle(stream, dev)
        _check(call(ctypes.c_void_p(raw)))
        if owned and stream is not None:
            current = _torch.cuda.current_stream(dev)
            if raw != current.cuda_stream:
                for t in owned:
                    t.record_stream(current)
    if given:
        _torch.autograd.graph.increment_version(given)


def _handles(lm, boost):
    return (lm.handle if lm is not None else None, boost.handle if boost is not None else None)


def _take(t, name, given):
    """An output of the caller's.  Refused where torch would refuse it as an
    ``out=``: gradients flow through it, but not through this library's calls."""
    if isinstance(t, _torch.Tensor):
        if t.requires_grad and _torch.is_grad_enabled():
            raise ValueError(f"{name} requires a gradient, which does not flow through this call: detach it")
        given.append(t)


def _alloc(t, shape, dtype, name, dev, stream, owned, given):
    if t is None:
        return _empty(shape, dtype, dev, stream, owned)
    _take(t, name, given)
    return t


def ctcbeam_decode_ex(logprobs, lengths, K: int, alpha: float = 0.0, beta: float = 0.0,
                      boost_w: float = 0.0, lm: Optional[LM] = None,
                      boost: Optional[Boost] = None, workspace=None, out_tokens=None,
                      out_lengths=None, out_scores=None, stream=None,
                      theta: float = math.inf, stats=None, logsumexp: bool = False,
                      boost_rollback: bool = False, row_cache: bool = True,
                      repeat_score: bool = False):
    """Enqueue one decode on ``stream`` (default: torch's current stream on the
    inputs' device; a torch.cuda.Stream or a raw hipStream_t handle).

    logprobs: float32 [B, T, V+1] device tensor (blank = V); lengths: int32 [B].
    Outputs are allocated when not given.  ``row_cache=False`` sets
    CTCBEAM_FLAG_NO_ROW_CACHE (same results); ``repeat_score=True`` sets
    CTCBEAM_FLAG_REPEAT_SCORE.  Returns (tokens [B,T] int32
    with -1 padding, lengths [B] int32, scores [B] float32, workspace uint8)."""
    import torch
    lib = _load()
    B, T, V, dev = _shape(logprobs)
    K = _size(K, "K")
    owned, given = [], [] if stats is None else [stats]
    out_tokens = _alloc(out_tokens, (B, T), torch.int32, "out_tokens", dev, stream, owned, given)
    out_lengths = _alloc(out_lengths, (B,), torch.int32, "out_lengths", dev, stream, owned, given)
    out_scores = _alloc(out_scores, (B,), torch.float32, "out_scores", dev, stream, owned, given)
    workspace = _alloc(workspace, (max(ctcbeam_workspace_bytes(B, T, K), 1),), torch.uint8, "workspace", dev, stream, owned, given)
    o = _opts(theta, stats, B, logsumexp, boost_rollback, row_cache, dev, repeat_score)
    args = (_dptr(logprobs, torch.float32, "logprobs", None, dev),
            _dptr(lengths, torch.int32, "lengths", (B,), dev),
            B, T, V, K, float(alpha), float(beta), float(boost_w), *_handles(lm, boost),
            _dptr(workspace, torch.uint8, "workspace", None, dev), int(workspace.numel()),
            _dptr(out_tokens, torch.int32, "out_tokens", (B, T), dev),
            _dptr(out_lengths, torch.int32, "out_lengths", (B,), dev),
            _dptr(out_scores, torch.float32, "out_scores", (B,), dev))
    _launch(lambda st: lib.ctcbeam_decode_ex(*args, st, None if o is None else ctypes.byref(o)),
            dev, stream, owned, given)
    return out_tokens, out_lengths, out_scores, workspace


def ctcbeam_decode(logprobs, lengths, K: int, alpha: float = 0.0, beta: float = 0.0,
                   boost_w: float = 0.0, lm: Optional[LM] = None, boost: Optional[Boost] = None,
                   workspace=None, out_tokens=None, out_lengths=None, out_scores=None,
                   stream=None):
    """``ctcbeam_decode_ex`` without options (no pruning, no statistics)."""
    return ctcbeam_decode_ex(logprobs, lengths, K, alpha, beta, boost_w, lm, boost, workspace,
                             out_tokens, out_lengths, out_scores, stream)


def ctcbeam_decode_nbest(logprobs, lengths, K: int, alpha: float = 0.0, beta: float = 0.0,
                         boost_w: float = 0.0, lm: Optional[LM] = None,
                         boost: Optional[Boost] = None, workspace=None, nbest_tokens=None,
                         nbest_lengths=None, nbest_scores=None, stream=None,
                         theta: float = math.inf, stats=None, logsumexp: bool = False,
                         boost_rollback: bool = False, row_cache: bool = True,
                         repeat_score: bool = False):
    """Enqueue one N-best decode on ``stream`` (as for ``ctcbeam_decode_ex``).

    Same inputs as ``ctcbeam_decode_ex``.  Returns (tokens [B,K,T] int32 with
    -1 padding, lengths [B,K] int32, scores [B,K] float32 descending,
    workspace uint8); row 0 of each utterance is the 1-best result."""
    import torch
    lib = _load()
    B, T, V, dev = _shape(logprobs)
    K = _size(K, "K")
    owned, given = [], [] if stats is None else [stats]
    nbest_tokens = _alloc(nbest_tokens, (B, K, T), torch.int32, "nbest_tokens", dev, stream, owned, given)
    nbest_lengths = _alloc(nbest_lengths, (B, K), torch.int32, "nbest_lengths", dev, stream, owned, given)
    nbest_scores = _alloc(nbest_scores, (B, K), torch.float32, "nbest_scores", dev, stream, owned, given)
    workspace = _alloc(workspace, (max(ctcbeam_workspace_bytes(B, T, K), 1),), torch.uint8, "workspace", dev, stream, owned, given)
    o = _opts(theta, stats, B, logsumexp, boost_rollback, row_cache, dev, repeat_score)
    args = (_dptr(logprobs, torch.float32, "logprobs", None, dev),
            _dptr(lengths, torch.int32, "lengths", (B,), dev),
            B, T, V, K, float(alpha), float(beta), float(boost_w), *_handles(lm, boost),
            _dptr(workspace, torch.uint8, "workspace", None, dev), int(workspace.numel()),
            _dptr(nbest_tokens, torch.int32, "nbest_tokens", (B, K, T), dev),
            _dptr(nbest_lengths, torch.int32, "nbest_lengths", (B, K), dev),
            _dptr(nbest_scores, torch.float32, "nbest_scores", (B, K), dev))
    _launch(lambda st: lib.ctcbeam_decode_nbest(*args, st, None if o is None else ctypes.byref(o)),
            dev, stream, owned, given)
    return nbest_tokens, nbest_lengths, nbest_scores, workspace


def ctcbeam_greedy_decode(logprobs, lengths, alpha: float = 0.0, beta: float = 0.0,
                          boost_w: float = 0.0, lm: Optional[LM] = None,
                          boost: Optional[Boost] = None, workspace=None, out_tokens=None,
                          out_lengths=None, out_scores=None, stream=None, stats=None,
                          boost_rollback: bool = False, repeat_score: bool = False):
    """Enqueue one greedy decode with fusion (Algorithm 1 with one hypothesis)
    on ``stream``.  Returns (tokens [B,T] int32 with -1 padding, lengths [B],
    scores [B], workspace uint8)."""
    import torch
    lib = _load()
    B, T, V, dev = _shape(logprobs)
    owned, given = [], [] if stats is None else [stats]
    out_tokens = _alloc(out_tokens, (B, T), torch.int32, "out_tokens", dev, stream, owned, given)
    out_lengths = _alloc(out_lengths, (B,), torch.int32, "out_lengths", dev, stream, owned, given)
    out_scores = _alloc(out_scores, (B,), torch.float32, "out_scores", dev, stream, owned, given)
    workspace = _alloc(workspace, (max(ctcbeam_workspace_bytes(B, 0, 1), 1),), torch.uint8, "workspace", dev, stream, owned, given)
    o = _opts(math.inf, stats, B, False, boost_rollback, True, dev, repeat_score)
    args = (_dptr(logprobs, torch.float32, "logprobs", None, dev),
            _dptr(lengths, torch.int32, "lengths", (B,), dev),
            B, T, V, float(alpha), float(beta), float(boost_w), *_handles(lm, boost),
            _dptr(workspace, torch.uint8, "workspace", None, dev), int(workspace.numel()),
            _dptr(out_tokens, torch.int32, "out_tokens", (B, T), dev),
            _dptr(out_lengths, torch.int32, "out_lengths", (B,), dev),
            _dptr(out_scores, torch.float32, "out_scores", (B,), dev))
    _launch(lambda st: lib.ctcbeam_greedy_decode(*args, st, None if o is None else ctypes.byref(o)),
            dev, stream, owned, given)
    return out_tokens, out_lengths, out_scores, workspace


NOALLOC_MAX_WORKSPACE = 16 << 20   # CTCBEAM_NOALLOC_MAX_WORKSPACE


def ctcbeam_decode_noalloc(logprobs, lengths, K: int, alpha: float = 0.0, beta: float = 0.0,
                           boost_w: float = 0.0, lm: Optional[LM] = None,
                           boost: Optional[Boost] = None, out_tokens=None, out_lengths=None,
                           out_scores=None, stream=None, theta: float = math.inf, stats=None,
                           logsumexp: bool = False, boost_rollback: bool = False,
                           row_cache: bool = True, repeat_score: bool = False):
    """``ctcbeam_decode_ex`` through the entry point that allocates nothing:
    the workspace is the library's fixed per-device array (calls that overlap
    on one device race).  Pass the outputs to keep the call allocation-free
    (they are allocated here when not given).  Returns (tokens, lengths,
    scores)."""
    import torch
    lib = _load()
    B, T, V, dev = _shape(logprobs)
    K = _size(K, "K")
    owned, given = [], [] if stats is None else [stats]
    out_tokens = _alloc(out_tokens, (B, T), torch.int32, "out_tokens", dev, stream, owned, given)
    out_lengths = _alloc(out_lengths, (B,), torch.int32, "out_lengths", dev, stream, owned, given)
    out_scores = _alloc(out_scores, (B,), torch.float32, "out_scores", dev, stream, owned, given)
    o = _opts(theta, stats, B, logsumexp, boost_rollback, row_cache, dev, repeat_score)
    args = (_dptr(logprobs, torch.float32, "logprobs", None, dev),
            _dptr(lengths, torch.int32, "lengths", (B,), dev),
            B, T, V, K, float(alpha), float(beta), float(boost_w), *_handles(lm, boost),
            _dptr(out_tokens, torch.int32, "out_tokens", (B, T), dev),
            _dptr(out_lengths, torch.int32, "out_lengths", (B,), dev),
            _dptr(out_scores, torch.float32, "out_scores", (B,), dev))
    _launch(lambda st: lib.ctcbeam_decode_noalloc(*args, st, None if o is None else ctypes.byref(o)),
            dev, stream, owned, given)
    return out_tokens, out_lengths, out_scores


def ctcbeam_query_status(workspace, stream=None) -> int:
    """Status bits (ORed over utterances) of the last decode that used
    ``workspace``; synchronises ``stream`` (default: torch's current one)."""
    lib = _load()
    dev = workspace.device
    bits = ctypes.c_uint32(0)
    with _torch.cuda.device(dev):
        raw = _stream_handle(stream, dev)
        _check(lib.ctcbeam_query_status(ctypes.c_void_p(workspace.data_ptr()),
                                        ctypes.c_void_p(raw), ctypes.byref(bits)))
    return int(bits.value)


def decode(logprobs, lengths, K: int, **kw):
    """Convenience: returns (tokens, lengths, scores) device tensors."""
    tok, ln, sc, _ = ctcbeam_decode_ex(logprobs, lengths, K, **kw)
    return tok, ln, sc


def decode_nbest(logprobs, lengths, K: int, **kw):
    """Convenience: returns N-best (tokens [B,K,T], lengths [B,K], scores [B,K])."""
    tok, ln, sc, _ = ctcbeam_decode_nbest(logprobs, lengths, K, **kw)
    return tok, ln, sc


# ------------------------------------------------ operators on rows of scores

class _Rows(ctypes.Structure):
    _fields_ = [("data", ctypes.c_void_p), ("type", ctypes.c_int), ("B", ctypes.c_int),
                ("T", ctypes.c_int), ("W", ctypes.c_int), ("stride_b", ctypes.c_int64),
                ("stride_t", ctypes.c_int64), ("lengths", ctypes.c_void_p)]


class _ProcessOpts(ctypes.Structure):
    _fields_ = [("history", ctypes.c_void_p), ("history_size", ctypes.c_int),
                ("history_stride", ctypes.c_int64), ("history_lengths", ctypes.c_void_p),
                ("penalties", ctypes.c_void_p), ("repetition", ctypes.c_float),
                ("presence", ctypes.c_float), ("frequency", ctypes.c_float),
                ("bias", ctypes.c_void_p), ("bias_stride", ctypes.c_int64),
                ("mask", ctypes.c_void_p), ("mask_stride_b", ctypes.c_int64),
                ("mask_stride_t", ctypes.c_int64), ("normalize", ctypes.c_int),
                ("reserved", ctypes.c_int * 3)]


_TYPES = {}   # CTCBEAM_TYPE_* by torch's type


def _need(t, dtype, name, dev):
    if not isinstance(t, _torch.Tensor) or not t.is_cuda:
        raise TypeError(f"{name} must be a device tensor")
    if t.device != dev:
        raise ValueError(f"{name} is on {t.device}, the inputs on {dev}")
    if dtype is not None and t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")


def _pointer(t, dtype, name, shape, dev):
    """Address of a contiguous device tensor (None stays None)."""
    if t is None:
        return None
    _need(t, dtype, name, dev)
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")
    return t.data_ptr()


def _rows_of(x, lengths, name):
    """(ctcbeam_rows, B, T, W, device) of scores [B, T, W] with adjacent labels."""
    _need(x, None, name, getattr(x, "device", None))
    if not _TYPES:
        _TYPES.update({_torch.float32: 0, _torch.float16: 1, _torch.bfloat16: 2})
    code = _TYPES.get(x.dtype)
    if code is None:
        raise TypeError(f"{name} must be float32, float16 or bfloat16, got {x.dtype}")
    if x.dim() != 3:
        raise ValueError(f"{name} must be [B, T, W]")
    B, T, W = x.shape
    if max(B, T, W) >= 1 << 31:
        _size(B, "B"), _size(T, "T"), _size(W, "W")
    sb, st, sl = x.stride()
    if sl != 1 and W > 1:
        raise ValueError(f"the labels of a row of {name} must be adjacent")
    dev = x.device
    return _Rows(x.data_ptr(), code, B, T, W, sb, st,
                 _pointer(lengths, _torch.int32, "lengths", (B,), dev)), B, T, W, dev


def _output(t, dtype, name, shape, dev, stream, owned, given):
    """(tensor, address) of an output: the given one, or a new one."""
    if t is None:
        t = _empty(shape, dtype, dev, stream, owned)
        return t, t.data_ptr()
    _take(t, name, given)
    return t, _pointer(t, dtype, name, shape, dev)


def _workspace(workspace, need, dev, stream, owned):
    """(tensor or None, address, bytes): the given workspace, or one of ``need`` bytes."""
    if workspace is None:
        if not need:
            return None, None, 0
        workspace = _empty((need,), _torch.uint8, dev, stream, owned)
        return workspace, workspace.data_ptr(), need
    return workspace, _dptr(workspace, _torch.uint8, "workspace", None, dev), workspace.numel()


def ctcbeam_process_logits(logits, lengths=None, history=None, history_lengths=None, penalties=None,
                           repetition: float = 1.0, presence: float = 0.0, frequency: float = 0.0,
                           bias=None, mask=None, normalize: bool = True, out=None, workspace=None,
                           stream=None):
    """Penalties for repeated tokens, biases and grammar masks on logits, on
    ``stream``: what the decode calls take as ``logprobs``.

    logits: float32, float16 or bfloat16 [B, T, W] with adjacent labels (any
    utterance and frame strides); lengths: int32 [B].  history: int32 [B, H],
    the tokens emitted before (ids outside 0..W-1 are ignored), of which the
    first ``history_lengths`` [B] count; penalties: float32 [B, 3] (repetition,
    presence, frequency of each utterance), else the three numbers.  bias:
    float32 [W] or [B, W].  mask: int32 [ceil(W/32)], [B, ceil(W/32)] or
    [B, T, ceil(W/32)], bit c%32 of word c/32 set where label c is allowed.
    ``normalize=False`` leaves out the log-softmax.  Frames behind an
    utterance's length are left as they were in ``out``, which may be the
    logits themselves where those are contiguous float32 (detached, if torch
    records a gradient for them).  No gradient flows through this call.
    Returns (float32 [B, T, W], workspace or None)."""
    lib = _load()
    rows, B, T, W, dev = _rows_of(logits, lengths, "logits")
    owned, given = [], []
    out, op = _output(out, _torch.float32, "out", (B, T, W), dev, stream, owned, given)
    o = _ProcessOpts(repetition=repetition, presence=presence, frequency=frequency, normalize=bool(normalize))
    if history is not None:
        _need(history, _torch.int32, "history", dev)
        if history.dim() != 2 or history.shape[0] != B:
            raise ValueError(f"history must be [{B}, H], got {tuple(history.shape)}")
        H = _size(history.shape[1], "history_size")
        if H > 1 and history.stride(1) != 1:
            raise ValueError("the tokens of a row of history must be adjacent")
        if H:
            o.history, o.history_size, o.history_stride = history.data_ptr(), H, history.stride(0)
            o.history_lengths = _pointer(history_lengths, _torch.int32, "history_lengths", (B,), dev)
    elif history_lengths is not None:
        raise ValueError("history_lengths without history")
    if penalties is not None:
        o.penalties = _pointer(penalties, _torch.float32, "penalties", (B, 3), dev)
    if bias is not None:
        _need(bias, _torch.float32, "bias", dev)
        if bias.shape != (W,) and bias.shape != (B, W):
            raise ValueError(f"bias must be [{W}] or [{B}, {W}], got {tuple(bias.shape)}")
        if W > 1 and bias.stride(-1) != 1:
            raise ValueError("the labels of a row of bias must be adjacent")
        o.bias, o.bias_stride = bias.data_ptr(), 0 if bias.dim() == 1 else bias.stride(0)
    if mask is not None:
        _need(mask, _torch.int32, "mask", dev)
        words = (W + 31) // 32
        if mask.shape != (words,) and mask.shape != (B, words) and mask.shape != (B, T, words):
            raise ValueError(f"mask must be [{words}], [{B}, {words}] or [{B}, {T}, {words}], got {tuple(mask.shape)}")
        if words > 1 and mask.stride(-1) != 1:
            raise ValueError("the words of a row of mask must be adjacent")
        o.mask = mask.data_ptr()
        o.mask_stride_b = mask.stride(0) if mask.dim() > 1 else 0
        o.mask_stride_t = mask.stride(1) if mask.dim() > 2 else 0
    workspace, wp, wn = _workspace(workspace, lib.ctcbeam_process_workspace_bytes(B, T, W), dev, stream, owned)
    _launch(lambda st: lib.ctcbeam_process_logits(ctypes.byref(rows), ctypes.byref(o), op, wp, wn, st),
            dev, stream, owned, given)
    return out, workspace


def ctcbeam_top_logits(logits, k: int, lengths=None, temperature: float = 1.0, values=None, ids=None,
                       tail=None, workspace=None, stream=None):
    """The k largest logits of every row, on ``stream``: (values float32
    [B, T, k] descending, ids int32 [B, T, k], tail float32 [B, T], workspace
    or None), tail the log-sum of exp(logit / temperature) over the labels that
    are not listed.  Equal values: the lowest label first; frames behind an
    utterance's length get -inf, -1 and -inf.  No gradient flows through this
    call."""
    lib = _load()
    rows, B, T, W, dev = _rows_of(logits, lengths, "logits")
    k = _size(k, "k")
    owned, given = [], []
    kk = max(k, 0)
    values, vp = _output(values, _torch.float32, "values", (B, T, kk), dev, stream, owned, given)
    ids, ip = _output(ids, _torch.int32, "ids", (B, T, kk), dev, stream, owned, given)
    tail, tp = _output(tail, _torch.float32, "tail", (B, T), dev, stream, owned, given)
    workspace, wp, wn = _workspace(workspace, lib.ctcbeam_top_workspace_bytes(B, T, W, k), dev, stream, owned)
    _launch(lambda st: lib.ctcbeam_top_logits(ctypes.byref(rows), k, temperature, vp, ip, tp, wp, wn, st),
            dev, stream, owned, given)
    return values, ids, tail, workspace


def ctcbeam_distill(student, values, ids, tail=None, lengths=None, temperature: float = 1.0, weights=1.0,
                    want_loss: bool = True, want_grad: bool = True, loss=None, grad=None, workspace=None,
                    stream=None):
    """Distillation from a teacher's top logits, on ``stream``: the divergence
    of every frame (float32 [B, T], unweighted) and, in the same pass over the
    student's logits, ``weights`` (a number, or float32 [B, T] of any strides)
    times its gradient, of the student's type.

    student: float32, float16 or bfloat16 [B, T, W]; values, ids, tail: as
    ``ctcbeam_top_logits`` gives them (``tail=None``: the list is renormalised).
    ``grad`` may have any utterance and frame strides whose rows do not
    overlap.  Returns (loss or None, grad or None, workspace or None)."""
    lib = _load()
    rows, B, T, W, dev = _rows_of(student, lengths, "student")
    owned, given = [], []
    _need(values, _torch.float32, "values", dev)
    if values.dim() != 3:
        raise ValueError("values must be [B, T, k]")
    k = _size(values.shape[2], "k")
    vp = _pointer(values, _torch.float32, "values", (B, T, k), dev)
    ip = _pointer(ids, _torch.int32, "ids", (B, T, k), dev)
    tp = _pointer(tail, _torch.float32, "tail", (B, T), dev)
    if ip is None:
        raise TypeError("ids must be a device tensor")
    weight, w, wsb, wst = 1.0, None, 0, 0
    if isinstance(weights, _torch.Tensor):
        _need(weights, _torch.float32, "weights", dev)
        if weights.shape != (B, T):
            raise ValueError(f"weights must have shape {(B, T)}, got {tuple(weights.shape)}")
        w, (wsb, wst) = weights.data_ptr(), weights.stride()
    elif weights is not None:
        weight = float(weights)
    lp = gp = None
    gsb = gst = 0
    if want_loss or loss is not None:
        loss, lp = _output(loss, _torch.float32, "loss", (B, T), dev, stream, owned, given)
    if grad is not None:
        _need(grad, student.dtype, "grad", dev)
        if grad.shape != (B, T, W):
            raise ValueError(f"grad must have shape {(B, T, W)}, got {tuple(grad.shape)}")
        gsb, gst, gsl = grad.stride()
        if W > 1 and gsl != 1:
            raise ValueError("the labels of a row of grad must be adjacent")
        _take(grad, "grad", given)
        gp = grad.data_ptr()
    elif want_grad:
        grad, gp = _output(None, student.dtype, "grad", (B, T, W), dev, stream, owned, given)
        gsb, gst = T * W, W
    workspace, wp, wn = _workspace(workspace, lib.ctcbeam_distill_workspace_bytes(B, T, W), dev, stream, owned)
    _launch(lambda st: lib.ctcbeam_distill(ctypes.byref(rows), vp, ip, tp, k, temperature, w, wsb, wst, weight,
                                           lp, gp, gsb, gst, wp, wn, st), dev, stream, owned, given)
    return loss, grad, workspace


def process_logits(logits, lengths=None, **kw):
    """Convenience: the processed scores alone."""
    return ctcbeam_process_logits(logits, lengths, **kw)[0]


def top_logits(logits, k: int, lengths=None, **kw):
    """Convenience: returns (values, ids, tail)."""
    return ctcbeam_top_logits(logits, k, lengths, **kw)[:3]


def distill(student, values, ids, tail=None, lengths=None, **kw):
    """Convenience: returns (loss or None, grad or None)."""
    return ctcbeam_distill(student, values, ids, tail, lengths, **kw)[:2]


_distill_function = None


def distill_loss(student, values, ids, tail=None, lengths=None, temperature: float = 1.0):
    """The divergence of every frame (float32 [B, T]) as a function that torch
    differentiates with respect to ``student``; the teacher's list is a
    constant.  Forward and backward read the student's logits once each
    (``distill`` gives both in one pass where the frames' weights are known).
    Not for capture into a graph while ``student`` needs a gradient: there
    ``distill`` gives loss and gradient without torch's bookkeeping, whose
    nodes belong to the stream they were made on."""
    import torch
    global _distill_function
    if _distill_function is None:
        class Distill(torch.autograd.Function):
            @staticmethod
            def forward(ctx, student, values, ids, tail, lengths, temperature):
                ctx.save_for_backward(student, values, ids, tail, lengths)
                ctx.temperature = temperature
                return distill(student, values, ids, tail, lengths, temperature=temperature, want_grad=False)[0]

            @staticmethod
            @torch.autograd.function.once_differentiable
            def backward(ctx, upstream):
                student, values, ids, tail, lengths = ctx.saved_tensors
                grad = distill(student, values, ids, tail, lengths, temperature=ctx.temperature,
                               weights=upstream, want_loss=False)[1]
                return grad, None, None, None, None, None
        _distill_function = Distill
    for name, t in (("values", values), ("tail", tail)):
        if isinstance(t, torch.Tensor) and t.requires_grad:
            raise ValueError(f"{name} is a constant of the loss: detach it")
    if isinstance(student, torch.Tensor) and student.requires_grad and torch.is_grad_enabled() and \
            student.is_cuda and torch.cuda.is_current_stream_capturing():
        raise RuntimeError("distill_loss is not captured with a gradient: use distill, which gives loss and gradient")
    return _distill_function.apply(student, values, ids, tail, lengths, float(temperature))
