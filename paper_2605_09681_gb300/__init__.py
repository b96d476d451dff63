"""Forcing-KV hot path on GB300: hybrid KV-cache compression (static structural pruning,
segment-similarity pruning) and chunk attention over the compressed cache; and a paged 8-bit cache of
many sequences (PagedKVCache) with the attention that reads it.

Every step runs in the CUDA kernels of libfk.so behind the C ABI of include/fk.h; this
module only marshals arguments (torch tensors for device memory and streams).
"""
from __future__ import annotations

import ctypes

import numpy as np

from . import _lib as L
from ._lib import FkError, KERNEL_KINDS, STATUS_NAMES

__all__ = ["ForcingKVCache", "PagedKVCache", "FkError", "KERNEL_KINDS", "STATUS_NAMES", "load_library",
           "head_profile", "classify_heads", "quantize_e4m3", "stream_read"]


def load_library():
    return L.load()


def _check(status: int, call: str) -> None:
    if status != L.FK_OK:
        raise FkError(status, call)


def _ptr(x) -> int:
    """Address of a bf16 tensor (torch, any device) or a uint16 numpy array of bf16 bits."""
    import torch
    if isinstance(x, torch.Tensor):
        if x.dtype != torch.bfloat16 or not x.is_contiguous():
            raise ValueError("expected a contiguous torch.bfloat16 tensor")
        return x.data_ptr()
    if isinstance(x, np.ndarray):
        if x.dtype != np.uint16 or not x.flags["C_CONTIGUOUS"]:
            raise ValueError("expected a C-contiguous uint16 array of bf16 bit patterns")
        return x.ctypes.data
    raise TypeError("unsupported tensor type %r" % type(x))


def _numel(x) -> int:
    return x.numel() if hasattr(x, "numel") and not isinstance(x, np.ndarray) else x.size


def _stream(stream) -> int | None:
    if stream is None:
        import torch
        if torch.cuda.is_initialized():
            # the current device's current stream without building a Stream object: 0.6 us a call,
            # torch.cuda.current_stream() 3.7
            try:
                return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
            except AttributeError:
                return torch.cuda.current_stream().cuda_stream
        if torch.cuda.is_available():
            return torch.cuda.current_stream().cuda_stream
        return None
    return getattr(stream, "cuda_stream", stream)


def head_profile(Q, K, n_generate: int, n_sink: int, n_transition: int, mass=None, status=None,
                 stream=None):
    """Offline head profiling (Sec. 4.1, Eq. 1) through fk_head_profile.

    Q [Nq, H, D] and K [Nk, H, D]: contiguous torch.bfloat16 CUDA tensors, keys ordered
    [generated | sink | other history | transition].  Adds each head's attention mass
    {A_Total, A_Generate, A_Transition, A_Sink} to `mass` (float64 [H, 4] on the device,
    created zeroed when None) and returns (mass, status); status is an int32 device tensor
    whose nonzero value means a bounded device wait expired."""
    import torch
    nq, H, D = Q.shape
    nk = K.shape[0]
    if tuple(K.shape[1:]) != (H, D):
        raise ValueError("Q and K disagree on heads / head_dim")
    # two zeroed tensors: a small window is paced by the host, and slicing both out of one costs it more than
    # a second fill (8 heads, 534 queries, 1246 keys: 31 us a call back to back, 37 with one buffer; a 480P window,
    # which the device paces, 383 against 379, but 429 against 442 for a first call)
    if mass is None:
        mass = torch.zeros((H, 4), dtype=torch.float64, device=Q.device)
    if status is None:
        status = torch.zeros(1, dtype=torch.int32, device=Q.device)
    lib = L.load()
    _check(lib.fk_head_profile(_ptr(Q), _ptr(K), nq, nk, H, D, n_generate, n_sink, n_transition,
                               mass.data_ptr(), status.data_ptr(), _stream(stream)),
           "fk_head_profile")
    return mass, status


def quantize_e4m3(X, row_scaled: bool, q8=None, exps=None, stream=None):
    """E4M3 codes of a bf16 CUDA tensor [..., dim] as the FP8 attention path forms them
    (fk_quantize_e4m3): row_scaled=True scales each row by its power-of-two exponent (queries),
    False rounds unscaled (keys).  Returns (q8 uint8 tensor of X's shape, int8 exponents per
    row or None)."""
    import torch
    dim = X.shape[-1]
    rows = X.numel() // dim if dim else 0
    if q8 is None:
        q8 = torch.empty(X.shape, dtype=torch.uint8, device=X.device)
    if row_scaled and exps is None:
        exps = torch.empty(rows, dtype=torch.int8, device=X.device)
    lib = L.load()
    _check(lib.fk_quantize_e4m3(_ptr(X), rows, dim, 1 if row_scaled else 0, q8.data_ptr(),
                                exps.data_ptr() if exps is not None else None, _stream(stream)),
           "fk_quantize_e4m3")
    return q8, exps


def stream_read(X, nbytes: int | None = None, stream=None) -> None:
    """Read the first `nbytes` (default: all) of a CUDA tensor once (fk_stream_read): the
    event-timed floor of a launch that must read that many bytes."""
    if not X.is_contiguous():
        raise ValueError("expected a contiguous tensor")
    n = X.numel() * X.element_size() if nbytes is None else int(nbytes)
    if n > X.numel() * X.element_size():
        raise ValueError("nbytes exceeds the tensor")
    _check(L.load().fk_stream_read(X.data_ptr(), n, _stream(stream)), "fk_stream_read")


def classify_heads(mass, alpha: float = 0.8) -> np.ndarray:
    """Eq. 1 on masses [H, 4] (host copy): 1 = static, 0 = dynamic (fk_classify_heads)."""
    m = np.ascontiguousarray(np.asarray(mass, dtype=np.float64))
    H = m.shape[0]
    out = np.zeros(H, dtype=np.uint8)
    lib = L.load()
    _check(lib.fk_classify_heads(m.ctypes.data_as(ctypes.POINTER(ctypes.c_double)), H,
                                 int(round(alpha * 1000)),
                                 out.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8))),
           "fk_classify_heads")
    return out


class ForcingKVCache:
    """One Forcing-KV cache (all layers of a model) on one GPU.

    Tensors are bf16 [tokens, n_heads, head_dim]; device or host memory.  Calls are
    asynchronous on `stream` (default: torch's current stream)."""

    def __init__(self, *, n_layers, n_heads, head_dim, tokens_per_frame, frames_per_chunk,
                 n_sink_frames, window_frames, n_segments, keep_budget_permille,
                 head_is_static, select_scope="per_frame", score_source="per_head",
                 incremental=False, max_history_frames=64, device=0, selection="similarity",
                 select_seed=0, static_drop_anchor=False, attn_precision="bf16"):
        self._lib = L.load()
        self._h = ctypes.c_void_p()
        hm = np.ascontiguousarray(np.asarray(head_is_static, dtype=np.uint8).reshape(-1))
        if hm.size != n_layers * n_heads:
            raise ValueError("head_is_static must have n_layers * n_heads entries")
        self._map = hm
        self.cfg = L.FkConfig(
            n_layers, n_heads, head_dim, tokens_per_frame, frames_per_chunk, n_sink_frames,
            window_frames, n_segments, keep_budget_permille,
            {"per_frame": L.FK_SCOPE_PER_FRAME, "pooled": L.FK_SCOPE_POOLED}[select_scope],
            {"per_head": L.FK_SCORE_PER_HEAD, "layer0_pooled": L.FK_SCORE_LAYER0_POOLED}[score_source],
            1 if incremental else 0, max_history_frames, device,
            hm.ctypes.data_as(ctypes.POINTER(ctypes.c_uint8)),
            L.FK_SELECT[selection], select_seed & 0xFFFFFFFF, 1 if static_drop_anchor else 0,
            L.FK_ATTN[attn_precision])
        self.n_layers, self.n_heads, self.head_dim = n_layers, n_heads, head_dim
        self.F, self.C, self.n_segments = tokens_per_frame, frames_per_chunk, n_segments
        self.device = device
        _check(self._lib.fk_create(ctypes.byref(self.cfg), ctypes.byref(self._h)), "fk_create")

    @classmethod
    def from_workload(cls, w, head_is_static, device=0, **over):
        kw = dict(n_layers=w.n_layers, n_heads=w.n_heads, head_dim=w.head_dim,
                  tokens_per_frame=w.tokens_per_frame, frames_per_chunk=w.frames_per_chunk,
                  n_sink_frames=w.n_sink_frames, window_frames=w.window_frames,
                  n_segments=w.n_segments, keep_budget_permille=w.keep_budget_permille,
                  head_is_static=head_is_static, select_scope=w.select_scope,
                  score_source=w.score_source, incremental=w.incremental,
                  max_history_frames=max(1, w.max_history_frames()), device=device,
                  selection=w.selection, select_seed=w.select_seed,
                  static_drop_anchor=w.static_drop_anchor, attn_precision=w.attn_precision)
        kw.update(over)
        return cls(**kw)

    # ---- lifetime
    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self._lib.fk_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    # ---- cache updates
    def append_frames(self, layer, K, V, stream=None):
        nf = _numel(K) // (self.F * self.n_heads * self.head_dim)
        _check(self._lib.fk_append_frames(self._h, layer, _ptr(K), _ptr(V), nf, _stream(stream)),
               "fk_append_frames")

    def append_chunk(self, layer, K, V, stream=None):
        _check(self._lib.fk_append_chunk(self._h, layer, _ptr(K), _ptr(V), _stream(stream)),
               "fk_append_chunk")

    def set_current(self, layer, K, V, stream=None):
        _check(self._lib.fk_set_current(self._h, layer, _ptr(K), _ptr(V), _stream(stream)),
               "fk_set_current")

    def compress(self, stream=None):
        _check(self._lib.fk_compress(self._h, _stream(stream)), "fk_compress")

    def attend(self, layer, Q, O=None, stream=None):
        if O is None:
            import torch
            O = torch.empty_like(Q)
        _check(self._lib.fk_attend(self._h, layer, _ptr(Q), _ptr(O), _stream(stream)), "fk_attend")
        return O

    # ---- inspection
    def kept(self, layer, head, stream=None) -> list:
        n = ctypes.c_int(0)
        st = self._lib.fk_get_kept(self._h, layer, head, None, 0, ctypes.byref(n), _stream(stream))
        if n.value == 0:
            _check(st, "fk_get_kept")
            return []
        buf = (ctypes.c_int32 * n.value)()
        _check(self._lib.fk_get_kept(self._h, layer, head, buf, n.value, ctypes.byref(n),
                                     _stream(stream)), "fk_get_kept")
        return list(buf)

    def scores(self, layer, head, stream=None):
        """(first_frame, fp32 array [n_frames, n_segments]) of the scoreable frames."""
        first, nfr = ctypes.c_int(0), ctypes.c_int(0)
        cap = 1 << 16
        buf = np.zeros(cap, dtype=np.float32)
        _check(self._lib.fk_get_scores(self._h, layer, head,
                                       buf.ctypes.data_as(ctypes.POINTER(ctypes.c_float)), cap,
                                       ctypes.byref(first), ctypes.byref(nfr), _stream(stream)),
               "fk_get_scores")
        return first.value, buf[: nfr.value * self.n_segments].reshape(nfr.value, self.n_segments).copy()

    def key_count(self, layer, head) -> int:
        n = ctypes.c_int(0)
        _check(self._lib.fk_key_count(self._h, layer, head, ctypes.byref(n)), "fk_key_count")
        return n.value

    def cache_bytes(self) -> int:
        return int(self._lib.fk_cache_bytes(self._h))

    def reserved_bytes(self) -> int:
        return int(self._lib.fk_reserved_bytes(self._h))

    def sync_status(self, stream=None) -> int:
        """Synchronize and return the device status (FK_OK, FK_ERR_RANGE, FK_ERR_TIMEOUT)."""
        return int(self._lib.fk_sync_status(self._h, _stream(stream)))

    # ---- timing
    def profile_enable(self, on=True):
        _check(self._lib.fk_profile_enable(self._h, 1 if on else 0), "fk_profile_enable")

    def profile_reset(self):
        _check(self._lib.fk_profile_reset(self._h), "fk_profile_reset")

    def profile_read(self, kind: str):
        ms, n = ctypes.c_double(0), ctypes.c_int64(0)
        _check(self._lib.fk_profile_read(self._h, KERNEL_KINDS[kind], ctypes.byref(ms),
                                         ctypes.byref(n)), "fk_profile_read")
        return ms.value, n.value

    def wait_selftest(self, limit_us: int = 20000, stream=None) -> None:
        """Run the bounded-wait self-test (fk_wait_selftest): the next sync_status() reports
        FK_ERR_TIMEOUT."""
        _check(self._lib.fk_wait_selftest(self._h, int(limit_us), _stream(stream)), "fk_wait_selftest")

    def force_attention_plan(self, query_tiles: int = 0, kv_splits: int = 0) -> None:
        """Fix the attention's query tiles per CTA and key splits, for tests and measurements
        (fk_force_attention_plan); 0, 0: chosen by the key counts."""
        _check(self._lib.fk_force_attention_plan(self._h, int(query_tiles), int(kv_splits)),
               "fk_force_attention_plan")

    def set_host_overlap(self, on: bool = True) -> None:
        """Overlap host transfers with queued work (see fk_set_host_overlap): host inputs must
        be final at call time; host outputs are complete after wait_outputs() (or
        sync_status()) and a synchronization of the stream."""
        _check(self._lib.fk_set_host_overlap(self._h, 1 if on else 0), "fk_set_host_overlap")

    def wait_outputs(self, stream=None) -> None:
        """Make the stream wait for pending host-output copies (fk_wait_outputs)."""
        _check(self._lib.fk_wait_outputs(self._h, _stream(stream)), "fk_wait_outputs")

    def launch_count(self) -> int:
        return int(self._lib.fk_launch_count(self._h))


def _ints(values, n=None):
    """A ctypes array of 32-bit whole numbers."""
    v = [int(x) for x in values]
    if n is not None and len(v) != n:
        raise ValueError("expected %d numbers, got %d" % (n, len(v)))
    if any(not -2 ** 31 <= x < 2 ** 31 for x in v):
        raise ValueError("numbers must fit 32 bits")
    return (ctypes.c_int32 * len(v))(*v)


class PagedKVCache:
    """Keys and values of many sequences in pages of E4M3 codes, one power-of-two scale for each page and
    head (fk_paged_*), on one GPU.

        cache.step(seqs, n_new)                      # which sequences append how many tokens
        for layer in range(n_layers):
            Q = cache.append(layer, K, V, cos, sin, Q=Q)   # keys and queries rotated, keys and values held
            O = cache.attend(layer, Q)

    Tensors are bf16 CUDA tensors [tokens, heads, head_dim], the step's sequences one after the other in its order;
    they may be slices of wider rows (a fused projection's output).  Calls are asynchronous on `stream`
    (default: torch's current stream of the cache's device), and tensors that they make are that stream's.  The step's
    tokens belong to their sequences from the next step on; until then append may be called again with other keys and
    values, which take their place."""

    def __init__(self, *, n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs,
                 max_seq_tokens, rope="half", device=0):
        self._lib = L.load()
        self._h = ctypes.c_void_p()
        self.cfg = L.FkPagedConfig(n_layers, n_q_heads, n_kv_heads, head_dim, page_tokens, n_pages, max_seqs,
                                   max_seq_tokens, L.FK_ROPE[rope], device)
        self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim = n_layers, n_q_heads, n_kv_heads, head_dim
        self.page_tokens, self.device = page_tokens, device
        import torch
        self._bf16, self._f32, self._rope = torch.bfloat16, torch.float32, L.FkRope()
        self._new = self._queries = 0
        self._count, self._dev = ctypes.byref(ctypes.c_int64(0)), torch.device("cuda", device)
        self._held = {}                              # tokens that a read of the current step gives
        _check(self._lib.fk_paged_create(ctypes.byref(self.cfg), ctypes.byref(self._h)), "fk_paged_create")

    # ---- lifetime
    def close(self):
        if getattr(self, "_h", None) and self._h.value:
            self._lib.fk_paged_destroy(self._h)
            self._h = ctypes.c_void_p()

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def __enter__(self):
        return self

    def __exit__(self, *exc):
        self.close()

    def _on(self, stream):
        if stream is None:
            import torch
            try:                                     # as _stream, of the cache's device
                return torch._C._cuda_getCurrentRawStream(self.device)
            except AttributeError:
                return torch.cuda.current_stream(self.device).cuda_stream
        return getattr(stream, "cuda_stream", stream)

    def _made(self, shape, stream):
        """An output tensor, of the memory of the stream that is to write it: the current stream may still have work
        queued on memory that it has given back."""
        import torch
        raw = self._on(stream)
        if raw == self._on(None):
            return torch.empty(shape, dtype=self._bf16, device=self._dev)
        own = torch.cuda.ExternalStream(raw, device=self._dev) if raw else torch.cuda.default_stream(self._dev)
        with torch.cuda.stream(own):
            return torch.empty(shape, dtype=self._bf16, device=self._dev)

    def _rows(self, x, tokens, heads, name):
        """(address, elements from token to token) of a [tokens, heads, head_dim] tensor.  (Few tensor properties are
        asked for: a small call is paced by the host.)"""
        D = self.head_dim
        if x.dtype is not self._bf16 or x.shape != (tokens, heads, D) or not x.is_cuda:
            raise ValueError("%s: expected a bf16 CUDA tensor of %d tokens (the step's) [%d, %d, %d], not %s %s"
                             % (name, tokens, tokens, heads, D, x.dtype, list(x.shape)))
        row, head, channel = x.stride()
        if tokens and (channel != 1 or (heads > 1 and head != D)):
            raise ValueError("%s: the heads of a token must lie contiguously" % name)
        return x.data_ptr(), row if tokens > 1 else heads * D

    # ---- steps
    def step(self, seqs, n_new, n_query=None, stream=None):
        """Begin a step: sequence seqs[i] appends n_new[i] tokens and asks n_query[i] queries (default: as
        many), which stand at its last positions."""
        s = _ints(seqs)
        n = _ints(n_new, len(s))
        q = None if n_query is None else _ints(n_query, len(s))
        _check(self._lib.fk_paged_step(self._h, len(s), s, n, q, self._on(stream)), "fk_paged_step")
        self._new = sum(n)
        self._queries = self._new if q is None else sum(q)
        self._held = {}

    def append(self, layer, K, V, cos=None, sin=None, positions=None, Q=None, Q_out=None, stream=None):
        """Append the step's keys and values to a layer, the keys rotated by the tables cos, sin [rows, dim / 2]
        (fp32) at rows `positions` (int32 [tokens]; default: each token's place in its sequence); without
        tables as they are.  With Q, the queries of the same tokens, returns them rotated (in Q_out, which
        may be Q)."""
        k, ks = self._rows(K, self._new, self.n_kv_heads, "K")
        v, vs = self._rows(V, self._new, self.n_kv_heads, "V")
        rope = q = o = None
        qs = os = 0
        if cos is not None:
            if sin is None or cos.dtype is not self._f32 or sin.dtype is not self._f32 or cos.dim() != 2 or \
                    cos.shape != sin.shape or not cos.is_contiguous() or not sin.is_contiguous():
                raise ValueError("cos, sin: expected contiguous fp32 tensors [rows, dim / 2]")
            rope = self._rope
            rope.rows, half = cos.shape
            rope.dim = 2 * half
            rope.cos, rope.sin, rope.positions = cos.data_ptr(), sin.data_ptr(), None
            if positions is not None:
                import torch
                if positions.dtype is not torch.int32 or positions.shape != (self._new,) or not positions.is_contiguous():
                    raise ValueError("positions: expected a contiguous int32 tensor [%d]" % self._new)
                rope.positions = positions.data_ptr()
            rope = ctypes.byref(rope)
        elif sin is not None or positions is not None:
            raise ValueError("sin and positions need cos")
        if Q is not None:
            q, qs = self._rows(Q, self._new, self.n_q_heads, "Q")
            if Q_out is None:
                import torch                         # (dense: rows of a wider tensor are not kept apart)
                Q_out = torch.empty_like(Q) if stream is None else self._made(Q.shape, stream)
                o, os = Q_out.data_ptr(), self.n_q_heads * self.head_dim
            else:
                o, os = self._rows(Q_out, self._new, self.n_q_heads, "Q_out")
        _check(self._lib.fk_paged_append(self._h, layer, k, ks, v, vs, rope, q, qs, o, os, self._on(stream)),
               "fk_paged_append")
        return Q_out

    def attend(self, layer, Q, O=None, causal=True, window=0, sinks=0, scale=None, stream=None):
        """Attention of the step's queries over what their sequences hold: query at position p sees key j when
        j <= p (causal) or any j, and under window > 0 only j > p - window or j < sinks; a query that sees
        none gives 0.  scale: default 1 / sqrt(head_dim)."""
        if scale is not None and not ctypes.c_float(scale).value > 0:      # (0 asks for the default)
            raise ValueError("scale must be positive in fp32")
        if window >= 2 ** 31 or sinks >= 2 ** 31:
            raise ValueError("window, sinks: at most 2^31 - 1")
        q, qs = self._rows(Q, self._queries, self.n_q_heads, "Q")
        if O is None:
            import torch
            O = torch.empty_like(Q) if stream is None else self._made(Q.shape, stream)
            o, os = O.data_ptr(), self.n_q_heads * self.head_dim
        else:
            o, os = self._rows(O, self._queries, self.n_q_heads, "O")
        _check(self._lib.fk_paged_attend(self._h, layer, q, qs, o, os, 1 if causal else 0, window, sinks,
                                         0.0 if scale is None else scale, self._on(stream)), "fk_paged_attend")
        return O

    def read(self, layer, whole=False, K=None, V=None, stream=None):
        """The held keys and values of the step's sequences as bf16 [tokens, n_kv_heads, head_dim]: all their
        tokens, or those from the start of the page that a sequence's first new token is in."""
        n = self._held.get(whole)
        if n is None:
            count = ctypes.c_int64(0)
            st = self._lib.fk_paged_read(self._h, layer, 1 if whole else 0, None, None, 0, ctypes.byref(count), None)
            if st != L.FK_OK and count.value == 0:
                _check(st, "fk_paged_read")
            n = self._held[whole] = count.value
        for x in (K, V):
            if x is not None:
                self._rows(x, n, self.n_kv_heads, "K, V")
                if not x.is_contiguous():
                    raise ValueError("K, V: expected contiguous tensors")
        shape = (n, self.n_kv_heads, self.head_dim)
        K = self._made(shape, stream) if K is None else K
        V = self._made(shape, stream) if V is None else V
        k, v = K.data_ptr(), V.data_ptr()
        _check(self._lib.fk_paged_read(self._h, layer, 1 if whole else 0, k, v, n, self._count, self._on(stream)),
               "fk_paged_read")
        return K, V

    def drop(self, seq):
        """End the current step and empty a sequence: its pages are free for the next step."""
        _check(self._lib.fk_paged_drop(self._h, seq), "fk_paged_drop")
        self._new = self._queries = 0
        self._held = {}

    # ---- inspection
    def length(self, seq) -> int:
        return int(self._lib.fk_paged_length(self._h, seq))

    def free_pages(self) -> int:
        return int(self._lib.fk_paged_free_pages(self._h))

    def reserved_bytes(self) -> int:
        return int(self._lib.fk_paged_reserved_bytes(self._h))

    def launch_count(self) -> int:
        return int(self._lib.fk_paged_launch_count(self._h))

    def sync_status(self, stream=None) -> int:
        """Synchronize and return the device status (FK_OK, FK_ERR_RANGE, FK_ERR_TIMEOUT)."""
        return int(self._lib.fk_paged_sync_status(self._h, self._on(stream)))
