"""ctypes binding of ``include/gsi.h`` (same names, argument marshalling only); the calls made once
per token go through an extension module (``csrc/torch_calls.cpp``), which does the same in a third of the time.

``Layer`` and ``Stack`` wrap a handle together with the torch tensors that back
its workspace; they add no computation.  If the CUDA library cannot be loaded
the import fails loudly: there is no fallback.
"""
from __future__ import annotations

import contextlib
import ctypes as C
import os

import torch

from . import build as _build

GSI_BF16, GSI_F32, GSI_F16 = 0, 1, 2
GSI_FLAG_NONE, GSI_FLAG_STATIC_PROJECTION, GSI_FLAG_DENSE, GSI_FLAG_FP8_IMAGE = 0, 1, 2, 4
GSI_MAX_MAPS, GSI_MAX_TOKENS = 8, 64
GSI_KV_MAX_SEQS, GSI_KV_MAX_DIM = 2048, 256

EXPORTED = [
    "gsi_status_string", "gsi_build_image", "gsi_workspace_bytes", "gsi_create",
    "gsi_forward", "gsi_forward_n", "gsi_forward_host", "gsi_forward_static", "gsi_extend_basis", "gsi_get_image", "gsi_get_image_fp8", "gsi_get_status",
    "gsi_set_spin_limit", "gsi_destroy", "gsi_stack_workspace_bytes", "gsi_stack_create", "gsi_stack_bind",
    "gsi_stack_set_mode", "gsi_stack_set_concurrent", "gsi_stack_is_persistent", "gsi_stack_set_trace", "gsi_stack_set_spin_limit", "gsi_stack_seek", "gsi_stack_step", "gsi_stack_launches_per_step",
    "gsi_stack_step_host", "gsi_stack_get_status", "gsi_stack_destroy",
    "gsi_kv_page_bytes", "gsi_kv_workspace_bytes", "gsi_kv_locate", "gsi_kv_create", "gsi_kv_plan", "gsi_kv_release",
    "gsi_kv_append", "gsi_kv_read", "gsi_kv_attend", "gsi_kv_attend_all", "gsi_kv_get_status", "gsi_kv_destroy",
]


class GsiDesc(C.Structure):
    _fields_ = [("d", C.c_int), ("k", C.c_int), ("n_maps", C.c_int),
                ("d_out", C.POINTER(C.c_int)), ("eps", C.c_float), ("max_tokens", C.c_int),
                ("p_dtype", C.c_int), ("flags", C.c_uint)]


class GsiStackIo(C.Structure):
    _fields_ = [("x", C.c_void_p), ("y", C.c_void_p)]


class GsiKvDesc(C.Structure):
    _fields_ = [(n, C.c_int) for n in ("n_heads", "head_dim", "page_tokens", "n_pages", "max_seqs", "max_pages", "max_tokens")]


class GsiError(RuntimeError):
    def __init__(self, code, where):
        self.code = int(code)
        super().__init__(f"{where}: {gsi_status_string(code)} ({int(code)})")


def lib_path() -> str:
    return _build.LIB


def _load():
    path = _build.build()   # no-op when the library matches the sources
    l = C.CDLL(path)
    vp, i, sz = C.c_void_p, C.c_int, C.c_size_t
    l.gsi_status_string.restype = C.c_char_p
    l.gsi_status_string.argtypes = [i]
    l.gsi_build_image.argtypes = [vp, vp, i, i, i, i, vp, vp]
    l.gsi_workspace_bytes.restype = sz
    l.gsi_workspace_bytes.argtypes = [C.POINTER(GsiDesc)]
    l.gsi_create.argtypes = [C.POINTER(GsiDesc), C.POINTER(vp), vp, vp, sz, vp, C.POINTER(vp)]
    l.gsi_forward.argtypes = [vp, vp, vp, vp, vp]
    l.gsi_forward_n.argtypes = [vp, vp, i, vp, vp, vp, vp]
    l.gsi_forward_host.argtypes = [vp, vp, i, vp, vp, vp, vp]
    l.gsi_forward_static.argtypes = [C.POINTER(vp), C.POINTER(i), i, vp, i, vp, i, i, C.c_float,
                                     vp, i, vp, vp, vp, vp]
    l.gsi_get_image.argtypes = [vp, i, C.POINTER(vp)]
    l.gsi_get_image_fp8.argtypes = [vp, C.POINTER(vp), C.POINTER(C.c_size_t)]
    l.gsi_extend_basis.argtypes = [vp, vp, C.c_float, vp, vp, vp, vp]
    l.gsi_get_status.argtypes = [vp, C.POINTER(i)]
    l.gsi_set_spin_limit.argtypes = [vp, C.c_uint]
    l.gsi_destroy.argtypes = [vp]
    l.gsi_stack_workspace_bytes.restype = sz
    l.gsi_stack_workspace_bytes.argtypes = [i]
    l.gsi_stack_create.argtypes = [i, C.POINTER(vp), vp, sz, vp, C.POINTER(vp)]
    l.gsi_stack_bind.argtypes = [vp, C.POINTER(GsiStackIo), i, vp, vp, vp]
    l.gsi_stack_set_mode.argtypes = [vp, i]
    l.gsi_stack_set_concurrent.argtypes = [vp, i, i]
    l.gsi_stack_is_persistent.argtypes = [vp, C.POINTER(i)]
    l.gsi_stack_set_trace.argtypes = [vp, vp]
    l.gsi_stack_set_spin_limit.argtypes = [vp, C.c_uint]
    l.gsi_stack_seek.argtypes = [vp, i, vp]
    l.gsi_stack_step.argtypes = [vp, vp]
    l.gsi_stack_launches_per_step.argtypes = [vp, C.POINTER(i)]
    l.gsi_stack_step_host.argtypes = [vp, C.POINTER(vp), C.POINTER(vp), vp, vp]
    l.gsi_stack_get_status.argtypes = [vp, C.POINTER(i)]
    l.gsi_stack_destroy.argtypes = [vp]
    kd, ll = C.POINTER(GsiKvDesc), C.c_longlong
    l.gsi_kv_page_bytes.restype = l.gsi_kv_workspace_bytes.restype = sz
    l.gsi_kv_page_bytes.argtypes = l.gsi_kv_workspace_bytes.argtypes = [kd]
    l.gsi_kv_locate.argtypes = [kd, i, i, i, i, C.POINTER(sz), C.POINTER(sz)]
    l.gsi_kv_create.argtypes = [kd, vp, sz, vp, C.POINTER(vp)]
    l.gsi_kv_plan.argtypes = [vp, vp, i, i, vp, vp, vp, vp, vp, vp, vp, vp, vp, vp]
    l.gsi_kv_release.argtypes = [vp, vp, i, vp, vp, vp, vp, vp]
    l.gsi_kv_append.argtypes = [vp, vp, vp, i, ll, ll, ll, ll, vp, i, vp, vp]
    l.gsi_kv_read.argtypes = [vp, vp, vp, i, i, vp, vp, vp]
    l.gsi_kv_attend.argtypes = l.gsi_kv_attend_all.argtypes = [vp, vp, i, ll, ll, i, i, C.c_float, vp, vp, vp, i, vp, vp, ll, ll, vp]
    l.gsi_kv_get_status.argtypes = [vp, C.POINTER(i)]
    l.gsi_kv_destroy.argtypes = [vp]
    for name in EXPORTED:
        if name not in ("gsi_status_string", "gsi_workspace_bytes", "gsi_stack_workspace_bytes", "gsi_kv_page_bytes",
                        "gsi_kv_workspace_bytes"):
            getattr(l, name).restype = i
    return l


def _load_calls():
    import importlib.util
    spec = importlib.util.spec_from_file_location("_torch_calls", _build.build_calls())
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    m.bind(*[C.cast(f, C.c_void_p).value for f in (lib.gsi_forward_n, lib.gsi_extend_basis, lib.gsi_forward_static)])
    m.bind_kv(*[C.cast(f, C.c_void_p).value for f in (lib.gsi_kv_plan, lib.gsi_kv_release, lib.gsi_kv_append, lib.gsi_kv_read,
                                                      lib.gsi_kv_attend, lib.gsi_kv_attend_all)])
    return m


lib = _load()
_calls = _load_calls()


def gsi_status_string(code) -> str:
    return lib.gsi_status_string(int(code)).decode()


def _check(code, where):
    if code != 0:
        raise GsiError(code, where)


def _stream_ptr(stream) -> int:
    if stream is None:   # (the raw handle: building a Stream object costs 3 us a call)
        return torch._C._cuda_getCurrentRawStream(torch._C._cuda_getDevice())
    return int(stream.cuda_stream) if hasattr(stream, "cuda_stream") else int(stream)


def _dtype_code(t: torch.Tensor) -> int:
    if t.dtype == torch.bfloat16:
        return GSI_BF16
    if t.dtype == torch.float32:
        return GSI_F32
    raise TypeError("basis must be bfloat16 or float32")


def make_desc(d, k, d_out, eps, max_tokens, p_dtype=GSI_BF16, flags=0):
    arr = (C.c_int * len(d_out))(*[int(v) for v in d_out])
    desc = GsiDesc(int(d), int(k), len(d_out), C.cast(arr, C.POINTER(C.c_int)), float(eps),
                   int(max_tokens), int(p_dtype), int(flags))
    desc._keep = arr
    return desc


def gsi_workspace_bytes(d, k, d_out, eps, max_tokens, p_dtype=GSI_BF16, flags=0) -> int:
    return int(lib.gsi_workspace_bytes(C.byref(make_desc(d, k, d_out, eps, max_tokens, p_dtype, flags))))


def gsi_build_image(W: torch.Tensor, P: torch.Tensor, out: torch.Tensor | None = None,
                    stream=None) -> torch.Tensor:
    """W_P = bf16(W P) on the device (Section 4.2 of the paper)."""
    assert W.is_cuda and P.is_cuda and W.dtype == torch.bfloat16
    assert W.is_contiguous() and P.is_contiguous()
    o, d = W.shape
    d2, k = P.shape
    assert d == d2
    if out is None:
        out = torch.empty((o, k), dtype=torch.bfloat16, device=W.device)
    _check(lib.gsi_build_image(W.data_ptr(), P.data_ptr(), o, d, k, _dtype_code(P),
                               out.data_ptr(), _stream_ptr(stream)), "gsi_build_image")
    return out


def gsi_forward_static(Ws, P, W_P, eps, x, y=None, gate=None, rho=None, stream=None):
    """Algorithm 1 through the entry point that allocates nothing inside the
    library: scratch comes from an array built into ``libgsi_b200.so``.  For
    callers that may not call cudaMalloc (see ``include/gsi.h``).  ``W_P`` is the
    concatenation of ``gsi_build_image(W_j, P)`` over the maps.  The output
    tensors are allocated HERE, by torch, only when the caller passes none."""
    status, y, gate, rho = _calls.forward_static(list(Ws), P, _dtype_code(P), W_P, float(eps), x, y, gate, rho, stream)
    _check(status, "gsi_forward_static")
    return y, gate, rho


class Layer:
    """One group: maps ``Ws`` (list of [d_out_j][d] bf16) sharing basis ``P``."""

    def __init__(self, Ws, P, eps: float, max_tokens: int = 1, flags: int = 0, stream=None):
        Ws = list(Ws)
        dense = bool(flags & GSI_FLAG_DENSE)
        dev = Ws[0].device
        assert dev.type == "cuda", "the gated subspace layer runs on a CUDA device only"
        for W in Ws:
            assert W.dtype == torch.bfloat16 and W.is_contiguous() and W.device == dev
        self.d = int(Ws[0].shape[1])
        self.d_out = [int(W.shape[0]) for W in Ws]
        self.O = sum(self.d_out)
        self.k = 8 if (dense and P is None) else int(P.shape[1])
        self.max_tokens = int(max_tokens)
        self.eps = float(eps)
        self.flags = int(flags)
        assert P is None or (P.is_contiguous() and P.device == dev and tuple(P.shape) == (self.d, self.k))
        self._Ws, self._P = Ws, P
        pd = GSI_BF16 if P is None else _dtype_code(P)
        self._desc = make_desc(self.d, self.k, self.d_out, eps, max_tokens, pd, flags)
        nbytes = int(lib.gsi_workspace_bytes(C.byref(self._desc)))
        if nbytes == 0:
            raise GsiError(2, "gsi_workspace_bytes (descriptor rejected)")
        self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
        warr = (C.c_void_p * len(Ws))(*[W.data_ptr() for W in Ws])
        h = C.c_void_p()
        _check(lib.gsi_create(C.byref(self._desc), warr, None if P is None else P.data_ptr(),
                              self.workspace.data_ptr(), nbytes, _stream_ptr(stream),
                              C.byref(h)), "gsi_create")
        self.handle = h
        self._handle = h.value   # ... as the extension module takes it
        self.device = dev

    def forward(self, x: torch.Tensor, y: torch.Tensor | None = None,
                gate: torch.Tensor | None = None, rho: torch.Tensor | None = None, stream=None):
        status, y, gate, rho = _calls.forward(self._handle, self.O, x, y, gate, rho, stream)
        if status:
            _check(status, "gsi_forward_n")
        return y, gate, rho

    def forward_host(self, x: torch.Tensor, stream=None):
        """Host tensors in, host tensors out (copies inside the call)."""
        assert not x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()
        n = int(x.shape[0])
        y = torch.empty((n, self.O), dtype=torch.float32).pin_memory()
        gate = torch.empty(n, dtype=torch.uint8).pin_memory()
        rho = torch.empty(n, dtype=torch.float32).pin_memory()
        _check(lib.gsi_forward_host(self.handle, x.data_ptr(), n, y.data_ptr(), gate.data_ptr(),
                                    rho.data_ptr(), _stream_ptr(stream)), "gsi_forward_host")
        return y, gate, rho

    def extend_basis(self, x: torch.Tensor, tau: float, k_active: torch.Tensor, stream=None):
        """gsi_extend_basis for one token x [d]; k_active is a device int32 tensor (in/out).
        Returns (appended, rho) as device tensors.  Writes the basis tensor given at creation."""
        assert x.numel() == self.d
        status, appended, rho = _calls.extend(self._handle, x, tau, k_active, stream)
        if status:
            _check(status, "gsi_extend_basis")
        return appended, rho

    def image(self, j: int) -> torch.Tensor:
        """Copy of the cached image of map j ([d_out_j][k] bf16)."""
        p = C.c_void_p()
        _check(lib.gsi_get_image(self.handle, j, C.byref(p)), "gsi_get_image")
        base = self.workspace.data_ptr()
        off = p.value - base
        nbytes = self.d_out[j] * self.k * 2
        return self.workspace[off:off + nbytes].view(torch.bfloat16).view(self.d_out[j], self.k).clone()

    def image_fp8(self):
        """The FP8 image of all maps as stored (GSI_FLAG_FP8_IMAGE handles): codes
        ``[sum d_out][k]`` uint8 and row scales ``[sum d_out]`` fp32, copied out of
        the tiled layout the header documents (a rearrangement of bytes only)."""
        p, n = C.c_void_p(), C.c_size_t()
        _check(lib.gsi_get_image_fp8(self.handle, C.byref(p), C.byref(n)), "gsi_get_image_fp8")
        off = p.value - self.workspace.data_ptr()
        raw = self.workspace[off:off + n.value]
        O, k = sum(self.d_out), self.k
        R, KT = (O + 15) // 16, k // 16
        raw = raw.view(R, KT * 256 + 64)
        # tile bytes [R][K][g][t][c8][r8][e]: element (row g + 8 r8, column 2 t + 8 c8 + e)
        tiles = raw[:, :KT * 256].reshape(R, KT, 8, 4, 2, 2, 2)
        codes = tiles.permute(0, 5, 2, 1, 4, 3, 6).reshape(R * 16, k)[:O].clone()
        scales = raw[:, KT * 256:].contiguous().view(torch.float32).reshape(R * 16)[:O].clone()
        return codes, scales

    def set_spin_limit(self, polls: int):
        """Polls a wait between the CTAs of one launch may take (0 = the default)."""
        _check(lib.gsi_set_spin_limit(self.handle, int(polls)), "gsi_set_spin_limit")

    def status(self) -> int:
        v = C.c_int()
        _check(lib.gsi_get_status(self.handle, C.byref(v)), "gsi_get_status")
        return v.value

    def close(self):
        if getattr(self, "handle", None):
            lib.gsi_destroy(self.handle)
            self.handle = None
            self._handle = 0

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class Stack:
    """An ordered chain of groups stepped as one decode step."""

    def __init__(self, layers, stream=None, mode: int = 0, concurrent=()):
        """concurrent: indices i such that groups i and i+1 do not read each other's outputs
        and may share a phase of the persistent kernel (gsi_stack_set_concurrent)."""
        self.layers = list(layers)
        self._mode = int(mode)
        n = len(self.layers)
        dev = self.layers[0].device
        self.B = self.layers[0].max_tokens
        nbytes = int(lib.gsi_stack_workspace_bytes(n))
        self.workspace = torch.zeros(nbytes, dtype=torch.uint8, device=dev)
        arr = (C.c_void_p * n)(*[l.handle for l in self.layers])
        h = C.c_void_p()
        _check(lib.gsi_stack_create(n, arr, self.workspace.data_ptr(), nbytes,
                                    _stream_ptr(stream), C.byref(h)), "gsi_stack_create")
        self.handle = h
        self.device = dev
        if self._mode:
            _check(lib.gsi_stack_set_mode(self.handle, self._mode), "gsi_stack_set_mode")
        for first in concurrent:
            _check(lib.gsi_stack_set_concurrent(self.handle, int(first), 1), "gsi_stack_set_concurrent")

    def is_persistent(self) -> bool:
        v = C.c_int()
        _check(lib.gsi_stack_is_persistent(self.handle, C.byref(v)), "gsi_stack_is_persistent")
        return bool(v.value)

    def bind(self, xs, ys=None, n_steps: int = 1, want_rho: bool = True, stream=None):
        """xs[g]: [n_steps][B][d] fp32 device tensors.  Allocates y and the logs."""
        n = len(self.layers)
        if ys is None:
            ys = [torch.empty((self.B, l.O), dtype=torch.float32, device=self.device)
                  for l in self.layers]
        self.xs, self.ys, self.n_steps = list(xs), list(ys), int(n_steps)
        for x, l in zip(self.xs, self.layers):
            assert x.is_cuda and x.dtype == torch.float32 and x.is_contiguous()
            assert x.numel() == n_steps * self.B * l.d
        self.gate_log = torch.zeros((n_steps, n, self.B), dtype=torch.uint8, device=self.device)
        self.rho_log = (torch.zeros((n_steps, n, self.B), dtype=torch.float32, device=self.device)
                        if want_rho else None)
        io = (GsiStackIo * n)(*[GsiStackIo(x.data_ptr(), y.data_ptr())
                                for x, y in zip(self.xs, self.ys)])
        _check(lib.gsi_stack_bind(self.handle, io, n_steps, self.gate_log.data_ptr(),
                                  None if self.rho_log is None else self.rho_log.data_ptr(),
                                  _stream_ptr(stream)), "gsi_stack_bind")

    def set_trace(self, on: bool = True):
        """Per-section SM-cycle counters, one row per CTA (persistent launch only); the
        sections are listed at gsi_stack_set_trace in the header."""
        self.trace = torch.zeros((256, 16), dtype=torch.int64, device=self.device) if on else None
        _check(lib.gsi_stack_set_trace(self.handle, self.trace.data_ptr() if on else None),
               "gsi_stack_set_trace")
        return self.trace

    def set_spin_limit(self, polls: int):
        """Polls a cross-CTA wait of the persistent kernel may take (0 = default)."""
        _check(lib.gsi_stack_set_spin_limit(self.handle, int(polls)), "gsi_stack_set_spin_limit")

    def seek(self, step: int, stream=None):
        _check(lib.gsi_stack_seek(self.handle, int(step), _stream_ptr(stream)), "gsi_stack_seek")

    def step(self, stream=None):
        _check(lib.gsi_stack_step(self.handle, _stream_ptr(stream)), "gsi_stack_step")

    def launches_per_step(self) -> int:
        v = C.c_int()
        _check(lib.gsi_stack_launches_per_step(self.handle, C.byref(v)),
               "gsi_stack_launches_per_step")
        return v.value

    def step_host(self, xs_host, ys_host, gate_host, stream=None):
        n = len(self.layers)
        xa = (C.c_void_p * n)(*[x.data_ptr() for x in xs_host])
        ya = (C.c_void_p * n)(*[y.data_ptr() for y in ys_host])
        _check(lib.gsi_stack_step_host(self.handle, xa, ya, gate_host.data_ptr(),
                                       _stream_ptr(stream)), "gsi_stack_step_host")

    def status(self) -> int:
        v = C.c_int()
        _check(lib.gsi_stack_get_status(self.handle, C.byref(v)), "gsi_stack_get_status")
        return v.value

    def close(self):
        if getattr(self, "handle", None):
            lib.gsi_stack_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass


class KVCache:
    """Keys and values in 4 bits, in pages, for up to ``max_seqs`` requests of up to ``max_len`` tokens, and
    attention over them (``include/gsi.h`` has the numbers' definition and the pages' layout).

        cache.plan(n_new)                         # once a step: pages, slots and positions of the new tokens
        cache.append(k, v, layer)                 # per layer: k, v [n][n_heads][head_dim], as columns of a group's y
        out = cache.attend(q, layer)              # q, out [n][q heads][head_dim]
        cache.release(done)                       # requests that have ended give their pages back

    Device tensors: the state ``lens``, ``table``, ``free``, ``n_free``, and what a plan leaves, ``q_start``,
    ``kv_len``, ``slots``, ``positions``, ``counts`` (new tokens, pages taken, pages left, requests refused).  None is
    read on the host, so a step can be captured into a CUDA graph.  ``pages`` (uint8, [n_layers][n_pages][bytes of a
    page]) may be the caller's memory.  A plan may be for the first few requests only; those behind have no rows then.  One cache may be used
    by one stream at a time.
    """

    def __init__(self, n_heads: int, head_dim: int, n_pages: int, max_seqs: int, max_len: int, page_tokens: int = 64,
                 n_layers: int = 1, max_tokens: int = GSI_MAX_TOKENS, device="cuda", pages: torch.Tensor | None = None,
                 stream=None):
        self.n_heads, self.head_dim, self.n_pages, self.page_tokens = int(n_heads), int(head_dim), int(n_pages), int(page_tokens)
        self.n_layers = int(n_layers)
        max_pages = -(-int(max_len) // max(1, self.page_tokens))
        self._desc = GsiKvDesc(self.n_heads, self.head_dim, self.page_tokens, self.n_pages, int(max_seqs), max_pages, int(max_tokens))
        self.page_bytes, nbytes = int(lib.gsi_kv_page_bytes(C.byref(self._desc))), int(lib.gsi_kv_workspace_bytes(C.byref(self._desc)))
        if nbytes == 0 or self.n_layers < 1:
            raise GsiError(2, "gsi_kv_workspace_bytes (descriptor rejected)")
        dev = torch.device(device) if pages is None else pages.device
        assert dev.type == "cuda", "the cache lives on a CUDA device"
        if dev.index is None:
            dev = torch.device("cuda", torch.cuda.current_device())
        whole = self.n_layers * self.n_pages * self.page_bytes
        # (what is made here is filled on the stream that gsi_kv_create waits for)
        on = contextlib.nullcontext() if stream is None else torch.cuda.stream(torch.cuda.ExternalStream(_stream_ptr(stream), dev))
        if pages is None:
            with on:
                pages = torch.empty((self.n_layers, self.n_pages, self.page_bytes), dtype=torch.uint8, device=dev)
        assert pages.dtype == torch.uint8 and pages.is_contiguous() and pages.numel() == whole and pages.data_ptr() % 16 == 0
        self.device, self.pages = dev, pages

        def ints(*shape, fill=0):
            return torch.full(shape, fill, dtype=torch.int32, device=dev)

        with torch.cuda.device(dev), on:
            self.workspace = torch.empty(nbytes, dtype=torch.uint8, device=dev)
            self.table, self.lens = ints(int(max_seqs), max_pages, fill=-1), ints(int(max_seqs))
            self.free = torch.arange(self.n_pages - 1, -1, -1, dtype=torch.int32, device=dev)
            self.n_free = ints(1, fill=self.n_pages)
            self.q_start, self.kv_len = ints(int(max_seqs) + 1), ints(int(max_seqs))
            self.slots, self.positions = ints(int(max_tokens), fill=-1), ints(int(max_tokens), fill=-1)
            self.counts = ints(4)
            h = C.c_void_p()
            _check(lib.gsi_kv_create(C.byref(self._desc), self.workspace.data_ptr(), nbytes, _stream_ptr(stream), C.byref(h)), "gsi_kv_create")
        self.handle = h
        self._state = _calls.kv_state(h.value, self.n_heads, self.head_dim, self.n_layers, pages, self.table, self.lens, self.free,
                                      self.n_free, self.q_start, self.kv_len, self.slots, self.positions, self.counts)
        self._like = {t: torch.empty(0, dtype=t) for t in (torch.float32, torch.bfloat16, torch.float16)}
        self._scale = float(self.head_dim) ** -0.5

    def plan(self, n_new: torch.Tensor, commit: bool = True, stream=None):
        """Room for ``n_new[s]`` more tokens of request s (int32, device), one launch.  ``commit=False`` leaves
        ``lens`` and ``n_free`` as they are: the next plan hands out the same pages again."""
        status = _calls.kv_plan(self._state, n_new, commit, stream)
        if status:
            _check(status, "gsi_kv_plan")

    def release(self, done: torch.Tensor, stream=None):
        """Requests s with ``done[s]`` (bool or uint8, device) give their pages back and are empty."""
        status = _calls.kv_release(self._state, done, stream)
        if status:
            _check(status, "gsi_kv_release")

    def append(self, k: torch.Tensor, v: torch.Tensor, layer: int = 0, slots: torch.Tensor | None = None, stream=None):
        """Row i of k and v to ``slots[i]`` (the plan's by default), rows with a negative slot nowhere."""
        status = _calls.kv_append(self._state, k, v, layer, slots, stream)
        if status:
            _check(status, "gsi_kv_append")

    def attend(self, q: torch.Tensor, layer: int = 0, scale: float | None = None, out: torch.Tensor | None = None, stream=None):
        """Attention of the plan's rows, each over its request's tokens up to its own; ``scale`` is
        ``head_dim ** -0.5`` by default.  ``out`` shares no element with ``q``; its rows behind the last request's are
        not written (without ``out``: zeros)."""
        status, out = _calls.kv_attend(self._state, q, layer, self._scale if scale is None else scale, out, stream)
        if status:
            _check(status, "gsi_kv_attend")
        return out

    def read(self, slots: torch.Tensor, layer: int = 0, dtype: torch.dtype = torch.float32, stream=None):
        """(k, v) [n][n_heads][head_dim]: the values that ``slots`` (int32, device) hold, zeros for a negative one."""
        status, k, v = _calls.kv_read(self._state, slots, layer, self._like[dtype], stream)
        if status:
            _check(status, "gsi_kv_read")
        return k, v

    def locate(self, slot: int, head: int, channel: int, is_v: bool):
        """(byte of the code, byte of the pair) of one element, from the first of a layer's pages."""
        code, pair = C.c_size_t(), C.c_size_t()
        _check(lib.gsi_kv_locate(C.byref(self._desc), slot, head, channel, int(is_v), C.byref(code), C.byref(pair)), "gsi_kv_locate")
        return code.value, pair.value

    def status(self) -> int:
        v = C.c_int()
        with torch.cuda.device(self.device):
            _check(lib.gsi_kv_get_status(self.handle, C.byref(v)), "gsi_kv_get_status")
        return v.value

    def close(self):
        if getattr(self, "handle", None):
            _calls.kv_close(self._state)
            lib.gsi_kv_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
