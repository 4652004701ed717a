"""Operators of the target model's verifying pass over the drafts of all paths (include/csd_verify.h).

Between Index.draft and Index.accept (binding.py) the target model sees every path's newest token and the draft
behind it.  PathCache holds the keys and values of the prompts, which the paths of a problem share, and of the paths, in 16
bits or quantised to 8 as they are written, and attends to them; targets() turns the logits into the tokens that
Index.accept compares with, and the probabilities that Index.append and Index.step take.  Argument marshalling only, in
native code (_csd_torch.so) where the arguments are the usual ones: all of it runs in the HIP kernels of libcsd.so, on the
current stream.  Serving only: there are no gradients, and a tensor that requires one is refused unless gradients are off.
"""
from __future__ import annotations

import ctypes
from typing import Optional

import torch

from . import binding
from .binding import CsdError, OK, _ptr, _stream, _vp

BF16, F16, F32 = 0, 1, 2
TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}

EXPORTS = ["csd_cache_bytes", "csd_cache_create", "csd_cache_destroy", "csd_cache_write", "csd_cache_write_prompt",
           "csd_cache_read", "csd_cache_read_prompt", "csd_attend", "csd_attend_form_of", "csd_targets_bytes", "csd_targets", "csd_cache_status"]


class CacheConfig(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in
                ("n_problems", "n_paths", "prompt_cap", "path_cap", "n_layers", "n_heads", "n_kv_heads", "head_dim",
                 "max_step", "type", "fp8")]


class Heads(ctypes.Structure):
    _fields_ = [("data", _vp)] + [(name, ctypes.c_int64) for name in ("row_stride", "token_stride", "head_stride")]


class AttendForm(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("joined", "solo", "prompt_splits", "path_splits", "groups")]


_lib = None
_native = None


def load() -> ctypes.CDLL:
    global _lib, _native
    if _lib is None:
        lib = binding.load()
        _native = binding._native
        i32, i64, size = ctypes.c_int32, ctypes.c_int64, ctypes.c_size_t
        cfgp, heads, f32 = ctypes.POINTER(CacheConfig), ctypes.POINTER(Heads), ctypes.c_float
        lib.csd_cache_bytes.argtypes = [cfgp, ctypes.POINTER(size)]
        lib.csd_cache_create.argtypes = [cfgp, _vp, size, _vp, ctypes.POINTER(_vp)]
        lib.csd_cache_destroy.argtypes = [_vp]
        for name in ("csd_cache_write", "csd_cache_write_prompt"):
            getattr(lib, name).argtypes = [_vp, i32, heads, heads, _vp, _vp, i32, _vp]
        for name in ("csd_cache_read", "csd_cache_read_prompt"):
            getattr(lib, name).argtypes = [_vp, i32, _vp, _vp, i32, _vp, _vp, _vp]
        lib.csd_attend.argtypes = [_vp, i32, heads, _vp, _vp, _vp, i32, f32, i32, i32, _vp, _vp, _vp]
        lib.csd_attend_form_of.argtypes = [cfgp, i32, i32, i32, ctypes.POINTER(AttendForm)]
        lib.csd_targets_bytes.argtypes = [i64, i32, ctypes.POINTER(size)]
        lib.csd_targets.argtypes = [_vp, i32, i64, i32, i64, _vp, i64, f32, _vp, _vp, _vp, size, _vp]
        lib.csd_cache_status.argtypes = [_vp, ctypes.POINTER(ctypes.c_uint32), _vp]
        for name in EXPORTS:
            getattr(lib, name).restype = ctypes.c_int
        _lib = lib
    return _lib


def _check(rc: int, what: str) -> None:
    if rc != OK:
        raise CsdError(rc, what)


def _no_gradients(*tensors) -> None:
    if torch.is_grad_enabled() and any(t is not None and t.requires_grad for t in tensors):
        raise TypeError("no gradients here: call under torch.no_grad(), or with detached tensors")


def _spacing(shape, stride) -> int:
    """The distance of the rows of leading axes that are evenly spaced (0: there is one row)."""
    rows, spacing = 1, 0
    for size, step in zip(reversed(shape), reversed(stride[:len(shape)])):
        if size > 1:
            spacing = step if rows == 1 else spacing
            if step != spacing * rows:
                raise TypeError("rows must be evenly spaced")
        rows *= size
    return spacing


def _heads(t: torch.Tensor, dtype, lead, n_heads: int, dim: int) -> Heads:
    """A tensor [*lead][n][heads][dim]: dense, or a slice of tokens or heads of a larger one."""
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError("expected a device tensor of dtype %s" % dtype)
    _no_gradients(t)
    shape, stride, at = tuple(t.shape), t.stride(), len(lead)
    if shape[:at] != tuple(lead) or len(shape) != at + 3 or shape[-2:] != (n_heads, dim):
        raise ValueError("tensor of shape %s, needs %s" % (shape, (*lead, "n", n_heads, dim)))
    if stride[-1] != 1:
        raise TypeError("a head's values must be contiguous")
    h = Heads(t.data_ptr(), _spacing(lead, stride), stride[at] if shape[at] > 1 else 0, stride[-2] if n_heads > 1 else 0)
    if (h.data or 0) % 16 or h.row_stride % 8 or h.token_stride % 8 or h.head_stride % 8:
        raise ValueError("heads must start at multiples of 16 bytes")
    return h


def attend_form(cfg: CacheConfig, n: int, prompt_bound: int = 0, path_bound: int = 0) -> AttendForm:
    """The form of the launch of PathCache.attend() for n tokens a path (host only: no GPU is needed)."""
    form = AttendForm()
    _check(load().csd_attend_form_of(ctypes.byref(cfg), n, prompt_bound, path_bound, ctypes.byref(form)), "csd_attend_form_of")
    return form


class PathCache:
    """Keys and values of P prompts and of P x N paths behind them, on the current device.

    prompt_cap, path_cap: tokens of a prompt, and of a path behind it.  max_step: most tokens a path of an attend() call.
    fp8: 8-bit codes (e4m3) with a power-of-two scale per token and kv head, quantised as they are written."""

    def __init__(self, n_problems, n_paths, prompt_cap, path_cap, n_heads, n_kv_heads, head_dim, max_step, n_layers=1,
                 dtype=torch.bfloat16, fp8=False, device="cuda"):
        if dtype not in (torch.bfloat16, torch.float16):
            raise TypeError("a cache is of bfloat16 or float16")
        self.cfg = CacheConfig(n_problems, n_paths, prompt_cap, path_cap, n_layers, n_heads, n_kv_heads, head_dim, max_step,
                               TYPES[dtype], int(bool(fp8)))
        self.P, self.N, self.dtype = n_problems, n_paths, dtype
        self.device = torch.device(device)
        self._h = _vp()
        nbytes = ctypes.c_size_t(0)
        _check(load().csd_cache_bytes(ctypes.byref(self.cfg), ctypes.byref(nbytes)), "csd_cache_bytes")
        # +256 so that a 256-byte aligned start always exists inside the buffer
        self._buf = torch.empty(nbytes.value + 256, dtype=torch.uint8, device=self.device)
        self._ws = (self._buf.data_ptr() + 255) // 256 * 256
        _check(load().csd_cache_create(ctypes.byref(self.cfg), self._ws, nbytes.value, _stream(), ctypes.byref(self._h)),
               "csd_cache_create")
        self._sizes = (-1 if self.device.index is None else self.device.index, n_problems, n_paths, n_heads, n_kv_heads, head_dim,
                       TYPES[dtype])
        self._scale = head_dim ** -0.5

    def _cache(self):
        """What every native call starts with."""
        return self._h.value if self._h else 0, _stream(), *self._sizes

    def close(self):
        if getattr(self, "_h", None):
            load().csd_cache_destroy(self._h)
            self._h = None

    def __del__(self):
        try:
            self.close()
        except Exception:       # interpreter shutdown: module globals may already be gone
            pass

    def _write(self, call, what, lead, layer, k, v, start, counts):
        rc = _native.cache_write(*self._cache(), len(lead) == 1, layer, k, v, start, counts)
        if rc is not None:
            return _check(rc, what)
        c, rows = self.cfg, 1
        for x in lead:
            rows *= x
        kh, vh = (_heads(t, self.dtype, lead, c.n_kv_heads, c.head_dim) for t in (k, v))
        n = k.shape[-3]
        if v.shape != k.shape:
            raise ValueError("keys of shape %s, values of shape %s" % (tuple(k.shape), tuple(v.shape)))
        _check(call(self._h, layer, ctypes.byref(kh), ctypes.byref(vh), _ptr(start, torch.int32, rows),
                    _ptr(counts, torch.int32, rows), n, _stream()), what)

    def write(self, layer, k, v, start=None, counts=None):
        """k, v [P][N][n][kv heads][head_dim] to positions start [P][N] int32 (None: 0) and on of the paths, the first counts
        [P][N] int32 of them (None: n).  Whatever was there is replaced."""
        self._write(_lib.csd_cache_write, "csd_cache_write", (self.P, self.N), layer, k, v, start, counts)

    def write_prompt(self, layer, k, v, start=None, counts=None):
        """k, v [P][n][kv heads][head_dim] to the prompts; start, counts [P]."""
        self._write(_lib.csd_cache_write_prompt, "csd_cache_write_prompt", (self.P,), layer, k, v, start, counts)

    def _read(self, call, what, lead, layer, n, start, counts):
        got = _native.cache_read(*self._cache(), len(lead) == 1, layer, n, start, counts)
        if got is not None:
            _check(got[0], what)
            return got[1], got[2]
        c, rows = self.cfg, 1
        for x in lead:
            rows *= x
        k, v = (torch.empty((*lead, n, c.n_kv_heads, c.head_dim), dtype=self.dtype, device=self.device) for _ in range(2))
        _check(call(self._h, layer, _ptr(start, torch.int32, rows), _ptr(counts, torch.int32, rows), n, k.data_ptr(), v.data_ptr(),
                    _stream()), what)
        return k, v

    def read(self, layer, n, start=None, counts=None):
        """Keys and values [P][N][n][kv heads][head_dim] of the paths, rows as in write(); zero beyond a row's count.  (8 bits of
        float16: 63488 and more are held as 65536, which attend() works with and read() gives as infinity.)"""
        return self._read(_lib.csd_cache_read, "csd_cache_read", (self.P, self.N), layer, n, start, counts)

    def read_prompt(self, layer, n, start=None, counts=None):
        """... [P][n][kv heads][head_dim] of the prompts."""
        return self._read(_lib.csd_cache_read_prompt, "csd_cache_read_prompt", (self.P,), layer, n, start, counts)

    def attend(self, layer, q, prompt_len, path_len, counts=None, scale=None, out=None, lse=None, prompt_bound=0, path_bound=0):
        """Attention of q [P][N][n][heads][head_dim], the paths' newest tokens (counts [P][N] of the n; None: all), to their prompts'
        first prompt_len [P] tokens (None: the capacity) and their own first path_len [P][N], the new ones among them.
        Token t of a path sees path_len - count + t + 1 of these.  Returns [P][N][n][heads][head_dim]; lse: a float32 tensor
        [P][N][n][heads] that takes the logarithms of the sums.  scale: 1 / sqrt(head_dim) where None.  prompt_bound,
        path_bound: what no length exceeds (0: the capacities), for the shape of the launch alone."""
        if out is None and lse is None:
            got = _native.attend(*self._cache(), layer, q, prompt_len, path_len, counts, self._scale if scale is None else scale,
                                 prompt_bound, path_bound)
            if got is not None:
                _check(got[0], "csd_attend")
                return got[1]
        _no_gradients(out, lse)
        c, rows = self.cfg, self.P * self.N
        heads = _heads(q, self.dtype, (self.P, self.N), c.n_heads, c.head_dim)
        n = q.shape[2]
        if out is None:
            out = torch.empty((self.P, self.N, n, c.n_heads, c.head_dim), dtype=self.dtype, device=self.device)
        _check(load().csd_attend(self._h, layer, ctypes.byref(heads), _ptr(prompt_len, torch.int32, self.P),
                                 _ptr(path_len, torch.int32, rows), _ptr(counts, torch.int32, rows), n,
                                 self._scale if scale is None else scale, prompt_bound, path_bound,
                                 _ptr(out, self.dtype, rows * n * c.n_heads * c.head_dim),
                                 _ptr(lse, torch.float32, rows * n * c.n_heads), _stream()), "csd_attend")
        return out

    def status(self) -> int:
        flags = ctypes.c_uint32(0)
        _check(load().csd_cache_status(self._h, ctypes.byref(flags), _stream()), "csd_cache_status")
        return flags.value


def targets(logits: torch.Tensor, noise: Optional[torch.Tensor] = None, inv_temperature: float = 1.0):
    """The model's tokens and their probabilities from logits [..., vocab] (bfloat16, float16, float32): tokens int32 [...], probs
    float32 [...].  Greedy, or a sample where noise [..., vocab] float32 (-ln(-ln u), u uniform) is given: the largest logit *
    inv_temperature + noise, the lowest of equals.  The probability is that of softmax(logits * inv_temperature)."""
    if logits.is_cuda:
        load()
        got = _native.targets(_stream(), logits, noise, inv_temperature)
        if got is not None:
            _check(got[0], "csd_targets")
            return got[1], got[2]
    if logits.dtype not in TYPES:
        raise TypeError("logits of dtype %s" % logits.dtype)
    if noise is not None and (noise.dtype != torch.float32 or noise.shape != logits.shape):
        raise TypeError("noise must be float32 of the logits' shape")
    for t in (logits,) if noise is None else (logits, noise):
        if not t.is_cuda or t.dim() == 0 or (t.stride(-1) != 1 and t.shape[-1] > 1):
            raise TypeError("expected a device tensor with contiguous rows")
    _no_gradients(logits, noise)
    lead, vocab = logits.shape[:-1], logits.shape[-1]
    rows, stride = lead.numel(), _spacing(lead, logits.stride())
    noise_stride = _spacing(lead, noise.stride()) if noise is not None else 0
    tokens = torch.empty(lead, dtype=torch.int32, device=logits.device)
    probs = torch.empty(lead, dtype=torch.float32, device=logits.device)
    nbytes = ctypes.c_size_t(0)
    _check(load().csd_targets_bytes(rows, vocab, ctypes.byref(nbytes)), "csd_targets_bytes")
    scratch = torch.empty(nbytes.value, dtype=torch.uint8, device=logits.device) if nbytes.value else None
    _check(load().csd_targets(logits.data_ptr(), TYPES[logits.dtype], rows, vocab, stride,
                              None if noise is None else noise.data_ptr(), noise_stride, inv_temperature, tokens.data_ptr(),
                              probs.data_ptr(), None if scratch is None else scratch.data_ptr(), nbytes.value, _stream()),
           "csd_targets")
    return tokens, probs
