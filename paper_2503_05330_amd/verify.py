"""Operators of the target model's verifying pass over the drafts of all paths (include/csd_verify.h).

Between Index.draft and Index.accept (binding.py) the target model sees every path's newest token and the draft
behind it.  PathCache holds the keys and values of the prompts, which the paths of a problem share, and of the paths, in 16
bits or quantised to 8 as they are written, and attends to them; targets() turns the logits into the tokens that
Index.accept compares with, and the probabilities that Index.append and Index.step take.  Around these: rotate() and PathCache.write_rotated()
turn queries and keys by their positions (Rotary), prompt_attend() is the prompts' own attention, which PathCache.write_packed()
takes the keys and values of, and adjust() applies penalties, biases and masks to logits before targets().  Argument marshalling only, in
native code (_csd_torch.so) where the arguments are the usual ones: all of it runs in the HIP kernels of libcsd.so, on the
current stream.  Serving only: there are no gradients, and a tensor that requires one is refused unless gradients are off.
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional

import torch

from . import binding
from .binding import CsdError, OK, _ptr, _stream, _vp

BF16, F16, F32 = 0, 1, 2
TYPES = {torch.bfloat16: BF16, torch.float16: F16, torch.float32: F32}

EXPORTS = ["csd_cache_bytes", "csd_cache_create", "csd_cache_destroy", "csd_cache_write", "csd_cache_write_prompt",
           "csd_cache_read", "csd_cache_read_prompt", "csd_rotary_turns", "csd_rotate", "csd_cache_write_rotated", "csd_cache_write_packed",
           "csd_prompt_attend", "csd_adjust", "csd_attend", "csd_attend_form_of", "csd_targets_bytes", "csd_targets", "csd_cache_status"]


class CacheConfig(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in
                ("n_problems", "n_paths", "prompt_cap", "path_cap", "n_layers", "n_heads", "n_kv_heads", "head_dim",
                 "max_step", "type", "fp8")]


class Heads(ctypes.Structure):
    _fields_ = [("data", _vp)] + [(name, ctypes.c_int64) for name in ("row_stride", "token_stride", "head_stride")]


class RotaryConfig(ctypes.Structure):
    _fields_ = [("turns", _vp), ("dim", ctypes.c_int32), ("interleaved", ctypes.c_int32), ("amplitude", ctypes.c_float)]


class Adjustment(ctypes.Structure):
    _fields_ = [(name, ctypes.c_int32) for name in ("n_problems", "n_paths", "n", "vocab", "type")] + [
        ("logits", _vp), ("logit_stride", ctypes.c_int64), ("out", _vp), ("out_stride", ctypes.c_int64), ("counts", _vp), ("penalties", _vp),
        ("tokens", _vp), ("token_stride", ctypes.c_int64), ("path_cap", ctypes.c_int32), ("path_len", _vp),
        ("prompt", _vp), ("prompt_stride", ctypes.c_int64), ("prompt_cap", ctypes.c_int32), ("prompt_len", _vp),
        ("bias", _vp), ("bias_stride", ctypes.c_int64), ("mask", _vp), ("mask_stride", ctypes.c_int64)]


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
        rotary, f64 = ctypes.POINTER(RotaryConfig), ctypes.c_double
        lib.csd_rotary_turns.argtypes = [i32, f64, f64, f64, f64, f64, _vp]
        lib.csd_rotate.argtypes = [rotary, heads, _vp, i64, i32, i32, i32, heads, _vp]
        lib.csd_cache_write_rotated.argtypes = [_vp, i32, rotary, heads, heads, heads, _vp, _vp, _vp, i32, _vp, _vp]
        lib.csd_cache_write_packed.argtypes = [_vp, i32, heads, heads, _vp, i64, _vp]
        lib.csd_prompt_attend.argtypes = [heads, heads, heads, i32, i32, i32, i32, _vp, i32, i64, f32, _vp, _vp, _vp]
        lib.csd_adjust.argtypes = [ctypes.POINTER(Adjustment), _vp]
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


class Rotary:
    """A rotation by position: the first dim values of a head in dim / 2 pairs, (i, i + dim / 2) or, interleaved, (2 i, 2 i + 1); pair i is
    turned by position * base^(-2i/dim).  For longer contexts than a model was trained on these are divided by factor; with
    original, the training's length, pairs of `high` turns over it and more stay, those of `low` turns and fewer are divided, and between
    them a share is.  amplitude: what the pairs are multiplied by.  frequencies [dim / 2], in radians a token, instead of all that."""

    def __init__(self, dim, base=10000.0, interleaved=False, factor=1.0, original=0, low=1.0, high=4.0, amplitude=1.0, frequencies=None,
                 device="cuda"):
        if frequencies is None:
            turns = (ctypes.c_double * max(dim // 2, 1))()
            _check(load().csd_rotary_turns(dim, base, factor, original, low, high, ctypes.addressof(turns)), "csd_rotary_turns")
            turns = torch.tensor(list(turns), dtype=torch.float64)
        else:
            turns = torch.as_tensor(frequencies, dtype=torch.float64, device="cpu") / (2 * math.pi)
            if turns.shape != (dim // 2,):
                raise ValueError("%d frequencies, needs %d" % (turns.numel(), dim // 2))
        if dim < 16 or dim % 16 or not math.isfinite(amplitude):
            raise ValueError("a rotation of %d values, amplitude %g" % (dim, amplitude))
        self.dim, self.interleaved, self.amplitude = dim, bool(interleaved), float(amplitude)
        self.turns = turns.to(device)
        self._cfg = RotaryConfig(self.turns.data_ptr(), dim, int(self.interleaved), self.amplitude)
        # what every native call starts with
        self._call = self._cfg.turns or 0, dim, self.interleaved, self.amplitude, self.turns.get_device()

    def _config(self):
        if not self.turns.is_cuda:
            raise TypeError("a rotation whose turns are not on the device")
        _here(self.turns)
        return ctypes.byref(self._cfg)


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
        self._place = self._buf.get_device()
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

    def write_rotated(self, layer, q, k, v, rotary, positions, start=None, counts=None):
        """What rotate() does to q [P][N][n][heads][head_dim] and k at positions [P][N][n] int32, and write() with the rotated keys and v, in
        one launch.  Returns the rotated queries, all n of each path."""
        here = torch._C._cuda_getDevice()
        got = None
        if here == self._place:
            got = _native.cache_write_rotated(*self._cache(), here, *rotary._call, layer, q, k, v, positions, start, counts)
        if got is not None:
            _check(got[0], "csd_cache_write_rotated")
            return got[1]
        c, lead = self.cfg, (self.P, self.N)
        rows = self.P * self.N
        qh = _heads(q, self.dtype, lead, c.n_heads, c.head_dim)
        kh, vh = (_heads(t, self.dtype, lead, c.n_kv_heads, c.head_dim) for t in (k, v))
        n = q.shape[-3]
        _here(self._buf, q, k, v, positions, start, counts)
        if v.shape != k.shape or k.shape[-3] != n:
            raise ValueError("queries of shape %s, keys of %s, values of %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
        if positions.shape != (*lead, n):
            raise ValueError("positions of shape %s, needs %s" % (tuple(positions.shape), (*lead, n)))
        out = torch.empty(q.shape, dtype=self.dtype, device=self.device)
        _check(load().csd_cache_write_rotated(self._h, layer, rotary._config(), ctypes.byref(qh), ctypes.byref(kh), ctypes.byref(vh),
                                              _ptr(positions, torch.int32, rows * n), _ptr(start, torch.int32, rows),
                                              _ptr(counts, torch.int32, rows), n, out.data_ptr(), _stream()), "csd_cache_write_rotated")
        return out

    def write_packed(self, layer, k, v, offsets):
        """k, v [tokens][kv heads][head_dim] of all prompts behind each other: problem p's are offsets[p] .. offsets[p + 1] - 1 (offsets [P + 1]
        int32, ascending), which become its prompt, from position 0 on."""
        c = self.cfg
        kh, vh = (_packed(t, self.dtype, c.n_kv_heads, c.head_dim) for t in (k, v))
        if v.shape != k.shape or k.dim() != 3:
            raise ValueError("keys of shape %s, values of shape %s" % (tuple(k.shape), tuple(v.shape)))
        _here(self._buf, offsets)
        if offsets.shape != (self.P + 1,):
            raise ValueError("offsets of shape %s, needs %s" % (tuple(offsets.shape), (self.P + 1,)))
        _check(load().csd_cache_write_packed(self._h, layer, ctypes.byref(kh), ctypes.byref(vh), _ptr(offsets, torch.int32, self.P + 1),
                                             len(k), _stream()), "csd_cache_write_packed")

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


def _here(*tensors) -> None:
    """The launches are of the current device."""
    for t in tensors:
        if t is not None and t.is_cuda and t.get_device() != torch._C._cuda_getDevice():
            raise ValueError("a tensor of cuda:%d while cuda:%d is the current device" % (t.get_device(), torch._C._cuda_getDevice()))


def _now():
    """The current stream and device, of a tensor's calls in native code."""
    if _native is None:
        load()
    device = torch._C._cuda_getDevice()
    return torch._C._cuda_getCurrentRawStream(device), device


def _packed(t: torch.Tensor, dtype, n_heads: int, dim: int) -> Heads:
    """A tensor [tokens][heads][dim], or one with several evenly spaced leading axes of tokens."""
    if not t.is_cuda or t.dtype != dtype:
        raise TypeError("expected a device tensor of dtype %s" % dtype)
    _here(t)
    _no_gradients(t)
    shape, stride = tuple(t.shape), t.stride()
    if len(shape) < 3 or shape[-2:] != (n_heads, dim):
        raise ValueError("tensor of shape %s, needs %s" % (shape, ("tokens", n_heads, dim)))
    if stride[-1] != 1:
        raise TypeError("a head's values must be contiguous")
    h = Heads(t.data_ptr(), 0, _spacing(shape[:-2], stride), stride[-2] if n_heads > 1 else 0)
    if (h.data or 0) % 16 or h.token_stride % 8 or h.head_stride % 8:
        raise ValueError("heads must start at multiples of 16 bytes")
    return h


def _overlap(a: torch.Tensor, b: torch.Tensor) -> bool:
    ends = lambda t: (t.data_ptr(), t.data_ptr() + (1 + sum((n - 1) * s for n, s in zip(t.shape, t.stride()))) * t.element_size())
    (x, y), (z, w) = ends(a), ends(b)
    return a.numel() > 0 and b.numel() > 0 and x < w and z < y


def rotate(x: torch.Tensor, positions: torch.Tensor, rotary: Rotary, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """Queries and keys x [..., heads, head_dim] (bfloat16, float16; a slice of a projection's output is fine) turned by their positions
    [...] int32: the first rotary.dim values of each head, the others as they are.  out: x itself, or another tensor of its shape."""
    if out is None and x.is_cuda:
        now = _now()
        got = _native.rotate(*now, *rotary._call, x, positions)
        if got is not None:
            _check(got[0], "csd_rotate")
            return got[1]
    if x.dim() < 3 or x.dtype not in (torch.bfloat16, torch.float16):
        raise TypeError("expected [..., heads, head_dim] of bfloat16 or float16")
    if positions.shape != x.shape[:-2]:
        raise ValueError("positions of shape %s, needs %s" % (tuple(positions.shape), tuple(x.shape[:-2])))
    H, D = x.shape[-2:]
    heads = _packed(x, x.dtype, H, D)
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    elif out.shape != x.shape:
        raise ValueError("out of shape %s, needs %s" % (tuple(out.shape), tuple(x.shape)))
    to = _packed(out, x.dtype, H, D)
    _here(positions)
    if _overlap(x, out) and (x.data_ptr() != out.data_ptr() or x.stride() != out.stride()):
        raise ValueError("out overlaps x")
    _check(load().csd_rotate(rotary._config(), ctypes.byref(heads), _ptr(positions, torch.int32, positions.numel()), positions.numel(),
                             H, D, TYPES[x.dtype], ctypes.byref(to), _stream()), "csd_rotate")
    return out


def prompt_attend(q, k, v, offsets, scale=None, out=None, lse=None):
    """Attention of packed sequences to themselves: q [tokens][heads][head_dim], k, v [tokens][kv heads][head_dim] (bfloat16, float16; slices of a
    projection's output are fine), sequence s the tokens offsets[s] .. offsets[s + 1] - 1 (offsets int32, ascending), each of which sees
    those up to itself.  Returns [tokens][heads][head_dim]; lse: a float32 tensor [tokens][heads] that takes the logarithms of the sums.
    scale: 1 / sqrt(head_dim) where None.  Tokens of no sequence are not written (where out is None they hold anything)."""
    if out is None and lse is None and q.is_cuda:
        now = _now()
        got = _native.prompt_attend(*now, q, k, v, offsets, scale)
        if got is not None:
            _check(got[0], "csd_prompt_attend")
            return got[1]
    if q.dim() != 3 or q.dtype not in (torch.bfloat16, torch.float16) or k.dim() != 3:
        raise TypeError("expected [tokens][heads][head_dim] of bfloat16 or float16")
    n, H, D = q.shape
    Hk = k.shape[1]
    heads = _packed(q, q.dtype, H, D), _packed(k, q.dtype, Hk, D), _packed(v, q.dtype, Hk, D)
    if len(k) != n or v.shape != k.shape:
        raise ValueError("queries of shape %s, keys of %s, values of %s" % (tuple(q.shape), tuple(k.shape), tuple(v.shape)))
    _no_gradients(out, lse)
    _here(out, lse, offsets)
    if out is None:
        out = torch.empty((n, H, D), dtype=q.dtype, device=q.device)
    if out.shape != q.shape or (lse is not None and lse.shape != (n, H)):
        raise ValueError("out of shape %s, lse of %s" % (tuple(out.shape), None if lse is None else tuple(lse.shape)))
    if offsets.dim() != 1 or len(offsets) < 2:
        raise ValueError("offsets of shape %s" % (tuple(offsets.shape),))
    if any(_overlap(out, t) for t in (q, k, v)):
        raise ValueError("out overlaps an input")
    _check(load().csd_prompt_attend(*map(ctypes.byref, heads), TYPES[q.dtype], H, Hk, D, _ptr(offsets, torch.int32), len(offsets) - 1, n,
                                    D ** -0.5 if scale is None else scale, _ptr(out, q.dtype, n * H * D), _ptr(lse, torch.float32, n * H),
                                    _stream()), "csd_prompt_attend")
    return out


def adjust(logits, tokens=None, path_len=None, counts=None, prompt=None, prompt_len=None, penalties=None, bias=None, mask=None, out=None):
    """Logits [P][N][n][vocab] (bfloat16, float16, float32) as they are sampled from, before targets().  Position t of a path has said the first path_len
    - counts + t + 1 of its tokens [P][N][any] int32 (path_len, counts [P][N] int32, as in attend(); counts None: n), and its prompt's first
    prompt_len [P] (None: all) of prompt [P][any].  penalties [P][3] float32, repetition, presence and frequency: the logit of a token that
    was said is divided by repetition where positive, else multiplied; one that the path said c times loses frequency * c + presence.
    bias [P][vocab] or [vocab] float32 is added.  mask [P][N][n][words] or [words] int32: bit v % 32 of word v / 32 is 0
    where token v becomes -inf.  Positions beyond a path's count become zeros.  out: logits itself, or another tensor of its shape."""
    if logits.is_cuda:
        now = _now()
        got = _native.adjust(*now, logits, tokens, path_len, counts, prompt, prompt_len, penalties, bias, mask, out)
        if got is not None:
            _check(got[0], "csd_adjust")
            return got[1]
    if logits.dtype not in TYPES or logits.dim() != 4:
        raise TypeError("expected logits [P][N][n][vocab]")
    _no_gradients(logits, penalties, bias, out)
    _here(logits, tokens, path_len, counts, prompt, prompt_len, penalties, bias, mask, out)
    P, N, n, V = logits.shape
    if out is None:
        out = torch.empty(logits.shape, dtype=logits.dtype, device=logits.device)
    if out.shape != logits.shape or out.dtype != logits.dtype:
        raise ValueError("out of shape %s and type %s" % (tuple(out.shape), out.dtype))

    def rows(t, dtype, lead, what):
        """(address, distance of the rows, row length) of [*lead][any]"""
        if t is None:
            return None, 0, 0
        if not t.is_cuda or t.dtype != dtype:
            raise TypeError("expected %s as a device tensor of dtype %s" % (what, dtype))
        if t.dim() != len(lead) + 1 or tuple(t.shape[:-1]) != tuple(lead) or (t.stride(-1) != 1 and t.shape[-1] > 1):
            raise ValueError("%s of shape %s, needs rows %s" % (what, tuple(t.shape), tuple(lead)))
        return t.data_ptr(), _spacing(t.shape[:-1], t.stride()), t.shape[-1]
    x, x_stride, _ = rows(logits, logits.dtype, (P, N, n), "logits")
    y, y_stride, _ = rows(out, logits.dtype, (P, N, n), "out")
    if _overlap(logits, out) and (x != y or logits.stride() != out.stride()):
        raise ValueError("out overlaps the logits")
    said, said_stride, path_cap = rows(tokens, torch.int32, (P, N), "tokens")
    asked, asked_stride, prompt_cap = rows(prompt, torch.int32, (P,), "prompt")
    b, b_stride, b_size = rows(bias, torch.float32, () if bias is not None and bias.dim() == 1 else (P,), "bias")
    m, m_stride, m_size = rows(mask, torch.int32, () if mask is not None and mask.dim() == 1 else (P, N, n), "mask")
    if (bias is not None and b_size != V) or (mask is not None and m_size < (V + 31) // 32):
        raise ValueError("bias or mask too short for %d tokens" % V)
    if tokens is not None and path_len is None:
        raise ValueError("tokens need path_len")
    if penalties is not None and penalties.shape != (P, 3):
        raise ValueError("penalties of shape %s, needs %s" % (tuple(penalties.shape), (P, 3)))
    if tokens is not None and path_cap == 0:
        said = None
    if prompt is not None and prompt_cap == 0:
        asked = None
    a = Adjustment(P, N, n, V, TYPES[logits.dtype], x, x_stride, y, y_stride, _ptr(counts, torch.int32, P * N), _ptr(penalties, torch.float32, 3 * P),
                   said, said_stride, path_cap, _ptr(path_len, torch.int32, P * N), asked, asked_stride, prompt_cap,
                   _ptr(prompt_len, torch.int32, P), b, b_stride, m, m_stride)
    _check(load().csd_adjust(ctypes.byref(a), _stream()), "csd_adjust")
    return out


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
