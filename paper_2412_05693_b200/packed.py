"""Packed caches: the ctypes layer of the bm_packed_* entry points of include/batchmax.h.

A packed cache holds its rows in 4 bits.  It is written token by token, block by block or out of a
:class:`~paper_2412_05693_b200.binding.BatchMaxCache`, read back, and attended to::

    cache = PackedCache(PackedConfig(batch=16, n_q_heads=32, n_kv_heads=8, head_dim=128, capacity=2048))
    cache.write_from(handle)                     # the pairs that an evicting prefill kept
    lens = torch.full((16,), n, dtype=torch.int32, device="cuda")
    ...                                          # per token: q (16, 1, 32, 128), k and v (16, 1, 8, 128)
    cache.write(k, v, start=lens)
    lens += 1
    out = cache.attend(q, lens)
"""
from __future__ import annotations

import ctypes as C
from dataclasses import dataclass

from .binding import BM_BF16, BM_F32, _check, _sz, _vp, bm_packed_config_t, fastcall, lib


@dataclass
class PackedConfig:
    batch: int
    n_q_heads: int
    n_kv_heads: int
    head_dim: int
    capacity: int                # rows a (sample, kv-head) cache may hold
    queries_max: int = 1         # largest number of queries per sample of an attend call
    dtype: str = "bf16"          # "bf16" | "f32": of keys, values, queries and outputs
    n_layers: int = 1
    softmax_scale: float = 0.0
    device: int = 0

    def c(self) -> bm_packed_config_t:
        return bm_packed_config_t(self.batch, self.n_layers, self.n_q_heads, self.n_kv_heads, self.head_dim, self.capacity,
                                  self.queries_max, BM_BF16 if self.dtype == "bf16" else BM_F32, self.softmax_scale, self.device)


def _size_query(fn_name: str, cfg: PackedConfig) -> int:
    out, c = _sz(0), cfg.c()
    _check(getattr(lib(), fn_name)(C.byref(c), C.byref(out)), fn_name)
    return out.value


def packed_bytes_per_sample(cfg: PackedConfig) -> int:
    return _size_query("bm_packed_bytes_per_sample", cfg)


def packed_arena_bytes(cfg: PackedConfig) -> int:
    return _size_query("bm_packed_arena_bytes", cfg)


def packed_workspace_bytes(cfg: PackedConfig) -> int:
    return _size_query("bm_packed_workspace_bytes", cfg)


def packed_max_batch(cfg: PackedConfig, hbm_budget_bytes: int) -> int:
    out, c = C.c_int32(0), cfg.c()
    _check(lib().bm_packed_max_batch(C.byref(c), hbm_budget_bytes, C.byref(out)), "bm_packed_max_batch")
    return out.value


def last_packed_path() -> int:
    """0: warps that share the caches' tiles took this thread's last attend call, 1: tiles of 128 query rows did."""
    return int(lib().bm_last_packed_path())


class PackedCache:
    """Handle of one bm_packed_t plus the torch tensors backing its arena and the workspace of its attend calls.

    Tensors are checked for the handle's dtype, device and shape (AssertionError); work goes to the device's current
    stream unless a stream is given.  attend calls that may overlap on the GPU need a workspace each.
    """

    def __init__(self, cfg: PackedConfig, arena=None, workspace=None, stream=None):
        import torch
        self.cfg, self.torch = cfg, torch
        self.device = torch.device("cuda", cfg.device)
        self.dtype = torch.bfloat16 if cfg.dtype == "bf16" else torch.float32
        need = packed_arena_bytes(cfg)
        with self._on(stream):   # (memory of the stream that will use it first)
            self.arena = arena if arena is not None else torch.empty(need, dtype=torch.uint8, device=self.device)
            self.workspace = workspace if workspace is not None else self.new_workspace()
        self._check_buffer(self.arena)
        h, c = _vp(None), cfg.c()
        _check(lib().bm_packed_create(C.byref(c), self.arena.data_ptr(), self.arena.numel(), self._stream(stream), C.byref(h)),
               "bm_packed_create")
        self.h = h
        self._fast = fastcall()   # calls of plain tensors on the current stream go through csrc/fastcall.cpp
        handle = (h.value, cfg.dtype == "bf16", cfg.device, cfg.n_q_heads, cfg.n_kv_heads, cfg.head_dim)
        address = lambda fn: C.cast(fn, _vp).value
        self._fast_write = (address(lib().bm_packed_write), *handle)
        self._fast_read = (address(lib().bm_packed_read), *handle)
        self._fast_attend = (address(lib().bm_packed_attend), *handle)

    def close(self):
        if getattr(self, "h", None) is not None and self.h:
            lib().bm_packed_destroy(self.h)
            self.h = self._fast = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def new_workspace(self):
        """A workspace for attend calls that may overlap others of this cache."""
        return self.torch.empty(packed_workspace_bytes(self.cfg), dtype=self.torch.uint8, device=self.device)

    # -- arguments ------------------------------------------------------------------------------------
    def _on(self, stream):
        return self.torch.cuda.stream(stream) if stream is not None else self.torch.cuda.device(self.device)

    def _stream(self, stream):
        if stream is not None:
            return stream.cuda_stream
        return self.torch._C._cuda_getCurrentRawStream(self.cfg.device)

    def _check_buffer(self, t):
        assert t.dtype == self.torch.uint8 and t.is_contiguous() and t.device == self.device, \
            "arena and workspace must be contiguous uint8 tensors on the handle's device"

    def _check_rows(self, t, heads):
        """(nsamples, I, heads, d); a sample's and a token's heads lie together, samples and tokens may be strided."""
        d = self.cfg.head_dim
        assert t.dim() == 4 and t.shape[2] == heads and t.shape[3] == d and t.shape[0] > 0 and t.shape[1] > 0 \
            and t.dtype == self.dtype and t.device == self.device, \
            "rows must be (nsamples, I, heads, head_dim) tensors of the handle's dtype on its device"
        s = t.stride()
        assert s[3] == 1 and (s[2] == d or heads == 1), "a token's heads must lie together"
        return (s[0] if t.shape[0] > 1 else 0), (s[1] if t.shape[1] > 1 else 0)

    def _index(self, t, n):
        if t is None:
            return None
        assert t.dtype == self.torch.int32 and t.dim() == 1 and t.shape[0] == n and t.is_contiguous() and t.device == self.device, \
            "lengths and rows must be contiguous int32 tensors of one entry per sample on the handle's device"
        return t.data_ptr()

    # -- the calls --------------------------------------------------------------------------------------
    def write(self, k, v, start=None, counts=None, layer: int = 0, sample0: int = 0, stream=None):
        """k, v (ns, I, Hkv, d): token i of sample s goes to row start[s] + i (start None: row i), the first counts[s] only."""
        if stream is None and self._fast is not None:
            rc = self._fast.packed_write(*self._fast_write, k, v, start, counts, layer, sample0)
            if rc is not None:
                if rc:
                    _check(rc, "bm_packed_write")
                return
        assert v.shape == k.shape, "k and v must have one shape"
        ns, I = k.shape[0], k.shape[1]
        strides = (C.c_int64 * 4)(*self._check_rows(k, self.cfg.n_kv_heads), *self._check_rows(v, self.cfg.n_kv_heads))
        _check(lib().bm_packed_write(self.h, layer, sample0, ns, k.data_ptr(), v.data_ptr(), strides, I, self._index(start, ns),
                                     self._index(counts, ns), self._stream(stream)), "bm_packed_write")

    def write_from(self, handle, layer: int = 0, sample0: int = 0, nsamples: int | None = None, from_layer: int = 0,
                   from_sample0: int = 0, stream=None):
        """The pairs that the caches of a BatchMaxCache hold become rows 0 .. n - 1; returns n."""
        ns = self.cfg.batch - sample0 if nsamples is None else nsamples
        _check(lib().bm_packed_write_from(self.h, layer, sample0, ns, handle.h, from_layer, from_sample0, self._stream(stream)),
               "bm_packed_write_from")
        return handle.length(from_layer, from_sample0)[0]

    def read(self, row0: int, rows: int, lens=None, out=None, layer: int = 0, sample0: int = 0, nsamples: int | None = None,
             stream=None):
        """(k, v), each (ns, rows, Hkv, d): what rows row0 .. stand for, zeros at and past lens[s]."""
        ns = self.cfg.batch - sample0 if nsamples is None else nsamples
        if not (0 <= row0 < row0 + rows <= self.cfg.capacity and 0 <= sample0 < sample0 + ns <= self.cfg.batch):
            _check(1, "bm_packed_read")   # (before memory is taken for them)
        if stream is None and out is None and self._fast is not None:
            got = self._fast.packed_read(*self._fast_read, row0, rows, layer, sample0, ns, lens)
            if got is not None:
                if type(got) is int:
                    _check(got, "bm_packed_read")
                return got
        shape = (ns, rows, self.cfg.n_kv_heads, self.cfg.head_dim)
        if out is None:
            with self._on(stream):
                k, v = (self.torch.empty(shape, dtype=self.dtype, device=self.device) for _ in range(2))
        else:
            k, v = out
            for t in out:
                assert t.shape == shape and t.is_contiguous() and t.dtype == self.dtype and t.device == self.device, \
                    "out must be two contiguous tensors (nsamples, rows, n_kv_heads, head_dim)"
        _check(lib().bm_packed_read(self.h, layer, sample0, ns, row0, rows, self._index(lens, ns), k.data_ptr(), v.data_ptr(),
                                    self._stream(stream)), "bm_packed_read")
        return k, v

    def attend(self, q, lens, first=None, max_len: int = 0, out=None, workspace=None, layer: int = 0, sample0: int = 0, stream=None):
        """q (ns, I, Hq, d) over rows first[s] .. of caches of lens[s] rows, causal among the I; returns out (ns, I, Hq, d)."""
        if stream is None and self._fast is not None:
            got = self._fast.packed_attend(*self._fast_attend, q, lens, first, out, self.workspace if workspace is None else workspace,
                                           max_len, layer, sample0)
            if got is not None:
                if type(got) is int:
                    _check(got, "bm_packed_attend")
                return got
        strides = (C.c_int64 * 2)(*self._check_rows(q, self.cfg.n_q_heads))
        ns, I = q.shape[0], q.shape[1]
        if out is None:
            with self._on(stream):
                out = self.torch.empty(q.shape, dtype=self.dtype, device=self.device)
        else:
            assert out.is_contiguous() and out.dtype == self.dtype and out.shape == q.shape and out.device == self.device, \
                "out must be a contiguous tensor of q's shape and dtype"
        if workspace is None:
            workspace = self.workspace
        self._check_buffer(workspace)
        _check(lib().bm_packed_attend(self.h, layer, sample0, ns, q.data_ptr(), strides, I, self._index(lens, ns),
                                      self._index(first, ns), max_len, out.data_ptr(), workspace.data_ptr(), workspace.numel(),
                                      self._stream(stream)), "bm_packed_attend")
        return out

    def status(self, stream=None) -> int:
        """The device status word: 0, 3 (a write met a row outside its cache) or 6 (a bounded wait expired)."""
        w = C.c_int32(0)
        _check(lib().bm_packed_status(self.h, C.byref(w), self._stream(stream)), "bm_packed_status")
        return w.value

    def clear_status(self, stream=None):
        _check(lib().bm_packed_clear_status(self.h, self._stream(stream)), "bm_packed_clear_status")

    def selftest_wait_timeout(self, stream=None):
        """Enqueue a warp whose bounded wait runs out: status() is 6 afterwards, until clear_status()."""
        _check(lib().bm_packed_selftest_wait_timeout(self.h, self._stream(stream)), "bm_packed_selftest_wait_timeout")
