"""Binding over the worker's part of the C-ABI HIP library (include/br_kv.h): block tables, the 8-bit cache of keys and
values, attention over it.

As in `binding`: argument marshalling only, every step runs in the library's kernels, PyTorch supplies device memory and
the stream, and nothing falls back to the CPU.  All `*_device` calls enqueue on the cache's stream and return; they check
types, shapes, strides and devices, since the C ABI takes bare pointers.  Tensors made or used on another stream are the
caller's to order against the cache's stream (`stream.wait_stream`, `Tensor.record_stream`).  Memory that a cache makes itself
(workspace, `new_layer`, `alloc_step`) is the cache's stream's, whatever stream is current; `lens` and `table` at the start may be the current one's.

    cfg = kv.KvConfig(rows=96, n_blocks=4096, max_blocks=512, n_kv_heads=8, n_q_heads=32, head_dim=128, fmt="fp8")
    cache = kv.KvCache(cfg)
    layers = [cache.new_layer() for _ in range(n_layers)]
    step = cache.alloc_step(token_cap=8192)
    ...
    cache.step_device(keep, add, step)                        # tables and slots of this decode step
    for layer in layers:
        cache.append_device(layer, k, v, step["slot"])        # k, v [token_cap, n_kv_heads, head_dim]
        cache.attend_device(layer, q, out, start=step["start"], count=step["count"], max_count=longest)
"""
from __future__ import annotations

import contextlib
import ctypes as C
import struct
from dataclasses import dataclass
from typing import Dict, Optional

from .binding import BR_OK, BrError, load as _load

FMT = dict(int8=0, fp8=1)
NSTATS = 8
ST = dict(tokens=0, used=1, free=2, rows=3, added=4, refused=5, no_blocks=6, taken=7)
STATUS = dict(taken=0, no_blocks=1, too_long=2, no_room=3)
EXPORTS = ("br_kv_workspace_bytes", "br_kv_init", "br_kv_step", "br_kv_append", "br_kv_read", "br_kv_attend", "br_kv_free",
           "br_kv_last_hip_error", "br_kv_get_layout")

_P, _I, _L = C.c_void_p, C.c_int32, C.c_int64


class _Config(C.Structure):
    _fields_ = [(k, _I) for k in ("n_workers", "rows", "block_tokens", "n_blocks", "max_blocks", "n_kv_heads", "n_q_heads", "head_dim", "fmt", "pad")] + \
               [("stream", _P), ("workspace", _P), ("workspace_bytes", C.c_uint64)]


class _State(C.Structure):
    _fields_ = [("lens", _P), ("table", _P)]


class _Lengths(C.Structure):
    _fields_ = [("keep", _P), ("add", _P)]


class _StepOut(C.Structure):
    _fields_ = [(k, _P) for k in ("slot", "pos", "start", "count", "status", "stats")] + [("token_cap", _I), ("pad", _I)]


class _Layer(C.Structure):
    _fields_ = [(k, _P) for k in ("k", "v", "k_scale", "v_scale")]


class _Tokens(C.Structure):
    _fields_ = [("k", _P), ("v", _P), ("slot", _P)] + [(k, _L) for k in ("k_token", "k_head", "v_token", "v_head")] + [("n_tokens", _I), ("dtype", _I)]


class _Attention(C.Structure):
    _fields_ = [(k, _P) for k in ("q", "out", "lse", "start", "count", "lens", "table")] + [(k, _L) for k in ("q_token", "q_head", "out_token", "out_head")] + \
               [("n_tokens", _I), ("max_count", _I), ("window", _I), ("dtype", _I), ("scale", C.c_float), ("pad", _I)]


class _Layout(C.Structure):
    _fields_ = [("lens", C.c_uint64), ("table", C.c_uint64), ("total_bytes", C.c_uint64)]


# The structs of the calls of a decode loop, packed in one go (a ctypes struct costs as much as the call): pointers, strides, numbers.
_PACK_LENGTHS, _PACK_STEP, _PACK_TOKENS, _PACK_ATTENTION = (struct.Struct(f) for f in ("@2P", "@6P2i", "@3P4q2i", "@7P4q4ifi"))
_lib = None


def load():
    """The library with the symbols of include/br_kv.h bound (raises if one is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _load()
    for name in EXPORTS:
        getattr(lib, name).restype = C.c_int32
    lib.br_kv_workspace_bytes.restype = C.c_uint64
    lib.br_kv_workspace_bytes.argtypes = [C.POINTER(_Config)]
    lib.br_kv_init.argtypes = [C.POINTER(_Config), C.POINTER(_State), C.POINTER(_P)]
    for name in ("br_kv_step", "br_kv_append", "br_kv_read", "br_kv_attend"):
        getattr(lib, name).argtypes = [_P, _P, _P]
    lib.br_kv_free.restype = None
    lib.br_kv_free.argtypes = [_P]
    lib.br_kv_last_hip_error.argtypes = [_P]
    lib.br_kv_get_layout.argtypes = [_P, C.POINTER(_Layout)]
    _lib = lib
    return lib


@dataclass(frozen=True)
class KvConfig:
    """Sizes of a cache (limits and meanings: br_kv_config)."""

    rows: int                 # requests a worker may hold: the router's slot limit B
    n_blocks: int             # blocks of each worker
    max_blocks: int           # entries of a row's table
    block_tokens: int = 16
    n_workers: int = 1
    n_kv_heads: int = 1
    n_q_heads: int = 1
    head_dim: int = 64
    fmt: str = "int8"         # "int8" or "fp8" (e4m3)


def _config(cfg: KvConfig, stream=0, workspace=0, workspace_bytes=0) -> _Config:
    return _Config(n_workers=cfg.n_workers, rows=cfg.rows, block_tokens=cfg.block_tokens, n_blocks=cfg.n_blocks, max_blocks=cfg.max_blocks,
                   n_kv_heads=cfg.n_kv_heads, n_q_heads=cfg.n_q_heads, head_dim=cfg.head_dim, fmt=FMT.get(cfg.fmt, -1), stream=stream, workspace=workspace,
                   workspace_bytes=workspace_bytes)


def workspace_bytes(cfg: KvConfig) -> int:
    return int(load().br_kv_workspace_bytes(C.byref(_config(cfg))))


class KvLayer:
    """One layer's cache: codes k [n_workers * n_blocks, n_kv_heads, block_tokens, head_dim] and v [.., head_dim, block_tokens]
    (uint8), scales k_scale, v_scale [n_workers * n_blocks, n_kv_heads] (float32)."""

    def __init__(self, k, v, k_scale, v_scale):
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.sizes = (k.shape, k.get_device())  # a cache takes layers of its own sizes only
        self.struct = _Layer(k=k.data_ptr(), v=v.data_ptr(), k_scale=k_scale.data_ptr(), v_scale=v_scale.data_ptr())
        self.ref, self.at = C.byref(self.struct), C.addressof(self.struct)


class KvCache:
    """Owns a workspace tensor and a br_kv_ctx; all methods only marshal arguments."""

    def __init__(self, cfg: KvConfig, lens=None, table=None, device="cuda:0", stream=None):
        """lens [n_workers, rows], table [n_workers, rows, max_blocks] (int32): requests held at the start."""
        import torch
        device = torch.device(device)
        if device.index is None:
            device = torch.device("cuda", torch.cuda.current_device())
        self._sizes(torch, load(), cfg, device)
        W, B = cfg.n_workers, cfg.rows
        nbytes = workspace_bytes(cfg)
        if nbytes == 0:
            raise BrError("invalid configuration")
        if (lens is None) != (table is None):
            raise BrError("lens and table come together")
        state = None
        if lens is not None:
            self._check(lens, "lens", (W, B), torch.int32)
            self._check(table, "table", (W, B, cfg.max_blocks), torch.int32)
            state = C.byref(_State(lens=lens.data_ptr(), table=table.data_ptr()))
        current = torch.cuda.current_stream(self.device)
        self.stream = stream if stream is not None else current
        if lens is not None and self.stream != current:  # what is on its way there comes first
            self.stream.wait_stream(current)
        with self._own():
            self.ws = torch.empty(nbytes // 4 + 64, dtype=torch.int32, device=self.device)
        assert self.ws.data_ptr() % 256 == 0
        c = _config(cfg, stream=self.stream.cuda_stream, workspace=self.ws.data_ptr(), workspace_bytes=self.ws.numel() * 4)
        ctx = _P()
        with torch.cuda.device(self.device):
            self._done(self.lib.br_kv_init(C.byref(c), state, C.byref(ctx)), "br_kv_init")
        self.ctx = ctx
        if lens is not None and self.stream != current:  # (their memory is not handed out again before they have been copied)
            lens.record_stream(self.stream), table.record_stream(self.stream)
        lay = _Layout()
        self._done(self.lib.br_kv_get_layout(ctx, C.byref(lay)), "br_kv_get_layout")
        #: cached tokens of every row and the block tables, as they are on the device: [n_workers, rows] and [n_workers, rows, max_blocks]
        self.lens = self.ws[lay.lens // 4:lay.lens // 4 + W * B].view(W, B)
        self.table = self.ws[lay.table // 4:lay.table // 4 + W * B * cfg.max_blocks].view(W, B, cfg.max_blocks)

    # -- checks ---------------------------------------------------------------
    def _sizes(self, torch, lib, cfg: KvConfig, device) -> None:
        """What the checks of every call go by, and room for the calls' structs."""
        self.torch, self.lib, self.cfg, self.device = torch, lib, cfg, device
        self._index = device.index if device.type == "cuda" else -1
        self._dtypes = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
        self._i32, self._f32, self._i64 = torch.int32, torch.float32, torch.int64
        W, B = cfg.n_workers, cfg.rows
        self._rows, self._stats, self._tables = torch.Size((W, B)), torch.Size((W, NSTATS)), torch.Size((W, B, cfg.max_blocks))
        self._scale = cfg.head_dim ** -0.5
        self._layer = (torch.Size((W * cfg.n_blocks, cfg.n_kv_heads, cfg.block_tokens, cfg.head_dim)), self._index)
        self._args = C.create_string_buffer(256)
        self._at = C.addressof(self._args)

    def _done(self, rc: int, what: str) -> None:
        if rc != BR_OK:
            ctx = getattr(self, "ctx", None)
            raise BrError(f"{what} failed: rc={rc} hip_error={self.lib.br_kv_last_hip_error(ctx) if ctx else 0}")

    def _check(self, x, name: str, shape, dtype) -> int:
        """The address of a contiguous tensor of that shape and type on this device."""
        if x.shape != shape or x.dtype is not dtype or x.get_device() != self._index or not x.is_contiguous():
            raise BrError(f"{name} must be a contiguous {dtype} tensor of shape {tuple(shape)} on {self.device}")
        return x.data_ptr()

    def _tokens(self, x, name: str, n, heads: int):
        """(type code, strides of tokens and heads) of keys, values, queries or outputs [n, heads, head_dim] with contiguous channels."""
        shape = x.shape
        if len(shape) != 3 or (n is not None and shape[0] != n) or shape[1] != heads or shape[2] != self.cfg.head_dim or x.get_device() != self._index:
            raise BrError(f"{name} must have shape {('tokens' if n is None else n, heads, self.cfg.head_dim)} on {self.device}")
        token, head, channel = x.stride()
        if channel != 1 and shape[0]:
            raise BrError(f"{name} must have contiguous channels")
        dtype = self._dtypes.get(x.dtype)
        if dtype is None:
            raise BrError(f"{name} must be float16, bfloat16 or float32, not {x.dtype}")
        return dtype, token, head

    # -- memory ---------------------------------------------------------------
    def _own(self):
        """Memory made in here belongs to the cache's stream: the allocator hands it out again behind that stream's work."""
        return self.torch.cuda.stream(self.stream) if self._index >= 0 else contextlib.nullcontext()

    def layer(self, k, v, k_scale, v_scale) -> KvLayer:
        """A layer over memory that is there (16-byte aligned)."""
        t, c = self.torch, self.cfg
        n, H, b, D = c.n_workers * c.n_blocks, c.n_kv_heads, c.block_tokens, c.head_dim
        self._check(k, "k", (n, H, b, D), t.uint8)
        self._check(v, "v", (n, H, D, b), t.uint8)
        self._check(k_scale, "k_scale", (n, H), t.float32)
        self._check(v_scale, "v_scale", (n, H), t.float32)
        return KvLayer(k, v, k_scale, v_scale)

    def new_layer(self) -> KvLayer:
        t, c = self.torch, self.cfg
        n, H, b, D = c.n_workers * c.n_blocks, c.n_kv_heads, c.block_tokens, c.head_dim
        e = lambda shape, dtype: t.empty(shape, dtype=dtype, device=self.device)
        with self._own():
            return self.layer(e((n, H, b, D), t.uint8), e((n, H, D, b), t.uint8), e((n, H), t.float32), e((n, H), t.float32))

    def alloc_step(self, token_cap: int) -> Dict[str, object]:
        """Output arrays of step_device, with room for token_cap new tokens per worker."""
        t, W, B = self.torch, self.cfg.n_workers, self.cfg.rows
        e = lambda *shape: t.empty(shape, dtype=t.int32, device=self.device)
        with self._own():
            return dict(slot=e(W, token_cap), pos=e(W, token_cap), start=e(W, B), count=e(W, B), status=e(W, B),
                        stats=t.empty((W, NSTATS), dtype=t.int64, device=self.device))

    # -- calls ----------------------------------------------------------------
    def step_device(self, keep, add, out) -> None:
        """Tables of the next step (br_kv_step): keep, add [n_workers, rows] int32; out: alloc_step's arrays."""
        check, i32, rows = self._check, self._i32, self._rows
        slot = out["slot"]
        if slot.dim() != 2 or slot.shape[0] != rows[0]:
            raise BrError("slot must have shape (n_workers, token_cap)")
        _PACK_LENGTHS.pack_into(self._args, 0, check(keep, "keep", rows, i32), check(add, "add", rows, i32))
        _PACK_STEP.pack_into(self._args, 16, check(slot, "slot", slot.shape, i32), check(out["pos"], "pos", slot.shape, i32), check(out["start"], "start", rows, i32),
                             check(out["count"], "count", rows, i32), check(out["status"], "status", rows, i32), check(out["stats"], "stats", self._stats, self._i64),
                             slot.shape[1], 0)
        rc = self.lib.br_kv_step(self.ctx, self._at, self._at + 16)
        if rc:
            self._done(rc, "br_kv_step")

    def _pack_tokens(self, layer, k, v, slot) -> None:
        if layer.sizes != self._layer:
            raise BrError("the layer is one of another cache's sizes")
        W, n = self._rows[0], slot.numel()
        if n % W or slot.dtype is not self._i32 or slot.get_device() != self._index or not slot.is_contiguous():
            raise BrError(f"slot must be a contiguous int32 tensor on {self.device} with the same number of tokens for each worker")
        dtype, k_token, k_head = self._tokens(k, "k", n, self.cfg.n_kv_heads)
        v_dtype, v_token, v_head = self._tokens(v, "v", n, self.cfg.n_kv_heads)
        if v_dtype != dtype:
            raise BrError("k and v must have one type")
        _PACK_TOKENS.pack_into(self._args, 0, k.data_ptr(), v.data_ptr(), slot.data_ptr(), k_token, k_head, v_token, v_head, n // W, dtype)

    def append_device(self, layer: KvLayer, k, v, slot) -> None:
        """Tokens into the cache (br_kv_append): k, v [tokens, n_kv_heads, head_dim], slot [tokens] (step_device's, or alike)."""
        self._pack_tokens(layer, k, v, slot)
        rc = self.lib.br_kv_append(self.ctx, layer.at, self._at)
        if rc:
            self._done(rc, "br_kv_append")

    def read_device(self, layer: KvLayer, slot, k, v) -> None:
        """Tokens out of the cache into k, v [tokens, n_kv_heads, head_dim] (br_kv_read)."""
        self._pack_tokens(layer, k, v, slot)
        rc = self.lib.br_kv_read(self.ctx, layer.at, self._at)
        if rc:
            self._done(rc, "br_kv_read")

    def attend_device(self, layer: KvLayer, q, out, lse=None, start=None, count=None, max_count: int = 1, scale: Optional[float] = None, window: int = 0,
                      lens=None, table=None) -> None:
        """Attention of q [tokens, n_q_heads, head_dim] over the rows' cached tokens into out (br_kv_attend).

        start, count [n_workers, rows] (step_device's): a row's query tokens; none: token r belongs to row r.  lse [tokens, n_q_heads] float32.
        scale: 1 / sqrt(head_dim) if not given.  lens, table: instead of the cache's own."""
        if layer.sizes != self._layer:
            raise BrError("the layer is one of another cache's sizes")
        heads = self.cfg.n_q_heads
        dtype, q_token, q_head = self._tokens(q, "q", None, heads)
        n = q.shape[0]
        if dtype == 2:
            raise BrError("q must be float16 or bfloat16")
        out_dtype, out_token, out_head = self._tokens(out, "out", n, heads)
        if out_dtype != dtype:
            raise BrError("q and out must have one type")
        if (start is None) != (count is None):
            raise BrError("start and count come together")
        check, i32, rows = self._check, self._i32, self._rows
        at = (q.data_ptr(), out.data_ptr(), 0 if lse is None else check(lse, "lse", (n, heads), self._f32),
              0 if start is None else check(start.view(rows) if start.shape != rows and start.numel() == rows.numel() else start, "start", rows, i32),
              0 if count is None else check(count.view(rows) if count.shape != rows and count.numel() == rows.numel() else count, "count", rows, i32),
              0 if lens is None else check(lens, "lens", rows, i32), 0 if table is None else check(table, "table", self._tables, i32), q_token, q_head, out_token, out_head, n)
        try:
            _PACK_ATTENTION.pack_into(self._args, 0, *at, max_count, window, dtype, self._scale if scale is None else scale, 0)
        except (struct.error, OverflowError):
            raise BrError("max_count and window must be whole numbers of 32 bits, scale a number of 32 bits") from None
        rc = self.lib.br_kv_attend(self.ctx, layer.at, self._at)
        if rc:
            self._done(rc, "br_kv_attend")

    def close(self) -> None:
        if getattr(self, "ctx", None):
            self.stream.synchronize()
            self.lib.br_kv_free(self.ctx)
            self.ctx = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass
