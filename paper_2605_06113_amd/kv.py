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

Of a cache with `shared=True` several rows may hold the same blocks (samples of one prompt, beams):

    cache.fork_device(rows, length)                           # row r goes on from the first length[r] tokens of row rows[r]
    cache.step_device(keep, add, step)                        # rows that write into a block that others hold get one of their own
    cache.plan_device(lead, members, start=step["start"], count=step["count"])   # for all layers of the step
    for layer in layers:
        cache.copy_device(layer, step["copy_src"], step["copy_dst"])   # ... with what it held, before anything is appended
        cache.append_device(layer, k, v, step["slot"])
        cache.attend_shared_device(layer, q, out)             # what rows hold together is read once
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
           "br_kv_last_hip_error", "br_kv_get_layout", "br_kv_shared_workspace_bytes", "br_kv_init_shared", "br_kv_get_shared_layout", "br_kv_fork", "br_kv_step_shared",
           "br_kv_compact", "br_kv_copy", "br_kv_plan", "br_kv_attend_shared", "br_kv_attend_diff")

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


class _SharedLayout(C.Structure):
    _fields_ = [("holders", C.c_uint64), ("total_bytes", C.c_uint64)]


class _Forks(C.Structure):
    _fields_ = [("from_", _P), ("len", _P)]


class _Families(C.Structure):
    _fields_ = [(k, _P) for k in ("lead", "start", "count")] + [("members", _I), ("pad", _I)]


class _Diff(C.Structure):
    _fields_ = [("lam", _P), ("lambda_token", _L)]


class _Moves(C.Structure):
    _fields_ = [(k, _P) for k in ("src", "dst", "src_worker")] + [("n", _I), ("pad", _I)]


# The structs of the calls of a decode loop, packed in one go (a ctypes struct costs as much as the call): pointers, strides, numbers.
_PACK_LENGTHS, _PACK_STEP, _PACK_TOKENS, _PACK_ATTENTION = (struct.Struct(f) for f in ("@2P", "@6P2i", "@3P4q2i", "@7P4q4ifi"))
_PACK_FORKS, _PACK_MOVES, _PACK_FAMILIES, _PACK_DIFF = (struct.Struct(f) for f in ("@2P", "@3P2i", "@3P2i", "@Pq"))
_lib = None


def load():
    """The library with the symbols of include/br_kv.h bound (raises if one is missing)."""
    global _lib
    if _lib is not None:
        return _lib
    lib = _load()
    for name in EXPORTS:
        getattr(lib, name).restype = C.c_int32
    for name in ("br_kv_workspace_bytes", "br_kv_shared_workspace_bytes"):
        getattr(lib, name).restype = C.c_uint64
        getattr(lib, name).argtypes = [C.POINTER(_Config)]
    for name in ("br_kv_init", "br_kv_init_shared"):
        getattr(lib, name).argtypes = [C.POINTER(_Config), C.POINTER(_State), C.POINTER(_P)]
    for name in ("br_kv_step", "br_kv_append", "br_kv_read", "br_kv_attend", "br_kv_copy", "br_kv_attend_shared"):
        getattr(lib, name).argtypes = [_P, _P, _P]
    for name in ("br_kv_step_shared", "br_kv_attend_diff"):
        getattr(lib, name).argtypes = [_P, _P, _P, _P]
    for name in ("br_kv_fork", "br_kv_compact", "br_kv_plan"):
        getattr(lib, name).argtypes = [_P, _P]
    lib.br_kv_get_shared_layout.argtypes = [_P, C.POINTER(_SharedLayout)]
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
    shared: bool = False      # several rows may hold a block (br_kv_init_shared)


def _config(cfg: KvConfig, stream=0, workspace=0, workspace_bytes=0) -> _Config:
    return _Config(n_workers=cfg.n_workers, rows=cfg.rows, block_tokens=cfg.block_tokens, n_blocks=cfg.n_blocks, max_blocks=cfg.max_blocks,
                   n_kv_heads=cfg.n_kv_heads, n_q_heads=cfg.n_q_heads, head_dim=cfg.head_dim, fmt=FMT.get(cfg.fmt, -1), stream=stream, workspace=workspace,
                   workspace_bytes=workspace_bytes)


def workspace_bytes(cfg: KvConfig) -> int:
    lib = load()
    return int((lib.br_kv_shared_workspace_bytes if cfg.shared else lib.br_kv_workspace_bytes)(C.byref(_config(cfg))))


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
            init = "br_kv_init_shared" if cfg.shared else "br_kv_init"
            self._done(getattr(self.lib, init)(C.byref(c), state, C.byref(ctx)), init)
        self.ctx = ctx
        if lens is not None and self.stream != current:  # (their memory is not handed out again before they have been copied)
            lens.record_stream(self.stream), table.record_stream(self.stream)
        lay = _Layout()
        self._done(self.lib.br_kv_get_layout(ctx, C.byref(lay)), "br_kv_get_layout")
        #: cached tokens of every row and the block tables, as they are on the device: [n_workers, rows] and [n_workers, rows, max_blocks]
        self.lens = self.ws[lay.lens // 4:lay.lens // 4 + W * B].view(W, B)
        self.table = self.ws[lay.table // 4:lay.table // 4 + W * B * cfg.max_blocks].view(W, B, cfg.max_blocks)
        if cfg.shared:
            own = _SharedLayout()
            self._done(self.lib.br_kv_get_shared_layout(ctx, C.byref(own)), "br_kv_get_shared_layout")
            #: how many entries of its worker's tables name each block: [n_workers, n_blocks]
            self.holders = self.ws[own.holders // 4:own.holders // 4 + W * cfg.n_blocks].view(W, cfg.n_blocks)

    # -- checks ---------------------------------------------------------------
    def _sizes(self, torch, lib, cfg: KvConfig, device) -> None:
        """What the checks of every call go by, and room for the calls' structs."""
        self.torch, self.lib, self.cfg, self.device = torch, lib, cfg, device
        self._index = device.index if device.type == "cuda" else -1
        self._dtypes = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2}
        self._i32, self._f32, self._i64 = torch.int32, torch.float32, torch.int64
        W, B = cfg.n_workers, cfg.rows
        self._rows, self._stats, self._tables = torch.Size((W, B)), torch.Size((W, NSTATS)), torch.Size((W, B, cfg.max_blocks))
        self._scale, self._half_scale = cfg.head_dim ** -0.5, (cfg.head_dim / 2) ** -0.5
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
        """Output arrays of step_device, with room for token_cap new tokens per worker (of a shared cache copy_src and copy_dst among them)."""
        t, W, B = self.torch, self.cfg.n_workers, self.cfg.rows
        e = lambda *shape: t.empty(shape, dtype=t.int32, device=self.device)
        with self._own():
            out = dict(slot=e(W, token_cap), pos=e(W, token_cap), start=e(W, B), count=e(W, B), status=e(W, B),
                       stats=t.empty((W, NSTATS), dtype=t.int64, device=self.device))
            if self.cfg.shared:
                out.update(copy_src=e(W, B), copy_dst=e(W, B))
            return out

    def alloc_moves(self, n: int) -> Dict[str, object]:
        """Output arrays of compact_device: at most n blocks of a worker move in a call."""
        t, W = self.torch, self.cfg.n_workers
        with self._own():
            return {k: t.empty((W, n), dtype=t.int32, device=self.device) for k in ("src", "dst")}

    # -- calls ----------------------------------------------------------------
    def step_device(self, keep, add, out) -> None:
        """Tables of the next step (br_kv_step, br_kv_step_shared): keep, add [n_workers, rows] int32; out: alloc_step's arrays."""
        check, i32, rows = self._check, self._i32, self._rows
        slot = out["slot"]
        if slot.dim() != 2 or slot.shape[0] != rows[0]:
            raise BrError("slot must have shape (n_workers, token_cap)")
        _PACK_LENGTHS.pack_into(self._args, 0, check(keep, "keep", rows, i32), check(add, "add", rows, i32))
        _PACK_STEP.pack_into(self._args, 16, check(slot, "slot", slot.shape, i32), check(out["pos"], "pos", slot.shape, i32), check(out["start"], "start", rows, i32),
                             check(out["count"], "count", rows, i32), check(out["status"], "status", rows, i32), check(out["stats"], "stats", self._stats, self._i64),
                             slot.shape[1], 0)
        if self.cfg.shared:
            _PACK_MOVES.pack_into(self._args, 96, check(out["copy_src"], "copy_src", rows, i32), check(out["copy_dst"], "copy_dst", rows, i32), 0, rows[1], 0)
            rc = self.lib.br_kv_step_shared(self.ctx, self._at, self._at + 16, self._at + 96)
        else:
            rc = self.lib.br_kv_step(self.ctx, self._at, self._at + 16)
        if rc:
            self._done(rc, "br_kv_step_shared" if self.cfg.shared else "br_kv_step")

    def _is_shared(self) -> None:
        if not self.cfg.shared:
            raise BrError("the cache's blocks have one holder each (shared=False)")

    def fork_device(self, rows, length=None) -> None:
        """Row r becomes the first length[r] tokens (below 0, or no length: all) of row rows[r] of its worker, by holding the same blocks (br_kv_fork).

        rows, length [n_workers, rows] int32, both as they are before the call; rows outside the worker's (-1): row r stays as it is."""
        self._is_shared()
        check, i32, shape = self._check, self._i32, self._rows
        _PACK_FORKS.pack_into(self._args, 0, check(rows, "rows", shape, i32), 0 if length is None else check(length, "length", shape, i32))
        rc = self.lib.br_kv_fork(self.ctx, self._at)
        if rc:
            self._done(rc, "br_kv_fork")

    def _pack_moves(self, src, dst, src_worker) -> None:
        if src.dim() != 2 or src.shape[0] != self._rows[0]:
            raise BrError("src must have shape (n_workers, n)")
        check, i32, shape = self._check, self._i32, src.shape
        _PACK_MOVES.pack_into(self._args, 0, check(src, "src", shape, i32), check(dst, "dst", shape, i32), 0 if src_worker is None else check(src_worker, "src_worker", shape, i32),
                              shape[1], 0)

    def compact_device(self, out) -> None:
        """The blocks in use move to the lowest ids, as many as out (alloc_moves) has room for (br_kv_compact); copy_device with out moves what they hold."""
        self._is_shared()
        self._pack_moves(out["src"], out["dst"], None)
        rc = self.lib.br_kv_compact(self.ctx, self._at)
        if rc:
            self._done(rc, "br_kv_compact")

    def copy_device(self, layer: KvLayer, src, dst, src_worker=None) -> None:
        """What blocks src hold to blocks dst (br_kv_copy): [n_workers, n] block ids of each worker, -1: none (but passed over one by one); src_worker: whose block src
        is, if another worker's."""
        if layer.sizes != self._layer:
            raise BrError("the layer is one of another cache's sizes")
        self._pack_moves(src, dst, src_worker)
        rc = self.lib.br_kv_copy(self.ctx, layer.at, self._at)
        if rc:
            self._done(rc, "br_kv_copy")

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
        self._pack_attention(layer, q, out, lse, (), start, count, max_count, scale, self._scale, window, lens, table)
        rc = self.lib.br_kv_attend(self.ctx, layer.at, self._at)
        if rc:
            self._done(rc, "br_kv_attend")

    def _pack_attention(self, layer, q, out, lse, lse_maps, start, count, max_count, scale, own_scale, window, lens, table) -> None:
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
        check, i32, rows = self._check, self._i32, self._rows
        at = (q.data_ptr(), out.data_ptr(), 0 if lse is None else check(lse, "lse", (n, heads, *lse_maps), self._f32), *self._check_lists(start, count),
              0 if lens is None else check(lens, "lens", rows, i32), 0 if table is None else check(table, "table", self._tables, i32), q_token, q_head, out_token, out_head, n)
        try:
            _PACK_ATTENTION.pack_into(self._args, 0, *at, max_count, window, dtype, own_scale if scale is None else scale, 0)
        except (struct.error, OverflowError):
            raise BrError("max_count and window must be whole numbers of 32 bits, scale a number of 32 bits") from None

    def _check_lists(self, start, count):
        """Addresses of a step's start and count, in any shape of as many numbers; 0 without them."""
        if (start is None) != (count is None):
            raise BrError("start and count come together")
        if start is None:
            return 0, 0
        check, i32, rows = self._check, self._i32, self._rows
        return (check(start.view(rows) if start.shape != rows and start.numel() == rows.numel() else start, "start", rows, i32),
                check(count.view(rows) if count.shape != rows and count.numel() == rows.numel() else count, "count", rows, i32))

    def plan_device(self, lead, members: int, start=None, count=None) -> None:
        """Which rows attend_shared_device reads together (br_kv_plan), for all layers of a step: behind step_device.

        lead [n_workers, rows] int32: the row that row r shares its first blocks with (its family's first, which may have left since, itself, or -1); at most `members` rows together:
        with 16 query rows of a key head short calls are fastest, with more those that read much.  Where rows hold little together (8 or 32 of them some 500 tokens)
        attend_device alone is faster than both calls; from some 1000 tokens, or for a hundred rows, reading together is.
        start, count: step_device's; rows whose count is not 1 are left out (attend_device serves them, with a count of 0 for the others); none: token r belongs to row r."""
        self._is_shared()
        at = (self._check(lead, "lead", self._rows, self._i32), *self._check_lists(start, count))
        try:
            _PACK_FAMILIES.pack_into(self._args, 0, *at, members, 0)
        except struct.error:
            raise BrError("members must be a whole number of 32 bits") from None
        rc = self.lib.br_kv_plan(self.ctx, self._at)
        if rc:
            self._done(rc, "br_kv_plan")

    def attend_shared_device(self, layer: KvLayer, q, out, lse=None, scale: Optional[float] = None, window: int = 0) -> None:
        """attend_device of the planned rows' tokens (br_kv_attend_shared): what rows hold together is read once for all of them.

        A plan holds until the next step_device or fork_device: behind those, without another plan_device, nothing is written."""
        self._is_shared()
        self._pack_attention(layer, q, out, lse, (), None, None, 1, scale, self._scale, window, None, None)
        rc = self.lib.br_kv_attend_shared(self.ctx, layer.at, self._at)
        if rc:
            self._done(rc, "br_kv_attend_shared")

    def attend_diff_device(self, layer: KvLayer, q, out, lam, lse=None, start=None, count=None, max_count: int = 1, scale: Optional[float] = None, window: int = 0,
                           lens=None, table=None) -> None:
        """Differential attention (br_kv_attend_diff): the first halves of the channels' map less lam times the second halves'.

        lam: float32 [n_q_heads], or [tokens, n_q_heads] with contiguous heads.  lse [tokens, n_q_heads, 2].  scale: 1 / sqrt(head_dim / 2) if not given.
        The rest as attend_device's."""
        n, heads = q.shape[0], self.cfg.n_q_heads
        self._pack_attention(layer, q, out, lse, (2,), start, count, max_count, scale, self._half_scale, window, lens, table)
        if lam.dtype is not self._f32 or lam.get_device() != self._index or lam.shape not in ((heads,), (n, heads)) or (lam.stride(-1) != 1 and heads > 1):
            raise BrError(f"lam must be a torch.float32 tensor of shape {(heads,)} or {(n, heads)} on {self.device}, its heads contiguous")
        _PACK_DIFF.pack_into(self._args, 160, lam.data_ptr(), lam.stride(0) if lam.dim() == 2 else 0)
        rc = self.lib.br_kv_attend_diff(self.ctx, layer.at, self._at, self._at + 160)
        if rc:
            self._done(rc, "br_kv_attend_diff")

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
