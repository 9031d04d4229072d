"""ctypes binding of the 8-bit KV cache and the rotary positions (include/sssd_kv8.h): same names as the C ABI, argument
marshalling only.  Tensors may have any strides as long as a head's channels lie in a row; nothing is copied or cast here."""
from __future__ import annotations

import ctypes as C
import struct
from typing import Optional

import torch

from .binding import SSSD_NO_WAIT, _check, _ptr, lib

FORMATS = {"e4m3": 0, "int8": 1}
SCALINGS = {"none": 0, "linear": 1, "bands": 2}
TYPES = {torch.float32: 0, torch.bfloat16: 1}


class Kv8Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("format", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "max_batch", "max_seq", "n_pages")]


class Kv8(C.Structure):
    _fields_ = [("cfg", Kv8Config), ("cache", C.c_void_p), ("cache_bytes", C.c_size_t), ("workspace", C.c_void_p),
                ("ws_bytes", C.c_size_t), ("block_table", C.c_void_p), ("status", C.c_void_p), ("flags", C.c_uint32)]


class RopeConfig(C.Structure):
    _fields_ = [("rotary_dims", C.c_int32), ("base", C.c_float), ("scaling", C.c_int32), ("factor", C.c_float), ("low", C.c_float),
                ("high", C.c_float), ("original", C.c_int32)]


class RopeArgs(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("rotary_dims", C.c_int32), ("pairs", C.c_int32), ("magnitude", C.c_float)]


class Kv8PagesArgs(C.Structure):
    _fields_ = [("table", C.c_void_p), ("refs", C.c_void_p), ("workspace", C.c_void_p), ("ws_bytes", C.c_size_t)]


ROWS = struct.Struct("@Piqqq").pack      # sssd_rows as bytes: half the time of a ctypes structure
_bound = None


def _lib() -> C.CDLL:
    global _bound
    if _bound is None:
        l = lib()
        vp, i32, p = C.c_void_p, C.c_int32, C.POINTER
        rows = vp                                # bytes, or NULL
        l.sssd_kv8_sizes.argtypes = [p(Kv8Config), p(C.c_size_t), p(C.c_size_t), p(i32), p(i32)]
        l.sssd_rope_frequencies.argtypes = [p(RopeConfig), p(C.c_double)]
        l.sssd_op_rope.argtypes = [rows, rows, i32, i32, i32, i32, vp, p(RopeArgs), vp]
        l.sssd_kv8_append.argtypes = [p(Kv8), i32, i32, i32, i32, rows, rows, vp, vp, p(RopeArgs), vp, rows, rows, vp]
        l.sssd_kv8_read.argtypes = [p(Kv8), i32, i32, i32, i32, vp, vp, rows, rows, vp]
        l.sssd_kv8_attention.argtypes = [p(Kv8), i32, i32, i32, rows, rows, vp, vp, vp, i32, i32, vp]
        l.sssd_kv8_commit_tree.argtypes = [p(Kv8), i32, i32, vp, vp, vp, vp]
        l.sssd_kv8_shared_sizes.argtypes = [p(Kv8Config), i32, i32, p(C.c_size_t)]
        l.sssd_kv8_attention_shared.argtypes = [p(Kv8), i32, i32, i32, rows, rows, vp, vp, vp, i32, vp, vp, vp, C.c_size_t, vp]
        l.sssd_kv8_pages_sizes.argtypes = [p(Kv8Config), p(C.c_size_t)]
        l.sssd_kv8_fork.argtypes = [p(Kv8), p(Kv8PagesArgs), vp, vp, vp]
        l.sssd_kv8_reserve.argtypes = [p(Kv8), p(Kv8PagesArgs), i32, i32, i32, vp, vp, vp]
        l.sssd_kv8_compact.argtypes = [p(Kv8), p(Kv8PagesArgs), p(Kv8), p(Kv8PagesArgs), vp, vp, vp]
        l.sssd_kv8_sync.argtypes = [p(Kv8), vp]
        _bound = l
    return _bound


def _rows(t: torch.Tensor, device: int) -> bytes:
    """[B][n][heads][channels], or [n][heads][channels], as the C ABI takes them; device: the number of the GPU, -1 for none."""
    stride = t.stride()
    kind = TYPES.get(t.dtype)
    assert kind is not None and len(stride) in (3, 4), "rows are [B][n][heads][head_dim], float32 or bfloat16"
    assert t.get_device() == device, f"rows on {t.device}, the cache (or the frequencies) on GPU {device}"
    assert stride[-1] == 1 or t.shape[-1] == 1, "a head's channels must lie in a row"
    if len(stride) == 3:
        return ROWS(t.data_ptr(), kind, 0, stride[0], stride[1])
    return ROWS(t.data_ptr(), kind, stride[0], stride[1], stride[2])


def _ints(t: Optional[torch.Tensor], shape, device: int) -> Optional[int]:
    if t is None:
        return None
    assert t.dtype is torch.int32 and t.shape == shape and t.get_device() == device and t.is_contiguous(), f"int32 {shape} on GPU {device}"
    return t.data_ptr()


def _enqueue(call, device: int, *args) -> None:
    """The call on the current stream of `device`, whichever device is the current one."""
    if torch._C._cuda_getDevice() == device:
        code = call(*args, torch._C._cuda_getCurrentRawStream(device))
    else:
        with torch.cuda.device(device):
            code = call(*args, torch._C._cuda_getCurrentRawStream(device))
    if code:
        _check(code, call.__name__)


def sssd_kv8_sizes(cfg: Kv8Config):
    cache, ws, per_seq, pages = C.c_size_t(), C.c_size_t(), C.c_int32(), C.c_int32()
    _check(_lib().sssd_kv8_sizes(C.byref(cfg), C.byref(cache), C.byref(ws), C.byref(per_seq), C.byref(pages)), "sssd_kv8_sizes")
    return cache.value, ws.value, per_seq.value, pages.value


def sssd_rope_frequencies(rotary_dims: int, base: float, scaling: str = "none", factor: float = 1.0, low: float = 1.0, high: float = 4.0,
                          original: int = 8192) -> torch.Tensor:
    """Turns per position of every pair, float64 on the host."""
    turns = torch.empty(max(rotary_dims // 2, 1), dtype=torch.float64)
    cfg = RopeConfig(rotary_dims, base, SCALINGS[scaling], factor, low, high, original)
    _check(_lib().sssd_rope_frequencies(C.byref(cfg), C.cast(turns.data_ptr(), C.POINTER(C.c_double))), "sssd_rope_frequencies")
    return turns


class Rope:
    """A rotation: its frequencies on the device, which channels form pairs, and what the rotated ones are multiplied by."""

    def __init__(self, rotary_dims: int, base: float, interleaved: bool = False, magnitude: float = 1.0, device: str = "cuda:0", **scaling):
        self.turns = sssd_rope_frequencies(rotary_dims, base, **scaling).to(device)
        self.args = RopeArgs(self.turns.data_ptr(), rotary_dims, int(interleaved), magnitude)
        self.ref, self.device = C.byref(self.args), self.turns.get_device()


def sssd_op_rope(x: torch.Tensor, positions: torch.Tensor, rope: Rope, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows][heads][head_dim] with positions [rows], or [B][n][heads][head_dim] with [B][n]; out may be x."""
    if out is None:
        out = torch.empty_like(x, memory_format=torch.contiguous_format)
    assert out.shape == x.shape and out.dtype == x.dtype
    shape = x.shape
    B, n = shape[:2] if len(shape) == 4 else (1, shape[0])
    _enqueue(_lib().sssd_op_rope, rope.device, _rows(x, rope.device), _rows(out, rope.device), B, n, shape[-2], shape[-1],
             _ints(positions, shape[:-2], rope.device), rope.ref)
    return out


class Kv8Cache:
    """Owns the device buffers (as torch tensors) of a cache in 8 bits."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_batch: int, max_seq: int, fmt: str = "e4m3",
                 n_pages: int = 0, device: str = "cuda:0", no_wait: bool = False):
        self.n_q_heads, self.n_kv_heads, self.head_dim = n_q_heads, n_kv_heads, head_dim
        self.cfg = Kv8Config(FORMATS[fmt], n_layers, n_q_heads, n_kv_heads, head_dim, max_batch, max_seq, n_pages)
        cache_bytes, ws_bytes, self.blocks_per_seq, self.n_pages = sssd_kv8_sizes(self.cfg)
        self.cache = torch.zeros(cache_bytes, dtype=torch.uint8, device=device)
        self.workspace = torch.zeros(ws_bytes, dtype=torch.uint8, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.device = self.cache.get_device()
        self._block_table = None
        self.args = Kv8(self.cfg, _ptr(self.cache), cache_bytes, _ptr(self.workspace), ws_bytes, None, _ptr(self.status),
                        SSSD_NO_WAIT if no_wait else 0)
        self._ref = C.byref(self.args)

    def _heads(self, t: torch.Tensor, like: torch.Tensor, shape) -> bytes:
        assert t.shape == shape and t.dtype is like.dtype, f"{tuple(t.shape)}, {t.dtype}: {shape}, {like.dtype} is wanted"
        return _rows(t, self.device)

    def sssd_kv8_set_block_table(self, block_table: Optional[torch.Tensor]) -> None:
        """The table is read on the device when each later call executes; None: contiguous runs of pages."""
        self.args.block_table = _ints(block_table, (self.cfg.max_batch, self.blocks_per_seq), self.device)
        self._block_table = block_table          # keep the tensor alive while the library reads it

    def sssd_kv8_append(self, layer: int, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, counts: Optional[torch.Tensor] = None,
                        first: int = 0, rope: Optional[Rope] = None, parents: Optional[torch.Tensor] = None,
                        q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> None:
        B, n = k.shape[:2]
        shape = (B, n, self.n_kv_heads, self.head_dim)
        turn = qq = to = None
        if rope is not None:
            assert rope.device == self.device
            turn = rope.ref
        assert (q is None) == (q_out is None), "q and q_out come together"
        if q is not None:
            of_q = (B, n, self.n_q_heads, self.head_dim)
            qq, to = self._heads(q, q, of_q), self._heads(q_out, q, of_q)
        _enqueue(_lib().sssd_kv8_append, self.device, self._ref, layer, first, B, n, self._heads(k, k, shape), self._heads(v, k, shape),
                 _ints(lens, (B,), self.device), _ints(counts, (B,), self.device), turn, _ints(parents, (B, n), self.device), qq, to)

    def sssd_kv8_read(self, layer: int, start: Optional[torch.Tensor], counts: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                      first: int = 0) -> None:
        B, n = k.shape[:2]
        shape = (B, n, self.n_kv_heads, self.head_dim)
        _enqueue(_lib().sssd_kv8_read, self.device, self._ref, layer, first, B, n, _ints(start, (B,), self.device), _ints(counts, (B,), self.device),
                 self._heads(k, k, shape), self._heads(v, k, shape))

    def sssd_kv8_attention(self, layer: int, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, counts: Optional[torch.Tensor] = None,
                           parents: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0) -> None:
        B, n = q.shape[:2]
        shape = (B, n, self.n_q_heads, self.head_dim)
        _enqueue(_lib().sssd_kv8_attention, self.device, self._ref, layer, B, n, self._heads(q, q, shape), self._heads(out, q, shape),
                 _ints(lens, (B,), self.device), _ints(counts, (B,), self.device), _ints(parents, (B, n), self.device), window, sinks)

    def sssd_kv8_shared_workspace(self, B: int, n: int) -> torch.Tensor:
        """What sssd_kv8_attention_shared takes for up to B sequences of up to n rows."""
        size = C.c_size_t()
        _check(_lib().sssd_kv8_shared_sizes(C.byref(self.cfg), B, n, C.byref(size)), "sssd_kv8_shared_sizes")
        return torch.empty(size.value, dtype=torch.uint8, device=self.cache.device)

    def sssd_kv8_attention_shared(self, layer: int, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, starts: torch.Tensor, shared: torch.Tensor,
                                  workspace: torch.Tensor, counts: Optional[torch.Tensor] = None, parents: Optional[torch.Tensor] = None) -> None:
        """Groups are sequences starts[g] .. starts[g+1]-1, whose first shared[g] positions are the same."""
        B, n = q.shape[:2]
        shape = (B, n, self.n_q_heads, self.head_dim)
        groups = shared.shape[0]
        assert workspace.get_device() == self.device and workspace.is_contiguous()
        _enqueue(_lib().sssd_kv8_attention_shared, self.device, self._ref, layer, B, n, self._heads(q, q, shape), self._heads(out, q, shape),
                 _ints(lens, (B,), self.device), _ints(counts, (B,), self.device), _ints(parents, (B, n), self.device), groups,
                 _ints(starts, (groups + 1,), self.device), _ints(shared, (groups,), self.device), workspace.data_ptr(),
                 workspace.numel() * workspace.element_size())

    def sssd_kv8_commit_tree(self, n: int, lens: torch.Tensor, accepted_len: torch.Tensor, accepted_path: Optional[torch.Tensor] = None) -> None:
        """n: rows of the step (accepted_path [B][n]); lens advances."""
        B = lens.numel()
        _enqueue(_lib().sssd_kv8_commit_tree, self.device, self._ref, B, n, _ints(lens, (B,), self.device), _ints(accepted_len, (B,), self.device),
                 _ints(accepted_path, (B, n), self.device))

    def sssd_kv8_sync(self) -> int:
        with torch.cuda.device(self.device):
            return _lib().sssd_kv8_sync(self._ref, torch.cuda.current_stream().cuda_stream)


class Kv8Pages:
    """Who has which pages of a cache's pool: owns the block table (set as the cache's), the pages' counts and the calls' workspace."""

    def __init__(self, cache: Kv8Cache):
        size = C.c_size_t()
        _check(_lib().sssd_kv8_pages_sizes(C.byref(cache.cfg), C.byref(size)), "sssd_kv8_pages_sizes")
        self.cache, where = cache, cache.cache.device
        self.table = torch.full((cache.cfg.max_batch, cache.blocks_per_seq), -1, dtype=torch.int32, device=where)
        self.refs = torch.zeros(cache.n_pages, dtype=torch.int32, device=where)
        self.workspace = torch.zeros(size.value, dtype=torch.uint8, device=where)
        self.args = Kv8PagesArgs(self.table.data_ptr(), self.refs.data_ptr(), self.workspace.data_ptr(), size.value)
        self._ref = C.byref(self.args)
        cache.sssd_kv8_set_block_table(self.table)

    def sssd_kv8_fork(self, origins: torch.Tensor, lens: torch.Tensor) -> None:
        """Slot b goes on from what slot origins[b] was (-1: empty); lens changes with it."""
        c, slots = self.cache, (self.cache.cfg.max_batch,)
        _enqueue(_lib().sssd_kv8_fork, c.device, c._ref, self._ref, _ints(origins, slots, c.device), _ints(lens, slots, c.device))

    def sssd_kv8_reserve(self, n: int, lens: torch.Tensor, counts: Optional[torch.Tensor] = None, first: int = 0) -> None:
        """Pages of their own for the next n (or counts[b]) rows of the sequences from slot `first` on."""
        c, B = self.cache, lens.numel()
        _enqueue(_lib().sssd_kv8_reserve, c.device, c._ref, self._ref, first, B, n, _ints(lens, (B,), c.device), _ints(counts, (B,), c.device))

    def sssd_kv8_compact(self, to: Optional["Kv8Pages"] = None, moved: Optional[torch.Tensor] = None, in_use: Optional[torch.Tensor] = None) -> None:
        """Pages in use to the front of the pool, or into another cache's."""
        c = self.cache
        assert to is None or to.cache.device == c.device
        _enqueue(_lib().sssd_kv8_compact, c.device, c._ref, self._ref, None if to is None else to.cache._ref, None if to is None else to._ref,
                 _ints(moved, (c.n_pages,), c.device), _ints(in_use, (1,), c.device))
