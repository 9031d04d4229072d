"""ctypes binding of the 8-bit KV cache and the rotary positions (include/sssd_kv8.h): same names as the C ABI, argument
marshalling only.  Tensors may have any strides as long as a head's channels lie in a row; nothing is copied or cast here."""
from __future__ import annotations

import ctypes as C
from typing import Optional

import torch

from .binding import _check, _ptr, lib

FORMATS = {"e4m3": 0, "int8": 1}
SCALINGS = {"none": 0, "linear": 1, "bands": 2}
TYPES = {torch.float32: 0, torch.bfloat16: 1}


class Kv8Config(C.Structure):
    _fields_ = [(n, C.c_int32) for n in ("format", "n_layers", "n_q_heads", "n_kv_heads", "head_dim", "max_batch", "max_seq", "n_pages")]


class Kv8(C.Structure):
    _fields_ = [("cfg", Kv8Config), ("cache", C.c_void_p), ("cache_bytes", C.c_size_t), ("workspace", C.c_void_p),
                ("ws_bytes", C.c_size_t), ("block_table", C.c_void_p), ("status", C.c_void_p)]


class Rows(C.Structure):
    _fields_ = [("data", C.c_void_p), ("type", C.c_int32), ("batch_stride", C.c_int64), ("row_stride", C.c_int64),
                ("head_stride", C.c_int64)]


class RopeConfig(C.Structure):
    _fields_ = [("rotary_dims", C.c_int32), ("base", C.c_float), ("scaling", C.c_int32), ("factor", C.c_float), ("low", C.c_float),
                ("high", C.c_float), ("original", C.c_int32)]


class RopeArgs(C.Structure):
    _fields_ = [("turns", C.c_void_p), ("rotary_dims", C.c_int32), ("pairs", C.c_int32), ("magnitude", C.c_float)]


_bound = None


def _lib() -> C.CDLL:
    global _bound
    if _bound is None:
        l = lib()
        vp, i32, p = C.c_void_p, C.c_int32, C.POINTER
        l.sssd_kv8_sizes.argtypes = [p(Kv8Config), p(C.c_size_t), p(C.c_size_t), p(i32), p(i32)]
        l.sssd_rope_frequencies.argtypes = [p(RopeConfig), p(C.c_double)]
        l.sssd_op_rope.argtypes = [p(Rows), p(Rows), i32, i32, i32, i32, vp, p(RopeArgs), vp]
        l.sssd_kv8_append.argtypes = [p(Kv8), i32, i32, i32, i32, p(Rows), p(Rows), vp, vp, p(RopeArgs), vp, p(Rows), p(Rows), vp]
        l.sssd_kv8_read.argtypes = [p(Kv8), i32, i32, i32, i32, vp, vp, p(Rows), p(Rows), vp]
        l.sssd_kv8_attention.argtypes = [p(Kv8), i32, i32, i32, p(Rows), p(Rows), vp, vp, vp, i32, i32, vp]
        l.sssd_kv8_commit_tree.argtypes = [p(Kv8), i32, i32, vp, vp, vp, vp]
        l.sssd_kv8_sync.argtypes = [p(Kv8), vp]
        _bound = l
    return _bound


def _rows(t: torch.Tensor, device: torch.device) -> Rows:
    """[B][n][heads][channels] as the C ABI takes them."""
    assert t.dim() == 4 and t.dtype in TYPES, "rows are [B][n][heads][head_dim], float32 or bfloat16"
    assert t.device == device, f"rows on {t.device}, the cache (or the frequencies) on {device}"
    assert t.stride(3) == 1 or t.shape[3] == 1, "a head's channels must lie in a row"
    return Rows(t.data_ptr(), TYPES[t.dtype], t.stride(0), t.stride(1), t.stride(2))


def _ints(t: Optional[torch.Tensor], shape, device: torch.device) -> Optional[int]:
    if t is None:
        return None
    assert t.dtype == torch.int32 and tuple(t.shape) == tuple(shape) and t.device == device, f"int32 {tuple(shape)} on {device}"
    return _ptr(t)


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


def sssd_op_rope(x: torch.Tensor, positions: torch.Tensor, rope: Rope, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x [rows][heads][head_dim] with positions [rows], or [B][n][heads][head_dim] with [B][n]; out may be x."""
    device = rope.turns.device
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    assert out.shape == x.shape and out.dtype == x.dtype
    four = (lambda t: t.unsqueeze(0)) if x.dim() == 3 else (lambda t: t)
    a, b = four(x), four(out)
    B, n, heads, d = a.shape
    with torch.cuda.device(device):
        _check(_lib().sssd_op_rope(C.byref(_rows(a, device)), C.byref(_rows(b, device)), B, n, heads, d, _ints(positions, x.shape[:-2], device),
                                   C.byref(rope.args), torch.cuda.current_stream().cuda_stream), "sssd_op_rope")
    return out


class Kv8Cache:
    """Owns the device buffers (as torch tensors) of a cache in 8 bits."""

    def __init__(self, n_layers: int, n_q_heads: int, n_kv_heads: int, head_dim: int, max_batch: int, max_seq: int, fmt: str = "e4m3",
                 n_pages: int = 0, device: str = "cuda:0"):
        self.cfg = Kv8Config(FORMATS[fmt], n_layers, n_q_heads, n_kv_heads, head_dim, max_batch, max_seq, n_pages)
        cache_bytes, ws_bytes, self.blocks_per_seq, self.n_pages = sssd_kv8_sizes(self.cfg)
        self.cache = torch.zeros(cache_bytes, dtype=torch.uint8, device=device)
        self.workspace = torch.zeros(ws_bytes, dtype=torch.uint8, device=device)
        self.status = torch.zeros(1, dtype=torch.int32, device=device)
        self.device = self.cache.device
        self._block_table = None
        self.args = Kv8(self.cfg, _ptr(self.cache), cache_bytes, _ptr(self.workspace), ws_bytes, None, _ptr(self.status))

    def _call(self, name: str, *args) -> None:
        with torch.cuda.device(self.device):
            _check(getattr(_lib(), name)(C.byref(self.args), *args, torch.cuda.current_stream().cuda_stream), name)

    def _heads(self, t: torch.Tensor, heads: int) -> Rows:
        assert tuple(t.shape[2:]) == (heads, self.cfg.head_dim), f"{tuple(t.shape)}: {heads} heads of {self.cfg.head_dim} channels are wanted"
        return _rows(t, self.device)

    def sssd_kv8_set_block_table(self, block_table: Optional[torch.Tensor]) -> None:
        """The table is read on the device when each later call executes; None: contiguous runs of pages."""
        self.args.block_table = _ints(block_table, (self.cfg.max_batch, self.blocks_per_seq), self.device)
        self._block_table = block_table          # keep the tensor alive while the library reads it

    def sssd_kv8_append(self, layer: int, k: torch.Tensor, v: torch.Tensor, lens: torch.Tensor, counts: Optional[torch.Tensor] = None,
                        first: int = 0, rope: Optional[Rope] = None, parents: Optional[torch.Tensor] = None,
                        q: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None) -> None:
        B, n = k.shape[:2]
        assert v.shape == k.shape and v.dtype == k.dtype
        assert rope is None or rope.turns.device == self.device
        kk, vv = self._heads(k, self.cfg.n_kv_heads), self._heads(v, self.cfg.n_kv_heads)
        qs = [None, None]
        if q is not None:
            assert q_out is not None and q.shape == q_out.shape and q.dtype == q_out.dtype and q.shape[:2] == k.shape[:2]
            qs = [C.byref(self._heads(t, self.cfg.n_q_heads)) for t in (q, q_out)]
        self._call("sssd_kv8_append", layer, first, B, n, C.byref(kk), C.byref(vv), _ints(lens, (B,), self.device),
                   _ints(counts, (B,), self.device), C.byref(rope.args) if rope is not None else None, _ints(parents, (B, n), self.device), *qs)

    def sssd_kv8_read(self, layer: int, start: Optional[torch.Tensor], counts: Optional[torch.Tensor], k: torch.Tensor, v: torch.Tensor,
                      first: int = 0) -> None:
        B, n = k.shape[:2]
        assert v.shape == k.shape and v.dtype == k.dtype
        kk, vv = self._heads(k, self.cfg.n_kv_heads), self._heads(v, self.cfg.n_kv_heads)
        self._call("sssd_kv8_read", layer, first, B, n, _ints(start, (B,), self.device), _ints(counts, (B,), self.device), C.byref(kk),
                   C.byref(vv))

    def sssd_kv8_attention(self, layer: int, q: torch.Tensor, lens: torch.Tensor, out: torch.Tensor, counts: Optional[torch.Tensor] = None,
                           parents: Optional[torch.Tensor] = None, window: int = 0, sinks: int = 0) -> None:
        B, n = q.shape[:2]
        assert out.shape == q.shape and out.dtype == q.dtype
        qq, oo = self._heads(q, self.cfg.n_q_heads), self._heads(out, self.cfg.n_q_heads)
        self._call("sssd_kv8_attention", layer, B, n, C.byref(qq), C.byref(oo), _ints(lens, (B,), self.device),
                   _ints(counts, (B,), self.device), _ints(parents, (B, n), self.device), window, sinks)

    def sssd_kv8_commit_tree(self, n: int, lens: torch.Tensor, accepted_len: torch.Tensor, accepted_path: Optional[torch.Tensor] = None) -> None:
        """n: rows of the step (accepted_path [B][n]); lens advances."""
        B = lens.numel()
        self._call("sssd_kv8_commit_tree", B, n, _ints(lens, (B,), self.device), _ints(accepted_len, (B,), self.device),
                   _ints(accepted_path, (B, n), self.device))

    def sssd_kv8_sync(self) -> int:
        with torch.cuda.device(self.device):
            return _lib().sssd_kv8_sync(C.byref(self.args), torch.cuda.current_stream().cuda_stream)
