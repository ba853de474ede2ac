"""ctypes binding of libminicache.so: argument marshalling only.

Every function here has the name of the C entry point it wraps (``include/minicache.h``)
and hands raw device pointers of torch tensors to it.  Nothing is computed in Python, and
there is no fallback: without the compiled library every call raises."""
from __future__ import annotations

import ctypes as C
import dataclasses
import os
from typing import Optional

import torch

MC_F16, MC_BF16 = 0, 1
MC_RETAIN_DISTINCT, MC_RETAIN_LITERAL, MC_RETAIN_TOPK = 0, 1, 2
MC_LAYER_LM1, MC_LAYER_L, MC_LAYER_BOTH = 0, 1, 2
MC_OP_MERGE, MC_OP_DECODE_ATTN = 0, 1
MC_OP_LAYER_ATTN, MC_OP_LAYER_OBSERVE, MC_OP_LAYER_EVICT = 2, 3, 4
MC_OP_LAYER_Q4_ATTN, MC_OP_LAYER_Q4_SELECT = 5, 6
MC_LAYER_APPEND, MC_LAYER_ACCUMULATE = 1, 2
MC_STATUS_WORDS = 4
MC_STATUS_FLAGS, MC_STATUS_RETAINED_TOTAL, MC_STATUS_NEAR_THRESHOLD = 0, 1, 2
MC_FLAG_RETAIN_OVERFLOW, MC_FLAG_WAIT_TIMEOUT, MC_FLAG_BAD_METADATA, MC_FLAG_BOUNDS = 1, 2, 4, 8
MC_FLAG_HINT_TOO_HIGH = 16
MC_BUILD_BOUNDS = 1

# MINICACHE_LIBRARY selects another build of the same library (the range-checked one, for instance)
_LIB_PATH = os.environ.get("MINICACHE_LIBRARY") or os.path.join(os.path.dirname(os.path.abspath(__file__)), "libminicache.so")


class McError(RuntimeError):
    def __init__(self, code: int, name: str, detail: str = ""):
        super().__init__(f"{name} ({code}){': ' + detail if detail else ''}")
        self.code = code
        self.name = name


class _Config(C.Structure):
    _fields_ = [("n_kv_heads", C.c_int32), ("n_q_heads", C.c_int32), ("head_dim", C.c_int32),
                ("page_size", C.c_int32), ("dtype", C.c_int32), ("retain_mode", C.c_int32),
                ("t", C.c_double), ("gamma", C.c_double), ("merge_fn", C.c_int32), ("cache_bits", C.c_int32),
                ("t_mode", C.c_int32), ("retain_union", C.c_int32), ("append_slack", C.c_int32)]


class _Batch(C.Structure):
    _fields_ = [("block_table", C.c_void_p), ("seq_lens", C.c_void_p), ("batch", C.c_int32),
                ("max_pages_per_seq", C.c_int32), ("max_seq_len", C.c_int32), ("reserved", C.c_int32),
                ("n_pages", C.c_int64)]


class _LayerKV(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p)]


class _LayerQ4(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_meta", C.c_void_p), ("v_codes", C.c_void_p), ("v_meta", C.c_void_p)]


class _Projection(C.Structure):
    _fields_ = [("x", C.c_void_p), ("w_k", C.c_void_p), ("w_v", C.c_void_p), ("d_model", C.c_int32), ("x_seq_stride", C.c_int32)]


class _PairCache(C.Structure):
    _fields_ = [("e_k", C.c_void_p), ("e_v", C.c_void_p), ("dist", C.c_void_p),
                ("ret_count", C.c_void_p), ("ret_offset", C.c_void_p), ("ret_index", C.c_void_p),
                ("ret_rows", C.c_void_p), ("ret_capacity", C.c_int64), ("ret_prefix", C.c_void_p),
                ("ret_prefix_stride", C.c_int64), ("seg_minmax", C.c_void_p),
                ("status", C.c_void_p), ("res_k", C.c_void_p), ("res_v", C.c_void_p)]


class _LayerCache(C.Structure):
    _fields_ = [("k_pool", C.c_void_p), ("v_pool", C.c_void_p), ("positions", C.c_void_p), ("weights", C.c_void_p),
                ("status", C.c_void_p)]


class _ScoreOpts(C.Structure):
    _fields_ = [("alibi_slopes", C.c_void_p), ("doc_start", C.c_void_p), ("prefix_len", C.c_void_p), ("q_pos", C.c_void_p),
                ("sm_scale", C.c_float), ("softcap", C.c_float), ("window", C.c_int32), ("reserved", C.c_int32)]


class _EvictOpts(C.Structure):
    _fields_ = [("q_pos", C.c_void_p), ("budget", C.c_int32), ("n_sink", C.c_int32), ("n_recent", C.c_int32), ("reserved", C.c_int32)]


class _LayerQ4Cache(C.Structure):
    _fields_ = [("k_codes", C.c_void_p), ("k_meta", C.c_void_p), ("v_codes", C.c_void_p), ("v_meta", C.c_void_p),
                ("res_k", C.c_void_p), ("res_v", C.c_void_p), ("status", C.c_void_p)]


class _PageSelection(C.Structure):
    _fields_ = [("budget", C.c_int32), ("n_sink", C.c_int32), ("n_recent", C.c_int32), ("reserved", C.c_int32)]


class _PairSizes(C.Structure):
    _fields_ = [("tile_bytes", C.c_size_t), ("e_bytes", C.c_size_t), ("dist_bytes", C.c_size_t),
                ("ret_count_bytes", C.c_size_t), ("ret_offset_bytes", C.c_size_t), ("ret_index_bytes", C.c_size_t),
                ("ret_rows_bytes", C.c_size_t), ("ret_prefix_bytes", C.c_size_t), ("seg_minmax_bytes", C.c_size_t),
                ("status_bytes", C.c_size_t), ("ret_prefix_stride", C.c_int64), ("total_bytes", C.c_size_t),
                ("res_bytes", C.c_size_t)]


class _Stats(C.Structure):
    _fields_ = [("flags", C.c_int32), ("reserved", C.c_int32), ("retained_total", C.c_int64),
                ("near_threshold", C.c_int64), ("token_heads", C.c_int64), ("full_bytes", C.c_int64),
                ("compressed_bytes", C.c_int64), ("stored_bytes", C.c_int64)]


EXPORTS = ("mc_decode_drain_host", "mc_decode_stage_host", "mc_decode_attn_append", "mc_prefill_merge_pair", "mc_admit_sequences", "mc_build_flags", "mc_merge_pairs", "mc_pair_bytes", "mc_get_stats", "mc_version", "mc_status_str", "mc_last_cuda_error", "mc_workspace_bytes", "mc_merge_pair",
           "mc_append_pair", "mc_restore", "mc_decode_attn", "mc_read_status", "mc_merge_pair_host",
           "mc_decode_attn_host", "mc_decode_io_bytes", "mc_decode_attn_static", "mc_merge_pair_q4", "mc_selftest_wait_timeout",
           "mc_layer_workspace_bytes", "mc_layer_attn", "mc_layer_observe", "mc_layer_evict", "mc_layer_read_status",
           "mc_layer_q4_append", "mc_layer_q4_read", "mc_layer_q4_select", "mc_layer_q4_attn", "mc_layer_q4_read_status")


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream) -> Optional[int]:
    if stream is None:
        stream = torch.cuda.current_stream()
    return stream.cuda_stream or None


_TORCH_DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


@dataclasses.dataclass
class McConfig:
    n_kv_heads: int
    n_q_heads: int
    page_size: int
    dtype: str  # "f16" | "bf16"
    t: float = 0.6
    gamma: float = 0.05
    retain_mode: int = MC_RETAIN_DISTINCT
    head_dim: int = 128
    merge_fn: int = 0  # MC_MERGE_SLERP (Eq. 3) | MC_MERGE_FMAX = 1 | MC_MERGE_MEAN = 2
    cache_bits: int = 16  # storage of the shared directions: 16 (the 16-bit type) or 4 (4-bit shared cache, pages of 32)
    t_mode: int = 0  # MC_T_FIXED | MC_T_MAGNITUDE_RATIO = 1 (per-token t from the two magnitudes)
    retain_union: int = 0  # 1: one retention set for keys and values (the union of Eq. 4's two sets)
    append_slack: int = 0  # > 0: free retained entries per segment; appended tokens are held against Eq. 4's stored threshold

    def c(self) -> _Config:
        return _Config(self.n_kv_heads, self.n_q_heads, self.head_dim, self.page_size,
                       {"f16": MC_F16, "bf16": MC_BF16}[self.dtype], self.retain_mode, float(self.t), float(self.gamma),
                       int(self.merge_fn), int(self.cache_bits), int(self.t_mode), int(self.retain_union),
                       int(self.append_slack))

    @property
    def torch_dtype(self):
        return _TORCH_DTYPES[self.dtype]


@dataclasses.dataclass
class Batch:
    """Device block table / sequence lengths plus the host-known bounds."""
    block_table: torch.Tensor  # int32 [batch][max_pages_per_seq]
    seq_lens: torch.Tensor  # int32 [batch]
    max_seq_len: int
    n_pages: int

    def c(self) -> _Batch:
        assert self.block_table.dtype == torch.int32 and self.seq_lens.dtype == torch.int32
        assert self.block_table.is_contiguous() and self.seq_lens.is_contiguous()
        b = self.seq_lens.shape[0]
        mp = self.block_table.shape[1] if self.block_table.dim() == 2 else 0
        return _Batch(_ptr(self.block_table), _ptr(self.seq_lens), b, mp, int(self.max_seq_len), 0, int(self.n_pages))

    def layer_c(self, dev: Optional[int] = None) -> _Batch:
        """c() for the mc_layer_* calls: a row of the block table for every sequence, both tensors on device dev."""
        bt, sl = self.block_table, self.seq_lens
        n, pages = sl.numel(), bt.size(1) if bt.dim() == 2 else -1
        if not (pages >= 0 and bt.size(0) >= n and bt.dtype is torch.int32 and sl.dtype is torch.int32 and bt.is_contiguous()
                and sl.is_contiguous() and (dev is None or (bt.get_device() == dev and sl.get_device() == dev))):
            _refuse(dev, block_table=(bt, torch.int32, 0), seq_lens=(sl, torch.int32, 0))
            raise AssertionError("block_table [batch][max_pages_per_seq] and seq_lens [batch] are wanted")
        return _Batch(bt.data_ptr(), sl.data_ptr(), n, pages, int(self.max_seq_len), 0, int(self.n_pages))



class PairCache:
    """Caller-owned device buffers of one compressed layer pair (allocated with torch)."""

    def __init__(self, cfg: McConfig, batch: int, n_pages: int, ret_capacity: int, device="cuda",
                 max_merge_len: Optional[int] = None):
        H, ps = cfg.n_kv_heads, cfg.page_size
        self.cfg = cfg
        if max_merge_len is None:  # bound of the sequence length at merge time: what the pages can hold at most
            max_merge_len = n_pages * ps
        cap = max(int(ret_capacity), 1)
        sz = lib().mc_pair_bytes(cfg, batch, n_pages, int(max_merge_len), cap)  # every size comes from the library
        self.sizes = sz
        self.tile_bytes = sz.tile_bytes
        nseg = 2 * batch * H
        z = lambda nbytes: torch.zeros(nbytes, dtype=torch.uint8, device=device)
        self.e_k = z(sz.e_bytes).view(n_pages, H, self.tile_bytes)
        self.e_v = z(sz.e_bytes).view(n_pages, H, self.tile_bytes)
        self.dist = z(sz.dist_bytes).view(torch.float32).view(n_pages, H, 2, ps)
        self.ret_count = z(sz.ret_count_bytes).view(torch.int32)
        self.ret_offset = z(sz.ret_offset_bytes).view(torch.int32)
        self.ret_index = z(sz.ret_index_bytes).view(torch.int32)
        self.ret_rows = z(sz.ret_rows_bytes).view(2, cap, 272)
        self.ret_capacity = int(ret_capacity)
        self.ret_prefix_stride = int(sz.ret_prefix_stride)
        self.ret_prefix = z(sz.ret_prefix_bytes).view(torch.int32).view(nseg, self.ret_prefix_stride)
        self.seg_minmax = z(sz.seg_minmax_bytes).view(torch.float32).view(nseg, 2)
        self.status = z(sz.status_bytes).view(torch.int32)
        self.q4 = cfg.cache_bits == 4
        self.res_k = self.res_v = None
        if self.q4:  # one 16-bit tile of 32 tokens per (sequence, head): the last, incomplete page
            self.res_k = z(sz.res_bytes).view(batch, H, sz.res_bytes // max(batch * H, 1))
            self.res_v = z(sz.res_bytes).view(batch, H, sz.res_bytes // max(batch * H, 1))

    def c(self) -> _PairCache:
        return _PairCache(_ptr(self.e_k), _ptr(self.e_v), _ptr(self.dist), _ptr(self.ret_count),
                          _ptr(self.ret_offset), _ptr(self.ret_index), _ptr(self.ret_rows), self.ret_capacity,
                          _ptr(self.ret_prefix), self.ret_prefix_stride, _ptr(self.seg_minmax), _ptr(self.status),
                          _ptr(self.res_k), _ptr(self.res_v))

    # -- decoding the tile layout (pure re-indexing, no arithmetic) ------------------------------
    def _rows16(self, pool: torch.Tensor) -> torch.Tensor:
        """16-bit tiles [n][H][tile] -> direction rows [n][H][page_size][128] (chunk permutation undone)."""
        ps = self.cfg.page_size
        n, H = pool.shape[:2]
        rows = pool[:, :, :ps * 256].reshape(n, H, ps, 16, 16)  # [..][row][chunk position][16 bytes]
        r = torch.arange(ps, device=pool.device)[:, None]
        c = torch.arange(16, device=pool.device)[None, :]
        pos = (c & 8) | ((c & 7) ^ (r & 7))  # where chunk c of row r is stored
        idx = pos[None, None, :, :, None].expand(n, H, ps, 16, 16)
        plain = torch.gather(rows, 3, idx).reshape(n, H, ps, 256)
        return plain.view(self.cfg.torch_dtype)

    def directions(self, tensor: str) -> torch.Tensor:
        """Stored directions of "k" or "v" as [n_pages][H][page_size][128] in the storage type
        (the 16-byte chunk permutation of the tile format undone).  16-bit cache only."""
        assert not self.q4, "a 4-bit cache holds codes: see q4_codes / q4_groups / residual_directions"
        return self._rows16(self.e_k if tensor == "k" else self.e_v)

    def scales(self, tensor: str) -> torch.Tensor:
        """Scales of "k" or "v" as [n_pages][H][2][page_size] fp32 ([..][0]: layer l-1, [1]: layer l)."""
        pool = self.e_k if tensor == "k" else self.e_v
        ps = self.cfg.page_size
        n_pages, H = pool.shape[:2]
        off = 2560 if self.q4 else ps * 256
        return pool[:, :, off:].contiguous().view(torch.float32).reshape(n_pages, H, 2, ps)

    # -- 4-bit shared cache: the tile's orders undone (pure re-indexing) -------------------------
    def q4_codes(self, tensor: str) -> torch.Tensor:
        """Codes of "k" or "v" as [n_pages][H][32][128] uint8, channels in natural order."""
        assert self.q4
        pool = self.e_k if tensor == "k" else self.e_v
        n_pages, H = pool.shape[:2]
        dev = pool.device
        words = pool[:, :, :2048].contiguous().view(torch.int32).reshape(n_pages, H, 512).long() & 0xFFFFFFFF
        nib = torch.stack([(words >> (4 * j)) & 15 for j in range(8)], dim=-1).to(torch.uint8)  # [..][word][nibble]
        out = torch.zeros(n_pages, H, 32, 128, dtype=torch.uint8, device=dev)
        if tensor == "k":
            # row r, word w, nibble j: channel 8 w + 2 (j % 4) + j // 4
            nib = nib.reshape(n_pages, H, 32, 16, 8)
            w = torch.arange(16, device=dev)[:, None]
            j = torch.arange(8, device=dev)[None, :]
            ch = (8 * w + 2 * (j % 4) + j // 4).reshape(-1)
            out[:, :, :, ch] = nib.reshape(n_pages, H, 32, 128)
        else:
            # block i (tokens 2i, 2i+1), chunk position cp, word k, nibble j: token 2i + j // 4,
            # channel 32 k + 16 ((j % 4) // 2) + 8 (j % 2) + (cp ^ ((i % 4) * 2))
            nib = nib.reshape(n_pages, H, 16, 8, 4, 8)
            i = torch.arange(16, device=dev)[:, None, None, None]
            cp = torch.arange(8, device=dev)[None, :, None, None]
            k = torch.arange(4, device=dev)[None, None, :, None]
            j = torch.arange(8, device=dev)[None, None, None, :]
            tok = (2 * i + j // 4).expand(16, 8, 4, 8).reshape(-1)
            ch = (32 * k + 16 * ((j % 4) // 2) + 8 * (j % 2) + (cp ^ ((i % 4) * 2))).expand(16, 8, 4, 8).reshape(-1)
            out[:, :, tok, ch] = nib.reshape(n_pages, H, -1)
        return out

    def q4_groups(self, tensor: str):
        """(scale, zero) of "k" ([n_pages][H][128], per channel) or "v" ([n_pages][H][32][4], per token and
        channel group) in the storage type."""
        assert self.q4
        pool = self.e_k if tensor == "k" else self.e_v
        n_pages, H = pool.shape[:2]
        dev = pool.device
        m = pool[:, :, 2048:2560].contiguous().view(self.cfg.torch_dtype)  # 256 values
        if tensor == "k":
            m = m.reshape(n_pages, H, 2, 16, 8)  # [scale|zero][chunk position][8 channels]
            o = torch.arange(16, device=dev)
            pos = 4 * (o & 3) + (o >> 2)  # where the chunk of channels [8 o, 8 o + 8) is stored
            m = m[:, :, :, pos].reshape(n_pages, H, 2, 128)
            return m[:, :, 0].contiguous(), m[:, :, 1].contiguous()
        m = m.reshape(n_pages, H, 16, 2, 4, 2)  # [token pair][scale|zero][group][token of the pair]
        m = m.permute(0, 1, 3, 2, 5, 4).reshape(n_pages, H, 2, 32, 4)
        return m[:, :, 0].contiguous(), m[:, :, 1].contiguous()

    def residual_directions(self, tensor: str) -> torch.Tensor:
        """The residual tiles' rows [batch][H][32][128] in the storage type (tokens of the last, incomplete page)."""
        assert self.q4
        return self._rows16(self.res_k if tensor == "k" else self.res_v)

    def residual_scales(self, tensor: str) -> torch.Tensor:
        """The residual tiles' scales [batch][H][2][32] fp32."""
        assert self.q4
        pool = self.res_k if tensor == "k" else self.res_v
        return pool[:, :, 32 * 256:].contiguous().view(torch.float32).reshape(pool.shape[0], pool.shape[1], 2, 32)

    def retained_rows(self, layer: int) -> torch.Tensor:
        """Raw retained rows of one layer (0: l-1, 1: l) as [ret_capacity][128] in the storage type."""
        return self.ret_rows[layer, :, :256].contiguous().view(self.cfg.torch_dtype)

    def retained_tokens(self, layer: int) -> torch.Tensor:
        """Token index stored with each retained entry of one layer: [ret_capacity] int32."""
        return self.ret_rows[layer, :, 256:260].contiguous().view(torch.int32).reshape(-1)

    def nbytes(self) -> int:
        ts = (self.e_k, self.e_v, self.dist, self.ret_count, self.ret_offset, self.ret_index,
              self.ret_rows, self.ret_prefix, self.seg_minmax, self.status) + ((self.res_k, self.res_v) if self.q4 else ())
        return sum(t.numel() * t.element_size() for t in ts)


# The mc_layer_* calls are made once per layer and decode step, where a microsecond counts: their tensors are checked in
# plain expressions, at every call, and _refuse finds out what was wrong.
def _good(t: Optional[torch.Tensor], dtype, n: int, dev: Optional[int]) -> bool:
    return t is None or (t.dtype is dtype and t.numel() >= n and t.is_contiguous() and (dev is None or t.get_device() == dev))


def _refuse(dev: Optional[int], **tensors) -> None:
    """tensors: name=(tensor, type, entries); raises AssertionError for the first that is not as wanted."""
    for name, (t, dtype, n) in tensors.items():
        assert t is None or (t.dtype is dtype and t.is_contiguous()), f"{name}: a contiguous {dtype} tensor is wanted"
        assert t is None or t.numel() >= n, f"{name}: at least {n} entries are wanted"
        assert t is None or dev is None or t.get_device() == dev, f"{name}: all tensors have to be on the current CUDA device"


def _layer_stream(stream, dev: int) -> Optional[int]:
    """The stream of a mc_layer_* call whose tensors are on device dev."""
    assert dev >= 0 and dev == torch._C._cuda_getDevice(), "all tensors have to be on the current CUDA device"
    # (the stream's handle itself: building a Stream object costs 1 us of a 10 us call)
    return (torch._C._cuda_getCurrentRawStream(dev) if stream is None else stream.cuda_stream) or None


_CFG = {}


def _cfg_c(cfg: "McConfig") -> _Config:
    """cfg.c(), remembered by the fields' values: the mc_layer_* calls are made once per layer and decode step."""
    key = tuple(cfg.__dict__.values())
    c = _CFG.get(key)
    if c is None:
        if len(_CFG) > 256:
            _CFG.clear()
        c = _CFG[key] = cfg.c()
    return c


@dataclasses.dataclass
class LayerCache:
    """One uncompressed layer's paged cache (caller-owned tensors, see mc_layer_cache): k_pool / v_pool
    [n_pages][n_kv_heads][page_size][128] in the storage type, positions int32 / weights float32
    [n_pages][n_kv_heads][page_size] or None, status int32 [MC_STATUS_WORDS] (zeros; made here if not given)."""
    cfg: McConfig
    k_pool: torch.Tensor
    v_pool: torch.Tensor
    positions: Optional[torch.Tensor] = None
    weights: Optional[torch.Tensor] = None
    status: Optional[torch.Tensor] = None

    def __post_init__(self):
        if self.status is None:
            self.status = torch.zeros(MC_STATUS_WORDS, dtype=torch.int32, device=self.k_pool.device)

    def c(self, n_pages: int, cfg: Optional[McConfig] = None, dev: Optional[int] = None) -> _LayerCache:
        """cfg: the call's configuration (default: the cache's own), which the pools have to hold n_pages pages of; dev: the
        device that the tensors have to be on."""
        cfg = cfg or self.cfg
        k, v, pos, w, st = self.k_pool, self.v_pool, self.positions, self.weights, self.status
        dt, rows = cfg.torch_dtype, n_pages * cfg.n_kv_heads * cfg.page_size
        if not (k.dtype is dt and v.dtype is dt and k.numel() >= 128 * rows and v.numel() >= 128 * rows and k.is_contiguous()
                and v.is_contiguous() and (dev is None or (k.get_device() == dev and v.get_device() == dev))
                and (pos is None or _good(pos, torch.int32, rows, dev)) and (w is None or _good(w, torch.float32, rows, dev))
                and _good(st, torch.int32, MC_STATUS_WORDS, dev)):
            _refuse(dev, k_pool=(k, dt, 128 * rows), v_pool=(v, dt, 128 * rows), positions=(pos, torch.int32, rows),
                    weights=(w, torch.float32, rows), status=(st, torch.int32, MC_STATUS_WORDS))
        return _LayerCache(k.data_ptr(), v.data_ptr(), None if pos is None else pos.data_ptr(), None if w is None else w.data_ptr(),
                           st.data_ptr())


@dataclasses.dataclass
class ScoreOpts:
    """How a score is formed and which tokens a query sees (see mc_score_opts).  Tensors live on the device:
    alibi_slopes float32 [n_q_heads]; doc_start, prefix_len, q_pos int32 [batch]."""
    sm_scale: float
    softcap: float = 0.0
    alibi_slopes: Optional[torch.Tensor] = None
    window: int = 0
    doc_start: Optional[torch.Tensor] = None
    prefix_len: Optional[torch.Tensor] = None
    q_pos: Optional[torch.Tensor] = None

    def c(self, cfg: McConfig, batch: int, dev: Optional[int] = None) -> _ScoreOpts:
        a, d, p, q = self.alibi_slopes, self.doc_start, self.prefix_len, self.q_pos
        if not ((a is None or _good(a, torch.float32, cfg.n_q_heads, dev)) and (d is None or _good(d, torch.int32, batch, dev))
                and (p is None or _good(p, torch.int32, batch, dev)) and (q is None or _good(q, torch.int32, batch, dev))):
            _refuse(dev, alibi_slopes=(a, torch.float32, cfg.n_q_heads), doc_start=(d, torch.int32, batch),
                    prefix_len=(p, torch.int32, batch), q_pos=(q, torch.int32, batch))
        return _ScoreOpts(None if a is None else a.data_ptr(), None if d is None else d.data_ptr(), None if p is None else p.data_ptr(),
                          None if q is None else q.data_ptr(), self.sm_scale, self.softcap, self.window, 0)


@dataclasses.dataclass
class EvictOpts:
    """What mc_layer_evict keeps (see mc_evict_opts); q_pos: device int32 [batch] or None."""
    budget: int
    n_sink: int = 0
    n_recent: int = 0
    q_pos: Optional[torch.Tensor] = None

    def c(self, batch: int, dev: Optional[int] = None) -> _EvictOpts:
        q = self.q_pos
        if not _good(q, torch.int32, batch, dev):
            _refuse(dev, q_pos=(q, torch.int32, batch))
        return _EvictOpts(None if q is None else q.data_ptr(), int(self.budget), int(self.n_sink), int(self.n_recent), 0)


@dataclasses.dataclass
class LayerQ4Cache:
    """One layer held in 4 bits (caller-owned tensors, see mc_layer_q4_cache): k_codes / v_codes uint8
    [n_pages][n_kv_heads][32][64], k_meta [n_pages][n_kv_heads][128][2] / v_meta [n_pages][n_kv_heads][32][4][2] float16
    (scale, zero), res_k / res_v [batch][n_kv_heads][32][128] in the storage type, status int32 [MC_STATUS_WORDS] (zeros;
    made here if not given)."""
    cfg: McConfig
    k_codes: torch.Tensor
    k_meta: torch.Tensor
    v_codes: torch.Tensor
    v_meta: torch.Tensor
    res_k: torch.Tensor
    res_v: torch.Tensor
    status: Optional[torch.Tensor] = None

    def __post_init__(self):
        if self.status is None:
            self.status = torch.zeros(MC_STATUS_WORDS, dtype=torch.int32, device=self.k_codes.device)

    @classmethod
    def empty(cls, cfg: McConfig, batch: int, n_pages: int, device="cuda") -> "LayerQ4Cache":
        """A cache of n_pages pages for `batch` sequences, its contents undefined."""
        h = cfg.n_kv_heads
        mk = lambda shape, dt: torch.empty(shape, dtype=dt, device=device)  # noqa: E731
        return cls(cfg, mk((n_pages, h, 32, 64), torch.uint8), mk((n_pages, h, 128, 2), torch.float16), mk((n_pages, h, 32, 64), torch.uint8),
                   mk((n_pages, h, 32, 4, 2), torch.float16), mk((batch, h, 32, 128), cfg.torch_dtype), mk((batch, h, 32, 128), cfg.torch_dtype))

    def c(self, batch: int, n_pages: int, cfg: Optional[McConfig] = None, dev: Optional[int] = None) -> _LayerQ4Cache:
        """cfg: the call's configuration (default: the cache's own), of which the pools have to hold n_pages pages and the
        begun pages `batch` sequences; dev: the device that the tensors have to be on."""
        cfg = cfg or self.cfg
        dt, tiles, begun = cfg.torch_dtype, n_pages * cfg.n_kv_heads, batch * cfg.n_kv_heads * 4096
        kc, km, vc, vm, rk, rv, st = self.k_codes, self.k_meta, self.v_codes, self.v_meta, self.res_k, self.res_v, self.status
        if not (kc.dtype is torch.uint8 and vc.dtype is torch.uint8 and km.dtype is torch.float16 and vm.dtype is torch.float16
                and rk.dtype is dt and rv.dtype is dt and st.dtype is torch.int32
                and kc.numel() >= 2048 * tiles and vc.numel() >= 2048 * tiles and km.numel() >= 256 * tiles and vm.numel() >= 256 * tiles
                and rk.numel() >= begun and rv.numel() >= begun and st.numel() >= MC_STATUS_WORDS
                and kc.is_contiguous() and vc.is_contiguous() and km.is_contiguous() and vm.is_contiguous() and rk.is_contiguous()
                and rv.is_contiguous() and st.is_contiguous()
                and (dev is None or (kc.get_device() == dev and vc.get_device() == dev and km.get_device() == dev and vm.get_device() == dev
                                     and rk.get_device() == dev and rv.get_device() == dev and st.get_device() == dev))):
            _refuse(dev, k_codes=(kc, torch.uint8, 2048 * tiles), k_meta=(km, torch.float16, 256 * tiles),
                    v_codes=(vc, torch.uint8, 2048 * tiles), v_meta=(vm, torch.float16, 256 * tiles), res_k=(rk, dt, begun),
                    res_v=(rv, dt, begun), status=(st, torch.int32, MC_STATUS_WORDS))
        return _LayerQ4Cache(kc.data_ptr(), km.data_ptr(), vc.data_ptr(), vm.data_ptr(), rk.data_ptr(), rv.data_ptr(), st.data_ptr())


@dataclasses.dataclass
class PageSelection:
    """Which pages mc_layer_q4_select keeps (see mc_page_selection)."""
    budget: int
    n_sink: int = 0
    n_recent: int = 0

    def c(self) -> _PageSelection:
        return _PageSelection(int(self.budget), int(self.n_sink), int(self.n_recent), 0)


def _row_stride(name: str, t: torch.Tensor, cfg: "McConfig", rows: int, dev: int) -> int:
    """Elements between two rows of [rows][n_kv_heads][128], whose heads have to be next to each other."""
    sh, st = t.shape, t.stride()
    if not (t.dtype is cfg.torch_dtype and len(sh) == 3 and sh[0] == rows and sh[1] == cfg.n_kv_heads and sh[2] == 128 and st[2] == 1
            and (st[1] == 128 or sh[1] == 1) and t.get_device() == dev):
        raise AssertionError(f"{name}: [rows][n_kv_heads][128] of {cfg.torch_dtype} with adjacent heads on device {dev} is wanted")
    return st[0] if rows > 1 else cfg.n_kv_heads * 128  # (no element of one row depends on its stride)


class MiniCacheLib:
    """Loads libminicache.so and exposes its entry points under their C names."""

    def __init__(self, path: str = _LIB_PATH):
        if not os.path.exists(path):
            raise McError(-1, "library missing",
                          f"{path} not built; run `python -m paper_2405_14366_b200.build` (there is no fallback path)")
        self.path = path
        self._lib = C.CDLL(path)
        L = self._lib
        L.mc_version.restype = C.c_int32
        L.mc_build_flags.restype = C.c_int32
        L.mc_status_str.restype = C.c_char_p
        L.mc_status_str.argtypes = [C.c_int32]
        L.mc_last_cuda_error.restype = C.c_char_p
        P, V = C.POINTER, C.c_void_p
        L.mc_workspace_bytes.argtypes = [P(_Config), P(_Batch), C.c_int32, C.c_int32, P(C.c_size_t)]
        L.mc_merge_pair.argtypes = [P(_Config), P(_Batch), P(_LayerKV), P(_LayerKV), P(_PairCache), C.c_int32, V,
                                    C.c_size_t, V]
        L.mc_merge_pairs.argtypes = [P(_Config), P(_Batch), C.c_int32, P(P(_LayerKV)), P(P(_LayerKV)), P(P(_PairCache)),
                                     C.c_int32, V, C.c_size_t, V]
        L.mc_merge_pairs.restype = C.c_int32
        L.mc_admit_sequences.argtypes = [P(_Config), P(_Batch), C.c_int32, C.c_int32, C.c_int32, P(P(_LayerKV)), P(P(_LayerKV)),
                                         P(P(_LayerQ4)), P(P(_LayerQ4)), P(P(_PairCache)), C.c_int64, C.c_int32, V, C.c_size_t, V]
        L.mc_admit_sequences.restype = C.c_int32
        L.mc_prefill_merge_pair.argtypes = [P(_Config), P(_Batch), P(_Projection), P(_LayerKV), P(_LayerKV), P(_PairCache),
                                            C.c_float, C.c_int32, V, C.c_size_t, V]
        L.mc_prefill_merge_pair.restype = C.c_int32
        L.mc_append_pair.argtypes = [P(_Config), P(_Batch), P(_PairCache), V, V, V, V, V]
        L.mc_restore.argtypes = [P(_Config), P(_Batch), P(_PairCache), C.c_int32, P(_LayerKV), C.c_int32, V]
        L.mc_pair_bytes.argtypes = [P(_Config), P(_Batch), C.c_int64, P(_PairSizes)]
        L.mc_pair_bytes.restype = C.c_int32
        L.mc_get_stats.argtypes = [P(_Config), P(_Batch), P(_PairCache), V, P(_Stats)]
        L.mc_get_stats.restype = C.c_int32
        L.mc_decode_attn.argtypes = [P(_Config), P(_Batch), P(_PairCache), C.c_int32, V, V, V, C.c_float, V, V, V,
                                     C.c_size_t, V]
        L.mc_decode_attn_append.argtypes = [P(_Config), P(_Batch), P(_PairCache), C.c_int32, V, V, V, C.c_float, V, V, V, V, V, V,
                                            V, C.c_size_t, V]
        L.mc_decode_attn_append.restype = C.c_int32
        L.mc_decode_stage_host.argtypes = [P(_Config), P(_Batch), C.c_int32, V, V, V, V, C.c_size_t, P(V), P(V), P(V), V]
        L.mc_decode_stage_host.restype = C.c_int32
        L.mc_decode_drain_host.argtypes = [P(_Config), P(_Batch), C.c_int32, V, V, V, V, V]
        L.mc_decode_drain_host.restype = C.c_int32
        L.mc_read_status.argtypes = [P(_PairCache), V, P(C.c_int32)]
        L.mc_merge_pair_host.argtypes = [P(_Config), P(_Batch), P(_LayerKV), P(_LayerKV), P(_LayerKV), P(_LayerKV),
                                         P(_PairCache), C.c_int32, V, C.c_size_t, V]
        L.mc_decode_attn_host.argtypes = [P(_Config), P(_Batch), P(_PairCache), C.c_int32, V, V, V, C.c_float, V, V,
                                          V, C.c_size_t, V, C.c_size_t, V]
        L.mc_decode_io_bytes.argtypes = [P(_Config), P(_Batch), C.c_int32, P(C.c_size_t)]
        L.mc_decode_attn_static.argtypes = [P(_Config), P(_Batch), P(_PairCache), C.c_int32, V, V, V, C.c_float, V, V, V]
        L.mc_decode_attn_static.restype = C.c_int32
        L.mc_merge_pair_q4.argtypes = [P(_Config), P(_Batch), P(_LayerQ4), P(_LayerQ4), P(_PairCache), C.c_int32, V,
                                       C.c_size_t, V]
        L.mc_merge_pair_q4.restype = C.c_int32
        L.mc_layer_workspace_bytes.argtypes = [P(_Config), P(_Batch), C.c_int32, C.c_int32, P(C.c_size_t)]
        L.mc_layer_attn.argtypes = [P(_Config), P(_Batch), P(_LayerCache), P(_ScoreOpts), V, V, V, C.c_int32, V, V, V, C.c_size_t, V]
        L.mc_layer_observe.argtypes = [P(_Config), P(_Batch), P(_LayerCache), P(_ScoreOpts), V, C.c_int32, C.c_int32, V, C.c_size_t, V]
        L.mc_layer_evict.argtypes = [P(_Config), P(_Batch), P(_LayerCache), P(_EvictOpts), V, V, C.c_size_t, V]
        L.mc_layer_read_status.argtypes = [P(_LayerCache), V, P(C.c_int32)]
        for f in ("mc_layer_workspace_bytes", "mc_layer_attn", "mc_layer_observe", "mc_layer_evict", "mc_layer_read_status"):
            getattr(L, f).restype = C.c_int32
        head = [P(_Config), P(_Batch), P(_LayerQ4Cache)]
        L.mc_layer_q4_append.argtypes = head + [V, V, C.c_int64, C.c_int64, V, C.c_int32, V]
        L.mc_layer_q4_read.argtypes = head + [V, V, V, C.c_int64, C.c_int64, V, C.c_int32, V]
        L.mc_layer_q4_select.argtypes = head + [P(_ScoreOpts), P(_PageSelection), V, V, V, V, C.c_size_t, V]
        L.mc_layer_q4_attn.argtypes = head + [P(_ScoreOpts), V, V, C.c_int32, V, V, V, C.c_int32, V, V, V, C.c_size_t, V]
        L.mc_layer_q4_read_status.argtypes = [P(_LayerQ4Cache), V, P(C.c_int32)]
        for f in ("mc_layer_q4_append", "mc_layer_q4_read", "mc_layer_q4_select", "mc_layer_q4_attn", "mc_layer_q4_read_status"):
            getattr(L, f).restype = C.c_int32
        L.mc_selftest_wait_timeout.argtypes = [P(_PairCache), C.c_int32, V]
        L.mc_selftest_wait_timeout.restype = C.c_int32
        for f in ("mc_workspace_bytes", "mc_merge_pair", "mc_append_pair", "mc_restore", "mc_decode_attn",
                  "mc_read_status", "mc_merge_pair_host", "mc_decode_attn_host", "mc_decode_io_bytes"):
            getattr(L, f).restype = C.c_int32

    # -- helpers ------------------------------------------------------------------------------
    def _check(self, code: int):
        if code != 0:
            name = self._lib.mc_status_str(code).decode()
            detail = self._lib.mc_last_cuda_error().decode() if code == 7 else ""
            raise McError(code, name, detail)

    def has_symbol(self, name: str) -> bool:
        return hasattr(self._lib, name)

    # -- entry points ---------------------------------------------------------------------------
    def mc_version(self) -> int:
        return self._lib.mc_version()

    def mc_build_flags(self) -> int:
        return self._lib.mc_build_flags()

    def mc_status_str(self, code: int) -> str:
        return self._lib.mc_status_str(code).decode()

    def mc_workspace_bytes(self, cfg: McConfig, batch: Batch, op: int, n_query_sets: int = 1) -> int:
        out = C.c_size_t(0)
        c, b = cfg.c(), batch.c()
        self._check(self._lib.mc_workspace_bytes(C.byref(c), C.byref(b), op, n_query_sets, C.byref(out)))
        return out.value

    def mc_merge_pair(self, cfg: McConfig, batch: Batch, k_lm1, v_lm1, k_l, v_l, pair: PairCache,
                      do_retention: bool, workspace: torch.Tensor, stream=None):
        c, b, pc = cfg.c(), batch.c(), pair.c()
        a, l = _LayerKV(_ptr(k_lm1), _ptr(v_lm1)), _LayerKV(_ptr(k_l), _ptr(v_l))
        self._check(self._lib.mc_merge_pair(C.byref(c), C.byref(b), C.byref(a), C.byref(l), C.byref(pc),
                                            1 if do_retention else 0, _ptr(workspace),
                                            workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_merge_pairs(self, cfg: McConfig, batch: Batch, layers, pairs, do_retention: bool, workspace: torch.Tensor,
                       stream=None):
        """layers: per pair a dict with k_lm1, v_lm1, k_l, v_l pools; pairs: the PairCache of each.
        workspace: len(pairs) * mc_workspace_bytes(MC_OP_MERGE) bytes."""
        n = len(pairs)
        c, b = cfg.c(), batch.c()
        a = [_LayerKV(_ptr(x["k_lm1"]), _ptr(x["v_lm1"])) for x in layers]
        l = [_LayerKV(_ptr(x["k_l"]), _ptr(x["v_l"])) for x in layers]
        pcs = [pc.c() for pc in pairs]
        arr = lambda items, T: (C.POINTER(T) * n)(*[C.pointer(x) for x in items])
        self._check(self._lib.mc_merge_pairs(C.byref(c), C.byref(b), n, arr(a, _LayerKV), arr(l, _LayerKV),
                                             arr(pcs, _PairCache), 1 if do_retention else 0, _ptr(workspace),
                                             workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_admit_sequences(self, cfg: McConfig, batch: Batch, seq_begin: int, seq_count: int, layers, pairs, rows_per_seq: int,
                           do_retention: bool, workspace: torch.Tensor, stream=None, q4: bool = False):
        """layers: per pair a dict with k_lm1, v_lm1, k_l, v_l pools, or (q4) with "_lm1" / "_l" dicts of
        k_codes, k_meta, v_codes, v_meta; pairs: the PairCache of each pair."""
        n = len(pairs)
        c, b = cfg.c(), batch.c()
        pcs = [pc.c() for pc in pairs]
        arr = lambda items, T: (C.POINTER(T) * n)(*[C.pointer(x) for x in items])
        if q4:
            mk = lambda d: _LayerQ4(_ptr(d["k_codes"]), _ptr(d["k_meta"]), _ptr(d["v_codes"]), _ptr(d["v_meta"]))
            a, l = [mk(x["_lm1"]) for x in layers], [mk(x["_l"]) for x in layers]
            args = (None, None, arr(a, _LayerQ4), arr(l, _LayerQ4))
        else:
            a = [_LayerKV(_ptr(x["k_lm1"]), _ptr(x["v_lm1"])) for x in layers]
            l = [_LayerKV(_ptr(x["k_l"]), _ptr(x["v_l"])) for x in layers]
            args = (arr(a, _LayerKV), arr(l, _LayerKV), None, None)
        self._check(self._lib.mc_admit_sequences(C.byref(c), C.byref(b), int(seq_begin), int(seq_count), n, *args,
                                                 arr(pcs, _PairCache), int(rows_per_seq), 1 if do_retention else 0,
                                                 _ptr(workspace), workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_prefill_merge_pair(self, cfg: McConfig, batch: Batch, x, w_k, w_v, k_lm1, v_lm1, k_l, v_l, pair: PairCache,
                              d_hint: float, do_retention: bool, workspace: torch.Tensor, stream=None):
        """x [batch][x_seq_stride][d_model], w_k / w_v [n_kv_heads * 128][d_model]: layer l's projection;
        k_l / v_l: pools that receive the raw rows of tokens with distance above d_hint."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        pj = _Projection(_ptr(x), _ptr(w_k), _ptr(w_v), int(x.shape[-1]), int(x.shape[1]))
        a, l = _LayerKV(_ptr(k_lm1), _ptr(v_lm1)), _LayerKV(_ptr(k_l), _ptr(v_l))
        self._check(self._lib.mc_prefill_merge_pair(C.byref(c), C.byref(b), C.byref(pj), C.byref(a), C.byref(l), C.byref(pc),
                                                    float(d_hint), 1 if do_retention else 0, _ptr(workspace),
                                                    workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_merge_pair_q4(self, cfg: McConfig, batch: Batch, q_lm1, q_l, pair: PairCache, do_retention: bool,
                         workspace: torch.Tensor, stream=None):
        """q_lm1 / q_l: dicts with k_codes, k_meta, v_codes, v_meta device tensors (4-bit layers)."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        a = _LayerQ4(_ptr(q_lm1["k_codes"]), _ptr(q_lm1["k_meta"]), _ptr(q_lm1["v_codes"]), _ptr(q_lm1["v_meta"]))
        l = _LayerQ4(_ptr(q_l["k_codes"]), _ptr(q_l["k_meta"]), _ptr(q_l["v_codes"]), _ptr(q_l["v_meta"]))
        self._check(self._lib.mc_merge_pair_q4(C.byref(c), C.byref(b), C.byref(a), C.byref(l), C.byref(pc),
                                               1 if do_retention else 0, _ptr(workspace),
                                               workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_append_pair(self, cfg: McConfig, batch: Batch, pair: PairCache, k_new_lm1, v_new_lm1, k_new_l, v_new_l,
                       stream=None):
        c, b, pc = cfg.c(), batch.c(), pair.c()
        self._check(self._lib.mc_append_pair(C.byref(c), C.byref(b), C.byref(pc), _ptr(k_new_lm1), _ptr(v_new_lm1),
                                             _ptr(k_new_l), _ptr(v_new_l), _stream(stream)))

    def mc_restore(self, cfg: McConfig, batch: Batch, pair: PairCache, layer_sel: int, dst_k, dst_v, stream=None):
        """dst_k / dst_v: pools in the storage type, or float32 pools (then the unrounded products are written)."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        d = _LayerKV(_ptr(dst_k), _ptr(dst_v))
        assert dst_k.dtype == dst_v.dtype and dst_k.dtype in (torch.float32, cfg.torch_dtype)
        f32 = 1 if dst_k.dtype == torch.float32 else 0
        self._check(self._lib.mc_restore(C.byref(c), C.byref(b), C.byref(pc), layer_sel, C.byref(d), f32, _stream(stream)))

    def mc_pair_bytes(self, cfg: McConfig, batch: int, n_pages: int, max_seq_len: int, ret_capacity: int) -> _PairSizes:
        c = cfg.c()
        b = _Batch(None, None, int(batch), 0, int(max_seq_len), 0, int(n_pages))
        out = _PairSizes()
        self._check(self._lib.mc_pair_bytes(C.byref(c), C.byref(b), int(ret_capacity), C.byref(out)))
        return out

    def mc_get_stats(self, cfg: McConfig, batch: Batch, pair: PairCache, stream=None, check: bool = True):
        """(dict of the mc_stats fields, return code); synchronises the stream."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        out = _Stats()
        code = self._lib.mc_get_stats(C.byref(c), C.byref(b), C.byref(pc), _stream(stream), C.byref(out))
        if check:
            self._check(code)
        return {f: getattr(out, f) for f, _ in _Stats._fields_ if f != "reserved"}, code

    def mc_decode_attn(self, cfg: McConfig, batch: Batch, pair: PairCache, layer_sel: int, q, k_new, v_new,
                       sm_scale: float, out, lse, workspace: torch.Tensor, stream=None):
        c, b, pc = cfg.c(), batch.c(), pair.c()
        self._check(self._lib.mc_decode_attn(C.byref(c), C.byref(b), C.byref(pc), layer_sel, _ptr(q), _ptr(k_new),
                                             _ptr(v_new), float(sm_scale), _ptr(out), _ptr(lse), _ptr(workspace),
                                             workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_decode_attn_append(self, cfg: McConfig, batch: Batch, pair: PairCache, layer_sel: int, q, k_new, v_new,
                              sm_scale: float, out, lse, k_new_lm1, v_new_lm1, k_new_l, v_new_l, workspace: torch.Tensor,
                              stream=None):
        """mc_decode_attn followed by mc_append_pair, in one call (the append rides on the attention's second launch)."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        self._check(self._lib.mc_decode_attn_append(C.byref(c), C.byref(b), C.byref(pc), layer_sel, _ptr(q), _ptr(k_new),
                                                    _ptr(v_new), float(sm_scale), _ptr(out), _ptr(lse), _ptr(k_new_lm1),
                                                    _ptr(v_new_lm1), _ptr(k_new_l), _ptr(v_new_l), _ptr(workspace),
                                                    workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_merge_pair_host(self, cfg: McConfig, batch: Batch, host, dev, pair: PairCache, do_retention: bool,
                           workspace: torch.Tensor, stream=None):
        """host / dev: dicts with k_lm1, v_lm1, k_l, v_l pools (pinned host tensors / device tensors)."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        ha, hl = _LayerKV(_ptr(host["k_lm1"]), _ptr(host["v_lm1"])), _LayerKV(_ptr(host["k_l"]), _ptr(host["v_l"]))
        da, dl = _LayerKV(_ptr(dev["k_lm1"]), _ptr(dev["v_lm1"])), _LayerKV(_ptr(dev["k_l"]), _ptr(dev["v_l"]))
        self._check(self._lib.mc_merge_pair_host(C.byref(c), C.byref(b), C.byref(ha), C.byref(hl), C.byref(da),
                                                 C.byref(dl), C.byref(pc), 1 if do_retention else 0, _ptr(workspace),
                                                 workspace.numel() * workspace.element_size(), _stream(stream)))

    def mc_decode_io_bytes(self, cfg: McConfig, batch: Batch, n_query_sets: int = 1) -> int:
        out = C.c_size_t(0)
        c, b = cfg.c(), batch.c()
        self._check(self._lib.mc_decode_io_bytes(C.byref(c), C.byref(b), n_query_sets, C.byref(out)))
        return out.value

    def mc_decode_attn_host(self, cfg: McConfig, batch: Batch, pair: PairCache, layer_sel: int, q_host, k_new_host,
                            v_new_host, sm_scale: float, out_host, lse_host, dev_io: torch.Tensor,
                            workspace: torch.Tensor, stream=None):
        c, b, pc = cfg.c(), batch.c(), pair.c()
        self._check(self._lib.mc_decode_attn_host(C.byref(c), C.byref(b), C.byref(pc), layer_sel, _ptr(q_host),
                                                  _ptr(k_new_host), _ptr(v_new_host), float(sm_scale), _ptr(out_host),
                                                  _ptr(lse_host), _ptr(dev_io), dev_io.numel() * dev_io.element_size(),
                                                  _ptr(workspace), workspace.numel() * workspace.element_size(),
                                                  _stream(stream)))

    def mc_decode_stage_host(self, cfg: McConfig, batch: Batch, n_query_sets: int, q_host, k_new_host, v_new_host,
                             dev_io: torch.Tensor, stream=None):
        """Stages q (and the new rows) from host tensors into `dev_io`; returns views of dev_io: (q, k_new, v_new)
        shaped [n_query_sets][batch][heads][128] in the storage type (k_new / v_new None if not given)."""
        c, b = cfg.c(), batch.c()
        qd, kd, vd = C.c_void_p(), C.c_void_p(), C.c_void_p()
        self._check(self._lib.mc_decode_stage_host(C.byref(c), C.byref(b), int(n_query_sets), _ptr(q_host), _ptr(k_new_host),
                                                   _ptr(v_new_host), _ptr(dev_io), dev_io.numel() * dev_io.element_size(),
                                                   C.byref(qd), C.byref(kd), C.byref(vd), _stream(stream)))
        base = dev_io.data_ptr()
        nb = batch.seq_lens.shape[0]

        def view(ptr, heads):
            if not ptr.value:
                return None
            n = n_query_sets * nb * heads * 256
            off = ptr.value - base
            return dev_io[off:off + n].view(cfg.torch_dtype).view(n_query_sets, nb, heads, 128)
        return view(qd, cfg.n_q_heads), view(kd, cfg.n_kv_heads), view(vd, cfg.n_kv_heads)

    def mc_decode_drain_host(self, cfg: McConfig, batch: Batch, n_query_sets: int, out_dev, lse_dev, out_host, lse_host,
                             stream=None):
        """Asynchronous copy of an attention result (and its log-sum-exps, if given) from device to host tensors."""
        c, b = cfg.c(), batch.c()
        self._check(self._lib.mc_decode_drain_host(C.byref(c), C.byref(b), int(n_query_sets), _ptr(out_dev), _ptr(lse_dev),
                                                   _ptr(out_host), _ptr(lse_host), _stream(stream)))

    def mc_decode_attn_static(self, cfg: McConfig, batch: Batch, pair: PairCache, layer_sel: int, q, k_new, v_new,
                              sm_scale: float, out, lse, stream=None):
        """mc_decode_attn for callers with no scratch memory to give: the split partials go to the
        library's built-in device array (at most MC_STATIC_SCRATCH_BYTES; larger geometries raise)."""
        c, b, pc = cfg.c(), batch.c(), pair.c()
        code = self._lib.mc_decode_attn_static(C.byref(c), C.byref(b), C.byref(pc), layer_sel, _ptr(q), _ptr(k_new),
                                               _ptr(v_new), float(sm_scale), _ptr(out), _ptr(lse), _stream(stream))
        if code == 5:
            raise McError(code, "MC_ERR_CAPACITY", self._lib.mc_last_cuda_error().decode())
        self._check(code)

    # -- one uncompressed layer -------------------------------------------------------------------
    def mc_layer_workspace_bytes(self, cfg: McConfig, batch: Batch, op: int, arg: int = 0) -> int:
        """arg: the call's flags (MC_OP_LAYER_ATTN, MC_OP_LAYER_Q4_ATTN), the number of observed queries (MC_OP_LAYER_OBSERVE),
        0 (MC_OP_LAYER_EVICT, MC_OP_LAYER_Q4_SELECT)."""
        out = C.c_size_t(0)
        c, b = cfg.c(), batch.c()
        self._check(self._lib.mc_layer_workspace_bytes(C.byref(c), C.byref(b), int(op), int(arg), C.byref(out)))
        return out.value

    def mc_layer_attn(self, cfg: McConfig, batch: Batch, layer: LayerCache, opts: ScoreOpts, q, k_new, v_new, flags: int, out, lse,
                      workspace: torch.Tensor, stream=None):
        """q, out [batch][n_q_heads][128], k_new / v_new [batch][n_kv_heads][128] or None; flags: MC_LAYER_APPEND |
        MC_LAYER_ACCUMULATE; lse [batch][n_q_heads] float32 or None.  Every tensor of a mc_layer_* call has to be on the
        device that is current (AssertionError)."""
        dev = q.get_device()
        c, b, dt = _cfg_c(cfg), batch.layer_c(dev), cfg.torch_dtype
        n = b.batch
        rows_q, rows_kv = n * cfg.n_q_heads * 128, n * cfg.n_kv_heads * 128
        if not (q.dtype is dt and out.dtype is dt and q.numel() == rows_q and out.numel() == rows_q and q.is_contiguous()
                and out.is_contiguous() and out.get_device() == dev and workspace.get_device() == dev):
            _refuse(dev, q=(q, dt, rows_q), out=(out, dt, rows_q), workspace=(workspace, workspace.dtype, 0))
            raise AssertionError("q and out: [batch][n_q_heads][128] are wanted")
        for t in (k_new, v_new):
            if t is not None and not (t.dtype is dt and t.numel() == rows_kv and t.is_contiguous() and t.get_device() == dev):
                _refuse(dev, k_new=(k_new, dt, rows_kv), v_new=(v_new, dt, rows_kv))
                raise AssertionError("k_new and v_new: [batch][n_kv_heads][128] are wanted")
        if lse is not None and not (_good(lse, torch.float32, 0, dev) and lse.numel() == n * cfg.n_q_heads):
            _refuse(dev, lse=(lse, torch.float32, n * cfg.n_q_heads))
            raise AssertionError("lse: [batch][n_q_heads] is wanted")
        l, o, at = layer.c(b.n_pages, cfg, dev), opts.c(cfg, n, dev), _layer_stream(stream, dev)
        code = self._lib.mc_layer_attn(c, b, l, o, q.data_ptr(), None if k_new is None else k_new.data_ptr(),
                                       None if v_new is None else v_new.data_ptr(), flags, out.data_ptr(),
                                       None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes, at)
        if code:
            self._check(code)

    def mc_layer_observe(self, cfg: McConfig, batch: Batch, layer: LayerCache, opts: ScoreOpts, q, flags: int, workspace: torch.Tensor,
                         stream=None):
        """q [batch][n_obs][n_q_heads][128]: the last n_obs queries of every sequence; flags: 0 (weights are written) or
        MC_LAYER_ACCUMULATE (added to)."""
        dev, shape = q.get_device(), q.shape
        c, b = _cfg_c(cfg), batch.layer_c(dev)
        assert len(shape) == 4 and shape[0] == b.batch and shape[2] == cfg.n_q_heads and shape[3] == 128, "q: [batch][n_obs][n_q_heads][128]"
        if not (_good(q, cfg.torch_dtype, 0, dev) and workspace.get_device() == dev):
            _refuse(dev, q=(q, cfg.torch_dtype, 0), workspace=(workspace, workspace.dtype, 0))
            raise AssertionError("all tensors have to be on the current CUDA device")
        l, o, at = layer.c(b.n_pages, cfg, dev), opts.c(cfg, b.batch, dev), _layer_stream(stream, dev)
        code = self._lib.mc_layer_observe(c, b, l, o, q.data_ptr(), shape[1], flags, workspace.data_ptr(), workspace.nbytes, at)
        if code:
            self._check(code)

    def mc_layer_evict(self, cfg: McConfig, batch: Batch, layer: LayerCache, opts: EvictOpts, new_lens: torch.Tensor,
                       workspace: torch.Tensor, stream=None):
        """new_lens int32 [batch] receives min(seq_lens, budget); it must not share memory with batch.seq_lens or opts.q_pos."""
        dev = new_lens.get_device()
        c, b = _cfg_c(cfg), batch.layer_c(dev)
        if not (_good(new_lens, torch.int32, 0, dev) and new_lens.numel() == b.batch and workspace.get_device() == dev):
            _refuse(dev, new_lens=(new_lens, torch.int32, b.batch), workspace=(workspace, workspace.dtype, 0))
            raise AssertionError("new_lens: int32 [batch] is wanted")
        l, o, at = layer.c(b.n_pages, cfg, dev), opts.c(b.batch, dev), _layer_stream(stream, dev)
        code = self._lib.mc_layer_evict(c, b, l, o, new_lens.data_ptr(), workspace.data_ptr(), workspace.nbytes, at)
        if code:
            self._check(code)

    def mc_layer_read_status(self, layer: LayerCache, stream=None, check: bool = True):
        words = (C.c_int32 * MC_STATUS_WORDS)()
        l = layer.c(0)
        code = self._lib.mc_layer_read_status(C.byref(l), _stream(stream), words)
        if check:
            self._check(code)
        return list(words), code

    # -- one layer held in 4 bits -----------------------------------------------------------------
    def _q4_rows(self, cfg, batch, layer, k, v, row_offsets, stream):
        """What mc_layer_q4_append and mc_layer_q4_read have in common: k, v [rows][n_kv_heads][128], row_offsets int32 [batch + 1]."""
        dev, rows = k.get_device(), k.size(0)
        b = batch.layer_c(dev)
        ks, vs = _row_stride("k", k, cfg, rows, dev), _row_stride("v", v, cfg, rows, dev)
        if not _good(row_offsets, torch.int32, b.batch + 1, dev):
            _refuse(dev, row_offsets=(row_offsets, torch.int32, b.batch + 1))
        return _cfg_c(cfg), b, layer.c(b.batch, b.n_pages, cfg, dev), ks, vs, rows, _layer_stream(stream, dev)

    def mc_layer_q4_append(self, cfg: McConfig, batch: Batch, layer: LayerQ4Cache, k, v, row_offsets: torch.Tensor, stream=None):
        """k, v [rows][n_kv_heads][128], parts of a wider row allowed; sequence b gets rows row_offsets[b] .. row_offsets[b + 1]."""
        c, b, l, ks, vs, rows, at = self._q4_rows(cfg, batch, layer, k, v, row_offsets, stream)
        code = self._lib.mc_layer_q4_append(c, b, l, k.data_ptr(), v.data_ptr(), ks, vs, row_offsets.data_ptr(), rows, at)
        if code:
            self._check(code)

    def mc_layer_q4_read(self, cfg: McConfig, batch: Batch, layer: LayerQ4Cache, begin: Optional[torch.Tensor], k, v,
                         row_offsets: torch.Tensor, stream=None):
        """Writes tokens begin[b] + i (begin int32 [batch] or None) to rows row_offsets[b] + i of k and v [rows][n_kv_heads][128]."""
        c, b, l, ks, vs, rows, at = self._q4_rows(cfg, batch, layer, k, v, row_offsets, stream)
        if begin is not None and not _good(begin, torch.int32, b.batch, k.get_device()):
            _refuse(k.get_device(), begin=(begin, torch.int32, b.batch))
        code = self._lib.mc_layer_q4_read(c, b, l, None if begin is None else begin.data_ptr(), k.data_ptr(), v.data_ptr(), ks, vs,
                                          row_offsets.data_ptr(), rows, at)
        if code:
            self._check(code)

    def mc_layer_q4_select(self, cfg: McConfig, batch: Batch, layer: LayerQ4Cache, opts: ScoreOpts, keep: PageSelection, q, pages,
                           counts, workspace: torch.Tensor, stream=None):
        """pages int32 [batch][n_kv_heads][budget], counts int32 [batch] receive the selection."""
        dev = q.get_device()
        c, b = _cfg_c(cfg), batch.layer_c(dev)
        n, rows_q, dt = b.batch, b.batch * cfg.n_q_heads * 128, cfg.torch_dtype
        if not (_good(q, dt, 0, dev) and q.numel() == rows_q and _good(pages, torch.int32, 0, dev)
                and pages.numel() == n * cfg.n_kv_heads * keep.budget and _good(counts, torch.int32, 0, dev) and counts.numel() == n
                and workspace.get_device() == dev):
            _refuse(dev, q=(q, dt, rows_q), pages=(pages, torch.int32, n * cfg.n_kv_heads * keep.budget), counts=(counts, torch.int32, n),
                    workspace=(workspace, workspace.dtype, 0))
            raise AssertionError("q [batch][n_q_heads][128], pages [batch][n_kv_heads][budget] and counts [batch] are wanted")
        l, o, at = layer.c(n, b.n_pages, cfg, dev), opts.c(cfg, n, dev), _layer_stream(stream, dev)
        code = self._lib.mc_layer_q4_select(c, b, l, o, keep.c(), q.data_ptr(), pages.data_ptr(), counts.data_ptr(),
                                            workspace.data_ptr(), workspace.nbytes, at)
        if code:
            self._check(code)

    def mc_layer_q4_attn(self, cfg: McConfig, batch: Batch, layer: LayerQ4Cache, opts: ScoreOpts, pages, counts, q, k_new, v_new,
                         flags: int, out, lse, workspace: torch.Tensor, stream=None):
        """As mc_layer_attn; pages int32 [batch][n_kv_heads][any], counts int32 [batch]: the pages to attend, or None, None."""
        dev = q.get_device()
        c, b, dt = _cfg_c(cfg), batch.layer_c(dev), cfg.torch_dtype
        n = b.batch
        rows_q, rows_kv = n * cfg.n_q_heads * 128, n * cfg.n_kv_heads * 128
        if not (q.dtype is dt and out.dtype is dt and q.numel() == rows_q and out.numel() == rows_q and q.is_contiguous()
                and out.is_contiguous() and out.get_device() == dev and workspace.get_device() == dev):
            _refuse(dev, q=(q, dt, rows_q), out=(out, dt, rows_q), workspace=(workspace, workspace.dtype, 0))
            raise AssertionError("q and out: [batch][n_q_heads][128] are wanted")
        for t in (k_new, v_new):
            if t is not None and not (t.dtype is dt and t.numel() == rows_kv and t.is_contiguous() and t.get_device() == dev):
                _refuse(dev, k_new=(k_new, dt, rows_kv), v_new=(v_new, dt, rows_kv))
                raise AssertionError("k_new and v_new: [batch][n_kv_heads][128] are wanted")
        if lse is not None and not (_good(lse, torch.float32, 0, dev) and lse.numel() == n * cfg.n_q_heads):
            _refuse(dev, lse=(lse, torch.float32, n * cfg.n_q_heads))
            raise AssertionError("lse: [batch][n_q_heads] is wanted")
        stride = 0
        if pages is not None:
            if not (_good(pages, torch.int32, 0, dev) and pages.dim() == 3 and pages.size(0) == n and pages.size(1) == cfg.n_kv_heads):
                _refuse(dev, pages=(pages, torch.int32, 0))
                raise AssertionError("pages: [batch][n_kv_heads][any] is wanted")
            if not (counts is not None and _good(counts, torch.int32, n, dev)):
                assert counts is not None, "counts are wanted with pages"
                _refuse(dev, counts=(counts, torch.int32, n))
            stride = pages.size(2)
        l, o, at = layer.c(n, b.n_pages, cfg, dev), opts.c(cfg, n, dev), _layer_stream(stream, dev)
        code = self._lib.mc_layer_q4_attn(c, b, l, o, None if pages is None else pages.data_ptr(),
                                          None if counts is None else counts.data_ptr(), stride, q.data_ptr(),
                                          None if k_new is None else k_new.data_ptr(), None if v_new is None else v_new.data_ptr(), flags,
                                          out.data_ptr(), None if lse is None else lse.data_ptr(), workspace.data_ptr(), workspace.nbytes, at)
        if code:
            self._check(code)

    def mc_layer_q4_read_status(self, layer: LayerQ4Cache, stream=None, check: bool = True):
        words = (C.c_int32 * MC_STATUS_WORDS)()
        l = layer.c(0, 0)
        code = self._lib.mc_layer_q4_read_status(C.byref(l), _stream(stream), words)
        if check:
            self._check(code)
        return list(words), code

    def mc_selftest_wait_timeout(self, pair: PairCache, poll_limit: int = 20000, stream=None):
        pc = pair.c()
        self._check(self._lib.mc_selftest_wait_timeout(C.byref(pc), int(poll_limit), _stream(stream)))

    def mc_read_status(self, pair: PairCache, stream=None, check: bool = True):
        words = (C.c_int32 * MC_STATUS_WORDS)()
        pc = pair.c()
        code = self._lib.mc_read_status(C.byref(pc), _stream(stream), words)
        if check:
            self._check(code)
        return list(words), code


_LIB: Optional[MiniCacheLib] = None


def lib() -> MiniCacheLib:
    """The process-wide library handle (raises if the shared object has not been built)."""
    global _LIB
    if _LIB is None:
        _LIB = MiniCacheLib()
    return _LIB
