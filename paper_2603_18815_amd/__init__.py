"""MI355X rollout attention: paged-KV decode, observation append and page writes.

Thin PyTorch-facing binding of the C ABI in include/rollout_attn.h. It only
checks tensor dtypes/devices, allocates outputs with torch and passes raw
device pointers plus torch's current HIP stream to the library; every step of
the computation runs in the library's HIP kernels. If the library is not built
the import of any function fails loudly: there is no fallback path.

Host-side sizes (max_kv_len, max_q_len, max_new, max_pos, total, ...) that are
left as None are read from the device tensors with .item(), which waits for the
GPU: such a call is neither asynchronous nor capturable into a HIP graph. Pass
them explicitly (and an output and workspace) to capture a call or to keep it
asynchronous. With stream= given, outputs and workspaces the wrapper allocates
come from that stream's own memory, so neither earlier work of other streams nor
a later reuse of the memory can overlap the call's kernels.

Layout (see the header): K pool [pages][Hkv][16][128] (token-major), V pool
[pages][Hkv][128][16] (dim-major), block table int32 [B][stride]. Pools are
bf16, or uint8 OCP FP8 E4M3 codes with one scale per pool (value = code * scale).
"""
from __future__ import annotations

import ctypes
import math
from typing import Optional, Tuple

import torch

from . import _lib
from ._lib import RolloutAttnError  # noqa: F401  (re-export)

PAGE_SIZE = 16
HEAD_DIM = 128

__all__ = ["PagedKV", "decode", "decode_noalloc", "decode_shared_prefix", "append", "append_write", "mixed",
           "kv_page_write",
           "kv_page_gather", "token_logprob", "decode_workspace_size",
           "decode_shared_prefix_workspace_size", "append_workspace_size", "mixed_workspace_size",
           "token_logprob_workspace_size", "token_logprob_pack_weight", "token_logprob_packed",
           "token_sample", "token_sample_workspace_size", "linear_decode", "linear_append",
           "linear_append_workspace_size", "block_table_extend", "block_table_release",
           "draft_tree_mask", "draft_tree_accept", "decode_tree", "decode_tree_workspace_size",
           "decode_tree_max_workspace_size",
           "token_logits_adjust", "block_table_fork", "block_table_release_shared",
           "block_table_release_shared_workspace_size", "kv_page_copy", "kv_page_compact",
           "abi_version", "RolloutAttnError"]


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _need(t: torch.Tensor, name: str, dtype: torch.dtype, device: torch.device) -> None:
    if t.is_cuda and t.dtype is dtype and t.device == device and t.is_contiguous():
        return
    # the kernels dereference every pointer on the GPU: host tensors are refused
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor, got one on {t.device}")
    if t.dtype != dtype:
        raise TypeError(f"{name} must be {dtype}, got {t.dtype}")
    if t.device != device:
        raise ValueError(f"{name} must be on {device}, got {t.device}")
    if not t.is_contiguous():
        raise ValueError(f"{name} must be contiguous")


def _shape(t: torch.Tensor, shape, name: str) -> None:
    if t.shape != shape:
        raise ValueError(f"{name} must have shape {tuple(shape)}, got {tuple(t.shape)}")


def _rows(kv: "PagedKV", B: int) -> None:
    if kv.block_table.shape[0] < B:
        raise ValueError(f"block_table has {kv.block_table.shape[0]} rows, batch has {B}")


def _stream(device: torch.device, stream) -> int:
    if stream is None:
        # the current stream's handle without building a torch.cuda.Stream (1.9 us)
        return torch._C._cuda_getCurrentRawStream(device.index)
    return stream.cuda_stream if hasattr(stream, "cuda_stream") else int(stream)


def _empty(shape, dtype: torch.dtype, device: torch.device, stream,
           scratch: bool = False) -> torch.Tensor:
    """torch.empty for an output or workspace (scratch) of a call launched on `stream`.

    torch's caching allocator orders the reuse of a block by the stream that was
    current when it was allocated: a block freed there may still have that stream's
    work pending on it when it is handed out again. When the call runs on another
    stream (stream= given), the block is therefore allocated as that stream's own, so
    that everything pending on it comes before the call's kernels; an output is also
    recorded on the current stream, where the caller may read it before dropping it."""
    if stream is None:
        return torch.empty(shape, dtype=dtype, device=device)
    s = stream if isinstance(stream, torch.cuda.Stream) else \
        torch.cuda.ExternalStream(int(stream), device=device)
    current = torch.cuda.current_stream(device)
    if s.cuda_stream == current.cuda_stream:
        return torch.empty(shape, dtype=dtype, device=device)
    with torch.cuda.stream(s):
        t = torch.empty(shape, dtype=dtype, device=device)
    if not scratch:
        t.record_stream(current)
    return t


class PagedKV:
    """A caller-owned paged KV cache: two pools and a block table, all on one GPU.

    bf16 pools, or fp8 pools (torch.uint8 or torch.float8_e4m3fn storage of E4M3
    codes) with k_scale / v_scale: an element's value is code * scale.
    """

    def __init__(self, k_pool: torch.Tensor, v_pool: torch.Tensor, block_table: torch.Tensor,
                 k_scale: Optional[float] = None, v_scale: Optional[float] = None):
        dev = k_pool.device
        if k_pool.dtype == torch.float8_e4m3fn:
            k_pool = k_pool.view(torch.uint8)
        if v_pool.dtype == torch.float8_e4m3fn:
            v_pool = v_pool.view(torch.uint8)
        self.fp8 = k_pool.dtype == torch.uint8
        dt = torch.uint8 if self.fp8 else torch.bfloat16
        _need(k_pool, "k_pool", dt, dev)
        _need(v_pool, "v_pool", dt, dev)
        if self.fp8 and (k_scale is None or v_scale is None):
            raise ValueError("fp8 pools need k_scale and v_scale")
        self.k_scale = float(k_scale) if self.fp8 else 1.0
        self.v_scale = float(v_scale) if self.fp8 else 1.0
        _need(block_table, "block_table", torch.int32, dev)
        if k_pool.dim() != 4 or k_pool.shape[2:] != (PAGE_SIZE, HEAD_DIM):
            raise ValueError(f"k_pool must be [pages][Hkv][16][128], got {tuple(k_pool.shape)}")
        n, hkv = k_pool.shape[:2]
        if tuple(v_pool.shape) != (n, hkv, HEAD_DIM, PAGE_SIZE):
            raise ValueError(f"v_pool must be [pages][Hkv][128][16], got {tuple(v_pool.shape)}")
        if block_table.dim() != 2:
            raise ValueError("block_table must be [B][stride]")
        self.k_pool, self.v_pool, self.block_table = k_pool, v_pool, block_table
        self.device = dev
        self.num_pages, self.num_kv_heads = int(n), int(hkv)
        self.bt_stride = int(block_table.shape[1])

    def with_table(self, block_table: torch.Tensor) -> "PagedKV":
        """Same pools, another block table (e.g. a sub-batch of rows)."""
        return PagedKV(self.k_pool, self.v_pool, block_table,
                       self.k_scale if self.fp8 else None, self.v_scale if self.fp8 else None)

    def struct(self) -> _lib.RaPagedKV:
        return _lib.RaPagedKV(self.k_pool.data_ptr(), self.v_pool.data_ptr(),
                              self.block_table.data_ptr(), self.num_pages, self.bt_stride,
                              self.num_kv_heads, PAGE_SIZE, HEAD_DIM,
                              _lib.RA_KV_FP8_E4M3 if self.fp8 else _lib.RA_KV_BF16,
                              self.k_scale, self.v_scale)


def abi_version() -> int:
    return _lib.load().ra_abi_version()


def decode_workspace_size(B: int, Hq: int, Hkv: int, max_kv_len: int) -> int:
    return int(_lib.load().rollout_attn_decode_workspace_size(B, Hq, Hkv, max_kv_len))


def decode(q: torch.Tensor, kv: PagedKV, kv_lens: torch.Tensor, max_kv_len: Optional[int] = None,
           scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
           lse: Optional[torch.Tensor] = None, want_lse: bool = False,
           workspace: Optional[torch.Tensor] = None, stream=None
           ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Decode attention; q bf16 [B][Hq][128] -> out fp32 [B][Hq][128] (, lse fp32 [B][Hq])."""
    lib = _lib.load()
    dev = kv.device
    _need(q, "q", torch.bfloat16, dev)
    _need(kv_lens, "kv_lens", torch.int32, dev)
    B, Hq, D = q.shape
    _shape(q, (B, Hq, HEAD_DIM), "q")
    _shape(kv_lens, (B,), "kv_lens")
    _rows(kv, B)
    if max_kv_len is None:
        max_kv_len = int(kv_lens.max().item()) if B else 0
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = _empty((B, Hq, D), torch.float32, dev, stream)
    _need(out, "out", torch.float32, dev)
    _shape(out, (B, Hq, HEAD_DIM), "out")
    if lse is None and want_lse:
        lse = _empty((B, Hq), torch.float32, dev, stream)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        _shape(lse, (B, Hq), "lse")
    if workspace is None:
        ws_bytes = lib.rollout_attn_decode_workspace_size(B, Hq, kv.num_kv_heads, max_kv_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    s = kv.struct()
    _lib.check("rollout_attn_decode", lib.rollout_attn_decode(
        q.data_ptr(), ctypes.byref(s), kv_lens.data_ptr(), B, Hq, max_kv_len, float(scale),
        out.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream(dev, stream)))
    return out, lse


def decode_noalloc(q: torch.Tensor, kv: PagedKV, kv_lens: torch.Tensor, max_kv_len: int,
                   out: torch.Tensor, scale: Optional[float] = None,
                   lse: Optional[torch.Tensor] = None, stream=None
                   ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """decode() without a workspace: the library's own per-GPU device scratch holds
    the split partials, so the call allocates nothing (the caller passes out, and
    lse if wanted, and the host-side max_kv_len). Plans needing more than
    RA_NOALLOC_SCRATCH_BYTES of partials are refused (RA_ERR_WORKSPACE). Calls
    that overlap on one GPU share that scratch and race: keep them on one stream."""
    lib = _lib.load()
    dev = kv.device
    _need(q, "q", torch.bfloat16, dev)
    _need(kv_lens, "kv_lens", torch.int32, dev)
    B, Hq, D = q.shape
    _shape(q, (B, Hq, HEAD_DIM), "q")
    _shape(kv_lens, (B,), "kv_lens")
    _rows(kv, B)
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    _need(out, "out", torch.float32, dev)
    _shape(out, (B, Hq, HEAD_DIM), "out")
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        _shape(lse, (B, Hq), "lse")
    s = kv.struct()
    _lib.check("rollout_attn_decode_noalloc", lib.rollout_attn_decode_noalloc(
        q.data_ptr(), ctypes.byref(s), kv_lens.data_ptr(), B, Hq, int(max_kv_len), float(scale),
        out.data_ptr(), _ptr(lse), _stream(dev, stream)))
    return out, lse


def decode_shared_prefix_workspace_size(B: int, Hq: int, Hkv: int, max_kv_len: int,
                                        max_prefix_len: int) -> int:
    return int(_lib.load().rollout_attn_decode_shared_prefix_workspace_size(
        B, Hq, Hkv, max_kv_len, max_prefix_len))


def decode_shared_prefix(q: torch.Tensor, kv: PagedKV, kv_lens: torch.Tensor,
                         group_start: torch.Tensor, prefix_len: torch.Tensor,
                         max_group_rows: int, max_prefix_len: int,
                         max_kv_len: Optional[int] = None, scale: Optional[float] = None,
                         out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                         want_lse: bool = False, workspace: Optional[torch.Tensor] = None,
                         stream=None) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Decode for groups of rows that share their first prefix_len[i] cached tokens.

    group_start int32 [G+1] (row offsets of the groups), prefix_len int32 [G];
    the result equals decode() on the same rows up to rounding.
    """
    lib = _lib.load()
    dev = kv.device
    _need(q, "q", torch.bfloat16, dev)
    _need(kv_lens, "kv_lens", torch.int32, dev)
    _need(group_start, "group_start", torch.int32, dev)
    _need(prefix_len, "prefix_len", torch.int32, dev)
    B, Hq, D = q.shape
    _shape(q, (B, Hq, HEAD_DIM), "q")
    _shape(kv_lens, (B,), "kv_lens")
    ng = prefix_len.shape[0]
    _shape(group_start, (ng + 1,), "group_start")
    _rows(kv, B)
    if max_kv_len is None:
        max_kv_len = int(kv_lens.max().item()) if B else 0
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = _empty((B, Hq, D), torch.float32, dev, stream)
    _need(out, "out", torch.float32, dev)
    _shape(out, (B, Hq, HEAD_DIM), "out")
    if lse is None and want_lse:
        lse = _empty((B, Hq), torch.float32, dev, stream)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        _shape(lse, (B, Hq), "lse")
    if workspace is None:
        ws_bytes = lib.rollout_attn_decode_shared_prefix_workspace_size(
            B, Hq, kv.num_kv_heads, max_kv_len, max_prefix_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    s = kv.struct()
    _lib.check("rollout_attn_decode_shared_prefix", lib.rollout_attn_decode_shared_prefix(
        q.data_ptr(), ctypes.byref(s), kv_lens.data_ptr(), group_start.data_ptr(),
        prefix_len.data_ptr(), B, Hq, ng, max_group_rows, max_prefix_len, max_kv_len,
        float(scale), out.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel(),
        _stream(dev, stream)))
    return out, lse


def append(q: torch.Tensor, cu_q: torch.Tensor, ctx_lens: torch.Tensor, kv: PagedKV,
           max_q_len: Optional[int] = None, max_kv_len: Optional[int] = None,
           scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
           lse: Optional[torch.Tensor] = None, want_lse: bool = False,
           workspace: Optional[torch.Tensor] = None, stream=None
           ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Append attention; q bf16 [total_q][Hq][128] -> out fp32 [total_q][Hq][128]."""
    lib = _lib.load()
    dev = kv.device
    _need(q, "q", torch.bfloat16, dev)
    _need(cu_q, "cu_q", torch.int32, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, dev)
    total_q, Hq, D = q.shape
    _shape(q, (total_q, Hq, HEAD_DIM), "q")
    B = ctx_lens.shape[0]
    _shape(cu_q, (B + 1,), "cu_q")
    _rows(kv, B)
    if max_q_len is None or max_kv_len is None:
        t = (cu_q[1:] - cu_q[:-1]) if B else cu_q[:0]
        if max_q_len is None:
            max_q_len = int(t.max().item()) if B else 0
        if max_kv_len is None:
            max_kv_len = int((t + ctx_lens).max().item()) if B else 0
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = _empty((total_q, Hq, D), torch.float32, dev, stream)
    _need(out, "out", torch.float32, dev)
    _shape(out, (total_q, Hq, HEAD_DIM), "out")
    if lse is None and want_lse:
        lse = _empty((total_q, Hq), torch.float32, dev, stream)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        _shape(lse, (total_q, Hq), "lse")
    if workspace is None:
        ws_bytes = lib.rollout_attn_append_workspace_size(B, Hq, kv.num_kv_heads, max_q_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    s = kv.struct()
    _lib.check("rollout_attn_append", lib.rollout_attn_append(
        q.data_ptr(), cu_q.data_ptr(), ctx_lens.data_ptr(), ctypes.byref(s), B, Hq, total_q,
        max_q_len, max_kv_len, float(scale), out.data_ptr(), _ptr(lse), workspace.data_ptr(),
        workspace.numel(), _stream(dev, stream)))
    return out, lse


def append_write(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, cu_q: torch.Tensor,
                 ctx_lens: torch.Tensor, kv: PagedKV, max_q_len: Optional[int] = None,
                 max_kv_len: Optional[int] = None, scale: Optional[float] = None,
                 out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                 want_lse: bool = False, workspace: Optional[torch.Tensor] = None, stream=None,
                 cos_sin: Optional[torch.Tensor] = None
                 ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Write the chunks' K/V (bf16 [total_q][Hkv][128], packed like q) at positions
    ctx_lens[b] + i and run the append attention, in one launch. With a rotary table
    cos_sin (fp32 [rows][128]) the chunk's keys and queries are rotated at their
    positions."""
    lib = _lib.load()
    dev = kv.device
    for t, n in ((q, "q"), (k_new, "k_new"), (v_new, "v_new")):
        _need(t, n, torch.bfloat16, dev)
    _need(cu_q, "cu_q", torch.int32, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, dev)
    total_q, Hq, D = q.shape
    _shape(q, (total_q, Hq, HEAD_DIM), "q")
    _shape(k_new, (total_q, kv.num_kv_heads, HEAD_DIM), "k_new")
    _shape(v_new, (total_q, kv.num_kv_heads, HEAD_DIM), "v_new")
    B = ctx_lens.shape[0]
    _shape(cu_q, (B + 1,), "cu_q")
    _rows(kv, B)
    if max_q_len is None or max_kv_len is None:
        t = (cu_q[1:] - cu_q[:-1]) if B else cu_q[:0]
        if max_q_len is None:
            max_q_len = int(t.max().item()) if B else 0
        if max_kv_len is None:
            max_kv_len = int((t + ctx_lens).max().item()) if B else 0
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out is None:
        out = _empty((total_q, Hq, D), torch.float32, dev, stream)
    _need(out, "out", torch.float32, dev)
    _shape(out, (total_q, Hq, HEAD_DIM), "out")
    if lse is None and want_lse:
        lse = _empty((total_q, Hq), torch.float32, dev, stream)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        _shape(lse, (total_q, Hq), "lse")
    if workspace is None:
        ws_bytes = lib.rollout_attn_append_workspace_size(B, Hq, kv.num_kv_heads, max_q_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    s = kv.struct()
    if cos_sin is None:
        _lib.check("rollout_attn_append_write", lib.rollout_attn_append_write(
            q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), cu_q.data_ptr(),
            ctx_lens.data_ptr(), ctypes.byref(s), B, Hq, total_q, max_q_len, max_kv_len,
            float(scale), out.data_ptr(), _ptr(lse), workspace.data_ptr(), workspace.numel(),
            _stream(dev, stream)))
    else:
        rows = _rope_table(cos_sin, dev)
        _lib.check("rollout_attn_append_write_rope", lib.rollout_attn_append_write_rope(
            q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), cu_q.data_ptr(),
            ctx_lens.data_ptr(), ctypes.byref(s), B, Hq, total_q, max_q_len, max_kv_len,
            float(scale), cos_sin.data_ptr(), rows, out.data_ptr(), _ptr(lse),
            workspace.data_ptr(), workspace.numel(), _stream(dev, stream)))
    return out, lse


def append_workspace_size(B: int, Hq: int, Hkv: int, max_q_len: int) -> int:
    return int(_lib.load().rollout_attn_append_workspace_size(B, Hq, Hkv, max_q_len))


def mixed_workspace_size(B_decode: int, B_append: int, Hq: int, Hkv_decode: int,
                         Hkv_append: int, max_kv_len_decode: int, max_q_len: int) -> int:
    return int(_lib.load().rollout_attn_mixed_workspace_size(
        B_decode, B_append, Hq, Hkv_decode, Hkv_append, max_kv_len_decode, max_q_len))


def mixed(q_decode: torch.Tensor, kv_decode: PagedKV, kv_lens: torch.Tensor,
          q_append: torch.Tensor, cu_q: torch.Tensor, ctx_lens: torch.Tensor,
          kv_append: PagedKV, max_kv_len_decode: Optional[int] = None,
          max_q_len: Optional[int] = None, max_kv_len_append: Optional[int] = None,
          scale: Optional[float] = None, out_decode: Optional[torch.Tensor] = None,
          out_append: Optional[torch.Tensor] = None, want_lse: bool = False,
          workspace: Optional[torch.Tensor] = None, stream=None):
    """Decode rows and append rows of one step in one launch.

    q_decode bf16 [Bd][Hq][128] -> out_decode fp32 [Bd][Hq][128];
    q_append bf16 [total_q][Hq][128] -> out_append fp32 [total_q][Hq][128].
    Returns (out_decode, out_append, lse_decode, lse_append); the lse entries
    are None unless want_lse.
    """
    lib = _lib.load()
    dev = q_decode.device
    _need(q_decode, "q_decode", torch.bfloat16, dev)
    _need(kv_lens, "kv_lens", torch.int32, dev)
    _need(q_append, "q_append", torch.bfloat16, dev)
    _need(cu_q, "cu_q", torch.int32, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, dev)
    for kv in (kv_decode, kv_append):
        if kv.device != dev:
            raise ValueError(f"caches must be on {dev}, got {kv.device}")
    Bd, Hq, D = q_decode.shape
    total_q = q_append.shape[0]
    _shape(q_decode, (Bd, Hq, HEAD_DIM), "q_decode")
    _shape(q_append, (total_q, Hq, HEAD_DIM), "q_append")
    _shape(kv_lens, (Bd,), "kv_lens")
    Ba = ctx_lens.shape[0]
    _shape(cu_q, (Ba + 1,), "cu_q")
    _rows(kv_decode, Bd)
    _rows(kv_append, Ba)
    if max_kv_len_decode is None:
        max_kv_len_decode = int(kv_lens.max().item()) if Bd else 0
    if max_q_len is None or max_kv_len_append is None:
        t = (cu_q[1:] - cu_q[:-1]) if Ba else cu_q[:0]
        if max_q_len is None:
            max_q_len = int(t.max().item()) if Ba else 0
        if max_kv_len_append is None:
            max_kv_len_append = int((t + ctx_lens).max().item()) if Ba else 0
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    if out_decode is None:
        out_decode = _empty((Bd, Hq, D), torch.float32, dev, stream)
    if out_append is None:
        out_append = _empty((total_q, Hq, D), torch.float32, dev, stream)
    _need(out_decode, "out_decode", torch.float32, dev)
    _shape(out_decode, (Bd, Hq, HEAD_DIM), "out_decode")
    _need(out_append, "out_append", torch.float32, dev)
    _shape(out_append, (total_q, Hq, HEAD_DIM), "out_append")
    lse_d = _empty((Bd, Hq), torch.float32, dev, stream) if want_lse else None
    lse_a = _empty((total_q, Hq), torch.float32, dev, stream) if want_lse else None
    if workspace is None:
        ws_bytes = lib.rollout_attn_mixed_workspace_size(
            Bd, Ba, Hq, kv_decode.num_kv_heads, kv_append.num_kv_heads, max_kv_len_decode,
            max_q_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    sd, sa = kv_decode.struct(), kv_append.struct()
    _lib.check("rollout_attn_mixed", lib.rollout_attn_mixed(
        q_decode.data_ptr(), ctypes.byref(sd), kv_lens.data_ptr(), Bd, max_kv_len_decode,
        out_decode.data_ptr(), _ptr(lse_d), q_append.data_ptr(), cu_q.data_ptr(),
        ctx_lens.data_ptr(), ctypes.byref(sa), Ba, total_q, max_q_len, max_kv_len_append,
        out_append.data_ptr(), _ptr(lse_a), Hq, float(scale), workspace.data_ptr(),
        workspace.numel(), _stream(dev, stream)))
    return out_decode, out_append, lse_d, lse_a


def _rope_table(cos_sin: torch.Tensor, dev) -> int:
    """Checks a rotary table (fp32 [rows][128]: cos | sin) and returns its rows."""
    _need(cos_sin, "cos_sin", torch.float32, dev)
    if cos_sin.dim() != 2 or cos_sin.shape[1] != HEAD_DIM:
        raise ValueError(f"cos_sin must have shape [rows][{HEAD_DIM}], got {tuple(cos_sin.shape)}")
    return int(cos_sin.shape[0])


def kv_page_write(k_new: torch.Tensor, v_new: torch.Tensor, cu_new: torch.Tensor,
                  start_pos: torch.Tensor, kv: PagedKV, max_new: Optional[int] = None,
                  max_pos: Optional[int] = None, stream=None,
                  cos_sin: Optional[torch.Tensor] = None) -> None:
    """Scatter packed new tokens (bf16 [N][Hkv][128]) into the pages (a bit copy into
    bf16 pools, quantized to E4M3 codes in fp8 pools). With a rotary table cos_sin
    (fp32 [rows][128], cos | sin per position) the keys are rotated at their
    positions as they are written."""
    lib = _lib.load()
    dev = kv.device
    _need(k_new, "k_new", torch.bfloat16, dev)
    _need(v_new, "v_new", torch.bfloat16, dev)
    _need(cu_new, "cu_new", torch.int32, dev)
    _need(start_pos, "start_pos", torch.int32, dev)
    B = start_pos.shape[0]
    _shape(cu_new, (B + 1,), "cu_new")
    _shape(k_new, (k_new.shape[0], kv.num_kv_heads, HEAD_DIM), "k_new")
    _shape(v_new, tuple(k_new.shape), "v_new")
    _rows(kv, B)
    if max_new is None or max_pos is None:
        n = (cu_new[1:] - cu_new[:-1]) if B else cu_new[:0]
        if max_new is None:
            max_new = int(n.max().item()) if B else 0
        if max_pos is None:
            max_pos = int((n + start_pos).max().item()) if B else 0
    s = kv.struct()
    if cos_sin is None:
        _lib.check("kv_page_write", lib.kv_page_write(
            k_new.data_ptr(), v_new.data_ptr(), cu_new.data_ptr(), start_pos.data_ptr(),
            ctypes.byref(s), B, k_new.shape[0], max_new, max_pos, _stream(dev, stream)))
    else:
        rows = _rope_table(cos_sin, dev)
        _lib.check("kv_page_write_rope", lib.kv_page_write_rope(
            k_new.data_ptr(), v_new.data_ptr(), cu_new.data_ptr(), start_pos.data_ptr(),
            ctypes.byref(s), B, k_new.shape[0], max_new, max_pos, cos_sin.data_ptr(), rows,
            _stream(dev, stream)))


def kv_page_gather(kv: PagedKV, lens: torch.Tensor, cu_out: torch.Tensor,
                   total: Optional[int] = None, max_len: Optional[int] = None, stream=None
                   ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Copy logical tokens [0, lens[b]) of every row out to packed [total][Hkv][128]
    (bf16, or uint8 E4M3 codes for fp8 pools)."""
    lib = _lib.load()
    dev = kv.device
    _need(lens, "lens", torch.int32, dev)
    _need(cu_out, "cu_out", torch.int32, dev)
    B = lens.shape[0]
    _shape(cu_out, (B + 1,), "cu_out")
    _rows(kv, B)
    if total is None:
        total = int(cu_out[-1].item()) if B else 0
    if max_len is None:
        max_len = int(lens.max().item()) if B else 0
    k_out = _empty((total, kv.num_kv_heads, HEAD_DIM),
                   torch.uint8 if kv.fp8 else torch.bfloat16, dev, stream)
    v_out = _empty(tuple(k_out.shape), k_out.dtype, dev, stream)
    s = kv.struct()
    _lib.check("kv_page_gather", lib.kv_page_gather(
        ctypes.byref(s), lens.data_ptr(), cu_out.data_ptr(), B, total, max_len,
        k_out.data_ptr(), v_out.data_ptr(), _stream(dev, stream)))
    return k_out, v_out


def token_logprob_workspace_size(N: int, V: int, D: int) -> int:
    return int(_lib.load().token_logprob_workspace_size(N, V, D))


def _token_logprob(h, W, targets, scale, out, lse, want_lse, workspace, stream, packed_V):
    """Shared marshalling of token_logprob / token_logprob_packed (packed_V: V of a
    packed matrix, None for a row-major one)."""
    lib = _lib.load()
    dev = h.device
    _need(h, "h", torch.bfloat16, dev)
    _need(W, "W", torch.bfloat16, dev)
    _need(targets, "targets", torch.int32, dev)
    N, D = h.shape
    if packed_V is None:
        V = W.shape[0]
        _shape(W, (V, D), "W")
    else:
        V = int(packed_V)
        need = lib.token_logprob_packed_weight_size(V, D)
        if W.dim() != 1 or W.numel() * 2 < need:
            raise ValueError(f"W_packed: expected a flat bf16 tensor of {need // 2} elements "
                             f"for V={V}, D={D}, got {tuple(W.shape)}")
    _shape(targets, (N,), "targets")
    if out is None:
        out = _empty((N,), torch.float32, dev, stream)
    _need(out, "out", torch.float32, dev)
    _shape(out, (N,), "out")
    if lse is None and want_lse:
        lse = _empty((N,), torch.float32, dev, stream)
    if lse is not None:
        _need(lse, "lse", torch.float32, dev)
        _shape(lse, (N,), "lse")
    if workspace is None:
        workspace = _empty(max(lib.token_logprob_workspace_size(N, V, D), 1), torch.uint8, dev,
                           stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    fn = lib.token_logprob if packed_V is None else lib.token_logprob_packed
    name = "token_logprob" if packed_V is None else "token_logprob_packed"
    _lib.check(name, fn(
        h.data_ptr(), W.data_ptr(), targets.data_ptr(), N, V, D, float(scale), out.data_ptr(),
        _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream(dev, stream)))
    return out, lse


def token_logprob(h: torch.Tensor, W: torch.Tensor, targets: torch.Tensor, scale: float = 1.0,
                  out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                  want_lse: bool = False, workspace: Optional[torch.Tensor] = None, stream=None
                  ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Log-probability of targets[n] under logits scale * h[n] . W^T.

    h bf16 [N][D], W bf16 [V][D], targets int32 [N] -> logprob fp32 [N] (, lse fp32 [N]).
    """
    return _token_logprob(h, W, targets, scale, out, lse, want_lse, workspace, stream, None)


def token_logprob_pack_weight(W: torch.Tensor, out: Optional[torch.Tensor] = None,
                              stream=None) -> torch.Tensor:
    """Packed copy of the LM-head matrix W bf16 [V][D] for token_logprob_packed
    (a flat bf16 tensor; rows past V are zeros)."""
    lib = _lib.load()
    dev = W.device
    _need(W, "W", torch.bfloat16, dev)
    V, D = W.shape
    n = lib.token_logprob_packed_weight_size(V, D) // 2
    if out is None:
        out = _empty((max(n, 1),), torch.bfloat16, dev, stream)
    _need(out, "out", torch.bfloat16, dev)
    _lib.check("token_logprob_pack_weight", lib.token_logprob_pack_weight(
        W.data_ptr(), V, D, out.data_ptr(), out.numel() * 2, _stream(dev, stream)))
    return out


def token_logprob_packed(h: torch.Tensor, W_packed: torch.Tensor, V: int, targets: torch.Tensor,
                         scale: float = 1.0, out: Optional[torch.Tensor] = None,
                         lse: Optional[torch.Tensor] = None, want_lse: bool = False,
                         workspace: Optional[torch.Tensor] = None, stream=None
                         ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """token_logprob with the packed matrix from token_logprob_pack_weight (V rows)."""
    return _token_logprob(h, W_packed, targets, scale, out, lse, want_lse, workspace, stream, V)


def token_sample_workspace_size(N: int, V: int) -> int:
    return int(_lib.load().token_sample_workspace_size(N, V))


def _per_row(t: Optional[torch.Tensor], name: str, dtype: torch.dtype, N: int, dev) -> None:
    if t is not None:
        _need(t, name, dtype, dev)
        _shape(t, (N,), name)


def token_sample(logits: torch.Tensor, uniform: torch.Tensor,
                 temperature: Optional[torch.Tensor] = None, top_k: Optional[torch.Tensor] = None,
                 top_p: Optional[torch.Tensor] = None, min_p: Optional[torch.Tensor] = None,
                 tokens: Optional[torch.Tensor] = None, logprob: Optional[torch.Tensor] = None,
                 want_logprob: bool = False, workspace: Optional[torch.Tensor] = None, stream=None
                 ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """One token a row, drawn from logits (bf16 or fp32 [N][V], rows any stride >= V apart)
    by the rows' temperature, top-k, top-p and min-p (fp32 / int32 / fp32 / fp32 [N], None:
    off) at the given uniform numbers (fp32 [N] in [0, 1)).

    Returns tokens int32 [N] and, if wanted, logprob fp32 [N] under the distribution drawn
    from. temperature <= 0 is greedy; a row of nothing but -inf gives -1.
    """
    lib = _lib.load()
    dev = logits.device
    bf16 = logits.dtype == torch.bfloat16
    if logits.device.type != "cuda":
        raise ValueError(f"logits must be a GPU tensor, got one on {logits.device}")
    if not bf16 and logits.dtype != torch.float32:
        raise TypeError(f"logits must be torch.float32 or torch.bfloat16, got {logits.dtype}")
    if logits.dim() != 2:
        raise ValueError(f"logits must be [N][V], got {tuple(logits.shape)}")
    N, V = logits.shape
    row_stride = logits.stride(0) if N > 1 else V
    if (V > 1 and logits.stride(1) != 1) or row_stride < V:
        raise ValueError("logits must have contiguous rows that do not overlap, got strides "
                         f"{tuple(logits.stride())}")
    _need(uniform, "uniform", torch.float32, dev)
    _shape(uniform, (N,), "uniform")
    _per_row(temperature, "temperature", torch.float32, N, dev)
    _per_row(top_k, "top_k", torch.int32, N, dev)
    _per_row(top_p, "top_p", torch.float32, N, dev)
    _per_row(min_p, "min_p", torch.float32, N, dev)
    if tokens is None:
        tokens = _empty((N,), torch.int32, dev, stream)
    _per_row(tokens, "tokens", torch.int32, N, dev)
    if logprob is None and want_logprob:
        logprob = _empty((N,), torch.float32, dev, stream)
    _per_row(logprob, "logprob", torch.float32, N, dev)
    if workspace is None:
        workspace = _empty(max(lib.token_sample_workspace_size(N, V), 1), torch.uint8, dev, stream,
                           scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    _lib.check("token_sample", lib.token_sample(
        logits.data_ptr(), _lib.RA_LOGITS_BF16 if bf16 else _lib.RA_LOGITS_FP32, N, V, row_stride,
        _ptr(temperature), _ptr(top_k), _ptr(top_p), _ptr(min_p), uniform.data_ptr(),
        tokens.data_ptr(), _ptr(logprob), workspace.data_ptr(), workspace.numel(),
        _stream(dev, stream)))
    return tokens, logprob


def _linear_inputs(q, k_new, v_new, states, slots, log_decay):
    """Checks the tensors of the linear attention; returns (dev, total, Hq, Hkv)."""
    dev = q.device
    for t, n in ((q, "q"), (k_new, "k_new"), (v_new, "v_new")):
        _need(t, n, torch.bfloat16, dev)
    _need(states, "states", torch.float32, dev)
    _need(slots, "slots", torch.int32, dev)
    _need(log_decay, "log_decay", torch.float32, dev)
    total, Hq, _ = q.shape
    _shape(q, (total, Hq, HEAD_DIM), "q")
    if states.dim() != 4 or tuple(states.shape[2:]) != (HEAD_DIM, HEAD_DIM):
        raise ValueError(f"states must be [slots][Hkv][128][128], got {tuple(states.shape)}")
    Hkv = states.shape[1]
    _shape(k_new, (total, Hkv, HEAD_DIM), "k_new")
    _shape(v_new, (total, Hkv, HEAD_DIM), "v_new")
    _shape(log_decay, (Hkv,), "log_decay")
    return dev, total, Hq, Hkv


def linear_decode(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, states: torch.Tensor,
                  slots: torch.Tensor, kv_lens: torch.Tensor, log_decay: torch.Tensor,
                  scale: Optional[float] = None, out: Optional[torch.Tensor] = None, stream=None
                  ) -> torch.Tensor:
    """Linear attention of one token a row: states[slots[b]] (fp32 [slots][Hkv][128][128]) is
    decayed by exp(log_decay), takes k_new v_new^T (bf16 [B][Hkv][128]) and is read by q
    (bf16 [B][Hq][128]) -> out bf16 [B][Hq][128]. kv_lens counts the row's tokens with this
    one (1: the state before is zero; <= 0: nothing happens, out is zero)."""
    lib = _lib.load()
    dev, B, Hq, Hkv = _linear_inputs(q, k_new, v_new, states, slots, log_decay)
    _need(kv_lens, "kv_lens", torch.int32, dev)
    _shape(slots, (B,), "slots")
    _shape(kv_lens, (B,), "kv_lens")
    if scale is None:
        scale = 1.0 / math.sqrt(HEAD_DIM)
    if out is None:
        out = _empty((B, Hq, HEAD_DIM), torch.bfloat16, dev, stream)
    _need(out, "out", torch.bfloat16, dev)
    _shape(out, (B, Hq, HEAD_DIM), "out")
    _lib.check("rollout_linear_attn_decode", lib.rollout_linear_attn_decode(
        q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), states.data_ptr(), slots.data_ptr(),
        states.shape[0], kv_lens.data_ptr(), log_decay.data_ptr(), B, Hq, Hkv, float(scale),
        out.data_ptr(), _stream(dev, stream)))
    return out


def linear_append_workspace_size(B: int, Hq: int, Hkv: int, total_q: int, max_q_len: int) -> int:
    return int(_lib.load().rollout_linear_attn_append_workspace_size(B, Hq, Hkv, total_q,
                                                                     max_q_len))


def linear_append(q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor, cu_q: torch.Tensor,
                  ctx_lens: torch.Tensor, states: torch.Tensor, slots: torch.Tensor,
                  log_decay: torch.Tensor, max_q_len: Optional[int] = None,
                  scale: Optional[float] = None, out: Optional[torch.Tensor] = None,
                  workspace: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Linear attention of new tokens (packed by cu_q like append's) after ctx_lens earlier
    ones whose state is states[slots[b]]: q bf16 [total_q][Hq][128], k_new and v_new bf16
    [total_q][Hkv][128] -> out bf16 [total_q][Hq][128]; the states are updated in place."""
    lib = _lib.load()
    dev, total_q, Hq, Hkv = _linear_inputs(q, k_new, v_new, states, slots, log_decay)
    _need(cu_q, "cu_q", torch.int32, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, dev)
    B = ctx_lens.shape[0]
    _shape(ctx_lens, (B,), "ctx_lens")
    _shape(cu_q, (B + 1,), "cu_q")
    _shape(slots, (B,), "slots")
    if max_q_len is None:
        max_q_len = int((cu_q[1:] - cu_q[:-1]).max().item()) if B else 0
    if scale is None:
        scale = 1.0 / math.sqrt(HEAD_DIM)
    if out is None:
        out = _empty((total_q, Hq, HEAD_DIM), torch.bfloat16, dev, stream)
    _need(out, "out", torch.bfloat16, dev)
    _shape(out, (total_q, Hq, HEAD_DIM), "out")
    if workspace is None:
        ws_bytes = lib.rollout_linear_attn_append_workspace_size(B, Hq, Hkv, total_q, max_q_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    _lib.check("rollout_linear_attn_append", lib.rollout_linear_attn_append(
        q.data_ptr(), k_new.data_ptr(), v_new.data_ptr(), cu_q.data_ptr(), ctx_lens.data_ptr(),
        states.data_ptr(), slots.data_ptr(), states.shape[0], log_decay.data_ptr(), B, Hq, Hkv,
        total_q, max_q_len, float(scale), out.data_ptr(), workspace.data_ptr(), workspace.numel(),
        _stream(dev, stream)))
    return out


def _table_inputs(block_table, free_pages, free_count, rows, names, rows_of_table=True):
    """Checks the tensors of the block-table calls; returns (dev, B, bt_stride)."""
    dev = block_table.device
    _need(block_table, "block_table", torch.int32, dev)
    _need(free_pages, "free_pages", torch.int32, dev)
    _need(free_count, "free_count", torch.int32, dev)
    if block_table.dim() != 2:
        raise ValueError("block_table must be [B][stride]")
    _shape(free_pages, (free_pages.numel(),), "free_pages")
    _shape(free_count, (1,), "free_count")
    B = rows[0].shape[0]
    for t, n in zip(rows, names):
        _need(t, n, torch.int32, dev)
        _shape(t, (B,), n)
    if rows_of_table and block_table.shape[0] < B:
        raise ValueError(f"block_table has {block_table.shape[0]} rows, batch has {B}")
    return dev, B, block_table.shape[1]


def block_table_extend(block_table: torch.Tensor, start_pos: torch.Tensor, num_new: torch.Tensor,
                       free_pages: torch.Tensor, free_count: torch.Tensor,
                       total_new: Optional[int] = None, cu_new: Optional[torch.Tensor] = None,
                       kv_lens: Optional[torch.Tensor] = None,
                       slot_map: Optional[torch.Tensor] = None,
                       taken: Optional[torch.Tensor] = None, stream=None
                       ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """Takes the pages that num_new more tokens a row need (after start_pos earlier ones) off
    the end of the free list (free_pages[:free_count], int32) into block_table, in place.

    Returns (cu_new int32 [B+1], kv_lens int32 [B], slot_map int64 [total_new], taken int32
    [1]): the arguments of kv_page_write and decode, each new token's page * 16 + slot (-1
    behind the last), and the pages taken, -1 if the call was refused as a whole (the list
    too short, a row past its table, more than total_new tokens, a length out of range):
    then nothing changed and the outputs are those of no new token.
    """
    lib = _lib.load()
    dev, B, stride = _table_inputs(block_table, free_pages, free_count, (start_pos, num_new),
                                   ("start_pos", "num_new"))
    if total_new is None:
        # a sum below 0, or past all rows' tables, is the call's to refuse
        total_new = slot_map.shape[0] if slot_map is not None else \
            min(max(int(num_new.sum().item()), 0), B * stride * PAGE_SIZE, 2**31 - 1)
    if total_new >= 2**31:
        raise ValueError(f"total_new must be below 2^31, got {total_new}")
    if cu_new is None:
        cu_new = _empty((B + 1,), torch.int32, dev, stream)
    if kv_lens is None:
        kv_lens = _empty((B,), torch.int32, dev, stream)
    if slot_map is None:
        slot_map = _empty((max(total_new, 0),), torch.int64, dev, stream)
    if taken is None:
        taken = _empty((1,), torch.int32, dev, stream)
    for t, n, dt, size in ((cu_new, "cu_new", torch.int32, B + 1),
                           (kv_lens, "kv_lens", torch.int32, B),
                           (slot_map, "slot_map", torch.int64, max(total_new, 0)),
                           (taken, "taken", torch.int32, 1)):
        _need(t, n, dt, dev)
        _shape(t, (size,), n)
    _lib.check("kv_block_table_extend", lib.kv_block_table_extend(
        start_pos.data_ptr(), num_new.data_ptr(), free_pages.data_ptr(), free_count.data_ptr(),
        free_pages.numel(), block_table.data_ptr(), B, stride, total_new, cu_new.data_ptr(),
        kv_lens.data_ptr(), slot_map.data_ptr(), taken.data_ptr(), _stream(dev, stream)))
    return cu_new, kv_lens, slot_map, taken


def block_table_release(block_table: torch.Tensor, lens: torch.Tensor, keep_lens: torch.Tensor,
                        free_pages: torch.Tensor, free_count: torch.Tensor,
                        max_pages: Optional[int] = None, released: Optional[torch.Tensor] = None,
                        stream=None) -> torch.Tensor:
    """Puts the pages of tokens keep_lens .. lens - 1 of every row (whole pages only) back on
    the free list. Returns the pages given back (int32 [1]), -1 if the call was refused as a
    whole. max_pages: how many to expect (sizes the launch; default: the whole table)."""
    lib = _lib.load()
    dev, B, stride = _table_inputs(block_table, free_pages, free_count, (lens, keep_lens),
                                   ("lens", "keep_lens"))
    if max_pages is None:
        max_pages = min(B * stride, 2**31 - 1)
    if released is None:
        released = _empty((1,), torch.int32, dev, stream)
    _need(released, "released", torch.int32, dev)
    _shape(released, (1,), "released")
    _lib.check("kv_block_table_release", lib.kv_block_table_release(
        lens.data_ptr(), keep_lens.data_ptr(), block_table.data_ptr(), B, stride,
        free_pages.data_ptr(), free_count.data_ptr(), free_pages.numel(), max_pages,
        released.data_ptr(), _stream(dev, stream)))
    return released


def _nodes(cu_q: torch.Tensor, max_q_len: Optional[int]) -> int:
    """Nodes of the largest tree, read from the device where they are not given."""
    if max_q_len is not None:
        return max_q_len
    return int((cu_q[1:] - cu_q[:-1]).max().item()) if cu_q.shape[0] > 1 else 0


def _out(t: Optional[torch.Tensor], name: str, shape, dtype: torch.dtype, dev, stream
         ) -> torch.Tensor:
    """The output given, checked, or a new one."""
    if t is None:
        t = _empty(shape, dtype, dev, stream)
    _need(t, name, dtype, dev)
    _shape(t, shape, name)
    return t


def _draft_inputs(cu_q, ctx_lens, nodes):
    """Checks the tensors of the calls on drafted trees; returns (dev, B, total)."""
    dev = cu_q.device
    _need(cu_q, "cu_q", torch.int32, dev)
    B = cu_q.shape[0] - 1
    _shape(cu_q, (max(B, 0) + 1,), "cu_q")
    if ctx_lens is not None:
        _need(ctx_lens, "ctx_lens", torch.int32, dev)
        _shape(ctx_lens, (B,), "ctx_lens")
    total = nodes[0][0].shape[0]
    for t, n in nodes:
        _need(t, n, torch.int32, dev)
        _shape(t, (total,), n)
    return dev, B, total


def draft_tree_mask(parents: torch.Tensor, cu_q: torch.Tensor,
                    ctx_lens: Optional[torch.Tensor] = None, max_q_len: Optional[int] = None,
                    tree_mask: Optional[torch.Tensor] = None,
                    positions: Optional[torch.Tensor] = None, stream=None
                    ) -> Tuple[torch.Tensor, torch.Tensor]:
    """Masks and positions of drafted trees (row b's nodes packed at cu_q[b] .. cu_q[b+1]-1):
    parents int32 [total] (a node's parent in its row, before it; -1: none) -> tree_mask int64
    [total][words], bit j of word j / 64 for the node itself and its ancestors, and positions
    int32 [total], ctx_lens[b] + the node's depth (where the caller rotates its key and query, in a
    model that does; kv_page_write's cos_sin= rotates at the place in the pages). words: those of
    the tree_mask given, or as many as max_q_len nodes need."""
    lib = _lib.load()
    dev, B, total = _draft_inputs(cu_q, ctx_lens, ((parents, "parents"),))
    max_q_len = _nodes(cu_q, max_q_len)
    words = tree_mask.shape[1] if tree_mask is not None else max(1, (max_q_len + 63) // 64)
    tree_mask = _out(tree_mask, "tree_mask", (total, words), torch.int64, dev, stream)
    positions = _out(positions, "positions", (total,), torch.int32, dev, stream)
    _lib.check("draft_tree_mask", lib.draft_tree_mask(
        parents.data_ptr(), cu_q.data_ptr(), _ptr(ctx_lens), B, total, max_q_len, words,
        tree_mask.data_ptr(), positions.data_ptr(), _stream(dev, stream)))
    return tree_mask, positions


def draft_tree_accept(parents: torch.Tensor, draft_tokens: torch.Tensor, chosen: torch.Tensor,
                      cu_q: torch.Tensor, ctx_lens: torch.Tensor,
                      max_q_len: Optional[int] = None, path: Optional[torch.Tensor] = None,
                      tokens: Optional[torch.Tensor] = None,
                      accepted: Optional[torch.Tensor] = None,
                      kv_lens: Optional[torch.Tensor] = None,
                      next_tokens: Optional[torch.Tensor] = None, stream=None
                      ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor,
                                 torch.Tensor]:
    """The walk down each tree from its root, node 0, along the children that hold the token
    chosen at their parent (int32 [total]; draft_tokens likewise).

    Returns (path int32 [total]: row b's nodes on the walk from cu_q[b] on, then -1; tokens int32
    [total]: the tokens chosen at them, which the step emits; accepted int32 [B]: how many;
    kv_lens int32 [B]: ctx_lens + accepted; next_tokens int32 [B]: the last one, the next root).
    """
    lib = _lib.load()
    dev, B, total = _draft_inputs(cu_q, ctx_lens, ((parents, "parents"),
                                                   (draft_tokens, "draft_tokens"),
                                                   (chosen, "chosen")))
    max_q_len = _nodes(cu_q, max_q_len)
    path = _out(path, "path", (total,), torch.int32, dev, stream)
    tokens = _out(tokens, "tokens", (total,), torch.int32, dev, stream)
    accepted = _out(accepted, "accepted", (B,), torch.int32, dev, stream)
    kv_lens = _out(kv_lens, "kv_lens", (B,), torch.int32, dev, stream)
    next_tokens = _out(next_tokens, "next_tokens", (B,), torch.int32, dev, stream)
    _lib.check("draft_tree_accept", lib.draft_tree_accept(
        parents.data_ptr(), draft_tokens.data_ptr(), chosen.data_ptr(), cu_q.data_ptr(),
        ctx_lens.data_ptr(), B, total, max_q_len, path.data_ptr(), tokens.data_ptr(),
        accepted.data_ptr(), kv_lens.data_ptr(), next_tokens.data_ptr(), _stream(dev, stream)))
    return path, tokens, accepted, kv_lens, next_tokens


def decode_tree_workspace_size(B: int, Hq: int, Hkv: int, total_q: int, max_q_len: int,
                               max_kv_len: int) -> int:
    return int(_lib.load().rollout_attn_decode_tree_workspace_size(B, Hq, Hkv, total_q, max_q_len,
                                                                   max_kv_len))


def decode_tree_max_workspace_size(B: int, Hq: int, Hkv: int, max_q_len: int,
                                   max_kv_len: int) -> int:
    """Bytes that are enough for every decode_tree call of up to B rows, max_q_len nodes a row and
    max_kv_len keys: decode_tree_workspace_size of a call can be less than that of a smaller one."""
    return int(_lib.load().rollout_attn_decode_tree_max_workspace_size(B, Hq, Hkv, max_q_len,
                                                                       max_kv_len))


def decode_tree(q: torch.Tensor, cu_q: torch.Tensor, ctx_lens: torch.Tensor,
                tree_mask: torch.Tensor, kv: PagedKV, max_q_len: Optional[int] = None,
                max_kv_len: Optional[int] = None, scale: Optional[float] = None,
                out: Optional[torch.Tensor] = None, lse: Optional[torch.Tensor] = None,
                want_lse: bool = False, workspace: Optional[torch.Tensor] = None, stream=None
                ) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """Attention of drafted trees: node i of row b (q bf16 [total_q][Hq][128], packed by cu_q;
    its key and value in the pages at ctx_lens[b] + i) over the row's ctx_lens[b] cached tokens
    and over the nodes j of its row whose bit is set in its tree_mask (int64 [total_q][words])
    -> out fp32 [total_q][Hq][128] (, lse fp32 [total_q][Hq])."""
    lib = _lib.load()
    dev = kv.device
    _need(q, "q", torch.bfloat16, dev)
    _need(cu_q, "cu_q", torch.int32, dev)
    _need(ctx_lens, "ctx_lens", torch.int32, dev)
    _need(tree_mask, "tree_mask", torch.int64, dev)
    total_q, Hq, D = q.shape
    _shape(q, (total_q, Hq, HEAD_DIM), "q")
    B = ctx_lens.shape[0]
    _shape(ctx_lens, (B,), "ctx_lens")
    _shape(cu_q, (B + 1,), "cu_q")
    if tree_mask.dim() != 2:
        raise ValueError(f"tree_mask must be [total_q][words], got {tuple(tree_mask.shape)}")
    words = tree_mask.shape[1]
    _shape(tree_mask, (total_q, words), "tree_mask")
    _rows(kv, B)
    max_q_len = _nodes(cu_q, max_q_len)
    if max_kv_len is None:
        max_kv_len = int((cu_q[1:] - cu_q[:-1] + ctx_lens).max().item()) if B else 0
    if scale is None:
        scale = 1.0 / math.sqrt(D)
    out = _out(out, "out", (total_q, Hq, HEAD_DIM), torch.float32, dev, stream)
    if lse is not None or want_lse:
        lse = _out(lse, "lse", (total_q, Hq), torch.float32, dev, stream)
    if workspace is None:
        ws_bytes = lib.rollout_attn_decode_tree_workspace_size(B, Hq, kv.num_kv_heads, total_q,
                                                               max_q_len, max_kv_len)
        workspace = _empty(max(ws_bytes, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    s = kv.struct()
    _lib.check("rollout_attn_decode_tree", lib.rollout_attn_decode_tree(
        q.data_ptr(), cu_q.data_ptr(), ctx_lens.data_ptr(), tree_mask.data_ptr(), words,
        ctypes.byref(s), B, Hq, total_q, max_q_len, max_kv_len, float(scale), out.data_ptr(),
        _ptr(lse), workspace.data_ptr(), workspace.numel(), _stream(dev, stream)))
    return out, lse


def _strided_rows(t: torch.Tensor, name: str, dev) -> int:
    """Elements between the rows of a matrix whose rows are contiguous and do not overlap."""
    if t.device.type != "cuda":
        raise ValueError(f"{name} must be a GPU tensor, got one on {t.device}")
    if t.device != dev:
        raise ValueError(f"{name} must be on {dev}, got {t.device}")
    if t.dim() != 2:
        raise ValueError(f"{name} must be a matrix, got {tuple(t.shape)}")
    n, w = t.shape
    stride = t.stride(0) if n > 1 else w
    if (w > 1 and t.stride(1) != 1) or stride < w:
        raise ValueError(f"{name} must have contiguous rows that do not overlap, got strides "
                         f"{tuple(t.stride())}")
    return stride


def token_logits_adjust(logits: torch.Tensor, history: Optional[torch.Tensor] = None,
                        history_lens: Optional[torch.Tensor] = None,
                        prompt_lens: Optional[torch.Tensor] = None,
                        repetition: Optional[torch.Tensor] = None,
                        frequency: Optional[torch.Tensor] = None,
                        presence: Optional[torch.Tensor] = None,
                        bias_tokens: Optional[torch.Tensor] = None,
                        bias_values: Optional[torch.Tensor] = None,
                        cu_bias: Optional[torch.Tensor] = None,
                        allowed: Optional[torch.Tensor] = None,
                        allowed_rows: Optional[torch.Tensor] = None,
                        cu_rows: Optional[torch.Tensor] = None,
                        draft_tokens: Optional[torch.Tensor] = None,
                        tree_mask: Optional[torch.Tensor] = None,
                        out: Optional[torch.Tensor] = None, stream=None) -> torch.Tensor:
    """Logits (bf16 or fp32 [N][V], rows any stride >= V apart) with penalties, biases and masks
    applied, for token_sample; out=logits works in place.

    history int32 [B][longest] with history_lens tokens a row, the first prompt_lens (None: 0) of
    them the prompt: tokens in it are divided by (or, below 0, multiplied with) repetition,
    those behind the prompt also lose frequency times their count, and presence (fp32 [B]).
    bias_tokens int32 / bias_values fp32 packed by cu_bias int32 [B+1] are added (a token's last
    entry). allowed int32 [M][>= ceil(V / 32)] holds masks of bits, allowed_rows int32 [N] a
    row's mask (outside [0, M): none; None: mask n): tokens whose bit is clear become -inf.
    Row n of the logits has history row n, or with cu_rows int32 [B+1] the b with cu_rows[b] <=
    n < cu_rows[b+1]; draft_tokens int32 [N] and tree_mask int64 [N][words] then add the drafted
    tokens of the nodes in row n's mask to its history. The root's token is one of them: history
    ends before it (history_lens = the step's ctx_lens), or it counts twice.
    """
    lib = _lib.load()
    dev = logits.device
    bf16 = logits.dtype == torch.bfloat16
    row_stride = _strided_rows(logits, "logits", dev)
    if not bf16 and logits.dtype != torch.float32:
        raise TypeError(f"logits must be torch.float32 or torch.bfloat16, got {logits.dtype}")
    N, V = logits.shape
    B = N if cu_rows is None else cu_rows.shape[0] - 1
    a = _lib.RaLogitsAdjust()

    def give(name, t, dtype, shape):
        if t is not None:
            _need(t, name, dtype, dev)
            _shape(t, shape, name)
            setattr(a, name, t.data_ptr())
    if (history is None) != (history_lens is None):
        raise ValueError("history and history_lens go together")
    if history is not None:
        a.history_stride = _strided_rows(history, "history", dev)
        if history.dtype != torch.int32:
            raise TypeError(f"history must be torch.int32, got {history.dtype}")
        _shape(history, (B, history.shape[1]), "history")
        a.history_width = history.shape[1]
        a.history = history.data_ptr()
    give("history_lens", history_lens, torch.int32, (B,))
    give("prompt_lens", prompt_lens, torch.int32, (B,))
    give("repetition", repetition, torch.float32, (B,))
    give("frequency", frequency, torch.float32, (B,))
    give("presence", presence, torch.float32, (B,))
    if bias_tokens is not None:
        if bias_values is None or cu_bias is None:
            raise ValueError("bias_tokens need bias_values and cu_bias")
        give("bias_tokens", bias_tokens, torch.int32, (bias_tokens.numel(),))
        a.num_bias = bias_tokens.numel()
        give("bias_values", bias_values, torch.float32, (bias_tokens.numel(),))
        give("cu_bias", cu_bias, torch.int32, (B + 1,))
    elif bias_values is not None or cu_bias is not None:
        raise ValueError("bias_values and cu_bias need bias_tokens")
    if allowed is not None:
        a.allowed_stride = _strided_rows(allowed, "allowed", dev)
        if allowed.dtype != torch.int32:
            raise TypeError(f"allowed must be torch.int32, got {allowed.dtype}")
        a.num_allowed = allowed.shape[0]
        if allowed.shape[1] * 32 < V:
            raise ValueError(f"allowed has {allowed.shape[1]} words a row, {V} logits need "
                             f"{(V + 31) // 32}")
        a.allowed = allowed.data_ptr()
    elif allowed_rows is not None:
        raise ValueError("allowed_rows need allowed")
    give("allowed_rows", allowed_rows, torch.int32, (N,))
    give("cu_rows", cu_rows, torch.int32, (max(B, 0) + 1,))
    if (draft_tokens is None) != (tree_mask is None):
        raise ValueError("draft_tokens and tree_mask go together")
    if draft_tokens is not None:
        if cu_rows is None:
            raise ValueError("draft_tokens need cu_rows")
        give("draft_tokens", draft_tokens, torch.int32, (N,))
        if tree_mask.dim() != 2:
            raise ValueError(f"tree_mask must be [N][words], got {tuple(tree_mask.shape)}")
        a.mask_words = tree_mask.shape[1]
        give("tree_mask", tree_mask, torch.int64, (N, a.mask_words))
    if out is None:
        out = _empty((N, V), logits.dtype, dev, stream)
    out_stride = _strided_rows(out, "out", dev)
    if out.dtype != logits.dtype:
        raise TypeError(f"out must be {logits.dtype}, got {out.dtype}")
    _shape(out, (N, V), "out")
    _lib.check("token_logits_adjust", lib.token_logits_adjust(
        logits.data_ptr(), _lib.RA_LOGITS_BF16 if bf16 else _lib.RA_LOGITS_FP32, N, V, row_stride,
        ctypes.byref(a), B, out.data_ptr(), out_stride, _stream(dev, stream)))
    return out


def block_table_fork(block_table: torch.Tensor, src_rows: torch.Tensor, dst_rows: torch.Tensor,
                     lens: torch.Tensor, shares: torch.Tensor, free_pages: torch.Tensor,
                     free_count: torch.Tensor, copy_src: Optional[torch.Tensor] = None,
                     copy_dst: Optional[torch.Tensor] = None,
                     taken: Optional[torch.Tensor] = None, stream=None
                     ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """Gives row dst_rows[i] of the table the first lens[i] tokens of row src_rows[i] (int32
    [n]): whole pages are shared (shares int32 [num_pages] counts a page's rows beyond the
    first), a partly filled last one comes off the free list.

    Returns (copy_src, copy_dst int32 [n]: the pages for kv_page_copy, -1 where there is none;
    taken int32 [1]: pages taken, -1 if the call was refused as a whole)."""
    lib = _lib.load()
    dev, n, stride = _table_inputs(block_table, free_pages, free_count,
                                   (src_rows, dst_rows, lens), ("src_rows", "dst_rows", "lens"),
                                   rows_of_table=False)
    _need(shares, "shares", torch.int32, dev)
    _shape(shares, (shares.numel(),), "shares")
    copy_src = _out(copy_src, "copy_src", (n,), torch.int32, dev, stream)
    copy_dst = _out(copy_dst, "copy_dst", (n,), torch.int32, dev, stream)
    taken = _out(taken, "taken", (1,), torch.int32, dev, stream)
    _lib.check("kv_block_table_fork", lib.kv_block_table_fork(
        src_rows.data_ptr(), dst_rows.data_ptr(), lens.data_ptr(), n, block_table.data_ptr(),
        block_table.shape[0], stride, shares.data_ptr(), shares.numel(), free_pages.data_ptr(),
        free_count.data_ptr(), free_pages.numel(), copy_src.data_ptr(), copy_dst.data_ptr(),
        taken.data_ptr(), _stream(dev, stream)))
    return copy_src, copy_dst, taken


def block_table_release_shared_workspace_size(B: int) -> int:
    return int(_lib.load().kv_block_table_release_shared_workspace_size(B))


def block_table_release_shared(block_table: torch.Tensor, lens: torch.Tensor,
                               keep_lens: torch.Tensor, shares: torch.Tensor,
                               free_pages: torch.Tensor, free_count: torch.Tensor,
                               released: Optional[torch.Tensor] = None,
                               workspace: Optional[torch.Tensor] = None, stream=None
                               ) -> torch.Tensor:
    """block_table_release for rows that share pages: a page goes back on the free list (which
    has room for all pages) when its last holder gives it up. Returns the pages put there
    (int32 [1]), -1 if the call was refused as a whole."""
    lib = _lib.load()
    dev, B, stride = _table_inputs(block_table, free_pages, free_count, (lens, keep_lens),
                                   ("lens", "keep_lens"))
    _need(shares, "shares", torch.int32, dev)
    _shape(shares, (shares.numel(),), "shares")
    released = _out(released, "released", (1,), torch.int32, dev, stream)
    if workspace is None:
        size = lib.kv_block_table_release_shared_workspace_size(B)
        workspace = _empty(max(size, 1), torch.uint8, dev, stream, scratch=True)
    _need(workspace, "workspace", torch.uint8, dev)
    _lib.check("kv_block_table_release_shared", lib.kv_block_table_release_shared(
        lens.data_ptr(), keep_lens.data_ptr(), block_table.data_ptr(), B, stride,
        shares.data_ptr(), shares.numel(), free_pages.data_ptr(), free_count.data_ptr(),
        free_pages.numel(), released.data_ptr(), workspace.data_ptr(), workspace.numel(),
        _stream(dev, stream)))
    return released


def kv_page_copy(kv: PagedKV, src_pages: torch.Tensor, dst_pages: torch.Tensor,
                 stream=None) -> None:
    """Copies pages src_pages[i] to dst_pages[i] (int32 [n]) of both pools; pairs that name no
    page (-1) are passed over."""
    lib = _lib.load()
    dev = kv.device
    n = src_pages.shape[0]
    for t, name in ((src_pages, "src_pages"), (dst_pages, "dst_pages")):
        _need(t, name, torch.int32, dev)
        _shape(t, (n,), name)
    s = kv.struct()
    _lib.check("kv_page_copy", lib.kv_page_copy(
        ctypes.byref(s), src_pages.data_ptr(), dst_pages.data_ptr(), n, _stream(dev, stream)))


def kv_page_compact(kv: PagedKV, start_pos: torch.Tensor, cu_src: torch.Tensor,
                    src_index: torch.Tensor, counts: Optional[torch.Tensor] = None,
                    max_count: Optional[int] = None, stream=None) -> None:
    """Moves row b's tokens start_pos[b] + src_index[cu_src[b] + i] to start_pos[b] + i, for i <
    counts[b] (None: all of the row's entries); a row's indices ascend. The accepted path of a
    tree: src_index = path, counts = accepted, cu_src = cu_q, start_pos = ctx_lens."""
    lib = _lib.load()
    dev = kv.device
    B = start_pos.shape[0]
    _need(start_pos, "start_pos", torch.int32, dev)
    _shape(start_pos, (B,), "start_pos")
    _need(cu_src, "cu_src", torch.int32, dev)
    _shape(cu_src, (B + 1,), "cu_src")
    _need(src_index, "src_index", torch.int32, dev)
    _shape(src_index, (src_index.numel(),), "src_index")
    _per_row(counts, "counts", torch.int32, B, dev)
    _rows(kv, B)
    if max_count is None:
        max_count = src_index.numel()
    s = kv.struct()
    _lib.check("kv_page_compact", lib.kv_page_compact(
        ctypes.byref(s), start_pos.data_ptr(), cu_src.data_ptr(), src_index.data_ptr(),
        _ptr(counts), B, src_index.numel(), max_count, _stream(dev, stream)))
