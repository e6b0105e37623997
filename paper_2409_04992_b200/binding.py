"""Thin ctypes layer over libinstinfer.so: argument marshalling only.

Function names mirror the C ABI (see include/instinfer.h for what each argument means).
Tensors are torch CUDA tensors used as device memory; every step of the path runs in the
library's kernels.  There is no fallback: if the library has not been built, loading fails.
"""
from __future__ import annotations

import array
import ctypes
import os
from pathlib import Path
from typing import Optional, Sequence, Tuple, Union

import torch

# INSTINFER_LIBRARY selects another build of the same library (the bounds-checking one, say).
LIBRARY = Path(os.environ.get("INSTINFER_LIBRARY") or Path(__file__).resolve().parent / "libinstinfer.so")

OK, ERR_INVALID_ARG, ERR_UNSUPPORTED, ERR_WORKSPACE, ERR_CUDA = range(5)
FLAG_SEQ_LEN_RANGE, FLAG_BLOCK_RANGE, FLAG_COPY_TIMEOUT, FLAG_BOUNDS_CHECK = 1, 2, 4, 8
FLAG_TREE_RANGE, FLAG_POOL, FLAG_TOKEN_RANGE = 16, 32, 64
MAX_VOCAB, MAX_BIAS = 262144, 256
MAX_TREE_TOKENS, MAX_TREE_ROWS, MAX_LAYERS, MAX_LATENT_ROWS = 128, 4096, 128, 16384
ROPE_SCALINGS = {"plain": 0, "linear": 1, "by_parts": 2}
STATIC_WORKSPACE_BYTES = 16 << 20

_lib: Optional[ctypes.CDLL] = None


class InstInferError(RuntimeError):
    def __init__(self, status: int):
        super().__init__(f"instinfer status {status}: {status_string(status)}")
        self.status = status


def load() -> ctypes.CDLL:
    """dlopen the CUDA library; raises if it is missing (build it with paper_2409_04992_b200.build)."""
    global _lib
    if _lib is None:
        if not LIBRARY.exists():
            raise RuntimeError(f"{LIBRARY} is missing: run `python -m paper_2409_04992_b200.build` "
                               "(there is no CPU or PyTorch fallback)")
        lib = ctypes.CDLL(str(LIBRARY))
        i32, i64, ptr, f32, sz = (ctypes.c_int32, ctypes.c_int64, ctypes.c_void_p,
                                  ctypes.c_float, ctypes.c_size_t)
        lib.instinfer_kv_append.restype = ctypes.c_int
        lib.instinfer_kv_append.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i64,
                                            i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_kv_append_bulk.restype = ctypes.c_int
        lib.instinfer_kv_append_bulk.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i64,
                                                 i32, i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_decode_attention.restype = ctypes.c_int
        lib.instinfer_decode_attention.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i32,
                                                   i32, i32, f32, ptr, sz, ptr, ptr]
        lib.instinfer_decode_attention_paged.restype = ctypes.c_int
        lib.instinfer_decode_attention_paged.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                         i32, i32, i32, i32, i32, i64, i32, f32,
                                                         ptr, sz, ptr, ptr]
        lib.instinfer_decode_attention_static.restype = ctypes.c_int
        lib.instinfer_decode_attention_static.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                          i32, i32, i32, i32, i32, i32, i64, i32,
                                                          f32, ptr, ptr]
        lib.instinfer_decode_attention_allgather.restype = ctypes.c_int
        lib.instinfer_decode_attention_allgather.argtypes = [ptr, i32, ptr, ptr, ptr, ptr, ptr, ptr,
                                                             i32, i32, i32, i32, i32, i32, i32, i32,
                                                             i64, i32, f32, ptr, sz, ptr, ptr]
        lib.instinfer_allgather_workspace_bytes.restype = sz
        lib.instinfer_allgather_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.instinfer_decode_attention_grouped.restype = ctypes.c_int
        lib.instinfer_decode_attention_grouped.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                           i32, i32, i32, i32, i32, i32, i32, i32,
                                                           i64, i32, f32, ptr, sz, ptr, ptr]
        lib.instinfer_grouped_workspace_bytes.restype = sz
        lib.instinfer_grouped_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
        lib.instinfer_tree_mask.restype = ctypes.c_int
        lib.instinfer_tree_mask.argtypes = [ptr, ptr, ptr, i32, i32, ptr, ptr]
        lib.instinfer_decode_attention_tree.restype = ctypes.c_int
        lib.instinfer_decode_attention_tree.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                        i32, i32, i32, i32, i32, i32, i32, i32,
                                                        i64, i32, f32, ptr, sz, ptr, ptr]
        lib.instinfer_tree_workspace_bytes.restype = sz
        lib.instinfer_tree_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
        lib.instinfer_verify_tree.restype = ctypes.c_int
        lib.instinfer_verify_tree.argtypes = [ptr, ptr, ptr, ptr, ptr, i32, i64, ptr, ptr, ptr, ptr,
                                              i32, i32, i32, ptr, ptr]
        lib.instinfer_kv_keep_path.restype = ctypes.c_int
        lib.instinfer_kv_keep_path.argtypes = [ptr, ptr, i32, ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i64,
                                               i32, i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_kv_fork.restype = ctypes.c_int
        lib.instinfer_kv_fork.argtypes = [ptr, ptr, ptr, ptr, ptr, i32, i32, i32, i64, i32, ptr, ptr]
        lib.instinfer_kv_resize.restype = ctypes.c_int
        lib.instinfer_kv_resize.argtypes = [ptr, ptr, i32, ptr, ptr, ptr, ptr, ptr, i32, i32, i64, i32, i32,
                                            i32, ptr, sz, ptr, ptr]
        lib.instinfer_kv_resize_workspace_bytes.restype = sz
        lib.instinfer_kv_resize_workspace_bytes.argtypes = [i32, i64]
        lib.instinfer_kv_defragment.restype = ctypes.c_int
        lib.instinfer_kv_defragment.argtypes = [ptr, ptr, i32, ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i64,
                                                i32, i32, i32, ptr, sz, ptr, ptr]
        lib.instinfer_kv_defragment_workspace_bytes.restype = sz
        lib.instinfer_kv_defragment_workspace_bytes.argtypes = [i64]
        f64 = ctypes.c_double
        lib.instinfer_rope_frequencies.restype = ctypes.c_int
        lib.instinfer_rope_frequencies.argtypes = [ptr, ptr, i32, f64, i32, f64, i32, f64, f64]
        lib.instinfer_rope_append.restype = ctypes.c_int
        lib.instinfer_rope_append.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, i32, i64, i64, i64, ptr, i32, i32, f32, ptr, ptr, ptr, ptr,
                                              i32, i32, i64, i32, i32, i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_latent_append.restype = ctypes.c_int
        lib.instinfer_latent_append.argtypes = [ptr, ptr, ptr, ptr, ptr, i32, i64, i64, i64, i64, ptr, i32, f32, ptr, ptr, ptr, ptr,
                                                i32, i32, i64, i32, i32, i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_decode_attention_latent.restype = ctypes.c_int
        lib.instinfer_decode_attention_latent.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i32, i32, i32, i32, i32,
                                                          i32, i32, i64, i32, f32, ptr, sz, ptr, ptr]
        lib.instinfer_latent_workspace_bytes.restype = sz
        lib.instinfer_latent_workspace_bytes.argtypes = [i32, i32, i32, i32, i32, i32]
        lib.instinfer_process_logits.restype = ctypes.c_int
        lib.instinfer_process_logits.argtypes = [ptr, i32, i64, ptr, i32, i64, ptr, ptr, ptr, i32, ptr, ptr, ptr, ptr, ptr, ptr, i32, ptr,
                                                 ptr, i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_decode_step_host.restype = ctypes.c_int
        lib.instinfer_decode_step_host.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                   i32, i32, i64, i32, i32, i32, i32, i32, f32,
                                                   ptr, sz, ptr, ptr]
        lib.instinfer_decode_step_host_overlapped.restype = ctypes.c_int
        lib.instinfer_decode_step_host_overlapped.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                              i32, i32, i64, i32, i32, i32, i32, i32, f32,
                                                              ptr, sz, ptr, ptr, ptr, ptr, ptr, ptr]
        lib.instinfer_sparf_append.restype = ctypes.c_int
        lib.instinfer_sparf_append.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, i32, i32, i64,
                                               ptr, i32, i32, i64, i32, i32, i32, ptr, ptr]
        lib.instinfer_sparf_append_bulk.restype = ctypes.c_int
        lib.instinfer_sparf_append_bulk.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, i32, i32,
                                                    i64, ptr, i32, i32, i64, i32, i32, i32, i32, ptr, ptr]
        lib.instinfer_sparf_decode_attention.restype = ctypes.c_int
        lib.instinfer_sparf_decode_attention.argtypes = [ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr, ptr,
                                                         ptr, ptr, i32, i32, i32, i32, i32, i64,
                                                         ptr, i32, i32, i64,
                                                         i32, i32, i32, i32, f32, ptr, sz, ptr, ptr]
        lib.instinfer_set_sparse_path.restype = ctypes.c_int
        lib.instinfer_set_sparse_path.argtypes = [i32]
        lib.instinfer_set_grouped_path.restype = ctypes.c_int
        lib.instinfer_set_grouped_path.argtypes = [i32]
        lib.instinfer_grouped_path_for.restype = i32
        lib.instinfer_grouped_path_for.argtypes = [i32, i32]
        lib.instinfer_sparf_workspace_bytes.restype = sz
        lib.instinfer_sparf_workspace_bytes.argtypes = [i32, i32, i32, i32, i32]
        lib.instinfer_workspace_bytes.restype = sz
        lib.instinfer_workspace_bytes.argtypes = [i32, i32, i32, i32]
        lib.instinfer_plan_chunk_tokens.restype = i32
        lib.instinfer_plan_chunk_tokens.argtypes = [i32, i32, i32]
        lib.instinfer_plan_num_splits.restype = i32
        lib.instinfer_plan_num_splits.argtypes = [i32, i32, i32]
        lib.instinfer_plan_merges_in_cluster.restype = i32
        lib.instinfer_plan_merges_in_cluster.argtypes = [i32, i32, i32]
        lib.instinfer_set_chunk_tokens.restype = ctypes.c_int
        lib.instinfer_set_chunk_tokens.argtypes = [i32]
        lib.instinfer_set_timing_events.restype = ctypes.c_int
        lib.instinfer_set_timing_events.argtypes = [ptr, ptr]
        lib.instinfer_status_string.restype = ctypes.c_char_p
        lib.instinfer_status_string.argtypes = [ctypes.c_int]
        _lib = lib
    return _lib


def _ptr(t: Optional[torch.Tensor]) -> Optional[int]:
    return None if t is None else t.data_ptr()


def _stream(stream: Optional[torch.cuda.Stream], device: Optional[int] = None) -> Optional[int]:
    if stream is not None:
        return stream.cuda_stream or None
    # (the raw handle: a Stream object per call costs as much as a short kernel)
    return torch._C._cuda_getCurrentRawStream(torch.cuda.current_device() if device is None else device) or None


def _here(*tensors: Optional[torch.Tensor]) -> int:
    """The current device, whose stream the call goes to; refuses tensors of another one (None: not given)."""
    # (the raw query, as in _stream: a microsecond less per call; -1 for tensors of the host)
    device = torch._C._cuda_getDevice()
    if {t.get_device() for t in tensors if t is not None} != {device}:
        raise InstInferError(ERR_INVALID_ARG)
    return device


def _check(status: int) -> None:
    if status != OK:
        raise InstInferError(status)


def status_string(status: int) -> str:
    return load().instinfer_status_string(int(status)).decode()


def workspace_bytes(batch: int, heads: int, head_dim: int, max_seq_len: int) -> int:
    return int(load().instinfer_workspace_bytes(batch, heads, head_dim, max_seq_len))


def plan_chunk_tokens(batch: int, heads: int, max_seq_len: int) -> int:
    return int(load().instinfer_plan_chunk_tokens(batch, heads, max_seq_len))


def plan_num_splits(batch: int, heads: int, max_seq_len: int) -> int:
    return int(load().instinfer_plan_num_splits(batch, heads, max_seq_len))


def plan_merges_in_cluster(batch: int, heads: int, max_seq_len: int) -> bool:
    return bool(load().instinfer_plan_merges_in_cluster(batch, heads, max_seq_len))


def set_chunk_tokens(chunk_tokens: int) -> None:
    _check(load().instinfer_set_chunk_tokens(int(chunk_tokens)))


def set_timing_events(before_split: Optional[torch.cuda.Event],
                      after_split: Optional[torch.cuda.Event]) -> None:
    """instinfer_set_timing_events with torch events (already created, i.e. recorded once)."""
    _check(load().instinfer_set_timing_events(
        None if before_split is None else before_split.cuda_event,
        None if after_split is None else after_split.cuda_event))


def kv_append(k_cache: torch.Tensor, v_cache: torch.Tensor, k_new: torch.Tensor,
              v_new: torch.Tensor, seq_lens: torch.Tensor,
              block_table: Optional[torch.Tensor] = None,
              status_flags: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_kv_append.  Caches: [B,H,s_max,D] (block_table None) or pools [P,H,T,D]."""
    batch, heads, head_dim = k_new.shape
    if block_table is None:
        max_blocks, block_tokens, phys, s_max = 0, 0, 0, k_cache.shape[2]
    else:
        max_blocks, block_tokens, phys, s_max = (block_table.shape[1], k_cache.shape[2],
                                                 k_cache.shape[0], 0)
    _check(load().instinfer_kv_append(
        _ptr(k_cache), _ptr(v_cache), _ptr(k_new), _ptr(v_new), _ptr(seq_lens),
        _ptr(block_table), max_blocks, block_tokens, phys, batch, heads, head_dim, s_max,
        _ptr(status_flags), _stream(stream)))


def kv_append_bulk(k_cache: torch.Tensor, v_cache: torch.Tensor, k_new: torch.Tensor,
                   v_new: torch.Tensor, seq_lens: torch.Tensor, new_lens: torch.Tensor,
                   block_table: Optional[torch.Tensor] = None,
                   status_flags: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_kv_append_bulk: k_new, v_new are [B, max_new, H, D] (token-major)."""
    batch, max_new, heads, head_dim = k_new.shape
    if block_table is None:
        max_blocks, block_tokens, phys, s_max = 0, 0, 0, k_cache.shape[2]
    else:
        max_blocks, block_tokens, phys, s_max = (block_table.shape[1], k_cache.shape[2],
                                                 k_cache.shape[0], 0)
    _check(load().instinfer_kv_append_bulk(
        _ptr(k_cache), _ptr(v_cache), _ptr(k_new), _ptr(v_new), _ptr(seq_lens), _ptr(new_lens),
        _ptr(block_table), max_blocks, block_tokens, phys, batch, max_new, heads, head_dim, s_max,
        _ptr(status_flags), _stream(stream)))


def decode_attention(out: torch.Tensor, lse: Optional[torch.Tensor], q: torch.Tensor,
                     k_cache: torch.Tensor, v_cache: torch.Tensor, seq_lens: torch.Tensor,
                     max_seq_len: int, scale: float, workspace: torch.Tensor,
                     status_flags: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention over contiguous caches [B,H,s_max,D]."""
    batch, heads, head_dim = q.shape
    _check(load().instinfer_decode_attention(
        _ptr(out), _ptr(lse), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(seq_lens),
        batch, heads, head_dim, k_cache.shape[2], int(max_seq_len), float(scale),
        _ptr(workspace), workspace.numel() * workspace.element_size(),
        _ptr(status_flags), _stream(stream)))


def decode_attention_paged(out: torch.Tensor, lse: Optional[torch.Tensor], q: torch.Tensor,
                           k_pool: torch.Tensor, v_pool: torch.Tensor,
                           block_table: torch.Tensor, seq_lens: torch.Tensor,
                           max_seq_len: int, scale: float, workspace: torch.Tensor,
                           status_flags: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention_paged over pools [P,H,T,D] with block_table [B,M]."""
    batch, heads, head_dim = q.shape
    _check(load().instinfer_decode_attention_paged(
        _ptr(out), _ptr(lse), _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(block_table),
        _ptr(seq_lens), batch, heads, head_dim, k_pool.shape[2], block_table.shape[1],
        k_pool.shape[0], int(max_seq_len), float(scale), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status_flags), _stream(stream)))


def decode_attention_static(out: torch.Tensor, lse: Optional[torch.Tensor], q: torch.Tensor,
                            k_cache: torch.Tensor, v_cache: torch.Tensor,
                            block_table: Optional[torch.Tensor], seq_lens: torch.Tensor,
                            max_seq_len: int, scale: float,
                            status_flags: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention_static: attention in the library's built-in scratch array,
    for callers that cannot provide a workspace (block_table None = contiguous caches)."""
    batch, heads, head_dim = q.shape
    if block_table is None:
        s_max, block_tokens, max_blocks, phys = k_cache.shape[2], 0, 0, 0
    else:
        s_max, block_tokens, max_blocks, phys = (0, k_cache.shape[2], block_table.shape[1],
                                                 k_cache.shape[0])
    _check(load().instinfer_decode_attention_static(
        _ptr(out), _ptr(lse), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
        _ptr(seq_lens), batch, heads, head_dim, s_max, block_tokens, max_blocks, phys,
        int(max_seq_len), float(scale), _ptr(status_flags), _stream(stream)))


def allgather_workspace_bytes(batch: int, heads: int, head_dim: int, max_seq_len: int) -> int:
    return int(load().instinfer_allgather_workspace_bytes(batch, heads, head_dim, max_seq_len))


def decode_attention_allgather(out_all: Sequence[Union[torch.Tensor, int]], lse: Optional[torch.Tensor],
                               q: torch.Tensor, k_cache: torch.Tensor, v_cache: torch.Tensor,
                               block_table: Optional[torch.Tensor], seq_lens: torch.Tensor,
                               head_offset: int, total_heads: int, max_seq_len: int, scale: float,
                               workspace: torch.Tensor,
                               status_flags: Optional[torch.Tensor] = None,
                               stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention_allgather: this rank's head shard (q [B, heads, D]), output
    rows stored into every rank's [B, total_heads, D] buffer.  out_all holds one entry per
    rank, a tensor or a raw device address of a peer mapping."""
    batch, heads, head_dim = q.shape
    if block_table is None:
        s_max, block_tokens, max_blocks, phys = k_cache.shape[2], 0, 0, 0
    else:
        s_max, block_tokens, max_blocks, phys = (0, k_cache.shape[2], block_table.shape[1],
                                                 k_cache.shape[0])
    addresses = [t.data_ptr() if isinstance(t, torch.Tensor) else int(t) for t in out_all]
    table = (ctypes.c_void_p * len(addresses))(*addresses)
    _check(load().instinfer_decode_attention_allgather(
        table, len(addresses), _ptr(lse), _ptr(q), _ptr(k_cache), _ptr(v_cache),
        _ptr(block_table), _ptr(seq_lens), batch, heads, int(head_offset), int(total_heads),
        head_dim, s_max, block_tokens, max_blocks, phys, int(max_seq_len), float(scale),
        _ptr(workspace), workspace.numel() * workspace.element_size(), _ptr(status_flags),
        _stream(stream)))


def grouped_workspace_bytes(batch: int, q_tokens: int, q_heads: int, kv_heads: int, head_dim: int,
                            max_seq_len: int) -> int:
    return int(load().instinfer_grouped_workspace_bytes(batch, q_tokens, q_heads, kv_heads,
                                                        head_dim, max_seq_len))


def decode_attention_grouped(out: torch.Tensor, lse: Optional[torch.Tensor], q: torch.Tensor,
                             k_cache: torch.Tensor, v_cache: torch.Tensor,
                             block_table: Optional[torch.Tensor], seq_lens: torch.Tensor,
                             max_seq_len: int, scale: float, workspace: torch.Tensor,
                             status_flags: Optional[torch.Tensor] = None,
                             stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention_grouped: q, out [B, Tq, Hq, D]; caches with Hkv heads
    ([B,Hkv,s_max,D], or pools [P,Hkv,T,D] with block_table)."""
    batch, q_tokens, q_heads, head_dim = q.shape
    kv_heads = k_cache.shape[1]
    if block_table is None:
        s_max, block_tokens, max_blocks, phys = k_cache.shape[2], 0, 0, 0
    else:
        s_max, block_tokens, max_blocks, phys = (0, k_cache.shape[2], block_table.shape[1],
                                                 k_cache.shape[0])
    _check(load().instinfer_decode_attention_grouped(
        _ptr(out), _ptr(lse), _ptr(q), _ptr(k_cache), _ptr(v_cache), _ptr(block_table),
        _ptr(seq_lens), batch, q_tokens, q_heads, kv_heads, head_dim, s_max, block_tokens,
        max_blocks, phys, int(max_seq_len), float(scale), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status_flags), _stream(stream)))


def rope_frequencies(rope_dim: int, base: float = 10000.0, scaling: str = "plain", factor: float = 1.0, trained_len: int = 0,
                     slow_turns: float = 1.0, fast_turns: float = 32.0,
                     device: torch.device | str = "cuda") -> Tuple[torch.Tensor, float]:
    """instinfer_rope_frequencies: the pairs' frequencies, fp64 [rope_dim / 2] on `device`, and the magnitude.
    scaling: "plain", "linear" or "by_parts"."""
    if scaling not in ROPE_SCALINGS:
        raise InstInferError(ERR_UNSUPPORTED)
    pairs = (ctypes.c_double * max(1, rope_dim // 2))()
    magnitude = ctypes.c_float()
    _check(load().instinfer_rope_frequencies(pairs, ctypes.byref(magnitude), int(rope_dim), float(base), ROPE_SCALINGS[scaling],
                                             float(factor), int(trained_len), float(slow_turns), float(fast_turns)))
    return torch.tensor(list(pairs), dtype=torch.float64, device=device), magnitude.value


# (The calls below are short next to Python's part of them: shapes and strides are asked for once, and devices, types
# and addresses in passes in C.)
_device_of, _type_of, _address_of, _is_contiguous = (torch.Tensor.get_device, torch.Tensor.dtype.__get__, torch.Tensor.data_ptr,
                                                     torch.Tensor.is_contiguous)


def _token_stride(shape, strides) -> int:
    """Elements from one token of a tensor [B, N, ...] to the next, all B * N of them evenly spaced."""
    if shape[1] <= 1:
        # (one token in all, or none: any stride that the library accepts will do)
        return strides[0] if shape[0] > 1 and shape[1] == 1 else 1 << 32
    if shape[0] > 1 and strides[0] != shape[1] * strides[1]:
        raise InstInferError(ERR_INVALID_ARG)
    return strides[1]


def _check_append(batch: int, max_new: int, frequencies: torch.Tensor, seq_lens: torch.Tensor, new_lens: Optional[torch.Tensor],
                  block_table: Optional[torch.Tensor], positions: Optional[torch.Tensor], tokens: int, shape):
    """What the two turning appends ask of their small tensors, for a cache of this shape whose dim `tokens` counts tokens;
    (s_max, block_tokens, max_blocks, blocks)."""
    ints = [t for t in (seq_lens, new_lens, positions, block_table) if t is not None]
    if frequencies.dtype is not torch.float64 or set(map(_type_of, ints)) != {torch.int32} or \
            not all(map(_is_contiguous, (frequencies, *ints))) or len(seq_lens) < batch or \
            (new_lens is not None and len(new_lens) < batch) or \
            (positions is not None and positions.shape != (batch, max_new)):
        raise InstInferError(ERR_INVALID_ARG)
    if block_table is None:
        if shape[0] < batch:
            raise InstInferError(ERR_INVALID_ARG)
        return shape[tokens], 0, 0, 0
    sequences, max_blocks = block_table.shape
    if sequences < batch:
        raise InstInferError(ERR_INVALID_ARG)
    return 0, shape[tokens], max_blocks, shape[0]


def rope_append(q_out: Optional[torch.Tensor], k_cache: torch.Tensor, v_cache: torch.Tensor, q: Optional[torch.Tensor],
                k_new: torch.Tensor, v_new: torch.Tensor, frequencies: torch.Tensor, seq_lens: torch.Tensor,
                new_lens: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                positions: Optional[torch.Tensor] = None, interleaved: bool = False, magnitude: float = 1.0,
                status_flags: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_rope_append: q [B, N, Hq, D] (None: keys and values only), k_new and v_new [B, N, H, D] in fp32, fp16 or
    bf16, slices of one projection if need be; q_out fp16 as q; frequencies fp64 [rope_dim / 2]; caches fp16 [B, H, s_max, D]
    or pools [P, H, T, D] with block_table; positions int32 [B, N]."""
    shape = k_new.shape
    batch, max_new, heads, head_dim = shape
    cache = k_cache.shape
    here = _here(q_out, k_cache, v_cache, q, k_new, v_new, frequencies, seq_lens, new_lens, block_table, positions, status_flags)
    kind = k_new.dtype
    if kind not in _TYPES:
        raise InstInferError(ERR_UNSUPPORTED)
    if v_cache.shape != cache or cache[1] != heads or cache[3] != head_dim or v_new.shape != shape or v_new.dtype is not kind or \
            (q is None) != (q_out is None) or not (k_cache.is_contiguous() and v_cache.is_contiguous()) or \
            k_cache.dtype is not torch.float16 or v_cache.dtype is not torch.float16:
        raise InstInferError(ERR_INVALID_ARG)
    k_strides, v_strides = k_new.stride(), v_new.stride()
    if k_strides[3] != 1 or v_strides[3] != 1 or (heads > 1 and (k_strides[2] != head_dim or v_strides[2] != head_dim)):
        raise InstInferError(ERR_INVALID_ARG)
    q_heads = q_stride = 0
    if q is not None:
        q_shape, q_strides = q.shape, q.stride()
        q_heads = q_shape[2]
        if q_shape != (batch, max_new, q_heads, head_dim) or q_out.shape != q_shape or q.dtype is not kind or \
                q_out.dtype is not torch.float16 or not q_out.is_contiguous() or q_strides[3] != 1 or (q_heads > 1 and q_strides[2] != head_dim):
            raise InstInferError(ERR_INVALID_ARG)
        q_stride = _token_stride(q_shape, q_strides)
    s_max, block_tokens, max_blocks, phys = _check_append(batch, max_new, frequencies, seq_lens, new_lens, block_table, positions, 2, cache)
    _check(load().instinfer_rope_append(
        _ptr(q_out), k_cache.data_ptr(), v_cache.data_ptr(), _ptr(q), k_new.data_ptr(), v_new.data_ptr(), _TYPES[kind],
        q_stride, _token_stride(shape, k_strides), _token_stride(shape, v_strides), frequencies.data_ptr(), 2 * len(frequencies),
        interleaved, magnitude, _ptr(positions), seq_lens.data_ptr(), _ptr(new_lens), _ptr(block_table), max_blocks,
        block_tokens, phys, batch, max_new, q_heads, heads, head_dim, s_max, _ptr(status_flags), _stream(stream, here)))


def latent_append(q_out: Optional[torch.Tensor], cache: torch.Tensor, q_rope: Optional[torch.Tensor], latent_new: torch.Tensor,
                  rope_new: torch.Tensor, frequencies: torch.Tensor, seq_lens: torch.Tensor,
                  new_lens: Optional[torch.Tensor] = None, block_table: Optional[torch.Tensor] = None,
                  positions: Optional[torch.Tensor] = None, interleaved: bool = False, magnitude: float = 1.0,
                  status_flags: Optional[torch.Tensor] = None, stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_latent_append: latent_new [B, N, L], rope_new [B, N, R], q_rope [B, N, H, R] (None: the cache's rows only),
    slices of projections if need be; q_out [B, N, H, L + R]; cache [B, s_max, L + R] or a pool [P, T, L + R] with
    block_table; all fp16 or all bf16."""
    shape, rope_shape, cache_shape = latent_new.shape, rope_new.shape, cache.shape
    batch, max_new, latent_dim = shape
    rope_dim = rope_shape[2]
    here = _here(q_out, cache, q_rope, latent_new, rope_new, frequencies, seq_lens, new_lens, block_table, positions, status_flags)
    kind = latent_new.dtype
    if kind not in _TYPES:
        raise InstInferError(ERR_UNSUPPORTED)
    strides, rope_strides = latent_new.stride(), rope_new.stride()
    if rope_shape[:2] != shape[:2] or cache_shape[2] != latent_dim + rope_dim or not cache.is_contiguous() or \
            (q_rope is None) != (q_out is None) or len(frequencies) * 2 != rope_dim or strides[2] != 1 or rope_strides[2] != 1 or \
            cache.dtype is not kind or rope_new.dtype is not kind:
        raise InstInferError(ERR_INVALID_ARG)
    q_heads = q_stride = head_stride = 0
    if q_rope is not None:
        q_shape, q_strides = q_rope.shape, q_rope.stride()
        q_heads = q_shape[2]
        head_stride = q_strides[2] if q_heads > 1 else rope_dim
        if q_shape != (batch, max_new, q_heads, rope_dim) or q_out.shape != (batch, max_new, q_heads, latent_dim + rope_dim) or \
                q_strides[3] != 1 or not q_out.is_contiguous() or q_rope.dtype is not kind or q_out.dtype is not kind:
            raise InstInferError(ERR_INVALID_ARG)
        q_stride = _token_stride(q_shape, q_strides)
    s_max, block_tokens, max_blocks, phys = _check_append(batch, max_new, frequencies, seq_lens, new_lens, block_table, positions, 1, cache_shape)
    _check(load().instinfer_latent_append(
        _ptr(q_out), cache.data_ptr(), _ptr(q_rope), latent_new.data_ptr(), rope_new.data_ptr(), _TYPES[kind],
        q_stride, head_stride, _token_stride(shape, strides), _token_stride(rope_shape, rope_strides),
        frequencies.data_ptr(), interleaved, magnitude, _ptr(positions), seq_lens.data_ptr(), _ptr(new_lens),
        _ptr(block_table), max_blocks, block_tokens, phys, batch, max_new, q_heads, latent_dim, rope_dim, s_max,
        _ptr(status_flags), _stream(stream, here)))


def latent_workspace_bytes(batch: int, q_tokens: int, q_heads: int, latent_dim: int, rope_dim: int, max_seq_len: int) -> int:
    return int(load().instinfer_latent_workspace_bytes(batch, q_tokens, q_heads, latent_dim, rope_dim, max_seq_len))


def decode_attention_latent(out: torch.Tensor, lse: Optional[torch.Tensor], q: torch.Tensor, cache: torch.Tensor,
                            block_table: Optional[torch.Tensor], seq_lens: torch.Tensor,
                            tree_lens: Optional[torch.Tensor], mask: Optional[torch.Tensor], max_seq_len: int,
                            scale: float, workspace: torch.Tensor, status_flags: Optional[torch.Tensor] = None,
                            stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention_latent: q [B, N, H, L + R], out [B, N, H, L], lse [B, N, H]; cache [B, s_max, L + R] or a pool
    [P, T, L + R] with block_table; mask as tree_mask writes it, or None for a chain; all fp16 or all bf16."""
    batch, q_tokens, q_heads, dims = q.shape
    out_shape, cache_shape = out.shape, cache.shape
    latent_dim = out_shape[3]
    here = _here(out, lse, q, cache, block_table, seq_lens, tree_lens, mask, workspace, status_flags)
    kind = q.dtype
    if kind not in _TYPES:
        raise InstInferError(ERR_UNSUPPORTED)
    ints = [t for t in (seq_lens, tree_lens, block_table) if t is not None]
    if out_shape != (batch, q_tokens, q_heads, latent_dim) or cache_shape[2] != dims or out.dtype is not kind or cache.dtype is not kind or \
            len(seq_lens) < batch or (tree_lens is not None and len(tree_lens) < batch) or set(map(_type_of, ints)) != {torch.int32} or \
            not all(map(_is_contiguous, (out, q, cache, *ints))) or \
            (lse is not None and (lse.numel() != batch * q_tokens * q_heads or lse.dtype is not torch.float32 or not lse.is_contiguous())) or \
            (mask is not None and (mask.shape[1:] != (q_tokens, (q_tokens + 63) // 64) or len(mask) < batch or mask.dtype is not torch.int64 or
                                  not mask.is_contiguous())):
        raise InstInferError(ERR_INVALID_ARG)
    if block_table is None:
        sequences, s_max, block_tokens, max_blocks, phys = cache_shape[0], cache_shape[1], 0, 0, 0
    else:
        (sequences, max_blocks), (phys, block_tokens, _), s_max = block_table.shape, cache_shape, 0
    if sequences < batch:
        raise InstInferError(ERR_INVALID_ARG)
    _check(load().instinfer_decode_attention_latent(
        out.data_ptr(), _ptr(lse), q.data_ptr(), cache.data_ptr(), _ptr(block_table), seq_lens.data_ptr(), _ptr(tree_lens), _ptr(mask),
        _TYPES[kind], batch, q_tokens, q_heads, latent_dim, dims - latent_dim, s_max, block_tokens, max_blocks, phys,
        int(max_seq_len), float(scale), workspace.data_ptr(), workspace.nbytes, _ptr(status_flags), _stream(stream, here)))


def tree_mask(mask: torch.Tensor, parents: torch.Tensor, tree_lens: Optional[torch.Tensor] = None,
              status_flags: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_tree_mask: mask int64 [B, T, ceil(T / 64)] (the bits of the header's uint64 words),
    parents int32 [B, T], tree_lens int32 [B] (None: T nodes each)."""
    batch, tree_tokens = parents.shape
    here = _here(mask, parents, tree_lens, status_flags)
    _check(load().instinfer_tree_mask(mask.data_ptr(), parents.data_ptr(), _ptr(tree_lens), batch, tree_tokens,
                                      _ptr(status_flags), _stream(stream, here)))


def tree_workspace_bytes(batch: int, tree_tokens: int, q_heads: int, kv_heads: int, head_dim: int,
                         max_seq_len: int) -> int:
    return int(load().instinfer_tree_workspace_bytes(batch, tree_tokens, q_heads, kv_heads, head_dim, max_seq_len))


def decode_attention_tree(out: torch.Tensor, lse: Optional[torch.Tensor], q: torch.Tensor,
                          k_cache: torch.Tensor, v_cache: torch.Tensor,
                          block_table: Optional[torch.Tensor], seq_lens: torch.Tensor,
                          tree_lens: Optional[torch.Tensor], mask: torch.Tensor, max_seq_len: int,
                          scale: float, workspace: torch.Tensor,
                          status_flags: Optional[torch.Tensor] = None,
                          stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_attention_tree: q, out [B, T, Hq, D]; mask as tree_mask writes it; caches
    with Hkv heads ([B,Hkv,s_max,D], or pools [P,Hkv,T,D] with block_table)."""
    batch, tree_tokens, q_heads, head_dim = q.shape
    shape = k_cache.shape
    sequences, kv_heads = shape[0] if block_table is None else block_table.shape[0], shape[1]
    here = _here(out, lse, q, k_cache, v_cache, block_table, seq_lens, tree_lens, mask, workspace, status_flags)
    if v_cache.shape != shape or shape[3] != head_dim or sequences < batch or \
            mask.numel() < batch * tree_tokens * ((tree_tokens + 63) // 64):
        raise InstInferError(ERR_INVALID_ARG)
    if block_table is None:
        s_max, block_tokens, max_blocks, phys = shape[2], 0, 0, 0
    else:
        s_max, block_tokens, max_blocks, phys = 0, shape[2], block_table.shape[1], shape[0]
    _check(load().instinfer_decode_attention_tree(
        out.data_ptr(), _ptr(lse), q.data_ptr(), k_cache.data_ptr(), v_cache.data_ptr(), _ptr(block_table), seq_lens.data_ptr(),
        _ptr(tree_lens), mask.data_ptr(), batch, tree_tokens, q_heads, kv_heads, head_dim, s_max, block_tokens,
        max_blocks, phys, int(max_seq_len), float(scale), workspace.data_ptr(),
        workspace.nbytes, _ptr(status_flags), _stream(stream, here)))


_TYPES = {torch.float32: 0, torch.float16: 1, torch.bfloat16: 2}
_INT32, _FLOAT32 = {torch.int32}, {torch.float32}


def verify_tree(path: torch.Tensor, path_lens: torch.Tensor, out_tokens: torch.Tensor,
                target_probs: torch.Tensor, draft_probs: Optional[torch.Tensor], tokens: torch.Tensor,
                parents: torch.Tensor, tree_lens: Optional[torch.Tensor], uniforms: torch.Tensor,
                status_flags: Optional[torch.Tensor] = None,
                stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_verify_tree: target_probs, draft_probs (None: drafts that were not sampled) fp32,
    fp16 or bf16 [B, T, V] with rows at one stride (a padded vocabulary sliced to V will do); the
    other tensors [B, T], path_lens and tree_lens [B]."""
    batch, tree_tokens, vocab = target_probs.shape
    stride = target_probs.stride(1) if tree_tokens > 1 else max(vocab, target_probs.stride(0))
    for probs in (target_probs, draft_probs):
        if probs is not None and (
                probs.dtype != target_probs.dtype or probs.shape != target_probs.shape or
                (vocab > 1 and probs.stride(2) != 1) or (tree_tokens > 1 and probs.stride(1) != stride) or
                (batch > 1 and probs.stride(0) != tree_tokens * stride)):
            raise InstInferError(ERR_INVALID_ARG)
    here = _here(path, path_lens, out_tokens, target_probs, draft_probs, tokens, parents, tree_lens, uniforms, status_flags)
    if target_probs.dtype not in _TYPES:
        raise InstInferError(ERR_UNSUPPORTED)
    _check(load().instinfer_verify_tree(
        path.data_ptr(), path_lens.data_ptr(), out_tokens.data_ptr(), target_probs.data_ptr(), _ptr(draft_probs),
        _TYPES[target_probs.dtype], stride, tokens.data_ptr(), parents.data_ptr(), _ptr(tree_lens),
        uniforms.data_ptr(), batch, tree_tokens, vocab, _ptr(status_flags), _stream(stream, here)))


def _row_stride(strides, batch: int, rows: int, vocab: int) -> int:
    """Elements from one row of a tensor [batch, rows, vocab] to the next, all evenly spaced (a padded vocabulary sliced to V will do)."""
    far, stride, near = strides
    if rows == 1:
        stride = far if batch > 1 else (vocab + 3) // 4 * 4
    if (vocab > 1 and near != 1) or (batch > 1 and far != rows * stride):
        raise InstInferError(ERR_INVALID_ARG)
    return stride


def process_logits(out: torch.Tensor, logits: torch.Tensor, tokens: Optional[torch.Tensor] = None,
                   token_lens: Optional[torch.Tensor] = None, prompt_lens: Optional[torch.Tensor] = None,
                   penalties: Optional[torch.Tensor] = None, draft_tokens: Optional[torch.Tensor] = None,
                   mask: Optional[torch.Tensor] = None, tree_lens: Optional[torch.Tensor] = None,
                   bias_tokens: Optional[torch.Tensor] = None, bias_values: Optional[torch.Tensor] = None,
                   allowed: Optional[torch.Tensor] = None, temperatures: Optional[torch.Tensor] = None,
                   probabilities: bool = True, status_flags: Optional[torch.Tensor] = None,
                   stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_process_logits: logits and out [B, T, V] in fp32, fp16 or bf16; tokens [B, M], token_lens and prompt_lens [B];
    penalties fp32 [B, 3]; draft_tokens [B, T] with mask as tree_mask writes it; bias_tokens and bias_values [B, n]; allowed
    int32 [B, T, ceil(V / 32)] (the bits of the header's uint32 words); temperatures fp32 [B]."""
    shape = logits.shape
    batch, tree_tokens, vocab = shape
    here = _here(out, logits, tokens, token_lens, prompt_lens, penalties, draft_tokens, mask, tree_lens, bias_tokens, bias_values, allowed,
                 temperatures, status_flags)
    ints = [t for t in (tokens, token_lens, prompt_lens, draft_tokens, tree_lens, bias_tokens, allowed) if t is not None]
    floats = [t for t in (penalties, bias_values, temperatures) if t is not None]
    if out.shape != shape or (bias_tokens is None) != (bias_values is None) or \
            not set(map(_type_of, ints)) <= _INT32 or not set(map(_type_of, floats)) <= _FLOAT32 or \
            not all(map(_is_contiguous, (*ints, *floats))) or (mask is not None and (mask.dtype is not torch.int64 or not mask.is_contiguous())):
        raise InstInferError(ERR_INVALID_ARG)
    each = (batch,)
    for t, rows in ((token_lens, each), (prompt_lens, each), (tree_lens, each), (temperatures, each), (penalties, (batch, 3)),
                    (draft_tokens, (batch, tree_tokens)), (mask, (batch, tree_tokens, (tree_tokens + 63) // 64)),
                    (allowed, (batch, tree_tokens, (vocab + 31) // 32))):
        # (more sequences than the batch has will do)
        if t is not None and t.shape != rows and (t.shape[1:] != rows[1:] or t.dim() == 0 or len(t) < batch):
            raise InstInferError(ERR_INVALID_ARG)
    max_tokens = max_bias = 0
    if tokens is not None:
        listed = tokens.shape
        if len(listed) != 2 or listed[0] < batch:
            raise InstInferError(ERR_INVALID_ARG)
        max_tokens = listed[1]
    if bias_tokens is not None:
        listed = bias_tokens.shape
        if len(listed) != 2 or listed[0] < batch or bias_values.shape != listed:
            raise InstInferError(ERR_INVALID_ARG)
        max_bias = listed[1]
    if out.dtype not in _TYPES or logits.dtype not in _TYPES:
        raise InstInferError(ERR_UNSUPPORTED)
    _check(load().instinfer_process_logits(
        out.data_ptr(), _TYPES[out.dtype], _row_stride(out.stride(), *shape), logits.data_ptr(), _TYPES[logits.dtype],
        _row_stride(logits.stride(), *shape), _ptr(tokens), _ptr(token_lens), _ptr(prompt_lens), max_tokens, _ptr(penalties), _ptr(draft_tokens), _ptr(mask), _ptr(tree_lens),
        _ptr(bias_tokens), _ptr(bias_values), max_bias, _ptr(allowed), _ptr(temperatures), int(probabilities), batch, tree_tokens, vocab,
        _ptr(status_flags), _stream(stream, here)))


_bytes_of = torch.Tensor.nbytes.__get__


def _layers(here: int, k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor]):
    """The two HOST pointer arrays of the calls that work on all layers at once, and the caches' shape: as many V as K
    caches, fp16, contiguous, of one size, all on the device `here`.  (Latent caches [B, s_max, 576] or pools [P, T, 576] come as
    cache.view(torch.float16).unsqueeze(1), half of the layers as K and half as V caches, an odd one as both of one place.)"""
    n = len(k_caches)
    caches = [*k_caches, *v_caches]
    # (whole passes in C: a model has some hundred caches, and a Python loop over them outlasts the kernel.  One shape
    # of another type has another number of bytes, so that the first cache's type speaks for all.)
    if n == 0 or len(caches) != 2 * n or not all(map(torch.Tensor.is_contiguous, caches)) or \
            len(set(map(_bytes_of, caches))) != 1 or set(map(torch.Tensor.get_device, caches)) != {here}:
        raise InstInferError(ERR_INVALID_ARG)
    shape = k_caches[0].shape
    if v_caches[0].shape != shape or k_caches[0].dtype is not torch.float16:
        raise InstInferError(ERR_INVALID_ARG)
    addresses = array.array("Q", map(torch.Tensor.data_ptr, caches))
    at, _ = addresses.buffer_info()
    return at, at + 8 * n, n, shape, addresses   # the caller keeps `addresses` alive during the call


def kv_keep_path(k_caches: Sequence[torch.Tensor], v_caches: Sequence[torch.Tensor], path: torch.Tensor,
                 path_lens: torch.Tensor, tree_lens: Optional[torch.Tensor], seq_lens: torch.Tensor,
                 new_lens: torch.Tensor, block_table: Optional[torch.Tensor] = None,
                 status_flags: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_kv_keep_path: one cache per layer ([B,H,s_max,D], or pools [P,H,T,D] with
    block_table); path [B, tree_tokens]."""
    batch, tree_tokens = path.shape
    here = _here(path, path_lens, tree_lens, seq_lens, new_lens, block_table, status_flags)
    k, v, n_layers, (blocks, heads, rows, head_dim), keep = _layers(here, k_caches, v_caches)
    if block_table is None:
        sequences, max_blocks, block_tokens, phys, s_max = blocks, 0, 0, 0, rows
    else:
        sequences, max_blocks = block_table.shape
        block_tokens, phys, s_max = rows, blocks, 0
    if sequences < batch:
        raise InstInferError(ERR_INVALID_ARG)
    _check(load().instinfer_kv_keep_path(
        k, v, n_layers, path.data_ptr(), path_lens.data_ptr(), _ptr(tree_lens), seq_lens.data_ptr(), new_lens.data_ptr(),
        _ptr(block_table), max_blocks, block_tokens, phys, batch, tree_tokens, heads, head_dim, s_max,
        _ptr(status_flags), _stream(stream, here)))


def kv_fork(block_table: torch.Tensor, block_refs: torch.Tensor, seq_lens: torch.Tensor, src: torch.Tensor,
            dst: torch.Tensor, block_tokens: int, status_flags: Optional[torch.Tensor] = None,
            stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_kv_fork: block_table [B, M], block_refs [P], seq_lens [B], src and dst [n]."""
    batch, max_blocks = block_table.shape
    here = _here(block_table, block_refs, seq_lens, src, dst, status_flags)
    if dst.numel() != src.numel():
        raise InstInferError(ERR_INVALID_ARG)
    _check(load().instinfer_kv_fork(block_table.data_ptr(), block_refs.data_ptr(), seq_lens.data_ptr(), src.data_ptr(), dst.data_ptr(),
                                    src.numel(), max_blocks, int(block_tokens), block_refs.numel(), batch,
                                    _ptr(status_flags), _stream(stream, here)))


def kv_resize_workspace_bytes(batch: int, num_phys_blocks: int) -> int:
    return int(load().instinfer_kv_resize_workspace_bytes(batch, num_phys_blocks))


def kv_resize(k_pools: Sequence[torch.Tensor], v_pools: Sequence[torch.Tensor], block_table: torch.Tensor,
              block_refs: torch.Tensor, seq_lens: torch.Tensor, want_lens: torch.Tensor, new_lens: torch.Tensor,
              workspace: torch.Tensor, status_flags: Optional[torch.Tensor] = None,
              stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_kv_resize: one pool [P,H,T,D] per layer; new_lens may be seq_lens."""
    batch, max_blocks = block_table.shape
    here = _here(block_table, block_refs, seq_lens, want_lens, new_lens, workspace, status_flags)
    k, v, n_layers, (phys, heads, block_tokens, head_dim), keep = _layers(here, k_pools, v_pools)
    if block_refs.numel() < phys:
        raise InstInferError(ERR_INVALID_ARG)
    _check(load().instinfer_kv_resize(
        k, v, n_layers, block_table.data_ptr(), block_refs.data_ptr(), seq_lens.data_ptr(), want_lens.data_ptr(), new_lens.data_ptr(),
        max_blocks, block_tokens, phys, batch, heads, head_dim, workspace.data_ptr(),
        workspace.nbytes, _ptr(status_flags), _stream(stream, here)))


def kv_defragment_workspace_bytes(num_phys_blocks: int) -> int:
    return int(load().instinfer_kv_defragment_workspace_bytes(num_phys_blocks))


def kv_defragment(k_pools: Sequence[torch.Tensor], v_pools: Sequence[torch.Tensor], block_table: torch.Tensor,
                  block_refs: torch.Tensor, seq_lens: torch.Tensor, new_block_table: torch.Tensor,
                  new_block_refs: torch.Tensor, blocks_used: torch.Tensor, workspace: torch.Tensor,
                  status_flags: Optional[torch.Tensor] = None,
                  stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_kv_defragment: one pool [P,H,T,D] per layer; the new table and counts may be the
    old ones; blocks_used int32 [1]."""
    batch, max_blocks = block_table.shape
    here = _here(block_table, block_refs, seq_lens, new_block_table, new_block_refs, blocks_used, workspace, status_flags)
    k, v, n_layers, (phys, heads, block_tokens, head_dim), keep = _layers(here, k_pools, v_pools)
    if block_refs.numel() < phys or new_block_refs.numel() < phys or new_block_table.shape != block_table.shape:
        raise InstInferError(ERR_INVALID_ARG)
    _check(load().instinfer_kv_defragment(
        k, v, n_layers, block_table.data_ptr(), new_block_table.data_ptr(), block_refs.data_ptr(), new_block_refs.data_ptr(),
        seq_lens.data_ptr(), blocks_used.data_ptr(), max_blocks, block_tokens, phys, batch, heads, head_dim,
        workspace.data_ptr(), workspace.nbytes, _ptr(status_flags), _stream(stream, here)))


def decode_step_host(out_host: torch.Tensor, qkv_host: torch.Tensor, qkv_dev: torch.Tensor,
                     out_dev: torch.Tensor, lse: Optional[torch.Tensor], k_cache: torch.Tensor,
                     v_cache: torch.Tensor, seq_lens: torch.Tensor,
                     block_table: Optional[torch.Tensor], max_seq_len: int, scale: float,
                     workspace: torch.Tensor, status_flags: Optional[torch.Tensor] = None,
                     stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_decode_step_host: qkv_host [3,B,H,D] and out_host [B,H,D] are (pinned) host
    tensors, qkv_dev / out_dev device staging buffers of the same shapes."""
    _, batch, heads, head_dim = qkv_host.shape
    if block_table is None:
        max_blocks, block_tokens, phys, s_max = 0, 0, 0, k_cache.shape[2]
    else:
        max_blocks, block_tokens, phys, s_max = (block_table.shape[1], k_cache.shape[2],
                                                 k_cache.shape[0], 0)
    _check(load().instinfer_decode_step_host(
        _ptr(out_host), _ptr(qkv_host), _ptr(qkv_dev), _ptr(out_dev), _ptr(lse), _ptr(k_cache),
        _ptr(v_cache), _ptr(seq_lens), _ptr(block_table), max_blocks, block_tokens, phys, batch,
        heads, head_dim, s_max, int(max_seq_len), float(scale), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status_flags), _stream(stream)))


def decode_step_host_overlapped(out_host: torch.Tensor, qkv_host: torch.Tensor, qkv_dev: torch.Tensor,
                                out_dev: torch.Tensor, lse: Optional[torch.Tensor], k_cache: torch.Tensor,
                                v_cache: torch.Tensor, seq_lens: torch.Tensor,
                                block_table: Optional[torch.Tensor], max_seq_len: int, scale: float,
                                workspace: torch.Tensor, status_flags: Optional[torch.Tensor],
                                compute: torch.cuda.Stream, upload: torch.cuda.Stream,
                                download: torch.cuda.Stream, uploaded: torch.cuda.Event,
                                attended: torch.cuda.Event) -> None:
    """instinfer_decode_step_host_overlapped: as decode_step_host, with the upload on `upload`
    and the download on `download`; `uploaded` and `attended` are events that have been
    recorded at least once (torch creates the CUDA event at its first record)."""
    _, batch, heads, head_dim = qkv_host.shape
    if block_table is None:
        max_blocks, block_tokens, phys, s_max = 0, 0, 0, k_cache.shape[2]
    else:
        max_blocks, block_tokens, phys, s_max = (block_table.shape[1], k_cache.shape[2],
                                                 k_cache.shape[0], 0)
    _check(load().instinfer_decode_step_host_overlapped(
        _ptr(out_host), _ptr(qkv_host), _ptr(qkv_dev), _ptr(out_dev), _ptr(lse), _ptr(k_cache),
        _ptr(v_cache), _ptr(seq_lens), _ptr(block_table), max_blocks, block_tokens, phys, batch,
        heads, head_dim, s_max, int(max_seq_len), float(scale), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status_flags), compute.cuda_stream or None,
        upload.cuda_stream or None, download.cuda_stream or None, uploaded.cuda_event or None,
        attended.cuda_event or None))


def sparf_append(k_pool: torch.Tensor, v_pool: torch.Tensor, kt_pool: torch.Tensor,
                 v_sum: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                 seq_lens: torch.Tensor, block_table: torch.Tensor, kt_block_table: torch.Tensor,
                 status_flags: Optional[torch.Tensor] = None,
                 stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_sparf_append: pools [P,H,T,D], kt_pool [Pk,H,D,Tk] with kt_block_table [B,Mk],
    v_sum fp32 [B,H,D]."""
    batch, heads, head_dim = k_new.shape
    _check(load().instinfer_sparf_append(
        _ptr(k_pool), _ptr(v_pool), _ptr(kt_pool), _ptr(v_sum), _ptr(k_new), _ptr(v_new),
        _ptr(seq_lens), _ptr(block_table), block_table.shape[1], k_pool.shape[2], k_pool.shape[0],
        _ptr(kt_block_table), kt_block_table.shape[1], kt_pool.shape[3], kt_pool.shape[0],
        batch, heads, head_dim, _ptr(status_flags), _stream(stream)))


def sparf_append_bulk(k_pool: torch.Tensor, v_pool: torch.Tensor, kt_pool: torch.Tensor,
                      v_sum: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                      seq_lens: torch.Tensor, new_lens: torch.Tensor, block_table: torch.Tensor,
                      kt_block_table: torch.Tensor, status_flags: Optional[torch.Tensor] = None,
                      stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_sparf_append_bulk: k_new, v_new are [B, max_new, H, D] (token-major)."""
    batch, max_new, heads, head_dim = k_new.shape
    _check(load().instinfer_sparf_append_bulk(
        _ptr(k_pool), _ptr(v_pool), _ptr(kt_pool), _ptr(v_sum), _ptr(k_new), _ptr(v_new),
        _ptr(seq_lens), _ptr(new_lens), _ptr(block_table), block_table.shape[1], k_pool.shape[2],
        k_pool.shape[0], _ptr(kt_block_table), kt_block_table.shape[1], kt_pool.shape[3],
        kt_pool.shape[0], batch, max_new, heads, head_dim, _ptr(status_flags), _stream(stream)))


def grouped_path_for(head_dim: int, block_tokens: int) -> int:
    """instinfer_grouped_path_for: 1 warp-level MMAs, 2 tcgen05, 0 unsupported (block_tokens 0: contiguous)."""
    return int(load().instinfer_grouped_path_for(int(head_dim), int(block_tokens)))


def set_grouped_path(path: int) -> None:
    """instinfer_set_grouped_path: 0 automatic, 1 warp-level MMAs, 2 tcgen05 where the shape allows."""
    _check(load().instinfer_set_grouped_path(int(path)))


def set_sparse_path(path: int) -> None:
    """instinfer_set_sparse_path: 0 automatic, 1 chunk-parallel, 2 one block per row."""
    _check(load().instinfer_set_sparse_path(int(path)))


def sparf_workspace_bytes(batch: int, heads: int, head_dim: int, max_seq_len: int, max_k: int) -> int:
    return int(load().instinfer_sparf_workspace_bytes(batch, heads, head_dim, max_seq_len, max_k))


def sparf_decode_attention(out: torch.Tensor, alpha: Optional[torch.Tensor],
                           selected: Optional[torch.Tensor], q: torch.Tensor,
                           k_pool: torch.Tensor, v_pool: torch.Tensor, kt_pool: torch.Tensor,
                           v_sum: torch.Tensor, block_table: torch.Tensor,
                           kt_block_table: torch.Tensor, seq_lens: torch.Tensor,
                           k_tokens: torch.Tensor, max_seq_len: int, max_k: int, r: int,
                           local_window: int, scale: float, workspace: torch.Tensor,
                           status_flags: Optional[torch.Tensor] = None,
                           stream: Optional[torch.cuda.Stream] = None) -> None:
    """instinfer_sparf_decode_attention (Algorithm 1) over paged pools."""
    batch, heads, head_dim = q.shape
    _check(load().instinfer_sparf_decode_attention(
        _ptr(out), _ptr(alpha), _ptr(selected), _ptr(q), _ptr(k_pool), _ptr(v_pool), _ptr(kt_pool),
        _ptr(v_sum), _ptr(block_table), _ptr(seq_lens), _ptr(k_tokens), batch, heads, head_dim,
        k_pool.shape[2], block_table.shape[1], k_pool.shape[0],
        _ptr(kt_block_table), kt_block_table.shape[1], kt_pool.shape[3], kt_pool.shape[0],
        int(max_seq_len), int(max_k), int(r), int(local_window), float(scale), _ptr(workspace),
        workspace.numel() * workspace.element_size(), _ptr(status_flags), _stream(stream)))


def alloc_workspace(batch: int, heads: int, head_dim: int, max_seq_len: int,
                    device: torch.device | str = "cuda") -> torch.Tensor:
    """A byte tensor of the size the library asks for under the current split plan."""
    need = workspace_bytes(batch, heads, head_dim, max_seq_len)
    if need == 0:
        raise InstInferError(ERR_INVALID_ARG)
    return torch.empty(need, dtype=torch.uint8, device=device)
