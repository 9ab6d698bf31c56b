"""GB300-native hot path of the hot-cold KV hierarchy for agentic LLM serving.

Baek et al., "Hot-Cold Tiering of HBM and High Bandwidth Flash for Agentic LLM
Serving": active sessions' KV (the hot set) stays in HBM and is read by every
decode step; paused sessions' KV (the cold pool) lives in a second tier and
moves only on pause (pack) and resume (unpack). Here both tiers are device
memory of one GB300; the CUDA kernels and the pool runtime are in
``libkvtier.so`` (C ABI: include/kvtier.h), bound by :mod:`.kvtier`.

:class:`Pool` is a convenience owner: it allocates the two arenas with torch
(device memory only) and forwards every operation to the C ABI.
"""
from __future__ import annotations

from . import kvtier
from .kvtier import KVError  # noqa: F401

__all__ = ["Pool", "kvtier", "KVError"]


class Pool:
    def __init__(self, *, num_layers: int, num_hot_blocks: int, cold_bytes: int,
                 num_q_heads: int = 32, num_kv_heads: int = 4, head_dim: int = 128,
                 block_tokens: int = 16, max_sessions: int = 64, max_batch: int = 64,
                 max_context: int = 32768, alloc_seed: int = 0, device: int = 0,
                 lru_residency: bool = False, cold_int8: bool = False):
        import torch
        self.device = torch.device("cuda", device)
        self.L, self.Hq, self.Hkv, self.D, self.bt = (num_layers, num_q_heads, num_kv_heads,
                                                      head_dim, block_tokens)
        self.num_hot_blocks = num_hot_blocks
        # The calls that a model makes per layer go to the library by the shortest way: a call on a few
        # tokens takes the GPU about as long as the host.
        self._prefill, self._tree = kvtier.lib.prefill_attention, kvtier.lib.tree_attention
        self._select, self._sparse = kvtier.lib.select_blocks, kvtier.lib.sparse_attention
        self._bf16, self._i32, self._masks, self._index = (torch.bfloat16, torch.int32,
                                                           (torch.int64, torch.uint64), device)
        self._f32 = torch.float32
        self._out_flags = {torch.float32: 0, torch.bfloat16: kvtier.KV_DECODE_OUT_BF16}
        probe = kvtier.make_config(num_layers=num_layers, num_q_heads=num_q_heads,
                                   num_kv_heads=num_kv_heads, head_dim=head_dim,
                                   block_tokens=block_tokens, num_hot_blocks=num_hot_blocks)
        self.block_bytes = kvtier.kv_block_bytes(probe)
        self.token_bytes = kvtier.kv_token_bytes(probe)
        self.bounds_bytes = kvtier.kv_bounds_bytes(probe)
        self.hot = torch.empty(num_hot_blocks * self.block_bytes // 2, dtype=torch.bfloat16,
                               device=self.device)
        self.cold_int8 = cold_int8
        self.cold = torch.empty(max(cold_bytes, 256) // 2, dtype=torch.bfloat16, device=self.device)
        cfg = kvtier.make_config(num_layers=num_layers, num_q_heads=num_q_heads,
                                 num_kv_heads=num_kv_heads, head_dim=head_dim,
                                 block_tokens=block_tokens, max_sessions=max_sessions,
                                 max_batch=max_batch, device=device, max_context=max_context,
                                 num_hot_blocks=num_hot_blocks, hot_base=self.hot,
                                 cold_bytes=cold_bytes, cold_base=self.cold, alloc_seed=alloc_seed,
                                 flags=(kvtier.KV_POOL_LRU_RESIDENCY if lru_residency else 0) |
                                 (kvtier.KV_POOL_COLD_INT8 if cold_int8 else 0))
        self.handle = kvtier.kv_pool_create(cfg)
        self.max_context = max_context
        self._calls = None
        if kvtier._calls is not None and head_dim == 128:
            self._calls = kvtier._calls.Calls(self.handle, device, num_q_heads, num_kv_heads, self.bounds_bytes, torch.bfloat16,
                                              torch.int32, torch.float32, *map(kvtier.address, (self._select, self._sparse)))

    def close(self) -> None:
        self._calls = None               # (it has the handle)
        if getattr(self, "handle", None):
            kvtier.kv_pool_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # views -----------------------------------------------------------------
    def hot_view(self):
        """The hot arena as [NB][L][2][Hkv][bt][D] bf16."""
        return self.hot.view(self.num_hot_blocks, self.L, 2, self.Hkv, self.bt, self.D)

    def image(self, sid: int):
        """A session's cold image as [L][2][Hkv][T_cap][D] bf16 (a view)."""
        if self.cold_int8:
            raise ValueError("the pool's images hold 8-bit rows: image_int8")
        info = kvtier.session_info(self.handle, sid)
        off = (info.image - self.cold.data_ptr()) // 2
        n = self.L * 2 * self.Hkv * info.capacity * self.D
        return self.cold[off:off + n].view(self.L, 2, self.Hkv, info.capacity, self.D)

    def image_int8(self, sid: int):
        """A session's 8-bit cold image (views): int8 codes [L][2][Hkv][T_cap][D] and uint8
        exponents [L][2][Hkv][T_cap]; value = code * 2^(exponent - 133), code -128 a NaN."""
        import torch
        if not self.cold_int8:
            raise ValueError("the pool's images hold bf16 rows: image")
        info = kvtier.session_info(self.handle, sid)
        off, shape = info.image - self.cold.data_ptr(), (self.L, 2, self.Hkv, info.capacity)
        rows = self.L * 2 * self.Hkv * info.capacity
        flat = self.cold.view(torch.int8)[off:off + rows * (self.D + 1)]
        return flat[:rows * self.D].view(*shape, self.D), flat[rows * self.D:].view(torch.uint8).view(shape)

    # C ABI forwards ------------------------------------------------------------
    def session_create(self, max_tokens: int) -> int:
        return kvtier.session_create(self.handle, max_tokens)

    def session_create_paused(self, max_tokens: int, tokens: int) -> int:
        return kvtier.session_create_paused(self.handle, max_tokens, tokens)

    def session_destroy(self, sid: int) -> None:
        kvtier.session_destroy(self.handle, sid)

    def session_append(self, sid: int, k, v, stream=None) -> None:
        """k, v: device bf16 [L][n][Hkv][D]."""
        kvtier.session_append(self.handle, sid, k, v, int(k.shape[1]), stream)

    def session_pause(self, sid: int, stream=None) -> None:
        kvtier.session_pause(self.handle, sid, stream)

    def session_resume(self, sid: int, stream=None) -> None:
        kvtier.session_resume(self.handle, sid, stream)

    def session_info(self, sid: int):
        return kvtier.session_info(self.handle, sid)

    def session_block_table(self, sid: int) -> list[int]:
        return kvtier.session_block_table(self.handle, sid)

    def session_ready_event(self, sid: int):
        return kvtier.session_ready_event(self.handle, sid)

    def batch_tables(self, sids, block_tables, max_blocks: int, seq_lens, stream=None) -> None:
        kvtier.kv_pool_batch_tables(self.handle, list(sids), block_tables, max_blocks, seq_lens,
                                    stream)

    def batch_reserve(self, sids, block_tables, max_blocks: int, seq_lens, stream=None,
                      counts=None) -> None:
        """One new position per session (filled by decode_append_attention), or
        counts[i] of them (filled by prefill_attention), then the batch's
        tables and lengths as batch_tables builds them."""
        if counts is not None:
            kvtier.kv_pool_batch_reserve_tokens(self.handle, list(sids), list(counts), block_tables,
                                                max_blocks, seq_lens, stream)
            return
        kvtier.kv_pool_batch_reserve(self.handle, list(sids), block_tables, max_blocks, seq_lens,
                                     stream)

    def prefetch(self, next_sids, busy=(), stream=None) -> None:
        """Fetch the next step's evicted blocks ahead of it (residency mode),
        victims outside next_sids and busy (the step still being decoded)."""
        kvtier.kv_pool_prefetch(self.handle, list(next_sids), list(busy), stream)

    def session_block_table_device(self, sid: int) -> tuple[int, int]:
        """(device address of the session's table row, logical blocks)."""
        return kvtier.session_block_table_device(self.handle, sid)

    def decode_attention(self, layer: int, q, block_tables, seq_lens, B: int, max_blocks: int,
                         scale: float, out, stream=None, overlap_previous: bool = False) -> None:
        """out: fp32, or bf16 (then the result is rounded to nearest even)."""
        import torch
        flags = (kvtier.KV_DECODE_OVERLAP_PREVIOUS if overlap_previous else 0) | \
            (kvtier.KV_DECODE_OUT_BF16 if getattr(out, "dtype", None) == torch.bfloat16 else 0)
        if flags:
            kvtier.decode_attention_ex(self.handle, layer, q, block_tables, seq_lens, B,
                                       max_blocks, scale, out, flags, stream)
        else:
            kvtier.decode_attention(self.handle, layer, q, block_tables, seq_lens, B, max_blocks,
                                    scale, out, stream)

    def decode_append_attention(self, layer: int, q, k_new, v_new, block_tables, seq_lens, B: int,
                                max_blocks: int, scale: float, out, stream=None,
                                overlap_previous: bool = False) -> None:
        """k_new, v_new: device bf16 [B][Hkv][D] (leading [L] for layer -1), the
        token at seq_lens[b] - 1 of each row, written to the pool and attended to."""
        import torch
        flags = (kvtier.KV_DECODE_OVERLAP_PREVIOUS if overlap_previous else 0) | \
            (kvtier.KV_DECODE_OUT_BF16 if getattr(out, "dtype", None) == torch.bfloat16 else 0)
        kvtier.decode_append_attention(self.handle, layer, q, k_new, v_new, block_tables, seq_lens,
                                       B, max_blocks, scale, out, flags, stream)

    def _turn(self, q, k, v, out, cu, tables, lens, B, max_blocks):
        """(token strides of q and of k and v, tokens, flags) of a call on packed tokens, checked: all
        on the pool's device; q, k and v bf16 [N][heads][D], heads contiguous, any token stride (k and
        v the same) but 0, which tokens that share storage have and which the library takes for
        contiguous rows; offsets, tables and lengths int32, contiguous, as long as the call reads."""
        total, D = q.shape[0], self.D
        kv_shape = (total, self.Hkv, D)
        q_stride, k_stride, v_stride = q.stride(), k.stride(), v.stride()
        # (What a single token or head has for a stride means nothing.)
        if q.dtype is not self._bf16 or k.dtype is not self._bf16 or v.dtype is not self._bf16 or \
                q.shape != (total, self.Hq, D) or k.shape != kv_shape or v.shape != kv_shape or \
                q_stride[2] != 1 or k_stride[2] != 1 or v_stride[2] != 1 or (q_stride[1] != D and self.Hq > 1) or \
                (self.Hkv > 1 and (k_stride[1] != D or v_stride[1] != D)) or \
                (total > 1 and (k_stride[0] != v_stride[0] or q_stride[0] == 0 or k_stride[0] == 0)):
            raise ValueError(f"need bf16 q [{total}][{self.Hq}][{D}], k and v {list(kv_shape)} with contiguous heads "
                             "and one token stride for k and v (not 0), got " +
                             ", ".join(f"{x.dtype} {tuple(x.shape)} strides {x.stride()}" for x in (q, k, v)))
        if out.shape != q.shape or not out.is_contiguous() or out.dtype not in self._out_flags:
            raise ValueError(f"out must be contiguous fp32 or bf16 [{total}][{self.Hq}][{D}]")
        i32, index = self._i32, self._index
        if cu.dtype is not i32 or tables.dtype is not i32 or lens.dtype is not i32 or cu.numel() <= B or \
                tables.numel() < B * max_blocks or lens.numel() < B or not cu.is_contiguous() or \
                not tables.is_contiguous() or not lens.is_contiguous():
            raise ValueError(f"need contiguous int32 offsets [{B + 1}], block tables [{B}][{max_blocks}] and lengths "
                             f"[{B}], got " + ", ".join(f"{x.dtype} {tuple(x.shape)} strides {x.stride()}"
                                                        for x in (cu, tables, lens)))
        if q.get_device() != index or k.get_device() != index or v.get_device() != index or \
                out.get_device() != index or cu.get_device() != index or tables.get_device() != index or \
                lens.get_device() != index:
            raise ValueError(f"all tensors must be on the pool's device, {self.device}")
        if total < 2:
            return 0, 0, total, self._out_flags[out.dtype]
        return q_stride[0], k_stride[0], total, self._out_flags[out.dtype]

    def prefill_attention(self, layer: int, q, k_new, v_new, cu_new, block_tables, seq_lens, B: int,
                          max_blocks: int, scale: float, out, stream=None) -> None:
        """Causal attention of a turn's new tokens (or whole prompts), packed: session b has rows
        cu_new[b]..cu_new[b+1]-1 of q [N][Hq][D] and k_new, v_new [N][Hkv][D] (bf16, any token
        stride, so views of one projection will do), the newest of its seq_lens[b] tokens; K and V
        go into the slots that batch_reserve(counts=...) allocated. out: fp32 or bf16."""
        q_stride, kv_stride, total, flags = self._turn(q, k_new, v_new, out, cu_new, block_tables, seq_lens, B,
                                                       max_blocks)
        rc = self._prefill(self.handle, layer, q.data_ptr(), q_stride, k_new.data_ptr(),
                           v_new.data_ptr(), kv_stride, cu_new.data_ptr(), total,
                           block_tables.data_ptr(), seq_lens.data_ptr(), B, max_blocks, scale,
                           out.data_ptr(), flags, kvtier._stream(stream))
        if rc:
            kvtier.raise_last(rc, "prefill_attention")

    def tree_attention(self, layer: int, q, k_draft, v_draft, ancestors, cu_draft, block_tables,
                       seq_lens, B: int, max_blocks: int, scale: float, out, stream=None) -> None:
        """Attention of drafted tokens (at most 64 per session, packed by cu_draft) over the
        session's seq_lens[b] cached tokens and the drafts in ancestors [N] (64-bit masks over the
        session's own drafts). Nothing is written to the pool."""
        q_stride, kv_stride, total, flags = self._turn(q, k_draft, v_draft, out, cu_draft, block_tables, seq_lens, B,
                                                       max_blocks)
        if ancestors.numel() != total or ancestors.dtype not in self._masks or not ancestors.is_contiguous() or \
                ancestors.get_device() != self._index:
            raise ValueError("need one contiguous 64-bit integer mask per draft, on the pool's device")
        rc = self._tree(self.handle, layer, q.data_ptr(), q_stride, k_draft.data_ptr(),
                        v_draft.data_ptr(), kv_stride, ancestors.data_ptr(), cu_draft.data_ptr(), total,
                        block_tables.data_ptr(), seq_lens.data_ptr(), B, max_blocks, scale,
                        out.data_ptr(), flags, kvtier._stream(stream))
        if rc:
            kvtier.raise_last(rc, "tree_attention")

    # attention over a part of the cache --------------------------------------------
    def new_bounds(self):
        """A buffer for the bounds of all blocks' keys (block_bounds), zeros."""
        import torch
        return torch.zeros(self.bounds_bytes, dtype=torch.int8, device=self.device)

    def bounds_views(self, bounds):
        """A buffer's int8 codes [L][Hkv][NB][2][D] (largest, smallest) and bf16 steps [L][Hkv][NB]
        (views); bound = code * step."""
        import torch
        shape = (self.L, self.Hkv, self.num_hot_blocks)
        n = self.L * self.Hkv * self.num_hot_blocks
        return (bounds[:n * 2 * self.D].view(*shape, 2, self.D),
                bounds[n * 2 * self.D:].view(torch.bfloat16).view(shape))

    def _rows(self, tables, lens, B, max_blocks, since=None):
        """Block tables, lengths and (or None) another int32 [B] of a call, checked."""
        i32, index = self._i32, self._index
        if tables.dtype is i32 and lens.dtype is i32 and tables.numel() >= B * max_blocks and lens.numel() >= B and \
                tables.is_contiguous() and lens.is_contiguous() and tables.get_device() == index == lens.get_device() \
                and (since is None or (since.dtype is i32 and since.numel() >= B and since.is_contiguous() and
                                       since.get_device() == index)):
            return
        raise ValueError(f"need contiguous int32 block tables [{B}][{max_blocks}] and lengths [{B}] on the pool's device, "
                         f"{self.device}, got " + ", ".join(f"{x.dtype} {tuple(x.shape)} strides {x.stride()}"
                                                            for x in (tables, lens, since) if x is not None))

    def _heads(self, x, B, heads, name):
        """The row stride of bf16 [B][heads][D] with contiguous heads, checked (0: one row)."""
        stride, D = x.stride(), self.D
        if x.dtype is not self._bf16 or x.shape != (B, heads, D) or stride[2] != 1 or \
                (heads > 1 and stride[1] != D) or (B > 1 and stride[0] == 0) or x.get_device() != self._index:
            raise ValueError(f"{name}: need bf16 [{B}][{heads}][{D}] with contiguous heads and a row stride that is "
                             f"not 0 on the pool's device, {self.device}, got {x.dtype} {tuple(x.shape)} strides {stride}")
        return stride[0] if B > 1 else 0

    def _list(self, selected, B):
        """Entries per row and head of a selection [B][Hkv][top], checked."""
        shape = selected.shape
        if selected.dtype is not self._i32 or len(shape) != 3 or shape[0] != B or shape[1] != self.Hkv or \
                not selected.is_contiguous() or selected.get_device() != self._index:
            raise ValueError(f"selected must be contiguous int32 [{B}][{self.Hkv}][top] on the pool's device, "
                             f"got {selected.dtype} {tuple(shape)} strides {selected.stride()}")
        return shape[2]

    def _whole_bounds(self, bounds):
        if bounds.numel() * bounds.element_size() < self.bounds_bytes or not bounds.is_contiguous() or \
                bounds.get_device() != self._index:
            raise ValueError(f"bounds must be a contiguous buffer of {self.bounds_bytes} bytes on the pool's "
                             "device (new_bounds)")

    def block_bounds(self, layer: int, block_tables, seq_lens, B: int, max_blocks: int, bounds, since=None,
                     stream=None) -> None:
        """Bounds of the keys of the rows' blocks that hold tokens from since[b] on (all without it), of
        one layer or (-1) all."""
        self._rows(block_tables, seq_lens, B, max_blocks, since)
        self._whole_bounds(bounds)
        kvtier.kv_pool_block_bounds(self.handle, layer, block_tables, seq_lens, since, B, max_blocks, bounds,
                                    stream)

    def select_blocks(self, layer: int, q, bounds, block_tables, seq_lens, B: int, max_blocks: int, selected,
                      first: int = 1, last: int = 1, scores=None, stream=None) -> None:
        """The `top` blocks of each row and KV head that q's [B][Hq][D] heads (any row stride) may need
        most, the row's `first` first and `last` last ones among them, into selected int32
        [B][Hkv][top]: ascending, -1 behind. scores: fp32 [B][Hkv][max_blocks] or None."""
        rc = self._calls and self._calls.select_blocks(layer, q, bounds, block_tables, seq_lens, B, max_blocks, selected, first,
                                                       last, scores, stream)
        if rc is None:                   # without the module, or something unusual about an argument
            self._rows(block_tables, seq_lens, B, max_blocks)
            self._whole_bounds(bounds)
            top, q_stride, at = self._list(selected, B), self._heads(q, B, self.Hq, "q"), None
            if scores is not None:
                at = scores.data_ptr()
                if scores.dtype is not self._f32 or scores.shape != (B, self.Hkv, max_blocks) or \
                        not scores.is_contiguous() or scores.get_device() != self._index:
                    raise ValueError(f"scores must be contiguous fp32 [{B}][{self.Hkv}][{max_blocks}] on the pool's device")
            rc = self._select(self.handle, layer, q.data_ptr(), q_stride, bounds.data_ptr(),
                              block_tables.data_ptr(), seq_lens.data_ptr(), B, max_blocks, first, last, top,
                              selected.data_ptr(), at, kvtier._stream(stream))
        if rc:
            kvtier.raise_last(rc, "select_blocks")

    def sparse_attention(self, layer: int, q, selected, block_tables, seq_lens, B: int, max_blocks: int,
                         scale: float, out, k_new=None, v_new=None, stream=None) -> None:
        """Attention of one new token per session over the listed blocks of each KV head (selected, as
        select_blocks leaves it, or any list). k_new, v_new: bf16 [B][Hkv][D] (any row stride), the
        token at seq_lens[b] - 1, written to its pool slot as well. out: fp32 or bf16 [B][Hq][D]."""
        rc = self._calls and self._calls.sparse_attention(layer, q, selected, block_tables, seq_lens, B, max_blocks, scale, out,
                                                          k_new, v_new, stream)
        if rc is None:
            self._rows(block_tables, seq_lens, B, max_blocks)
            top, q_stride, kv_stride, k, v = self._list(selected, B), self._heads(q, B, self.Hq, "q"), 0, None, None
            if (k_new is None) != (v_new is None):
                raise ValueError("k_new and v_new come together")
            if k_new is not None:
                kv_stride = self._heads(k_new, B, self.Hkv, "k_new")
                if self._heads(v_new, B, self.Hkv, "v_new") != kv_stride:
                    raise ValueError("k_new and v_new need the same row stride")
                k, v = k_new.data_ptr(), v_new.data_ptr()
            if out.shape != (B, self.Hq, self.D) or not out.is_contiguous() or out.dtype not in self._out_flags or \
                    out.get_device() != self._index:
                raise ValueError(f"out must be contiguous fp32 or bf16 [{B}][{self.Hq}][{self.D}] on the pool's device")
            rc = self._sparse(self.handle, layer, q.data_ptr(), q_stride, k, v, kv_stride, selected.data_ptr(), top,
                              block_tables.data_ptr(), seq_lens.data_ptr(), B, max_blocks, scale, out.data_ptr(),
                              self._out_flags[out.dtype], kvtier._stream(stream))
        if rc:
            kvtier.raise_last(rc, "sparse_attention")

    # pages of sessions ---------------------------------------------------------------
    def session_fork(self, sid: int, n: int = 1, tokens: int | None = None, max_tokens: int | None = None,
                     stream=None) -> list[int]:
        """n sessions of max_tokens (the parent's capacity) that begin with its first `tokens` (all):
        full blocks are shared, the partly filled one copied (residency mode: all copied)."""
        if tokens is None or max_tokens is None:
            info = kvtier.session_info(self.handle, sid)
            tokens = info.tokens if tokens is None else tokens
            max_tokens = info.capacity if max_tokens is None else max_tokens
        return kvtier.session_fork(self.handle, sid, tokens, max_tokens, n, stream)

    def session_truncate(self, sid: int, tokens: int, stream=None) -> None:
        """Forget all but the first `tokens` tokens."""
        kvtier.session_truncate(self.handle, sid, tokens, stream)

    def session_compact(self, sid: int, keep, prefix: int = 0, stream=None) -> None:
        """Keep the first `prefix` tokens and, behind them, those that `keep` names: ascending positions,
        int32 [n] for all heads, or [L][Hkv][n] (expanded dimensions will do)."""
        if keep.dtype is not self._i32 or keep.get_device() != self._index or \
                (keep.dim() != 1 and (keep.dim() != 3 or keep.shape[:2] != (self.L, self.Hkv))) or \
                (keep.shape[-1] > 1 and keep.stride(-1) != 1):
            raise ValueError(f"keep must be int32 [n] or [{self.L}][{self.Hkv}][n] with contiguous lists on the pool's "
                             f"device, got {keep.dtype} {tuple(keep.shape)} strides {keep.stride()}")
        strides = (0, 0) if keep.dim() == 1 else (keep.stride(0) if self.L > 1 else 0,
                                                  keep.stride(1) if self.Hkv > 1 else 0)
        kvtier.session_compact(self.handle, sid, keep, *strides, keep.shape[-1], prefix, stream)

    def shuffle_free(self, seed: int) -> None:
        kvtier.kv_pool_shuffle_free(self.handle, seed)

    def free_list(self) -> list[int]:
        return kvtier.kv_pool_free_list(self.handle)

    def stats(self) -> dict:
        return kvtier.kv_pool_get_stats(self.handle)

    def check_device(self) -> int:
        return kvtier.kv_pool_check_device(self.handle)
