"""Device-buffer bookkeeping around the C-ABI calls for one compaction event.

PyTorch is used for device memory and streams only; every step of the path
(planning, prefill, append, decode, merge) runs inside libcompact_attn.
"""
from __future__ import annotations

from typing import Optional, Sequence

import numpy as np
import torch

from . import binding as B


def bits_to_tensor(bits: np.ndarray, device=None, pin: bool = False) -> torch.Tensor:
    """uint16 bf16 bit patterns -> torch.bfloat16 tensor (same bits)."""
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).view(torch.bfloat16)
    if pin:
        t = t.pin_memory()
    return t.to(device, non_blocking=pin) if device is not None else t


def tensor_to_bits(t: torch.Tensor) -> np.ndarray:
    """torch.bfloat16 tensor -> uint16 bit patterns on the host."""
    return t.detach().contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


class CompactionSession:
    """One history cut into blocks, one summary sequence per block (paper, Section 4).

    Owns the plan handle, the device index buffer, the K/V page pools and the
    decode workspace.  All calls are enqueued on the current torch stream of
    `device` unless a stream is given.  With kv_bits = 8 the cache holds e4m3 codes with a scale per page, head and K or
    V (half the bytes of a decode step, twice the tokens in a pool of given size); append, decode, decode_append and
    append_prefill are then the calls of that cache, and lengths live on the device.  What differs from the bf16 cache:
      - `lens` is another tensor after every append and every fused step, and the one before is overwritten by the next:
        read it anew, and let a captured graph that is replayed as a loop hold an even number of such calls;
      - a block without room for its rows is left out and its length stays; status() says so (CPA_ENOSPC), where the bf16
        cache's call raises;
      - the decode's split is made on the device, pages_per_split is not used;
      - decode_append_steps makes one call per step.
    """

    def __init__(self, block_lens: Sequence[int], max_new_tokens: int, num_q_heads: int,
                 num_kv_heads: int, head_dim: int, free_pages: Sequence[int], num_pages: int,
                 scale: Optional[float] = None, device: str = "cuda:0", pages_per_split: int = 0,
                 poison_pools: bool = False, page_size: int = 16, q_tile_rows: int = 0,
                 prefix_lens: Optional[Sequence[int]] = None, shared_pages: Optional[Sequence[int]] = None,
                 pools=None, num_sms: int = 0, chunk_tokens: int = 0, decode_sms: int = 0, dynamic_pages: bool = False,
                 decode_steps_per_chunk: int = 1, kv_bits: int = 16):
        if kv_bits not in (8, 16):
            raise ValueError(f"kv_bits is 8 or 16, not {kv_bits}")
        if kv_bits == 8 and (prefix_lens is not None or chunk_tokens or dynamic_pages or pools is not None):
            raise ValueError("a cache of 8 bits takes whole blocks: no cached prefix, chunks, pages on demand or shared pools")
        self.kv_bits = kv_bits
        self.device = torch.device(device)
        self.Hq, self.Hkv, self.d, self.P = num_q_heads, num_kv_heads, head_dim, page_size
        self.B = len(block_lens)
        self.block_lens = np.asarray(block_lens, dtype=np.int32)
        self.scale = float(scale if scale is not None else head_dim ** -0.5)
        props = torch.cuda.get_device_properties(self.device)
        # num_sms is the SM budget of this event: the persistent prefill grid and the decode wave are sized
        # from it (all SMs unless the caller wants to leave room for other work on the device)
        self.cfg = B.cpa_config(num_q_heads, num_kv_heads, head_dim, page_size, self.scale, q_tile_rows,
                                pages_per_split, num_sms or props.multi_processor_count)
        self.prefix_aware = prefix_lens is not None
        self.chunk_tokens = chunk_tokens
        self.dynamic_pages = dynamic_pages
        if dynamic_pages:       # no pages reserved for the summaries: blocks draw from a common reserve as they grow
            assert prefix_lens is None and not chunk_tokens
            self.plan = B.cpa_plan_create_dynamic(self.cfg, self.block_lens, max_new_tokens, free_pages)
        elif chunk_tokens and self.prefix_aware:   # both: cached history prefix, own tokens in chunks
            self.plan = B.cpa_plan_create_prefix_chunked(self.cfg, self.block_lens, prefix_lens, shared_pages,
                                                         max_new_tokens, chunk_tokens, free_pages, decode_sms,
                                                         decode_steps_per_chunk)
        elif chunk_tokens:      # prefill in chunks, mixed with the decode of blocks that are past their prompt
            self.plan = B.cpa_plan_create_chunked(self.cfg, self.block_lens, max_new_tokens, chunk_tokens, free_pages,
                                                  decode_sms, decode_steps_per_chunk)
        elif self.prefix_aware:   # the paper's layout: cached history prefix + own tokens per worker
            self.plan = B.cpa_plan_create_prefix(self.cfg, self.block_lens, prefix_lens, shared_pages,
                                                 max_new_tokens, free_pages)
        else:
            self.plan = B.cpa_plan_create(self.cfg, self.block_lens, max_new_tokens, free_pages)
        self.total_tokens = B.cpa_plan_param(self.plan, B.PARAM_TOTAL_TOKENS)
        nbytes = B.cpa_plan_param(self.plan, B.PARAM_INDEX_BYTES)
        self.index_buf = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        pool_shape = (num_pages, num_kv_heads, page_size, head_dim)
        if kv_bits == 8:
            self._init_q8(max_new_tokens, free_pages, num_pages, poison_pools)
        elif pools is not None:   # pools that already hold a cached history (shared with another session)
            self.k_pool, self.v_pool = pools
            assert tuple(self.k_pool.shape) == pool_shape and tuple(self.v_pool.shape) == pool_shape
        elif poison_pools:   # unused slots hold NaN: the kernels must mask by index, not by value
            self.k_pool = torch.full(pool_shape, float("nan"), dtype=torch.bfloat16, device=self.device)
            self.v_pool = torch.full(pool_shape, float("nan"), dtype=torch.bfloat16, device=self.device)
        else:  # no initialisation needed: slots are masked by index until they are written
            self.k_pool = torch.empty(pool_shape, dtype=torch.bfloat16, device=self.device)
            self.v_pool = torch.empty(pool_shape, dtype=torch.bfloat16, device=self.device)
        ws = (B.cpa_decode_q8_workspace_bytes(self.cfg) if kv_bits == 8
              else B.cpa_plan_param(self.plan, B.PARAM_DECODE_WORKSPACE_BYTES))
        self.workspace = torch.empty(max(ws, 256), dtype=torch.uint8, device=self.device)
        self._check(B.cpa_plan_upload(self.plan, self.index_buf, nbytes, self._stream()), "cpa_plan_upload")

    # -- the cache in 8 bits --------------------------------------------------
    def _init_q8(self, max_new_tokens: int, free_pages, num_pages: int, poison: bool) -> None:
        """Pool and scales of the 8-bit cache, and its tables, which the device builds from the block lengths with the
        plan's own rules (so that page lists and slots are the plan's)."""
        self.k_pool = self.v_pool = None
        free = torch.as_tensor(np.ascontiguousarray(free_pages, dtype=np.int32), device=self.device)
        self.dims = B.cpa_table_dims(self.B, max_new_tokens, num_pages, max(1, self.param(B.PARAM_PAGES_USED)),
                                     self.total_tokens)
        nbytes = B.cpa_tables_bytes(self.cfg, self.dims)
        if nbytes < 0:
            raise B.CpaError(nbytes, "cpa_tables_bytes")
        self.tables = torch.empty(nbytes, dtype=torch.uint8, device=self.device)
        shape = (num_pages, self.Hkv, 2, self.P, self.d)
        if poison:   # unused slots hold NaN: the kernels must mask by index, not by value
            self.kv_pool = torch.full(shape, 0x7F, dtype=torch.uint8, device=self.device).view(torch.float8_e4m3fn)
            self.kv_scales = torch.full(shape[:3], float("nan"), device=self.device)
        else:
            self.kv_pool = torch.empty(shape, dtype=torch.float8_e4m3fn, device=self.device)
            self.kv_scales = torch.empty(shape[:3], device=self.device)
        # cached tokens per block before and after a step: every call reads one array and writes the other
        self.lens = torch.zeros(self.B, dtype=torch.int32, device=self.device)
        self._lens_next = torch.empty_like(self.lens)
        lens = torch.as_tensor(self.block_lens, device=self.device)
        self._q8("cpa_tables_build", lens, free, len(free_pages), tables_last=True)
        at = B.cpa_tables_offset(self.cfg, self.dims, B.ARR_CU_SEQLENS)
        self._cu = self.tables[at:at + 4 * (self.B + 1)].view(torch.int32)

    def _q8(self, what: str, *args, tables_last: bool = False) -> None:
        args = (*args, self.tables) if tables_last else (self.tables, *args)
        if torch.cuda.current_device() == self.lens.device.index:
            rc = getattr(B, what)(self.cfg, self.dims, *args, self._stream())
        else:
            with torch.cuda.device(self.device):
                rc = getattr(B, what)(self.cfg, self.dims, *args, self._stream())
        self._check(rc, what)

    def _q8_rows(self, heads: int, rows: int, **tensors) -> None:
        """Refuses tensors that the kernels would misread: they take packed bf16 [rows, heads, head_dim]."""
        for name, t in tensors.items():
            if (t.dtype != torch.bfloat16 or t.device != self.lens.device or t.shape != (rows, heads, self.d) or
                    not t.is_contiguous()):
                raise ValueError(f"{name}: contiguous bf16 [{rows}, {heads}, {self.d}] on {self.lens.device} is wanted, "
                                 f"not {t.dtype} {tuple(t.shape)} on {t.device}")

    def _swap_lens(self) -> None:
        self.lens, self._lens_next = self._lens_next, self.lens

    def _append_q8(self, k: torch.Tensor, v: torch.Tensor, cu: Optional[torch.Tensor], rows: int) -> None:
        self._q8_rows(self.Hkv, rows, k=k, v=v)
        self._q8("cpa_kv_append_q8", k, v, cu, rows, self.lens, self._lens_next, self.kv_pool, self.kv_scales)
        self._swap_lens()

    def _decode_q8(self, q: torch.Tensor, k_new, v_new, active, out: Optional[torch.Tensor]) -> torch.Tensor:
        if out is None:
            out = torch.empty_like(q)
        self._q8_rows(self.Hq, self.B, q=q, out=out)
        if active is not None and (active.dtype != torch.int32 or active.device != self.lens.device or
                                   active.shape != (self.B,) or not active.is_contiguous()):
            raise ValueError(f"active: contiguous int32 [{self.B}] on {self.lens.device} is wanted")
        if k_new is None:
            self._q8("cpa_decode_q8", q, self.lens, active, self.kv_pool, self.kv_scales, out, self.workspace)
            return out
        self._q8_rows(self.Hkv, self.B, k_new=k_new, v_new=v_new)
        self._q8("cpa_decode_append_q8", q, k_new, v_new, self.lens, self._lens_next, active, self.kv_pool, self.kv_scales,
                 out, self.workspace)
        self._swap_lens()
        return out

    def read_cache(self, first: Sequence[int], counts: Sequence[int]):
        """K and V rows [sum(counts), Hkv, d] in bf16 of positions first[b] .. first[b] + counts[b] of every block of an
        8-bit cache (to hand a history on to calls that take bf16 rows).  The range has to lie in the block's pages;
        positions behind the block's tokens (`lens`, which live on the device and are not looked at here) have no
        defined value."""
        self._only(8, "read_cache")
        first, counts = np.asarray(first), np.asarray(counts)
        if any(a.shape != (self.B,) or a.dtype.kind not in "iu" or (a < 0).any() or (a > 2 ** 31).any() for a in (first, counts)):
            raise ValueError(f"first and counts: {self.B} whole numbers each, none negative or beyond int32")
        first, counts = first.astype(np.int64), counts.astype(np.int64)
        room = (self.block_lens.astype(np.int64) + self.dims.max_new_tokens + self.P - 1) // self.P * self.P
        if (first > room).any() or (counts > room - first).any():
            b = int(np.argmax((first > room) | (counts > room - first)))
            raise ValueError(f"block {b}: {counts[b]} positions from {first[b]} on leave its pages, which hold {room[b]}")
        cu = torch.as_tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), device=self.device)
        rows = int(counts.sum())
        k, v = (torch.empty((rows, self.Hkv, self.d), dtype=torch.bfloat16, device=self.device) for _ in range(2))
        self._q8("cpa_kv_read_q8", torch.as_tensor(first.astype(np.int32), device=self.device), cu, rows, self.kv_pool,
                 self.kv_scales, k, v)
        return k, v

    def _only(self, bits: int, what: str) -> None:
        if self.kv_bits != bits:
            raise B.CpaError(B.CPA_EUNSUPPORTED, f"{what} on a cache of {self.kv_bits} bits")

    # -- helpers ------------------------------------------------------------
    def _stream(self) -> int:
        return int(torch.cuda.current_stream(self.device).cuda_stream)

    @staticmethod
    def _check(rc: int, where: str) -> None:
        if rc != B.CPA_OK:
            raise B.CpaError(rc, where)

    def export(self, which: int) -> np.ndarray:
        if self.kv_bits == 8 and which == B.ARR_SEQ_LENS:   # (the plan does not follow the 8-bit cache)
            return self.lens.cpu().numpy()
        return B.cpa_plan_export(self.plan, which)

    def param(self, which: int) -> int:
        return B.cpa_plan_param(self.plan, which)

    # -- the hot path -------------------------------------------------------
    def prefill(self, q: torch.Tensor, k: torch.Tensor, v: torch.Tensor,
                out: Optional[torch.Tensor] = None, variant: Optional[int] = None) -> torch.Tensor:
        """Causal attention of every block over itself; q/out [tokens,Hq,d], k/v [tokens,Hkv,d]."""
        if out is None:
            out = torch.empty_like(q)
        if self.prefix_aware:
            self._check(B.cpa_prefill_prefix(self.plan, q, k, v, self.k_pool, self.v_pool, out, self._stream()),
                        "cpa_prefill_prefix")
        elif variant is None:
            self._check(B.cpa_prefill(self.plan, q, k, v, out, None, self._stream()), "cpa_prefill")
        else:
            self._check(B.cpa_prefill_variant(self.plan, q, k, v, out, self._stream(), variant),
                        "cpa_prefill_variant")
        return out

    def append_prefill(self, k: torch.Tensor, v: torch.Tensor) -> None:
        """Store the prefill K/V of every block in its pages."""
        if self.kv_bits == 8:
            return self._append_q8(k, v, self._cu, self.total_tokens)
        self._check(B.cpa_kv_append(self.plan, k, v, self.block_lens, self.k_pool, self.v_pool,
                                    self._stream()), "cpa_kv_append")

    def append(self, k_new: torch.Tensor, v_new: torch.Tensor, new_lens=None) -> None:
        """One token per block (new_lens None) or new_lens[b] tokens per block."""
        if self.kv_bits == 8:
            if new_lens is None:
                return self._append_q8(k_new, v_new, None, self.B)
            counts = np.asarray(new_lens, dtype=np.int64)
            if counts.shape != (self.B,) or (counts < 0).any():
                raise B.CpaError(B.CPA_EINVAL, "cpa_kv_append_q8")
            cu = torch.as_tensor(np.concatenate([[0], np.cumsum(counts)]).astype(np.int32), device=self.device)
            return self._append_q8(k_new, v_new, cu, int(counts.sum()))
        self._check(B.cpa_kv_append(self.plan, k_new, v_new, new_lens, self.k_pool, self.v_pool,
                                    self._stream()), "cpa_kv_append")

    def decode(self, q: torch.Tensor, out: Optional[torch.Tensor] = None, active=None) -> torch.Tensor:
        """q/out [B,Hq,d]: newest token of every block over that block's cache.  `active` (8-bit cache only): device
        int32 [B], blocks whose flag is 0 sit out."""
        if self.kv_bits == 8:
            return self._decode_q8(q, None, None, active, out)
        if active is not None:
            raise B.CpaError(B.CPA_EUNSUPPORTED, "active on a cache of 16 bits")
        if out is None:
            out = torch.empty_like(q)
        self._check(B.cpa_decode(self.plan, q, self.k_pool, self.v_pool, out, self.workspace,
                                 self._stream()), "cpa_decode")
        return out

    def decode_append(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                      out: Optional[torch.Tensor] = None, active=None) -> torch.Tensor:
        """One decode step with its append fused in (same result as append() then decode()).  `active` as for decode."""
        if self.kv_bits == 8:
            return self._decode_q8(q, k_new, v_new, active, out)
        if active is not None:
            raise B.CpaError(B.CPA_EUNSUPPORTED, "active on a cache of 16 bits")
        if out is None:
            out = torch.empty_like(q)
        self._check(B.cpa_decode_append(self.plan, q, k_new, v_new, self.k_pool, self.v_pool, out,
                                        self.workspace, self._stream()), "cpa_decode_append")
        return out

    def decode_append_steps(self, q: torch.Tensor, k_new: torch.Tensor, v_new: torch.Tensor,
                            out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """q/out [n,B,Hq,d], k_new/v_new [n,B,Hkv,d]: n consecutive fused decode steps (enqueued by one call of the library
        for the bf16 cache, by one call per step for the 8-bit cache)."""
        if out is None:
            out = torch.empty_like(q)
        if self.kv_bits == 8:
            if not q.shape[0] == k_new.shape[0] == v_new.shape[0] == out.shape[0]:
                raise ValueError(f"steps: {q.shape[0]} of q, {k_new.shape[0]} of k_new, {v_new.shape[0]} of v_new, {out.shape[0]} of out")
            for t in range(q.shape[0]):
                self._decode_q8(q[t], k_new[t], v_new[t], None, out[t])
            return out
        assert q.is_contiguous() and k_new.is_contiguous() and v_new.is_contiguous() and out.is_contiguous()
        self._check(B.cpa_decode_append_steps(self.plan, q, k_new, v_new, self.k_pool, self.v_pool, out,
                                              self.workspace, q.shape[0], self._stream()), "cpa_decode_append_steps")
        return out

    def step_mixed(self, step: int, q, k, v, out, q_dec=None, k_new=None, v_new=None, out_dec=None) -> None:
        """Step `step` of a chunked plan: the chunk that starts at this step, if any (rows of the whole-event
        tensors q/k/v/out), beside one decode token of the blocks whose turn it is."""
        self._only(16, "step_mixed")
        self._check(B.cpa_step_mixed(self.plan, step, q, k, v, out, q_dec, k_new, v_new, out_dec, self.k_pool,
                                     self.v_pool, self.workspace, self._stream()), "cpa_step_mixed")

    def event_from_host(self, h_q, h_k, h_v, h_out, h_q_dec=None, h_k_dec=None, h_v_dec=None, h_out_dec=None,
                        stage: Optional[torch.Tensor] = None) -> torch.Tensor:
        """The whole event from host tensors (page-locked ones overlap with the kernels): prompts [tokens,H,d],
        decode steps' inputs [T,B,H,d]; h_out / h_out_dec are written.  Everything is enqueued on the current
        stream; synchronise it before reading the outputs.  Returns the device staging buffer (uint8,
        PARAM_HOST_STAGE_BYTES), which a later event of the same shape may be given again."""
        self._only(16, "event_from_host")
        need = self.param(B.PARAM_HOST_STAGE_BYTES)
        if stage is None:
            stage = torch.empty(max(need, 256), dtype=torch.uint8, device=self.device)
        assert stage.numel() >= need and stage.device == self.device
        self._check(B.cpa_event_host(self.plan, h_q, h_k, h_v, h_out, h_q_dec, h_k_dec, h_v_dec, h_out_dec, stage,
                                     self.k_pool, self.v_pool, self.workspace, self._stream()), "cpa_event_host")
        return stage

    def step_mixed_range(self, first_step: int, num_steps: int, q, k, v, out, q_dec=None, k_new=None, v_new=None,
                         out_dec=None) -> None:
        """Steps first_step .. first_step + num_steps - 1 of a chunked plan by one call; the decode tensors are
        [num_steps, B, H, d], slice i for step first_step + i."""
        self._only(16, "step_mixed_range")
        self._check(B.cpa_step_mixed_range(self.plan, first_step, num_steps, q, k, v, out, q_dec, k_new, v_new,
                                           out_dec, self.k_pool, self.v_pool, self.workspace, self._stream()),
                    "cpa_step_mixed_range")

    def decode_append_dynamic(self, q, k_new, v_new, active=None, out=None):
        """One decode step of a plan with pages on demand; `active` is a device int32 [B] tensor of stop flags."""
        self._only(16, "decode_append_dynamic")
        if out is None:
            out = torch.empty_like(q)
        self._check(B.cpa_decode_append_dynamic(self.plan, q, k_new, v_new, active, self.k_pool, self.v_pool, out,
                                                self.workspace, self._stream()), "cpa_decode_append_dynamic")
        return out

    def release(self, active) -> None:
        """Blocks whose flag is 0 give their pages back to the reserve."""
        self._check(B.cpa_release_blocks(self.plan, active, self._stream()), "cpa_release_blocks")

    def sync(self) -> None:
        """Read the device's lengths, page table and reserve back into the plan's host copies."""
        self._check(B.cpa_plan_sync(self.plan, self._stream()), "cpa_plan_sync")

    def status(self) -> int:
        rc = B.cpa_plan_status(self.plan, self._stream())
        return rc if rc or self.kv_bits == 16 else B.cpa_tables_status(self.tables, self._stream())

    def close(self) -> None:
        if self.plan:
            torch.cuda.synchronize(self.device)
            B.cpa_plan_destroy(self.plan)
            self.plan = None

    def __del__(self):  # pragma: no cover
        try:
            self.close()
        except Exception:
            pass
