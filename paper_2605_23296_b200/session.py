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


def _with_index(device) -> torch.device:
    """The device by its number: "cuda" alone would follow the current device from call to call."""
    d = torch.device(device)
    return torch.device("cuda", torch.cuda.current_device()) if d.type == "cuda" and d.index is None else d


class Rotary:
    """Rotary positions of one configuration on one device: the frequencies, computed once (cpa_rope_turns)."""

    def __init__(self, rope_dim: int, interleaved: bool = False, base: float = 10000.0, scaling: int = B.ROPE_UNSCALED,
                 factor: float = 1.0, trained_len: int = 0, fast: float = 32.0, slow: float = 1.0, amplitude: float = 1.0,
                 device: str = "cuda:0"):
        self.device = _with_index(device)
        self.cfg = B.cpa_rope_config(rope_dim, B.ROPE_INTERLEAVED if interleaved else B.ROPE_HALF, scaling, trained_len, base, factor,
                                     fast, slow, amplitude)
        self.turns = torch.from_numpy(B.cpa_rope_turns(self.cfg).view(np.int64)).to(self.device)

    def turn(self, positions: torch.Tensor, q: torch.Tensor, k: Optional[torch.Tensor] = None, q_out: Optional[torch.Tensor] = None,
             k_out: Optional[torch.Tensor] = None, inverse: bool = False, offset: Optional[int] = None) -> None:
        """Turns the rows q [rows, heads, head_dim] and, if given, k to `positions` (int32 [rows]), in place or into q_out and
        k_out; the rotated part is a head's last rope_dim elements, or those at `offset`.  On the current stream of the device."""
        rows = q.shape[0]
        if positions.dtype != torch.int32 or positions.device != self.turns.device or positions.shape != (rows,) or not positions.is_contiguous():
            raise ValueError(f"positions: contiguous int32 [{rows}] on {self.turns.device} is wanted")
        if q.device != positions.device or (k is not None and (k.device != positions.device or k.shape[0] != rows)):
            raise ValueError(f"q and k: {rows} rows each on {positions.device} are wanted")
        args = [B.rope_rows(q, q_out, self.cfg.rope_dim, offset), None if k is None else B.rope_rows(k, k_out, self.cfg.rope_dim, offset)]
        with torch.cuda.device(self.device):
            rc = B.cpa_rope(self.cfg, self.turns, positions, rows, *args, inverse, int(torch.cuda.current_stream(self.device).cuda_stream))
        if rc != B.CPA_OK:
            raise B.CpaError(rc, "cpa_rope")


class LatentSession:
    """A compaction event of a model with latent attention: one history cut into blocks, one summary sequence per block, the
    cache one row [latent | positional key] per token for all heads.

    Owns the plan of the prompts' prefill, the tables, the pool of rows and the decode's workspace.  All calls are enqueued on
    the current torch stream of `device`.  As with CompactionSession's 8-bit cache the lengths live on the device: `lens` is
    another tensor after every append and every step (read it anew; a captured graph that is replayed as a loop holds an even
    number of such calls), and a block without room is left out, which status() reports.  `rope` turns queries and keys to
    first[b] + their place in block b; without it they are taken as they are."""

    def __init__(self, block_lens: Sequence[int], max_new_tokens: int, num_heads: int, free_pages: Sequence[int], num_pages: int,
                 latent_dim: int = 512, scale: Optional[float] = None, rope: Optional[Rotary] = None,
                 norm_weight: Optional[torch.Tensor] = None, norm_eps: float = 1e-6, first: Optional[Sequence[int]] = None,
                 device: str = "cuda:0", poison_pools: bool = False, num_sms: int = 0):
        self.device = _with_index(device)
        self.plan = None
        self.H, self.L, self.rope, self.norm_weight = num_heads, latent_dim, rope, norm_weight
        self.B = len(block_lens)
        self.block_lens = np.asarray(block_lens, dtype=np.int32)
        self.total_tokens = int(self.block_lens.sum())
        self.scale = float(scale if scale is not None else (128 + 64) ** -0.5)
        if norm_weight is not None and (norm_weight.dtype != torch.bfloat16 or norm_weight.shape != (latent_dim,) or
                                        not norm_weight.is_contiguous()):
            raise ValueError(f"norm_weight: contiguous bf16 [{latent_dim}] is wanted")
        if rope is not None and rope.cfg.rope_dim != 64:
            raise ValueError(f"rope: 64 rotated elements are wanted, not {rope.cfg.rope_dim}")
        start = np.zeros(self.B, dtype=np.int64) if first is None else np.asarray(first, dtype=np.int64)
        # (the kernels read one position per block, and add to it in 32 bits)
        if start.shape != (self.B,) or (start < -2 ** 31).any() or (start + self.block_lens + max_new_tokens > 2 ** 31 - 1).any():
            raise ValueError(f"first: {self.B} positions are wanted, one per block, which stay within 32 bits for all of its tokens")
        self.cfg = B.cpa_latent_config(num_heads, latent_dim, 64, 128, 128, 16, self.scale, norm_eps, num_sms)
        tables_cfg = B.cpa_latent_tables_config(self.cfg)
        plan_cfg = B.cpa_latent_plan_config(self.cfg)
        # The plan is there for the prefill's schedule, which reads no pages: it gets as many as there are, but not their ids, which
        # it would hold against the rows of a grouped cache (num_heads times as many as a page of this one has).
        free = np.ascontiguousarray(free_pages, dtype=np.int32)
        with torch.cuda.device(self.device):             # (whose SMs the plan counts)
            self.plan = B.cpa_plan_create(plan_cfg, self.block_lens, max_new_tokens, np.zeros_like(free))
        used = B.cpa_plan_param(self.plan, B.PARAM_PAGES_USED)
        if (free[:used] < 0).any():
            self.close()
            raise B.CpaError(B.CPA_EINVAL, "free_pages")
        self.dims = B.cpa_table_dims(self.B, max_new_tokens, num_pages, used, 0)
        on = dict(device=self.device)
        self.index_buf = torch.empty(B.cpa_plan_param(self.plan, B.PARAM_INDEX_BYTES), dtype=torch.uint8, **on)
        self.tables = torch.empty(B.cpa_tables_bytes(tables_cfg, self.dims), dtype=torch.uint8, **on)
        self.pool = torch.empty((num_pages, 16, latent_dim + 64), dtype=torch.bfloat16, **on)
        if poison_pools:   # unused slots hold NaN: the kernels must mask by index, not by value
            self.pool.fill_(float("nan"))
        self.workspace = torch.empty(B.cpa_latent_decode_workspace_bytes(self.cfg), dtype=torch.uint8, **on)
        self.lens = torch.zeros(self.B, dtype=torch.int32, **on)
        self._lens_next = torch.empty_like(self.lens)
        for name, t in (("norm_weight", norm_weight), ("rope", rope and rope.turns)):
            if t is not None and t.device != self.lens.device:
                B.cpa_plan_destroy(self.plan)
                self.plan = None
                raise ValueError(f"{name}: on {self.lens.device}, not on {t.device}")
        self.first = None if first is None else torch.as_tensor(start.astype(np.int32), **on)
        self.cu = torch.as_tensor(np.concatenate([[0], np.cumsum(self.block_lens)]).astype(np.int32), **on)
        self.positions = torch.as_tensor(np.concatenate([s + np.arange(n) for s, n in zip(start, self.block_lens)]).astype(np.int32), **on)
        lens, d_free = torch.as_tensor(self.block_lens, **on), torch.as_tensor(free, **on)
        self._call("cpa_plan_upload", self.plan, self.index_buf, self.index_buf.numel())
        self._call("cpa_tables_build", tables_cfg, self.dims, lens, d_free, len(free), self.tables)

    def _call(self, what: str, *args) -> None:
        with torch.cuda.device(self.device):
            rc = getattr(B, what)(*args, int(torch.cuda.current_stream(self.device).cuda_stream))
        if rc != B.CPA_OK:
            raise B.CpaError(rc, what)

    def _rows(self, rows: int, row: int, **tensors) -> None:
        for name, t in tensors.items():
            if (t.dtype != torch.bfloat16 or t.device != self.lens.device or t.shape != (rows, row) or
                    (t.numel() and t.stride(1) != 1)):
                raise ValueError(f"{name}: bf16 [{rows}, {row}] with whole rows on {self.lens.device} is wanted, not {t.dtype} "
                                 f"{tuple(t.shape)} on {t.device}")

    def _packed(self, **tensors) -> None:
        for name, (t, shape) in tensors.items():
            if t.dtype != torch.bfloat16 or t.device != self.lens.device or t.shape != shape or not t.is_contiguous():
                raise ValueError(f"{name}: contiguous bf16 {list(shape)} on {self.lens.device} is wanted, not {t.dtype} "
                                 f"{tuple(t.shape)} on {t.device}")

    def _rope(self):
        return (None, None) if self.rope is None else (self.rope.cfg, self.rope.turns)

    def append(self, x: torch.Tensor, counts: Optional[Sequence[int]] = None, packed: bool = False) -> Optional[torch.Tensor]:
        """New rows x [rows, latent_dim + 64] (packed block-major, any row stride), counts[b] per block or one each: normalised,
        turned and stored behind the blocks' tokens.  With `packed` the stored rows come back too.  (Their queries meet the
        cache through decode() and step() alone, a token per block at a time; prefill() is over the prompts themselves.)"""
        if counts is None:
            cu, rows = None, self.B
        else:
            n = np.asarray(counts, dtype=np.int64)
            if n.shape != (self.B,) or (n < 0).any():
                raise ValueError(f"counts: {self.B} whole numbers, none negative")
            cu, rows = torch.as_tensor(np.concatenate([[0], np.cumsum(n)]).astype(np.int32), device=self.device), int(n.sum())
        return self._append(x, cu, rows, packed)

    def append_prefill(self, x: torch.Tensor) -> torch.Tensor:
        """The prompts' rows x [total_tokens, latent_dim + 64] into the cache; returns the stored rows, packed, which the up
        projections of the expanded form and prefill() read."""
        return self._append(x, self.cu, self.total_tokens, True)

    def _append(self, x, cu, rows, packed):
        self._rows(rows, self.L + 64, x=x)
        out = torch.empty((rows, self.L + 64), dtype=torch.bfloat16, device=self.device) if packed else None
        self._call("cpa_latent_append", self.cfg, self.dims, self.tables, *self._rope(), x, x.stride(0) if rows > 1 else self.L + 64,
                   self.norm_weight, cu, rows, self.first, self.lens, self._lens_next, self.pool, out)
        self.lens, self._lens_next = self._lens_next, self.lens
        return out

    def turn_queries(self, q: torch.Tensor) -> torch.Tensor:
        """Turns the positional part (the last 64 elements) of the prompts' queries [total_tokens, heads, 192], in place."""
        if self.rope is not None:
            self.rope.turn(self.positions, q)
        return q

    def prefill(self, q: torch.Tensor, kv: torch.Tensor, packed: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
        """Expanded form, causal over every block: q [tokens, heads, 128 + 64] (turned), kv [tokens, heads, 128 + 128], and
        append_prefill's packed rows, of which the positional keys are read.  Returns [tokens, heads, 128]."""
        T = self.total_tokens
        if out is None:
            out = torch.empty((T, self.H, 128), dtype=torch.bfloat16, device=self.device)
        self._packed(q=(q, (T, self.H, 192)), kv=(kv, (T, self.H, 256)), packed=(packed, (T, self.L + 64)), out=(out, (T, self.H, 128)))
        self._call("cpa_latent_prefill", self.cfg, self.plan, q, kv, packed[:, self.L:], self.L + 64, out)
        return out

    def _io(self, q_latent, q_rope, out):
        if out is None:
            out = torch.empty((self.B, self.H, self.L), dtype=torch.bfloat16, device=self.device)
        for name, t, e in (("q_latent", q_latent, self.L), ("q_rope", q_rope, 64), ("out", out, self.L)):
            if t.device != self.lens.device or t.shape != (self.B, self.H, e):
                raise ValueError(f"{name}: [{self.B}, {self.H}, {e}] on {self.lens.device} is wanted, not {tuple(t.shape)} on {t.device}")
        return B.latent_io(q_latent, q_rope, out), out

    def _active(self, active):
        if active is not None and (active.dtype != torch.int32 or active.device != self.lens.device or active.shape != (self.B,) or
                                   not active.is_contiguous()):
            raise ValueError(f"active: contiguous int32 [{self.B}] on {self.lens.device} is wanted")
        return active

    def decode(self, q_latent: torch.Tensor, q_rope: torch.Tensor, out: Optional[torch.Tensor] = None, active=None) -> torch.Tensor:
        """Absorbed form: q_latent [B, heads, latent_dim], q_rope [B, heads, 64] (turned) over the blocks' cached rows; returns
        [B, heads, latent_dim].  Blocks whose flag in `active` (device int32 [B]) is 0 sit out."""
        io, out = self._io(q_latent, q_rope, out)
        self._call("cpa_latent_decode", self.cfg, self.dims, self.tables, io, self.lens, self._active(active), self.pool, self.workspace)
        return out

    def step(self, q_latent: torch.Tensor, q_rope: torch.Tensor, x: torch.Tensor, out: Optional[torch.Tensor] = None,
             active=None) -> torch.Tensor:
        """One decode step: x [B, latent_dim + 64] appended, q_rope turned to the new token's position, then decode()."""
        io, out = self._io(q_latent, q_rope, out)
        self._rows(self.B, self.L + 64, x=x)
        self._call("cpa_latent_step", self.cfg, self.dims, self.tables, *self._rope(), io, x, x.stride(0) if self.B > 1 else self.L + 64,
                   self.norm_weight, self.first, self.lens, self._lens_next, self._active(active), self.pool, self.workspace)
        self.lens, self._lens_next = self._lens_next, self.lens
        return out

    def status(self) -> int:
        stream = int(torch.cuda.current_stream(self.device).cuda_stream)
        return B.cpa_plan_status(self.plan, stream) or B.cpa_tables_status(self.tables, stream)

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
