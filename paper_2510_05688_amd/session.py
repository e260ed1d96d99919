"""Device buffers for one plan: allocation and upload only (PyTorch as the memory allocator).

No arithmetic of the method happens here; every call goes straight to the C ABI.
"""
from __future__ import annotations

import math
from typing import Dict, Optional

import numpy as np
import torch

from . import binding as vb


def _bf16_from_bits(bits: np.ndarray, device) -> torch.Tensor:
    t = torch.from_numpy(np.ascontiguousarray(bits).view(np.int16))
    return t.to(device).view(torch.bfloat16)


class DecodeSession:
    """Owns a plan, its workspace and output buffers on one GPU."""

    # where the tokens of the last write() begin, and whether that still holds (the buffer stays, for captured writes)
    first: Optional[torch.Tensor] = None
    written = False

    def __init__(self, params: Dict, device: int = 0, q_len: int = 1, kv_format: int = vb.VATT_KV_BF16,
                 block_tokens: Optional[int] = None, rotary: Optional[Dict] = None):
        """kv_format, block_tokens, rotary: the cache's format (VATT_KV_*), the tokens per block and the rotation
        (fields of vatt_rotary) of the cache calls below.  q_len > 1: a plan for multi-query steps; q is then
        [B, q_len, Hq, d] and every output has one row per (sequence, query token) pair, b * q_len + t, where the
        single-token shapes have one per sequence."""
        if not torch.cuda.is_available():
            raise RuntimeError("DecodeSession needs a GPU; there is no CPU path")
        self.device = torch.device("cuda", device)
        torch.cuda.set_device(self.device)
        self.params = dict(params)
        self.q_len = int(q_len)
        self.kv_format, self.block_tokens, self.plain = int(kv_format), block_tokens, None
        self.plan = self._new_plan()
        if rotary is not None:
            vb.vatt_plan_set_rotary(self.plan, rotary)
        p = self.params
        self.Hq, self.Hkv, self.d = p["n_q_heads"], p["n_kv_heads"], p["head_dim"]
        self.B = p["batch"] * self.q_len  # rows of every per-query buffer
        self.n_max = p["n_max"]
        self.paged = p.get("kv_layout", 0) == vb.VATT_LAYOUT_PAGED
        self.idx_cap = vb.vatt_plan_index_capacity(self.plan)
        self.seg = [vb.vatt_plan_index_segment(self.plan, s) for s in range(5)]
        self.ws_bytes = vb.vatt_plan_workspace_bytes(self.plan)
        dev = self.device
        self.workspace = torch.empty(self.ws_bytes, dtype=torch.uint8, device=dev)
        assert self.workspace.data_ptr() % 256 == 0
        self.out_o = torch.empty(self.B, self.Hq, self.d, dtype=torch.float32, device=dev)
        self.out_lse = torch.empty(self.B, self.Hq, dtype=torch.float32, device=dev)
        self.out_idx = torch.empty(self.B, self.Hq, self.idx_cap, dtype=torch.int32, device=dev)
        self.out_counts = torch.empty(self.B, self.Hq, 8, dtype=torch.int32, device=dev)
        self.out_budget_raw = torch.empty(self.B, self.Hq, dtype=torch.float64, device=dev)
        self.out_stats = torch.empty(self.B, self.Hq, 4, dtype=torch.float32, device=dev)
        self.dense_o = torch.empty(self.B, self.Hq, self.d, dtype=torch.float32, device=dev)
        self.dense_lse = torch.empty(self.B, self.Hq, dtype=torch.float32, device=dev)
        self.block_table: Optional[torch.Tensor] = None
        self.q = self.k = self.v = self.seq_lens = self.seq_seeds = self.rcache = self.cache_seeds = None
        self.summary = self.blocks = self.block_count = None
        self.first = torch.zeros(p["batch"], dtype=torch.int32, device=dev)

    def _new_plan(self):
        device = -1 if self.device.type == "cpu" else self.device.index
        plan = (vb.vatt_plan_create(self.params, device) if self.q_len == 1
                else vb.vatt_plan_create_chunk(self.params, self.q_len, device))
        vb.vatt_plan_set_option(plan, vb.VATT_OPT_KV_FORMAT, self.kv_format)
        if self.block_tokens is not None:
            vb.vatt_plan_set_option(plan, vb.VATT_OPT_BLOCK_TOKENS, int(self.block_tokens))
        return plan

    def close(self):
        for plan in (self.plan, self.plain):
            if plan:
                vb.vatt_plan_destroy(plan)
        self.plan = self.plain = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    # ---- uploads -----------------------------------------------------------
    def upload(self, q_bits, k_bits, v_bits, seq_lens, seeds, block_table=None):
        """k_bits, v_bits: bf16 rows in the plan's layout; on a quantised plan codes and scales, vatt_kv_cache_bytes in all."""
        dev = self.device
        want = vb.vatt_kv_cache_bytes(self.plan)
        if vb.vatt_kv_scale_offset(self.plan) < want:  # (there are scales)
            if np.asarray(k_bits).nbytes != want or np.asarray(v_bits).nbytes != want:
                raise ValueError(f"K and V of this plan's format have {want} bytes each, got {np.asarray(k_bits).nbytes} and {np.asarray(v_bits).nbytes}")
        self.q = _bf16_from_bits(q_bits, dev)
        self.k = _bf16_from_bits(k_bits, dev)
        self.v = _bf16_from_bits(v_bits, dev)
        self.seq_lens = torch.from_numpy(np.ascontiguousarray(seq_lens, dtype=np.int32)).to(dev)
        self.seq_seeds = torch.from_numpy(np.ascontiguousarray(seeds, dtype=np.uint64).view(np.int64)).to(dev)
        self.block_table = None
        self.summary = self.blocks = self.block_count = None  # (of make_cache's cache only)
        self.written = False
        if block_table is not None:
            self.block_table = torch.from_numpy(np.ascontiguousarray(block_table, dtype=np.int32)).to(dev)
        return self

    def move_kv_to_host(self):
        """Moves the uploaded K and V to pinned host memory; self.k / self.v become the addresses the kernels
        read them at (vatt_host_kv_device_pointer), and the pinned tensors stay alive in self.k_host / v_host."""
        torch.cuda.synchronize(self.device)
        self.k_host = torch.empty(self.k.shape, dtype=self.k.dtype, pin_memory=True).copy_(self.k)
        self.v_host = torch.empty(self.v.shape, dtype=self.v.dtype, pin_memory=True).copy_(self.v)
        self.k = vb.vatt_host_kv_device_pointer(self.k_host)
        self.v = vb.vatt_host_kv_device_pointer(self.v_host)
        return self

    def set_seeds(self, seeds):
        self.seq_seeds = torch.from_numpy(np.ascontiguousarray(seeds, dtype=np.uint64).view(np.int64)).to(self.device)

    def _stream(self):
        return torch.cuda.current_stream(self.device).cuda_stream

    # ---- calls ---------------------------------------------------------------
    def decode(self, q=None, k=None, v=None):
        vb.vatt_decode(self.plan, self._query(q), self.k if k is None else k,
                       self.v if v is None else v, self.block_table, self.seq_lens, self.seq_seeds,
                       self.workspace, self.out_o, self.out_lse, self.out_idx, self.out_counts,
                       self.out_budget_raw, self.out_stats, self._stream())

    def decode_given_topk(self, topk_idx, topk_cnt, k=None, v=None, q=None):
        """vatt_decode_given_topk with int32 device tensors topk_idx [B, Hq, k_max], topk_cnt [B, Hq].  After make_cache() its seeds
        come from set_seeds()."""
        vb.vatt_decode_given_topk(self.plan, self._query(q), self.k if k is None else k, self.v if v is None else v,
                                  self.block_table, self.seq_lens, self.seq_seeds, topk_idx, topk_cnt,
                                  self.workspace, self.out_o, self.out_lse, self.out_idx, self.out_counts,
                                  self.out_budget_raw, self.out_stats, self._stream())

    # ---- random cache of base-sample rows ------------------------------------
    def make_random_cache(self, cache_seeds, slots: Optional[int] = None):
        """Allocates the cache buffer and fills it from the sequences as uploaded (vatt_random_cache_fill)."""
        if slots is not None:
            vb.vatt_plan_set_option(self.plan, vb.VATT_OPT_CACHE_SLOTS, int(slots))
        self.cache_slots = vb.vatt_random_cache_slots(self.plan)
        self.cache_seeds = torch.from_numpy(np.ascontiguousarray(cache_seeds, dtype=np.uint64).view(np.int64)).to(self.device)
        self.rcache = torch.empty(vb.vatt_random_cache_bytes(self.plan), dtype=torch.uint8, device=self.device)
        assert self.rcache.data_ptr() % 256 == 0
        vb.vatt_random_cache_fill(self.plan, self.k, self.v, self.block_table, self.seq_lens, self.cache_seeds,
                                  self.rcache, self._stream())

    def random_cache_host(self):
        """(tokens int32 [B, Hkv, slots] with -1 in unused slots, counts int32 [B, Hkv]) of the cache."""
        B = self.params["batch"]
        tok = torch.empty(B, self.Hkv, self.cache_slots, dtype=torch.int32, device=self.device)
        cnt = torch.empty(B, self.Hkv, dtype=torch.int32, device=self.device)
        vb.vatt_random_cache_read(self.plan, self.rcache, tok, cnt, self._stream())
        torch.cuda.synchronize(self.device)
        return tok.cpu().numpy(), cnt.cpu().numpy()

    def append_device_cached(self, k_new, v_new):
        self.written = False
        self._renew_summary(k_new, v_new)
        vb.vatt_append_kv_cached(self.plan, k_new, v_new, self.k, self.v, self.block_table, self.seq_lens,
                                 self.cache_seeds, self.rcache, self._stream())

    def decode_given_topk_cached(self, topk_idx, topk_cnt, k=None, v=None, q=None):
        vb.vatt_decode_given_topk_cached(self.plan, self._query(q), self.k if k is None else k,
                                         self.v if v is None else v, self.block_table, self.seq_lens,
                                         self.seq_seeds, topk_idx, topk_cnt, self.rcache, self.workspace,
                                         self.out_o, self.out_lse, self.out_idx, self.out_counts,
                                         self.out_budget_raw, self.out_stats, self._stream())

    def dense(self, q=None, k=None, v=None):
        vb.vatt_dense_decode(self.plan, self._query(q), self.k if k is None else k,
                             self.v if v is None else v, self.block_table, self.seq_lens, self.workspace,
                             self.dense_o, self.dense_lse, self._stream())

    def score(self, q=None, k=None):
        vb.vatt_score(self.plan, self._query(q), self.k if k is None else k, self.block_table,
                      self.seq_lens, self.workspace, self._stream())

    def append(self, k_new_bits, v_new_bits):
        kn = _bf16_from_bits(k_new_bits, self.device)
        vn = _bf16_from_bits(v_new_bits, self.device)
        self.append_device(kn, vn)

    def append_device(self, k_new, v_new):
        """Append one token per sequence from tensors that are already on the device (bf16 [B, Hkv, d]).  The summaries
        of their blocks follow, if there are any."""
        self.written = False
        self._renew_summary(k_new, v_new)
        vb.vatt_append_kv(self.plan, k_new, v_new, self.k, self.v, self.block_table, self.seq_lens, self._stream())

    # ---- the cache from the projections' outputs to attention over blocks -----
    def make_cache(self, block_table=None):
        """Allocates an empty cache in the plan's format, summaries of its blocks and lists for the chosen ones.
        block_table: [B, ceil(n_max / page_size)] on a paged plan."""
        dev = self.device
        if self.paged and block_table is not None:
            want = self.params["batch"] * -(-self.n_max // self.params["page_size"])
            if np.size(block_table) != want:
                raise ValueError(f"block_table: a paged plan's has {want} entries, got {np.shape(block_table)}")
        self.q = self.seq_seeds = self.rcache = self.cache_seeds = None  # (of other sequences)
        self.written = False
        self.k, self.v = (torch.zeros(vb.vatt_kv_cache_bytes(self.plan), dtype=torch.uint8, device=dev) for _ in range(2))
        self.block_table = None
        if block_table is not None:
            self.block_table = torch.from_numpy(np.ascontiguousarray(block_table, dtype=np.int32)).to(dev)
        self.seq_lens = torch.zeros(self.params["batch"], dtype=torch.int32, device=dev)
        self._make_summary()
        return self

    def _make_summary(self):
        self.block_capacity = vb.vatt_block_list_capacity(self.plan)
        self.summary = self.blocks = self.block_count = None
        if self.block_capacity:
            dev = self.device
            self.summary = torch.zeros(vb.vatt_block_summary_bytes(self.plan) // 2, dtype=torch.bfloat16, device=dev)
            self.blocks = torch.zeros(self.B, self.Hkv, self.block_capacity, dtype=torch.int32, device=dev)
            self.block_count = torch.zeros(self.B, self.Hkv, dtype=torch.int32, device=dev)
            self._make_plain()

    def _make_plain(self):
        """A plan like the session's without a rotation: appended rows are the caller's as they are, and bf16."""
        self.plain = self.plain or self._new_plan()
        vb.vatt_plan_set_option(self.plain, vb.VATT_OPT_KV_FORMAT, vb.VATT_KV_BF16)
        for tokens in (16, 32, 64, 128, 256):  # (the number may have been set on the plan itself; the size says which)
            if vb.vatt_block_summary_bytes(self.plain) == vb.vatt_block_summary_bytes(self.plan):
                break
            vb.vatt_plan_set_option(self.plain, vb.VATT_OPT_BLOCK_TOKENS, tokens)

    def fill_summary(self):
        """Summaries of all blocks of the cache as it is, from one pass over K: what select_blocks needs of an uploaded cache, or of one
        that was written to without write() or append_device()."""
        if self.summary is None:
            self._make_summary()
        vb.vatt_block_summary_fill(self.plan, self.k, self.block_table, self.seq_lens, self.summary, self._stream())
        return self

    def _renew_summary(self, k_new, v_new):
        """The row that an append is about to write, written with the summary of its block."""
        if self.summary is not None and vb.vatt_kv_scale_offset(self.plan) == vb.vatt_kv_cache_bytes(self.plan):  # (quantised plans do not append)
            row = self.Hkv * self.d
            vb.vatt_write_kv(self.plain, None, k_new, v_new, 0, row, row, 1, self.seq_lens, None, self.k, self.v, self.block_table,
                             self.summary, None, None, self._stream())

    def write(self, q, k_new, v_new, new_lens=None, out_q=None):
        """Appends the tokens k_new, v_new (bf16 [B, n_new, Hkv, d], as far as new_lens says) to every sequence; returns the
        rotated queries (bf16 [B, n_new, Hq, d]), zeros for tokens that are not written, or None without q.  With out_q they go there, and
        rows of tokens that are not written stay as they are (clearing those of 2 x 16K tokens of 32 heads takes 51 of 196 us).
        seq_lens stays the same tensor, so that a captured write goes on where the last replay ended."""
        for x, heads in ((q, self.Hq), (k_new, self.Hkv), (v_new, self.Hkv)):
            want = (self.params["batch"], k_new.shape[1], heads, self.d)
            if x is not None and (x.shape != want or x.dtype != torch.bfloat16 or x.device != self.device):
                raise ValueError(f"expected bfloat16 {want} on {self.device}, got {x.dtype} {tuple(x.shape)} on {x.device}")
        self._check("new_lens", new_lens, torch.int32, self.params["batch"])
        if out_q is not None:
            if q is None:
                raise ValueError("out_q without q")
            self._check("out_q", out_q, torch.bfloat16, *q.shape)
        elif q is not None:
            out_q = torch.zeros(q.shape, dtype=torch.bfloat16, device=self.device)
        strides = [0 if x is None else vb.token_stride(x) for x in (q, k_new, v_new)]
        self.written = False
        if self.first is None:
            self.first = torch.empty_like(self.seq_lens)
        if new_lens is not None and any(self._overlap(new_lens, x) for x in (self.seq_lens, self.first)):
            new_lens = new_lens.clone()  # (both are written to)
        self.first.copy_(self.seq_lens)
        vb.vatt_write_kv(self.plan, q, k_new, v_new, *strides, k_new.shape[1], self.first, new_lens, self.k, self.v, self.block_table,
                         self.summary, out_q, self.seq_lens, self._stream())
        self.written = True
        return out_q

    def attend(self, q, new_lens=None, sink=0, window=0, dtype=torch.bfloat16, out=None, lse=None, first=None):
        """Attention of the tokens of the last write() over the cache, each over all tokens up to itself or (window > 0) over the first
        `sink` and the last `window` of them.  q: their rotated queries, bf16 [B, n_new, Hq, d]; new_lens: as in that write.  Returns
        (output in `dtype`, bfloat16 or float32, [B, n_new, Hq, d]; ln of the sums, float32 [B, n_new, Hq]), zeros for tokens that do
        not count; with `out` (its type counts) or `lse` they go there, and such rows stay as they are.  first: int32 [B], where the
        tokens begin, if they are not those of the last write()."""
        want = (self.params["batch"], q.shape[1] if q.dim() == 4 else 0, self.Hq, self.d)
        if q.shape != want or q.dtype != torch.bfloat16 or q.device != self.device:
            raise ValueError(f"expected bfloat16 [{want[0]}, n_new, {want[2]}, {want[3]}] on {self.device}, got {q.dtype} {tuple(q.shape)} on {q.device}")
        if first is None and not self.written:
            raise ValueError("no write() to go by: give the tokens' first positions")
        self._check("new_lens", new_lens, torch.int32, want[0])
        self._check("first", first, torch.int32, want[0])
        dtype = dtype if out is None else out.dtype
        if dtype not in (torch.bfloat16, torch.float32):
            raise ValueError(f"output in bfloat16 or float32, not {dtype}")
        self._check("out", out, dtype, *want)
        self._check("lse", lse, torch.float32, *want[:3])
        out = torch.zeros(want, dtype=dtype, device=self.device) if out is None else out
        lse = torch.zeros(want[:3], dtype=torch.float32, device=self.device) if lse is None else lse
        need = vb.vatt_chunk_workspace_bytes(self.plan, want[1])
        workspace = torch.empty(need, dtype=torch.uint8, device=self.device) if need else None
        vb.vatt_chunk_attend(self.plan, q, vb.token_stride(q), want[1], self.first if first is None else first, new_lens, self.k, self.v,
                             self.block_table, sink, window, workspace, vb.VATT_OUT_BF16 if dtype == torch.bfloat16 else vb.VATT_OUT_F32,
                             out, lse, self._stream())
        return out, lse

    def window_decode(self, sink: int, window: int, q=None):
        """A decode step over the first `sink` and the last `window` tokens, into out_o and out_lse."""
        vb.vatt_window_decode(self.plan, self._query(q), self.k, self.v, self.block_table, self.seq_lens, sink, window, self.workspace,
                              self.out_o, self.out_lse, self._stream())

    @staticmethod
    def _overlap(x, y):
        """Whether two tensors, each one value behind the other, share memory."""
        a, b = x.data_ptr(), y.data_ptr()
        return a < b + y.numel() * y.element_size() and b < a + x.numel() * x.element_size()

    def _check(self, name, x, dtype, *shape):
        """A kernel gets x as an address: x has to be a tensor of so many values, one behind the other, on this device (None is left to
        the call)."""
        if x is None:
            return
        if not isinstance(x, torch.Tensor):
            raise ValueError(f"{name}: expected a tensor, got {type(x).__name__}")
        if x.numel() != math.prod(shape) or x.dtype != dtype or x.device != self.device or not x.is_contiguous():
            raise ValueError(f"{name}: expected contiguous {dtype} {shape} on {self.device}, got {x.dtype} {tuple(x.shape)} on {x.device}")

    def _query(self, q):
        if q is None:
            return self.q
        self._check("q", q, torch.bfloat16, self.B, self.Hq, self.d)
        return q

    def read_rows(self, first, n_rows: int):
        """(K, V) rows first[b] .. first[b] + n_rows - 1 in bf16 [B, Hkv, n_rows, d]; zeros where a sequence has none.  first: int32 [B]
        on the device, or one number for all (None: 0)."""
        if isinstance(first, int):
            first = torch.full((self.params["batch"],), first, dtype=torch.int32, device=self.device)
        self._check("first", first, torch.int32, self.params["batch"])
        out = [torch.zeros(self.params["batch"], self.Hkv, n_rows, self.d, dtype=torch.bfloat16, device=self.device) for _ in range(2)]
        vb.vatt_read_kv(self.plan, self.k, self.v, self.block_table, self.seq_lens, first, n_rows, out[0], out[1], self._stream())
        return out

    def select_blocks(self, q=None, topk_idx=None, topk_cnt=None):
        """Fills self.blocks and self.block_count (and the token lists for decode_given_topk, if given)."""
        k_max = self.seg[3] - self.seg[2]
        self._check("topk_idx", topk_idx, torch.int32, self.B, self.Hq, max(k_max, 1))  # (with none an entry that nobody writes)
        self._check("topk_cnt", topk_cnt, torch.int32, self.B, self.Hq)
        vb.vatt_select_blocks(self.plan, self._query(q), self.summary, self.block_table, self.seq_lens, self.workspace,
                              self.blocks, self.block_count, topk_idx, topk_cnt, self._stream())

    def block_decode(self, q=None):
        """Attention over the chosen blocks, into out_o and out_lse."""
        vb.vatt_block_decode(self.plan, self._query(q), self.k, self.v, self.block_table, self.seq_lens, self.blocks,
                             self.block_count, self.workspace, self.out_o, self.out_lse, self._stream())

    # ---- read-back -----------------------------------------------------------
    def scores_host(self) -> np.ndarray:
        """float32 [B, Hq, n_max] view of the score region of the workspace (copied to host)."""
        off = vb.vatt_plan_workspace_offset(self.plan, vb.VATT_WS_SCORES)
        stride = vb.vatt_plan_score_stride(self.plan)
        nbytes = self.B * self.Hq * stride * 4
        t = self.workspace[off:off + nbytes].view(torch.float32).view(self.B, self.Hq, stride)
        return t[:, :, :self.n_max].cpu().numpy()

    def results_host(self) -> Dict[str, np.ndarray]:
        torch.cuda.synchronize(self.device)
        return dict(
            O=self.out_o.cpu().numpy(), lse=self.out_lse.cpu().numpy(), idx=self.out_idx.cpu().numpy(),
            counts=self.out_counts.cpu().numpy(), b_star=self.out_budget_raw.cpu().numpy(),
            stats=self.out_stats.cpu().numpy(), seg=list(self.seg),
        )
