"""Device-side plumbing around libcommvq: torch tensors for memory, nothing of the method itself."""
from __future__ import annotations

from typing import Optional

import numpy as np

from . import binding as B


def _torch():
    import torch

    if not torch.cuda.is_available():
        raise RuntimeError("libcommvq needs a GPU (gfx950); no CPU fallback exists")
    return torch


def to_device(arr: np.ndarray, bf16: bool = False):
    """Upload a numpy array; uint16 arrays flagged bf16 become torch.bfloat16 views of the same bits."""
    torch = _torch()
    if bf16:
        assert arr.dtype == np.uint16
        return torch.from_numpy(np.ascontiguousarray(arr).view(np.int16)).cuda().view(torch.bfloat16)
    return torch.from_numpy(np.ascontiguousarray(arr)).cuda()


class DeviceWorkload:
    """A synth.Workload resident in HBM (one copy of every input buffer)."""

    def __init__(self, w):
        bf = w.dtype == "bf16"
        self.w = w
        self.q = to_device(w.q, bf)
        self.key_codes = to_device(w.key_codes)
        self.val_codes = to_device(w.val_codes)
        self.key_codebooks = to_device(w.key_codebooks, bf)
        self.val_codebooks = to_device(w.val_codebooks, bf)
        self.cu_seqlens = to_device(w.cu_seqlens)
        self.q_pos = to_device(w.q_pos)
        self.key_pos = None if w.key_pos is None else to_device(w.key_pos)
        self.positions = B.make_positions(w.B, self.cu_seqlens, self.q_pos, self.key_pos, w.total_tokens, w.max_seqlen)


class DecodeAttention:
    """Owns a libcommvq handle, a workspace and an output buffer for one batch shape."""

    def __init__(self, w, max_position: Optional[int] = None, softmax_scale: float = 0.0, position_free: bool = False,
                 q_dtype: Optional[str] = None):
        torch = _torch()
        dt = B.COMMVQ_BF16 if w.dtype == "bf16" else B.COMMVQ_F32
        qdt = dt if q_dtype is None else (B.COMMVQ_BF16 if q_dtype == "bf16" else B.COMMVQ_F32)
        if max_position is None:
            max_position = max(int(w.q_pos.max()), w.max_seqlen, 0 if w.key_pos is None else int(w.key_pos.max()))
        paired = getattr(w, "key_format", "indexed") == "paired"
        vbin = getattr(w, "val_format", "indexed") == "binary"
        self.cfg = B.Config(w.Hq, w.Hkv, w.d, 16 if paired else w.Mk, 16 if vbin else w.Mv, w.K, qdt, dt, float(w.rope_base),
                            float(softmax_scale), int(max_position),
                            B.COMMVQ_KEYS_PAIRED if paired else B.COMMVQ_KEYS_INDEXED, w.key_levels if paired else 0,
                            1 if position_free else 0,
                            B.COMMVQ_VALUES_BINARY if vbin else B.COMMVQ_VALUES_INDEXED, w.val_bits if vbin else 0)
        self.handle = B.commvq_create(self.cfg)
        self.plan = B.commvq_plan_query(self.handle, w.B, w.total_tokens, w.max_seqlen)
        self.workspace_bytes = B.commvq_workspace_bytes(self.handle, w.B, w.total_tokens, w.max_seqlen)
        self.workspace = torch.empty(self.workspace_bytes, dtype=torch.uint8, device="cuda")
        assert self.workspace.data_ptr() % 256 == 0
        self.out = torch.empty((w.B, w.Hq, w.d), dtype=torch.float32, device="cuda")
        self.n_scores = w.total_tokens * w.Hq
        self._packed = {}

    def pack_key_codebooks(self, dw: DeviceWorkload):
        """One-time re-layout of dw's (static) key codebooks; later calls with dw skip the per-call re-layout."""
        torch = _torch()
        buf = torch.empty(B.commvq_packed_key_codebook_bytes(self.handle), dtype=torch.uint8, device="cuda")
        B.commvq_pack_key_codebooks(self.handle, dw.key_codebooks, buf, self.stream_ptr())
        self._packed[dw.key_codebooks.data_ptr()] = (buf, dw.key_codebooks)  # keep both alive while registered

    def pack_value_codebooks(self, dw: DeviceWorkload):
        """One-time re-layout of dw's (static) value codebooks for the batched output kernel."""
        torch = _torch()
        buf = torch.empty(B.commvq_packed_value_codebook_bytes(self.handle), dtype=torch.uint8, device="cuda")
        B.commvq_pack_value_codebooks(self.handle, dw.val_codebooks, buf, self.stream_ptr())
        self._packed[("v", dw.val_codebooks.data_ptr())] = (buf, dw.val_codebooks)

    def close(self):
        if self.handle is not None:
            B.commvq_destroy(self.handle)
            self.handle = None

    def __del__(self):
        try:
            self.close()
        except Exception:
            pass

    def stream_ptr(self) -> int:
        return int(_torch().cuda.current_stream().cuda_stream)

    def __call__(self, dw: DeviceWorkload, out=None):
        """Enqueue commvq_decode_attn on torch's current stream; returns the (asynchronous) output tensor."""
        out = self.out if out is None else out
        B.commvq_decode_attn(self.handle, dw.q, dw.key_codes, dw.val_codes, dw.key_codebooks, dw.val_codebooks,
                             dw.positions, out, self.workspace, self.workspace_bytes, self.stream_ptr())
        return out

    def scores(self, dw: DeviceWorkload):
        """Run the score stage alone and return the logits [T*Hq] (ragged (b, h, i) layout)."""
        torch = _torch()
        s = torch.empty(self.n_scores, dtype=torch.float32, device="cuda")
        B.commvq_stage_scores(self.handle, dw.q, dw.key_codes, dw.key_codebooks, dw.positions, self.workspace,
                              self.workspace_bytes, s, self.stream_ptr())
        return s

    def staged(self, dw: DeviceWorkload):
        """scores -> bins -> output through the three stage entry points."""
        st = self.stream_ptr()
        B.commvq_stage_scores(self.handle, dw.q, dw.key_codes, dw.key_codebooks, dw.positions, self.workspace,
                              self.workspace_bytes, None, st)
        B.commvq_stage_bins(self.handle, dw.val_codes, dw.positions, self.workspace, self.workspace_bytes, st)
        B.commvq_stage_output(self.handle, dw.val_codebooks, dw.positions, self.out, self.workspace,
                              self.workspace_bytes, st)
        return self.out


def _expect(name: str, t, shape, dtype):
    """The calls take addresses: a tensor of another shape, type, order or place would be misread."""
    if t is None or tuple(t.shape) != tuple(shape) or t.dtype != dtype or not t.is_cuda or not t.is_contiguous():
        raise ValueError(f"{name}: a contiguous {dtype} tensor {tuple(shape)} on the GPU")


class PagedCache:
    """The pages of one layer for up to `batch` sequences: records in index form, block tables, free pages.

    Lengths and the pages that a sequence owns are kept on the host; one object's calls belong on one stream."""

    def __init__(self, cfg: B.Config, handle, n_blocks: int, block_size: int, batch: int, max_blocks: int, n_axes: int = 1):
        torch = _torch()
        self.cfg, self.handle, self.batch = cfg, handle, batch
        self.pages = B.make_pages(block_size, n_blocks, max_blocks, n_axes)
        heads = cfg.n_kv_heads
        self.key_pages = torch.zeros((n_blocks, heads, block_size, cfg.m_key), dtype=torch.uint8, device="cuda")
        self.val_pages = torch.zeros((n_blocks, heads, block_size, cfg.m_val), dtype=torch.uint8, device="cuda")
        self.key_pos = torch.zeros((n_blocks * block_size, n_axes), dtype=torch.int32, device="cuda") if n_axes > 1 else None
        self.block_tables = torch.full((batch, max_blocks), -1, dtype=torch.int32, device="cuda")
        self.seq_lens = torch.zeros(batch, dtype=torch.int32, device="cuda")
        self.lens = [0] * batch
        self.free = list(range(n_blocks))
        self.owned = [[] for _ in range(batch)]

    def append(self, new_lens, key_codes, val_codes, token_pos=None):
        """Takes pages for new_lens[b] more tokens of every sequence and stores their records, [sum of new_lens][heads][codebooks], sequence by sequence."""
        torch = _torch()
        size, total = self.pages.block_size, sum(new_lens)
        pages_of = lambda n: -(-n // size)
        if len(new_lens) != self.batch or min(new_lens) < 0:
            raise ValueError("new_lens: one number >= 0 per sequence")
        want = [pages_of(c + n) - pages_of(c) for c, n in zip(self.lens, new_lens)]
        need = sum(want)
        if need > len(self.free) or any(pages_of(c + n) > self.pages.max_blocks for c, n in zip(self.lens, new_lens)):
            raise RuntimeError("the cache has no room for the new tokens")
        if total:
            _expect("key_codes", key_codes, (total, self.cfg.n_kv_heads, self.cfg.m_key), torch.uint8)
            _expect("val_codes", val_codes, (total, self.cfg.n_kv_heads, self.cfg.m_val), torch.uint8)
            if self.key_pos is not None:
                _expect("token_pos", token_pos, (total, self.pages.n_axes), torch.int32)
        ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        stream = int(torch.cuda.current_stream().cuda_stream)
        cached, new, free = ints(self.lens), ints(list(new_lens)), ints(self.free[:need] or [-1])
        cu, slots, taken = (torch.empty(n, dtype=torch.int32, device="cuda") for n in (self.batch + 1, max(1, total), 2))
        B.commvq_page_tables(self.pages, self.batch, cached, new, free, need, self.block_tables, self.seq_lens, cu, slots, None, total, taken, stream)
        if total:
            B.commvq_store_pages(self.handle, self.pages, total, slots, key_codes, val_codes, token_pos if self.key_pos is not None else None,
                                 self.key_pages, self.val_pages, self.key_pos, stream)
        for b, n in enumerate(want):
            self.owned[b] += self.free[:n]
            del self.free[:n]
        self.lens = [c + n for c, n in zip(self.lens, new_lens)]
        return slots

    def release(self, b: int):
        """Sequence b is done: its pages are free again, its place is empty."""
        self.free += self.owned[b]
        self.owned[b], self.lens[b] = [], 0
        self.seq_lens[b] = 0


class TreeAttention:
    """Attention of drafted trees over a PagedCache: the layer's codebooks, laid out once, and a workspace that grows with the batch.

    One object's calls belong on one stream (they share the workspace)."""

    def __init__(self, cfg: B.Config, handle, key_codebooks, val_codebooks):
        torch = _torch()
        self.cfg, self.handle, self.key_codebooks, self.val_codebooks = cfg, handle, key_codebooks, val_codebooks
        self.tables = None
        if cfg.codebook_dtype == B.COMMVQ_BF16:
            self.tables = torch.empty(B.commvq_tree_table_bytes(handle), dtype=torch.uint8, device="cuda")
            B.commvq_tree_prepare(handle, key_codebooks, val_codebooks, self.tables, int(torch.cuda.current_stream().cuda_stream))
        self.workspace = torch.empty(0, dtype=torch.uint8, device="cuda")

    def __call__(self, cache: PagedCache, q, node_keys, node_vals, nodes, node_pos, node_mask=None, pair_axis=None, out=None):
        """nodes[b]: drafted tokens of sequence b (host); the other arguments are the call's device tensors."""
        torch = _torch()
        total, most, longest = sum(nodes), max(nodes), max(cache.lens)
        if len(nodes) != cache.batch or min(nodes) < 0:
            raise ValueError("nodes: one number >= 0 per sequence")
        kind = torch.bfloat16 if self.cfg.q_dtype == B.COMMVQ_BF16 else torch.float32
        _expect("q", q, (total, self.cfg.n_q_heads, 128), kind)
        _expect("node_keys", node_keys, (total, self.cfg.n_kv_heads, 128), kind)
        _expect("node_vals", node_vals, (total, self.cfg.n_kv_heads, 128), kind)
        _expect("node_pos", node_pos, (total, cache.pages.n_axes), torch.int32)
        if node_mask is not None:
            _expect("node_mask", node_mask, (total,), torch.int64)
        if out is not None:
            _expect("out", out, tuple(q.shape), kind)
        if total == 0:
            return torch.empty_like(q) if out is None else out
        ends = [0]
        for n in nodes:
            ends.append(ends[-1] + n)
        cu = torch.tensor(ends, dtype=torch.int32, device="cuda")
        need = B.commvq_tree_workspace_bytes(self.handle, cache.batch, total, most, longest)
        if self.workspace.numel() < need:
            self.workspace = torch.empty(need, dtype=torch.uint8, device="cuda")
        out = torch.empty_like(q) if out is None else out
        tree = B.make_tree(cache.batch, total, most, longest, cache.seq_lens, cache.block_tables, cu, node_pos, node_mask, cache.key_pos, pair_axis,
                           total_tokens=sum(cache.lens))
        B.commvq_tree_attn(self.handle, cache.pages, tree, q, node_keys, node_vals, cache.key_pages, cache.val_pages, self.key_codebooks,
                           self.val_codebooks, self.tables, out, self.workspace, self.workspace.numel(), int(torch.cuda.current_stream().cuda_stream))
        return out
