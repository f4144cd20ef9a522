"""Buffer holder for one layer of a paged cache (allocation + call order only)."""
from __future__ import annotations

import torch

from . import binding as B


def rope_table(rope_len: int, rot_dim: int, base: float = 10000.0, device=None) -> torch.Tensor:
    """[rope_len, rot_dim] float: cosines, then sines, of position * base^(-2i / rot_dim); angles in double."""
    half = rot_dim // 2
    turn = base ** (-torch.arange(half, dtype=torch.float64, device=device) / max(half, 1))
    angle = torch.arange(rope_len, dtype=torch.float64, device=device)[:, None] * turn
    return torch.cat([angle.cos(), angle.sin()], dim=1).float()


class PagedLayer:
    """Owns one layer's pages (and their scales), abstracts, score / selection / output / workspace buffers.  What the
    layers of a model share comes from the caller: `page_table` [B, max_pages] and `seq_len` [B] int32 (both brought up to
    date by whoever schedules, seq_len with the step's tokens counted in) and the rotation's table.

      append      kv_page_append: new tokens into the pages; returns the rotated queries
      step        append, then attention of one token per sequence: over all pages, or - with `token_budget` or
                  `max_chunks` - chunk_score, chunk_topk_select with the pages as chunks, attention over the kept ones
      prompt      append, then causal attention of the new tokens

and, for caches that are shared and kept within bounds,

      attend_shared  attention of one token per sequence where groups of sequences begin with the same pages (`groups`: the most
                     groups of a call)
      weigh          what each cached token got of the attention of some rows, added to `weight`
      evict          the sequences brought down to `keep_len` tokens, by `weight` (`evicts`: the most rows of a sequence that
                     may move in a call); returns the new lengths, which become seq_len once all layers have evicted
                     (tokens of pages that several sequences list have to be among the first ones, which stay: `n_first`)

After an eviction a token's place is not its position: `append`, `step` and `prompt` then want `position` ([axes, rows]; with several
axes `axis` [rot_dim / 2] says whose each pair is).  `n_seen` [B] int32 is how many tokens a sequence ever had, brought up to date by
whoever schedules, as seq_len is.  A place in the batch that another sequence takes over needs nothing: `weigh` starts its new tokens
anew.  A sequence whose tokens were not all weighed (`weigh` of a prompt's last queries only) has `weight` and `token_id` of the
others set by the caller: to 0 and to their places.

    Sequences may list pages that others filled, and tokens may be taken back (`seq_len` lowered before the next append).
    Under a budget a place in the batch that another sequence takes over must be idle (length 0) for a step in between, or
    have its `n_chunks` set to 0: the rows of abstracts are the place's, and are made anew from the pages then.

    Calls of one layer must not overlap, on two streams or as two graphs: they share its buffers.  Workspaces hold nothing between
    calls: `workspaces_of` another layer makes this one use that one's where they are large enough, as the layers of a model can, whose
    calls follow one another on one stream.  The leoam_page_*workspace_bytes calls say how large they are: attend's a few MiB, prompt's
    up to 66, attend_shared's 65 and a KiB for every query head of every sequence; evict's 16 KiB for every 4096 or 8192 places that the
    table has for a (sequence, kv head), where these are too many for a workgroup (32 sequences of up to 131072 tokens, 8 heads: 74 MiB).
    """

    def __init__(self, page_table: torch.Tensor, seq_len: torch.Tensor, n_q_heads: int, n_kv_heads: int, n_pages: int,
                 page_size: int, dtype: torch.dtype, kv_dtype=None, rope: torch.Tensor = None, interleaved: bool = False,
                 k_max: int = 0, max_chunks: int = 0, token_budget: int = 0, head_dim: int = 128, workspaces_of: "PagedLayer" = None,
                 axis: torch.Tensor = None, groups: int = 0, evicts: int = 0):
        batch, max_pages = page_table.shape
        rope_len, rot_dim = rope.shape if rope is not None else (0, 0)
        self.page_table, self.seq_len, self.rope = page_table, seq_len, rope
        self.pages = p = B.make_pages(batch, n_q_heads, n_kv_heads, head_dim, n_pages, page_size, max_pages, dtype, kv_dtype,
                                      rot_dim, interleaved, rope_len)
        dev = page_table.device
        store = torch.float8_e4m3fn if p.kv_dtype == B.E4M3 else dtype
        self.k_pages = torch.zeros(n_pages, n_kv_heads, page_size, head_dim, dtype=store, device=dev)
        self.v_pages = torch.zeros_like(self.k_pages)
        self.k_scale = self.v_scale = None
        if p.kv_dtype == B.E4M3:
            self.k_scale = torch.zeros(n_pages, n_kv_heads, dtype=torch.float32, device=dev)
            self.v_scale = torch.zeros_like(self.k_scale)
        self.status = torch.zeros(batch, dtype=torch.int32, device=dev)
        self.out = torch.empty(batch, n_q_heads, head_dim, dtype=torch.float32, device=dev)
        self.lse = torch.empty(batch, n_q_heads, dtype=torch.float32, device=dev)
        self.lse_of_all = False      # what stands there is the last attention's, over all pages
        self.max_chunks, self.token_budget = int(max_chunks), int(token_budget)
        self.selects = self.max_chunks > 0 or self.token_budget > 0
        self.abstract = self.chunk_off = self.n_chunks = self.sel_idx = self.sel_count = None
        if self.selects:
            k_max = min(max_pages, int(k_max) or max_pages)
            self.shape = B.make_shape(batch, n_q_heads, n_kv_heads, head_dim, max_pages * page_size, max_pages, k_max, dtype)
            self.abstract = torch.zeros(batch, n_kv_heads, max_pages, 2, head_dim, dtype=dtype, device=dev)
            self.chunk_off = torch.zeros(batch, max_pages + 1, dtype=torch.int32, device=dev)
            self.n_chunks = torch.zeros(batch, dtype=torch.int32, device=dev)
            self.score = torch.empty(batch, n_kv_heads, max_pages, dtype=torch.float32, device=dev)
            self.sel_idx = torch.empty(batch, n_kv_heads, k_max, dtype=torch.int32, device=dev)
            self.sel_count = torch.empty(batch, n_kv_heads, dtype=torch.int32, device=dev)
        need = B.leoam_page_workspace_bytes(self.pages, 0)
        if workspaces_of is not None and workspaces_of.workspace.numel() >= need:
            self.workspace = workspaces_of.workspace
        else:
            self.workspace = self._new(need, torch.uint8, None)
        # the last is the largest; earlier ones stay, a captured graph may use them
        self.prompt_workspaces = [] if workspaces_of is None else workspaces_of.prompt_workspaces
        self.scale = B.default_scale(head_dim)
        self.axis, self.groups, self.evicts = axis, int(groups), int(evicts)
        self.weight = self.token_id = self.shared_workspace = self.evict_workspace = None
        if self.groups:
            need = B.leoam_page_shared_workspace_bytes(self.pages, self.groups)
            other = getattr(workspaces_of, "shared_workspace", None)
            self.shared_workspace = other if other is not None and other.numel() >= need else self._new(need, torch.uint8, None)
        if self.evicts:
            places = (batch, n_kv_heads, max_pages * page_size)
            self.weight = torch.zeros(places, dtype=torch.float32, device=dev)
            self.token_id = torch.zeros(places, dtype=torch.int32, device=dev)
            self.moves = torch.empty(batch, n_kv_heads, self.evicts, 2, dtype=torch.int32, device=dev)
            self.move_count = torch.empty(batch, n_kv_heads, dtype=torch.int32, device=dev)
            self.new_len = torch.zeros(batch, dtype=torch.int32, device=dev)
            self.evict_status = torch.zeros(batch, dtype=torch.int32, device=dev)
            need = B.leoam_page_evict_workspace_bytes(self.pages)
            other = getattr(workspaces_of, "evict_workspace", None)
            self.evict_workspace = other if other is not None and other.numel() >= need else self._new(need, torch.uint8, None)

    def _new(self, shape, dtype, stream) -> torch.Tensor:
        """Of the stream's own memory: freed before its kernels have run, it is given to later ones of that stream only."""
        device = self.page_table.device
        if stream is not None and not isinstance(stream, torch.cuda.Stream):
            stream = torch.cuda.ExternalStream(int(getattr(stream, "cuda_stream", stream)), device=device)
        with torch.cuda.stream(stream):      # (None: as it is)
            return torch.empty(shape, dtype=dtype, device=device)

    def append(self, q, k, v, new_off=None, q_out=None, stream=None, position=None) -> torch.Tensor:
        if q_out is None:
            q_out = self._new(q.shape, q.dtype, stream)
        if position is not None:
            B.kv_page_append_at(self.pages, q, k, v, new_off, self.seq_len, self.page_table, self.rope, position, self.axis, q_out,
                                self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.abstract, self.chunk_off, self.n_chunks,
                                self.status, stream)
            return q_out
        B.kv_page_append(self.pages, q, k, v, new_off, self.seq_len, self.page_table, self.rope, q_out, self.k_pages,
                         self.v_pages, self.k_scale, self.v_scale, self.abstract, self.chunk_off, self.n_chunks, self.status,
                         stream)
        return q_out

    def attend(self, q, stream=None) -> torch.Tensor:
        """q [B, Hq, 128], rotated; out [B, Hq, 128] float."""
        idx = count = None
        if self.selects:
            B.chunk_score(self.shape, q, self.abstract, self.n_chunks, self.score, None, stream)
            B.chunk_topk_select(self.shape, self.score, self.chunk_off, self.n_chunks, self.max_chunks, self.token_budget,
                                self.sel_idx, self.sel_count, None, None, stream)
            idx, count = self.sel_idx, self.sel_count
        B.page_attention_decode(self.pages, q, self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.page_table,
                                self.seq_len, idx, count, self.scale, self.out, self.lse, self.workspace, stream)
        self.lse_of_all = not self.selects
        return self.out

    def attend_shared(self, q, group_off, group_pages, stream=None) -> torch.Tensor:
        """As attend over all pages; sequences group_off[g] .. group_off[g + 1] - 1 list the same group_pages[g] pages first."""
        if self.shared_workspace is None or group_pages.numel() > self.groups:
            raise ValueError("PagedLayer was made for %d groups" % self.groups)
        B.page_attention_decode_shared(self.pages, q, self.k_pages, self.v_pages, self.k_scale, self.v_scale, self.page_table, self.seq_len,
                                       group_off, group_pages, self.scale, self.out, self.lse, self.shared_workspace, stream)
        self.lse_of_all = True
        return self.out

    def weigh(self, q, n_seen, new_off=None, lse=None, decay: float = 1.0, stream=None) -> None:
        """q (rotated) and lse of an attention call of this step, over all pages.  lse None: what attend or attend_shared left; refused
        after prompt, which leaves its logarithms in the lse that it is given, and after attend under a budget: that is over the kept
        pages, and the other pages' tokens would get weight that nobody gave them."""
        if self.weight is None:
            raise ValueError("PagedLayer was made without evictions")
        if lse is None and not self.lse_of_all:
            raise ValueError("lse: the layer's last attention was over kept pages or a prompt's, or there was none")
        B.page_weight_add(self.pages, q, new_off, self.k_pages, self.k_scale, self.page_table, self.seq_len, self.scale,
                          self.lse if lse is None else lse, decay, self.weight, self.weight, n_seen, self.token_id, stream)

    def evict(self, keep_len, n_seen, n_first=None, n_recent: int = 0, stream=None) -> torch.Tensor:
        """keep_len, n_seen, n_first [B] int32; new lengths [B] int32 (evict_status says where nothing could be done).  The first n_first
        tokens stay where they are.  Pages that several sequences list must be among them, or one sequence's rows would be moved into
        what the others read: n_first says at least how many tokens those hold, and a layer made with `groups` wants it given."""
        if self.weight is None:
            raise ValueError("PagedLayer was made without evictions")
        if n_first is None and self.groups:
            raise ValueError("n_first: tokens of shared pages must stay where they are")
        B.page_evict_select(self.pages, self.weight, self.token_id, n_seen, self.seq_len, keep_len, n_first, n_recent, self.moves,
                            self.move_count, self.new_len, self.evict_status, self.evict_workspace, stream)
        B.kv_page_move(self.pages, self.moves, self.move_count, self.seq_len, self.new_len, self.page_table, self.k_pages, self.v_pages,
                       self.k_scale, self.v_scale, self.weight, self.token_id, self.abstract, self.chunk_off, self.n_chunks, stream)
        return self.new_len

    def step(self, q, k, v, q_out=None, stream=None, position=None) -> torch.Tensor:
        """One new token per sequence: q [B, Hq, 128], k, v [B, Hkv, 128]."""
        return self.attend(self.append(q, k, v, None, q_out, stream, position), stream)

    def prompt(self, q, k, v, new_off, out=None, lse=None, q_out=None, stream=None, position=None) -> torch.Tensor:
        """Sequence b's new tokens are rows new_off[b] .. new_off[b + 1]; out [n, Hq, 128] in q's type."""
        q_out = self.append(q, k, v, new_off, q_out, stream, position)
        out = self._new(q_out.shape, q_out.dtype, stream) if out is None else out
        need = B.leoam_page_workspace_bytes(self.pages, q_out.shape[0])
        if not self.prompt_workspaces or self.prompt_workspaces[-1].numel() < need:
            # (a longer prompt needs a few bytes more: whole MiB, so that such steps do not pile up)
            self.prompt_workspaces.append(self._new(-(-need >> 20) << 20, torch.uint8, stream))
        B.page_attention_prefill(self.pages, q_out, new_off, self.k_pages, self.v_pages, self.k_scale, self.v_scale,
                                 self.page_table, self.seq_len, self.scale, out, lse, self.prompt_workspaces[-1], stream)
        self.lse_of_all = False      # (self.lse is an earlier step's)
        return out
