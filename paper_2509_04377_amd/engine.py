"""Host-side sequencing of C-ABI calls: the state of one paged cache, the decode step, and a multi-layer driver.

Nothing here computes a step of the path; every operation is a call into libpe through binding.py.  What
lives here is the control flow that belongs to the caller of the library: which calls a decode step makes
(Alg. 3: score + evict when a sequence's newest page has just filled at budget, then append, then attend),
and an integer mirror of the sequence lengths, so that the host can tell trigger steps without reading
anything back from the device (the kernels evaluate the same predicate on the device lengths).

Multi-layer driver: all layers' pages live in one physical pool; the block table is
[layers * S, Hk, max_blocks] with layer l owning rows l*S .. (l+1)*S - 1 ("layers folded into the sequence
dimension").  Scoring, eviction and the prefill prune see the folded table in ONE launch each; append and
attention are launched per layer, in layer order, because in a model layer l+1's query depends on layer l's
output.

Beside the paper's step there are three more: a verification of drafted tokens (tree_decode, then accept_path, which scores and
evicts between the accepted tokens where single steps would have), attention over the pages with the highest bounds
(select_pages) and eviction by the attention that pages got (evict_by_attention).
"""
from dataclasses import dataclass, replace
from typing import List, Optional

import torch

from . import binding as pe


class HostOnly:
    """While active, the drivers below advance their host-side bookkeeping (length mirror, which lengths array is
    current) without calling the library: the launches of such a step are replayed from a captured HIP graph."""
    active = False

    def __enter__(self):
        HostOnly.active = True

    def __exit__(self, *exc):
        HostOnly.active = False


def host_only():
    return HostOnly()


def _launch(fn, *args):
    """Call a binding function unless the step's launches come from a graph replay."""
    if not HostOnly.active:
        fn(*args)


def triggers(host_lens, block_size: int, budget: int) -> List[bool]:
    """Alg. 3's branch per sequence: the newest page has just filled (L % B == 0) and the sequence holds at
    least the budget (with a budget >= context nothing is ever evicted: Sec. 4.3)."""
    return [n > 0 and n % block_size == 0 and n >= budget for n in host_lens]


def evicts_within(n, tokens, block_size: int, budget: int) -> bool:
    """Whether a sequence of n cached tokens that takes on so many more is to lose a page on the way."""
    full = max(-(-max(n, budget) // block_size), 1) * block_size   # the first length from n on at which a page goes
    return tokens > full - n


@dataclass
class PagedCache:
    """Device-side state of one paged KV cache (one layer, or several layers folded into num_seqs).

    Owns nothing but tensors; every operation is a C-ABI call."""
    desc: pe.pe_cache_desc
    k_pool: torch.Tensor       # [P, B, D]
    v_pool: torch.Tensor       # [P, B, D]
    block_table: torch.Tensor  # [S, Hk, max_blocks] int32
    seq_lens: torch.Tensor     # [S] int32
    spare: torch.Tensor        # [S, Hk, n_spare] int32
    spare_used: torch.Tensor   # [S, Hk] int32
    freed_phys: torch.Tensor   # [S, Hk] int32
    evicted_logical: torch.Tensor  # [S, Hk] int32
    scores: torch.Tensor       # [S, Hk, max_blocks] fp32
    budget: int
    decode_ws: torch.Tensor = None
    host_lens: list = None     # host mirror of seq_lens (pure integer bookkeeping, never read back)
    seq_lens_alt: torch.Tensor = None  # second lengths array for pe_append_paged_decode (swapped after each call)
    cached_scores: bool = False    # keep `scores` alive across steps and score only newly filled pages
    host_scored: list = None       # per sequence: full pages whose score is in `scores` (host bookkeeping)
    evict_opts: pe.pe_evict_opts = None  # eviction variant (policy, protected pages, shared heads); None = Alg. 3
    fused_evict: bool = False  # score + evict of a trigger step in one pass over the pages (pe_score_evict)
    selection: "Selection" = None  # attend to selected pages only (select_pages)
    attention: "Attention" = None  # `scores` are the attention that pages got (evict_by_attention)

    @staticmethod
    def create(dtype, num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, layout, budget, device="cuda",
               k_pool=None, v_pool=None, shared=False, decode_opts=None):
        """`layout`: block table, spare lists and pool size (synth.page_layout).  shared=True builds the
        head-shared cache (pe.PE_LAYOUT_SHARED): `layout` then describes ONE row per sequence (a layout made for a
        single KV head), pools are [P, B, Hk, D] and the per-row arrays lose their head dimension.  decode_opts:
        decode_splits / decode_shape / decode_flat_order of the descriptor (launch shape of the attention)."""
        desc = pe.make_desc(dtype, num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, layout.max_blocks,
                            layout.num_phys_blocks, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD,
                            **(decode_opts or {}))
        table, spare = layout.block_table, layout.spare
        if shared:
            assert table.shape[1] == 1, "a shared cache takes a layout with one row per sequence"
            table, spare = table[:, 0], spare[:, 0]
            shape = (layout.num_phys_blocks, block_size, num_kv_heads, head_dim)
            per_row = (num_seqs,)
        else:
            shape = (layout.num_phys_blocks, block_size, head_dim)
            per_row = (num_seqs, num_kv_heads)
        if k_pool is None:
            k_pool = torch.zeros(shape, dtype=dtype, device=device)
            v_pool = torch.zeros(shape, dtype=dtype, device=device)
        i32 = dict(dtype=torch.int32, device=device)
        cache = PagedCache(desc, k_pool, v_pool, table.to(device).contiguous(),
                           torch.zeros(num_seqs, **i32), spare.to(device).contiguous(),
                           torch.zeros(per_row, **i32), torch.full(per_row, -1, **i32),
                           torch.full(per_row, -1, **i32),
                           torch.empty((num_seqs, num_kv_heads, layout.max_blocks), dtype=torch.float32, device=device),
                           int(budget))
        cache.decode_ws = pe.alloc_workspace(pe.PE_OP_PAGED_DECODE, desc, device=device)
        cache.host_lens = [0] * num_seqs
        return cache

    @property
    def shared(self) -> bool:
        return self.desc.layout == pe.PE_LAYOUT_SHARED

    def prefill_prune(self, k_in, v_in, cu_seqlens, max_seqlen, kept_idx_out=None, workspace=None):
        total = k_in.shape[0]
        if workspace is None:
            workspace = pe.alloc_workspace(pe.PE_OP_PREFILL_PRUNE, self.desc, total, device=k_in.device)
        _launch(pe.pe_prefill_prune, self.desc, k_in, v_in, cu_seqlens, total, max_seqlen, self.budget, self.k_pool, self.v_pool,
                         self.block_table, self.seq_lens, kept_idx_out, workspace)

    def set_host_lens(self, prompt_lens):
        """Tell the host mirror what the prune was given: cached length = min(L, C)."""
        self.host_lens = [min(int(L), self.budget) for L in prompt_lens]
        if self.selection is not None:
            self.selection.seen = None
        if self.attention is not None:
            self.attention.started = False

    def triggers(self) -> List[bool]:
        return triggers(self.host_lens, self.desc.block_size, self.budget)

    def any_trigger(self) -> bool:
        return any(self.triggers())

    def append_paged_decode(self, new_k, new_v, q, out, softmax_scale=None):
        if softmax_scale is None:
            softmax_scale = float(self.desc.head_dim) ** -0.5
        if self.seq_lens_alt is None:
            self.seq_lens_alt = torch.empty_like(self.seq_lens)
        _launch(pe.pe_append_paged_decode, self.desc, new_k, new_v, q, self.k_pool, self.v_pool, self.block_table,
                self.seq_lens, self.seq_lens_alt, self.freed_phys, self.spare, self.spare_used, softmax_scale, out,
                self.decode_ws)
        self.seq_lens, self.seq_lens_alt = self.seq_lens_alt, self.seq_lens

    def decode_step(self, new_k, new_v, q, out, softmax_scale=None, fused=True):
        """One decode iteration of one layer (Alg. 3): score + evict when some sequence's newest page has
        filled at budget, append the new token, attend.  Which steps trigger follows from the lengths
        alone, so the host decides it without reading anything back."""
        trig = self.triggers()
        if self.selection is not None:
            self.bound_pages()
        if any(trig):
            if self.attention is not None and not self.attention.started:   # nothing seen yet: this step's queries look first
                self.paged_decode_weights(q, torch.empty_like(q), softmax_scale)   # (out may be q, which is needed again)
            self.score_and_evict()
            self.evicted(trig)
        self.append_and_attend(new_k, new_v, q, out, softmax_scale, fused)
        self.host_lens = [n + 1 for n in self.host_lens]

    def evicted(self, which):
        """Bookkeeping behind an eviction of these sequences."""
        self.host_lens = [n - self.desc.block_size if t else n for n, t in zip(self.host_lens, which)]
        if self.selection is not None and self.selection.seen is not None:
            self.selection.seen = [n - t for n, t in zip(self.selection.seen, which)]

    def append_and_attend(self, new_k, new_v, q, out, softmax_scale=None, fused=True):
        """What a step launches behind an eviction.  Selected pages and attention weights have no fused form."""
        if self.selection is not None or self.attention is not None:
            self.append_kv(new_k, new_v)
            (self.selected_decode if self.selection is not None else self.paged_decode_weights)(q, out, softmax_scale)
        elif fused:
            self.append_paged_decode(new_k, new_v, q, out, softmax_scale)
        else:
            self.append_kv(new_k, new_v)
            self.paged_decode(q, out, softmax_scale)

    def score_blocks(self):
        _launch(pe.pe_score_blocks, self.desc, self.k_pool, self.v_pool, self.block_table, self.seq_lens, self.scores)

    def score_triggered_blocks(self):
        _launch(pe.pe_score_triggered_blocks, self.desc, self.k_pool, self.v_pool, self.block_table, self.seq_lens, self.budget,
                                  self.scores)

    def evict_blocks(self):
        _launch(pe.pe_evict_blocks, self.desc, self.scores, self.block_table, self.seq_lens, self.budget, self.evicted_logical,
                        self.freed_phys)

    def score_and_evict(self):
        """Score + evict of a trigger step.  With cached scores only the pages filled since the last call are
        scored (all of them the first time) and the eviction keeps the score rows aligned with the table."""
        B = self.desc.block_size
        if self.attention is not None:   # the scores are there; the newest page, which has had no time to be attended to, stays
            if not self.attention.started:
                raise RuntimeError("no attention step before the first eviction: nothing to choose a page by")
            o = self.evict_opts or pe.pe_evict_opts(pe.PE_POLICY_LOWEST_SCORE, 0, 1, 0, 0)
            opts = pe.pe_evict_opts(o.policy, o.protect_first, o.protect_last, o.share_heads, 1)
            _launch(pe.pe_evict_blocks_ex, self.desc, opts, self.scores, self.block_table, self.seq_lens, self.budget,
                    self.evicted_logical, self.freed_phys)
            return
        if self.evict_opts is not None:
            o = self.evict_opts
            opts = pe.pe_evict_opts(o.policy, o.protect_first, o.protect_last, o.share_heads, 0)
            if o.policy != pe.PE_POLICY_OLDEST:
                self.score_triggered_blocks()
            _launch(pe.pe_evict_blocks_ex, self.desc, opts, self.scores if o.policy != pe.PE_POLICY_OLDEST else None,
                               self.block_table, self.seq_lens, self.budget, self.evicted_logical, self.freed_phys)
            return
        if self.fused_evict and not self.cached_scores:
            _launch(pe.pe_score_evict, self.desc, self.k_pool, self.v_pool, self.block_table, self.seq_lens, self.budget, None,
                           self.evicted_logical, self.freed_phys)
            return
        if not self.cached_scores:   # Alg. 3: score the pages of the sequences that evict now, then evict
            self.score_triggered_blocks()
            self.evict_blocks()
            return
        full = [n // B for n in self.host_lens]
        if self.host_scored is None:
            self.score_blocks()
        else:
            recent = max(f - sc for f, sc in zip(full, self.host_scored))
            if recent > 0:
                _launch(pe.pe_score_recent_blocks, self.desc, self.k_pool, self.v_pool, self.block_table, self.seq_lens, recent,
                                       self.scores)
        _launch(pe.pe_evict_blocks_cached, self.desc, self.scores, self.block_table, self.seq_lens, self.budget,
                               self.evicted_logical, self.freed_phys)
        self.host_scored = [f - 1 if t else f for f, t in zip(full, self.triggers())]

    def append_kv(self, new_k, new_v):
        _launch(pe.pe_append_kv, self.desc, new_k, new_v, self.k_pool, self.v_pool, self.block_table, self.seq_lens,
                self.freed_phys, self.spare, self.spare_used)

    def paged_decode(self, q, out, softmax_scale=None):
        if softmax_scale is None:
            softmax_scale = float(self.desc.head_dim) ** -0.5
        _launch(pe.pe_paged_decode, self.desc, q, self.k_pool, self.v_pool, self.block_table, self.seq_lens, softmax_scale,
                out, self.decode_ws)


    # ---- verification of drafted tokens ----

    def tree_decode(self, q, k_draft, v_draft, tree_mask, out, draft_lens=None, softmax_scale=None, workspace=None):
        """Attention of q [S, T, Hq, D] over the cache and the drafts that tree_mask [S, T] names (int64 words); the cache is read only,
        and all of it also where steps attend to selected pages."""
        if softmax_scale is None:
            softmax_scale = float(self.desc.head_dim) ** -0.5
        T = int(q.shape[1])
        if workspace is None:
            workspace = pe.alloc_workspace(pe.PE_OP_TREE_DECODE, self.desc, T, device=q.device)
        _launch(pe.pe_tree_decode, self.desc, T, q, k_draft, v_draft, draft_lens, tree_mask, self.k_pool, self.v_pool,
                self.block_table, self.seq_lens, softmax_scale, out, workspace)

    def accept_path(self, k_draft, v_draft, path, path_lens, host_path_lens):
        """Append the drafts path[s][:path_lens[s]] (path [S, P] and path_lens [S] int32 on the device, host_path_lens the latter's
        values, at most P; every named draft exists).  The effect on the cache is that of as many single steps: before a token joins a
        sequence whose newest page is full and which is at budget, a page of that sequence goes, and of no other: a sequence
        whose path ends with a full page keeps its pages until it goes on.  With evict_by_attention a decode step has to come before
        a path on which pages go (a tree leaves no weights); what is refused leaves the cache as it was."""
        B = self.desc.block_size
        left = [int(n) for n in host_path_lens]
        if len(left) != len(self.host_lens) or min(left) < 0 or max(left) > path.shape[-1]:
            raise ValueError("host_path_lens: one length per sequence, 0 to path.shape[-1]")
        room = self.desc.max_blocks * B
        if self.budget > room and any(n + m > room for n, m in zip(self.host_lens, left)):
            raise ValueError("the path is longer than what is left of a table row, and nothing is evicted below the budget")
        if self.attention is not None and not self.attention.started and any(evicts_within(n, m, B, self.budget)
                                                                             for n, m in zip(self.host_lens, left)):
            raise RuntimeError("no attention step before the first eviction: nothing to choose a page by")
        path_done = torch.zeros_like(path_lens)
        while any(left):
            trig = self.triggers()
            now = [t and n > 0 for t, n in zip(trig, left)]
            if any(now):
                if now == trig:
                    self.score_and_evict()
                else:
                    self._score_and_evict_of(now)
                self.evicted(now)
            _launch(pe.pe_append_path, self.desc, k_draft, v_draft, path, path_lens, path_done, self.k_pool, self.v_pool,
                    self.block_table, self.seq_lens, self.freed_phys, self.spare, self.spare_used)
            taken = [min(m, B - n % B) for n, m in zip(self.host_lens, left)]
            self.host_lens = [n + t for n, t in zip(self.host_lens, taken)]
            left = [m - t for m, t in zip(left, taken)]

    def _score_and_evict_of(self, now):
        """score_and_evict for some sequences only: a call for each run of neighbours."""
        if self.cached_scores and self.host_scored is None and self.evict_opts is None and self.attention is None:
            self.score_blocks()
            self.host_scored = [n // self.desc.block_size for n in self.host_lens]
        first = 0
        while first < len(now):
            end = first + 1
            while end < len(now) and now[end] == now[first]:
                end += 1
            if now[first]:
                part = self.rows(first, end)
                part.score_and_evict()
                if part.host_scored is not None:
                    self.host_scored[first:end] = part.host_scored
            first = end

    def rows(self, first, end):
        """The same cache's sequences first .. end - 1, as a cache (views; host_lens and host_scored are copies)."""
        d, sl = self.desc, slice(first, end)
        fields = {name: getattr(d, name) for name, _ in d._fields_}
        views = {name: getattr(self, name)[sl] for name in ("block_table", "seq_lens", "spare", "spare_used", "freed_phys",
                                                            "evicted_logical", "scores", "host_lens")}
        return replace(self, desc=pe.pe_cache_desc(**{**fields, "num_seqs": end - first}), **views, seq_lens_alt=None, selection=None,
                       host_scored=None if self.host_scored is None else self.host_scored[sl])

    # ---- attention over selected pages ----

    def select_pages(self, num_pages, bounds=None):
        """From now on a step attends to the num_pages pages with the highest bounds only (the newest among them); 0: to all.
        bounds: as pe_page_bounds keeps them (several layers of one pool share them)."""
        if num_pages and self.attention is not None:
            raise ValueError("attention weights are kept over all pages, not over selected ones")
        self.selection = Selection.create(self, int(num_pages), bounds) if num_pages else None

    def bound_pages(self):
        """Bounds of the pages that have filled since the last call (the first time: of all full ones).  Due before a selection that
        has a newer page; a selection never asks for the newest page's."""
        sel, B = self.selection, self.desc.block_size
        recent = sel.recent(self.host_lens, B)
        if recent != 0:
            _launch(pe.pe_page_bounds, self.desc, self.k_pool, self.block_table, self.seq_lens, max(recent, 0), sel.bounds)
        sel.seen = [n // B for n in self.host_lens]

    def selected_decode(self, q, out, softmax_scale=None):
        if softmax_scale is None:
            softmax_scale = float(self.desc.head_dim) ** -0.5
        sel = self.selection
        _launch(pe.pe_select_pages, self.desc, q, sel.bounds, self.block_table, self.seq_lens, sel.num_pages, sel.table, sel.lens,
                None, sel.select_ws)
        _launch(pe.pe_paged_decode, sel.desc, q, self.k_pool, self.v_pool, sel.table, sel.lens, softmax_scale, out, sel.decode_ws)

    # ---- eviction by the attention that pages got ----

    def evict_by_attention(self, decay=1.0):
        """From now on `scores` hold the attention weight of each page (decay: what is left of it a step later), and the page with
        the least goes.  The choice, protected pages and shared heads are evict_opts'; without them the newest page is protected.
        The weights are those of decode steps (one that has to evict before there are any looks with its own queries first)."""
        if self.selection is not None:
            raise ValueError("attention weights are kept over all pages, not over selected ones")
        self.attention = Attention(float(decay), pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, self.desc, device=self.k_pool.device))

    def paged_decode_weights(self, q, out, softmax_scale=None):
        if softmax_scale is None:
            softmax_scale = float(self.desc.head_dim) ** -0.5
        att = self.attention
        _launch(pe.pe_paged_decode_weights, self.desc, q, self.k_pool, self.v_pool, self.block_table, self.seq_lens, softmax_scale,
                att.decay, self.scores if att.started else None, self.scores, out, att.workspace)
        att.started = True


@dataclass
class Selection:
    """What a step over selected pages keeps."""
    num_pages: int
    bounds: torch.Tensor       # [P, 2, D] (shared: [P, 2, Hk, D])
    table: torch.Tensor        # [S, Hk, num_pages] int32 (shared: [S, num_pages])
    lens: torch.Tensor         # [S] int32
    desc: pe.pe_cache_desc     # of the cache with that table
    select_ws: torch.Tensor
    decode_ws: torch.Tensor
    seen: list = None          # full pages per sequence at the last bound_pages; None before the first

    @staticmethod
    def create(cache, num_pages, bounds=None):
        d, dev = cache.desc, cache.k_pool.device
        desc = pe.pe_cache_desc(**{**{name: getattr(d, name) for name, _ in d._fields_}, "max_blocks": num_pages})
        if bounds is None:
            heads = (d.num_kv_heads,) if cache.shared else ()
            bounds = torch.empty((d.num_phys_blocks, 2) + heads + (d.head_dim,), dtype=cache.k_pool.dtype, device=dev)
        return Selection(num_pages, bounds, torch.empty(cache.block_table.shape[:-1] + (num_pages,), dtype=torch.int32, device=dev),
                         torch.empty_like(cache.seq_lens), desc, pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, d, device=dev),
                         pe.alloc_workspace(pe.PE_OP_PAGED_DECODE, desc, device=dev))

    def recent(self, lens, B):
        """How many of the newest full pages may have no bounds; -1: all.  (An eviction takes one off both counts, so that it is one
        too many where a page without bounds went.)"""
        if self.seen is None:
            return -1
        return max([n // B - s for n, s in zip(lens, self.seen)] + [0])


@dataclass
class Attention:
    """What a step that keeps attention weights needs beside the scores."""
    decay: float
    workspace: torch.Tensor
    started: bool = False      # the scores hold weights


class LayeredCache:
    def __init__(self, dtype, layers, num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, layout, budget,
                 device="cuda", shared=False, decode_opts=None):
        self.layers, self.S = layers, num_seqs
        self.Hk, self.Hq, self.D, self.B = num_kv_heads, num_q_heads, head_dim, block_size
        self.dtype, self.budget, self.device = dtype, int(budget), device
        R = layers * num_seqs
        assert layout.block_table.shape[0] == R
        self.folded = PagedCache.create(dtype, R, num_kv_heads, num_q_heads, head_dim, block_size, layout, budget,
                                        device, shared=shared)
        f = self.folded
        self.per_layer: List[PagedCache] = []
        for l in range(layers):
            sl = slice(l * num_seqs, (l + 1) * num_seqs)
            desc = pe.make_desc(dtype, num_seqs, num_kv_heads, num_q_heads, head_dim, block_size, layout.max_blocks,
                                layout.num_phys_blocks, pe.PE_LAYOUT_SHARED if shared else pe.PE_LAYOUT_PER_HEAD,
                                **(decode_opts or {}))
            c = PagedCache(desc, f.k_pool, f.v_pool, f.block_table[sl], f.seq_lens[sl], f.spare[sl],
                              f.spare_used[sl], f.freed_phys[sl], f.evicted_logical[sl], f.scores[sl], int(budget))
            self.per_layer.append(c)
        # one split workspace serves every layer: launches are ordered on one stream
        self.decode_ws = pe.alloc_workspace(pe.PE_OP_PAGED_DECODE, self.per_layer[0].desc, device=device)
        # second lengths array for the fused append + attention call; all layers swap in lockstep
        f.seq_lens_alt = torch.empty_like(f.seq_lens)
        for l, c in enumerate(self.per_layer):
            c.decode_ws = self.decode_ws
            c.seq_lens_alt = f.seq_lens_alt[l * num_seqs:(l + 1) * num_seqs]
        self.fused = True
        self.native_layers = True   # fused mode: the per-layer launches are issued by one native call
        self.host_lens = [0] * num_seqs   # the same in every layer

    def prefill_prune_layer(self, layer, k_in, v_in, cu_seqlens, max_seqlen, kept_idx_out=None, workspace=None):
        self.per_layer[layer].prefill_prune(k_in, v_in, cu_seqlens, max_seqlen, kept_idx_out, workspace)

    def set_host_lens(self, prompt_lens):
        self.host_lens = [min(int(L), self.budget) for L in prompt_lens]
        for c in [self.folded] + self.per_layer:
            c.set_host_lens(list(prompt_lens) * (self.layers if c is self.folded else 1))

    def _triggers(self):
        return triggers(self.host_lens, self.B, self.budget)

    def decode_step(self, new_k, new_v, q, out, softmax_scale: Optional[float] = None, layer_hook=None):
        """new_k, new_v [layers, S, Hk, D]; q, out [layers, S, Hq, D].  One decode iteration of all layers."""
        trig = self._triggers()
        f = self.folded
        f.host_lens = self.host_lens * self.layers
        if f.selection is not None:
            f.bound_pages()
        if any(trig):
            if f.attention is not None and not f.attention.started:
                for l, c in enumerate(self.per_layer):
                    c.paged_decode_weights(q[l], torch.empty_like(q[l]), softmax_scale)   # (out may be q, which is needed again)
                f.attention.started = True
            f.score_and_evict()
            f.evicted(trig * self.layers)
            self.host_lens = f.host_lens[:self.S]
        fused = self.fused and f.selection is None and f.attention is None
        if fused and self.native_layers:
            # one native call issues the fused append + attention launch of every layer, in layer order
            if layer_hook is not None:
                layer_hook(0, 0)
            _launch(pe.pe_append_paged_decode_layers, self.per_layer[0].desc, self.layers, new_k, new_v, q, f.k_pool, f.v_pool,
                                             f.block_table, f.seq_lens, f.seq_lens_alt, f.freed_phys, f.spare,
                                             f.spare_used, float(self.D) ** -0.5 if softmax_scale is None
                                             else softmax_scale, out, self.decode_ws)
            if layer_hook is not None:
                layer_hook(self.layers - 1, 1)
            for c in self.per_layer:
                c.seq_lens, c.seq_lens_alt = c.seq_lens_alt, c.seq_lens
        for l, c in enumerate(self.per_layer if not (fused and self.native_layers) else ()):
            if fused or f.selection is not None or f.attention is not None:
                if layer_hook is not None:
                    layer_hook(l, 0)
                c.append_and_attend(new_k[l], new_v[l], q[l], out[l], softmax_scale)
            else:
                c.append_kv(new_k[l], new_v[l])
                if layer_hook is not None:
                    layer_hook(l, 0)
                c.paged_decode(q[l], out[l], softmax_scale)
            if layer_hook is not None:
                layer_hook(l, 1)
        if f.attention is not None:
            f.attention.started = True
        if fused:   # every layer wrote its new lengths into the other array
            f.seq_lens, f.seq_lens_alt = f.seq_lens_alt, f.seq_lens
        self.host_lens = [n + 1 for n in self.host_lens]
        return any(trig)

    def tree_decode_layer(self, layer, q, k_draft, v_draft, tree_mask, out, draft_lens=None, softmax_scale=None, workspace=None):
        self.per_layer[layer].tree_decode(q, k_draft, v_draft, tree_mask, out, draft_lens, softmax_scale, workspace)

    def accept_path(self, k_draft, v_draft, path, path_lens, host_path_lens):
        """PagedCache.accept_path in every layer at once: k_draft, v_draft [layers, S, T, Hk, D]; path [S, P], path_lens [S]."""
        f = self.folded
        f.host_lens = self.host_lens * self.layers
        try:
            f.accept_path(k_draft.flatten(0, 1), v_draft.flatten(0, 1), path.repeat(self.layers, 1), path_lens.repeat(self.layers),
                          list(host_path_lens) * self.layers)
        finally:
            self.host_lens = f.host_lens[:self.S]

    def select_pages(self, num_pages):
        """PagedCache.select_pages in every layer; the pool's bounds are kept by one launch for all of them."""
        self.folded.select_pages(num_pages)
        one = None
        if num_pages:   # launches are ordered on one stream: one set of tables and workspaces serves every layer
            one = Selection.create(self.per_layer[0], int(num_pages), self.folded.selection.bounds)
        for c in self.per_layer:
            c.selection = one

    def evict_by_attention(self, decay=1.0):
        """PagedCache.evict_by_attention in every layer."""
        self.folded.evict_by_attention(decay)
        one = pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, self.per_layer[0].desc, device=self.device)
        for c in self.per_layer:
            c.attention = Attention(float(decay), one)


class GraphedStepper:
    """Replays the launches of a decode step from captured HIP graphs (one per distinct launch sequence).

    The inputs live in fixed buffers (new_k, new_v, q, out), as a serving loop would keep them.  A step's
    launch sequence depends only on host-side integers (which lengths array is current, whether this is a
    trigger step, how many pages the cached-score mode has to score) and on what select_pages and evict_by_attention
    have put into the caches, so that these key the graph.  The first step with a new key is captured and then
    replayed; later ones advance the host bookkeeping with the launches switched off and replay the stored graph.
    A graph's selection or attention, whose tensors it points into, is held beside it; when another one (or none) has
    taken its place, the next step lets go of both."""

    def __init__(self, eng: "LayeredCache", new_k, new_v, q, out, softmax_scale: Optional[float] = None):
        self.eng, self.args = eng, (new_k, new_v, q, out, softmax_scale)
        self.graphs = {}   # key: (graph, selections and attentions of all caches)
        self.modes = (None, None)   # the folded cache's at the last step: they change in all caches together

    def _key(self):
        e, f = self.eng, self.eng.folded
        trig = any(e._triggers())
        recent = None
        if trig and f.cached_scores:
            if f.host_scored is None:
                recent = -1
            else:
                recent = max(n // e.B - sc for n, sc in zip(e.host_lens * e.layers, f.host_scored))
        fresh = None if f.selection is None else (id(f.selection), f.selection.recent(e.host_lens * e.layers, e.B))
        seen = None if f.attention is None else (id(f.attention), f.attention.decay, f.attention.started)
        opts = f.evict_opts and tuple(getattr(f.evict_opts, name) for name, _ in f.evict_opts._fields_)
        return (f.seq_lens.data_ptr(), trig, e.fused, f.cached_scores, f.fused_evict, recent, fresh, seen, opts)

    def _forget(self):
        """Drop the graphs that point into a selection or an attention that is no longer in use."""
        f = self.eng.folded
        if f.selection is self.modes[0] and f.attention is self.modes[1]:
            return
        self.modes = (f.selection, f.attention)
        stale = [k for k, (_, of) in self.graphs.items() if any(m is not None and m is not now for m, now in zip(of, self.modes))]
        if stale:
            torch.cuda.synchronize()   # a replay may be on its way
            for k in stale:
                del self.graphs[k]

    def step(self) -> bool:
        self._forget()
        key = self._key()
        g, _ = self.graphs.get(key, (None, None))
        if g is None:
            g = torch.cuda.CUDAGraph()
            with torch.cuda.graph(g):
                trig = self.eng.decode_step(*self.args)
            self.graphs[key] = (g, [m for c in [self.eng.folded] + self.eng.per_layer for m in (c.selection, c.attention)])
        else:
            with host_only():
                trig = self.eng.decode_step(*self.args)
        g.replay()
        return trig
