"""Attention over the paged cache beyond one dense query a sequence, as cases that can be timed and checked.

  tree     pe_tree_decode: the attention of a tree of drafted tokens, each of which attends to the whole cache and to
           the drafts that its mask names (speculative decoding: one call verifies all drafts of every sequence).
  commit   pe_append_path, twice, with an eviction of the oldest page between: the accepted path of a tree joins the
           cache at its budget. The path has as many tokens as a page, so the cache is as long afterwards as before.
  weights  pe_paged_decode_weights: one query a sequence, and the softmax weight that each page got added up for an
           eviction by accumulated attention.
  sparse   pe_select_pages, then pe_paged_decode on the selected pages: a long cache of which each query reads the
           pages whose keys can give the largest products. `bounds` says what the step does in front of it: "none";
           "recent", the bounds of the page that has just filled (pe_page_bounds); "all", those of a whole prompt.

A case is a dict of plain values: `kind`; `dtype`, `layout`, `seqs`, `kv_heads`, `q_heads`, `head_dim`, `page`,
`min_len`, `max_len` everywhere (lengths are spread evenly between the two, in an order that the seed gives); `drafts`
for tree; `pages` (selected ones) and `bounds` for sparse.
"""
import math

import numpy as np
import torch

own = False   # True: run() calls the library; False: the same in plain torch operations, in 32 bits and more

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
DECAY = 0.9375
INF = float("inf")


def _case(name, kind, dtype, layout, seqs, kv_heads, q_heads, head_dim, page, min_len, max_len, **more):
    return dict({"name": name, "kind": kind, "dtype": dtype, "layout": layout, "seqs": seqs, "kv_heads": kv_heads,
                 "q_heads": q_heads, "head_dim": head_dim, "page": page, "min_len": min_len, "max_len": max_len}, **more)


def _unnamed(*args, **more):
    case = _case("", *args, **more)
    del case["name"]
    return case


def listed():
    return [
        # four drafts of one sequence of the 1B shape: the smallest verification, bound by latency
        _case("tree_1b_one", "tree", "bf16", "per_head", 1, 8, 32, 64, 16, 1000, 1000, drafts=4),
        # a serving batch of the 8B shape at its budget, a small tree for each sequence: still bound by the cache
        _case("tree_8b_batch", "tree", "bf16", "per_head", 32, 8, 32, 128, 16, 1024, 2048, drafts=8),
        # the widest trees over long ragged caches: 256 query rows share a KV head, the matrix products count
        _case("tree_8b_wide", "tree", "bf16", "per_head", 8, 8, 32, 128, 16, 4001, 8192, drafts=64),
        # fp32, head-shared pages, an odd number of drafts, three query heads a KV head
        _case("tree_f32_shared", "tree", "f32", "shared", 4, 4, 12, 64, 32, 37, 1500, drafts=7),
        # accepted paths of a small model's batch (one layer): a few launches
        _case("commit_1b_layer", "commit", "bf16", "per_head", 8, 8, 32, 64, 16, 1024, 1024),
        # all layers of the 8B shape at once, layers folded into the sequences
        _case("commit_8b_model", "commit", "bf16", "per_head", 256, 8, 32, 128, 16, 1024, 1024),
        # one layer of the 1B shape: bound by the chain of a launch
        _case("weights_1b_layer", "weights", "bf16", "per_head", 8, 8, 32, 64, 16, 1024, 1024),
        # the 8B shape at full batch and budget: bound by the cache's traffic
        _case("weights_8b_batch", "weights", "bf16", "per_head", 32, 8, 32, 128, 16, 2033, 2048),
        # fp32, head-shared, ragged, larger pages
        _case("weights_f32_ragged", "weights", "f32", "shared", 6, 4, 8, 128, 32, 1, 3001),
        # an eighth of a 1B cache is read, a page has just filled
        _case("sparse_1b_step", "sparse", "bf16", "per_head", 8, 8, 32, 64, 16, 4096, 4096, pages=32, bounds="recent"),
        # few long sequences: 4096 of 65536 tokens each
        _case("sparse_8b_long", "sparse", "bf16", "per_head", 4, 8, 32, 128, 16, 60001, 65536, pages=256, bounds="none"),
        # behind a batch of long prompts: the bounds of the whole cache, one decision a sequence
        _case("sparse_8b_prompt", "sparse", "bf16", "shared", 16, 8, 32, 128, 32, 8000, 16384, pages=64, bounds="all"),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the ranges above: any supported type, layout, head size, page size and number of query heads a KV head;
    lengths from one token on, odd ones among them; none costs more than the largest listed ones."""
    kind = rng.choice(("tree", "tree", "weights", "sparse", "sparse", "commit"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    layout = rng.choice(("per_head", "shared"))
    group = rng.choice((1, 2, 3, 4, 4, 5, 7, 8))
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    head_dim = rng.choice((64, 128))
    page = rng.choice((16, 16, 32, 64, 128))
    seqs = _log_int(rng, 1, 32)
    if kind == "commit":
        max_len = page * rng.randint(1, max(1, 1024 // page))
        return _unnamed(kind, dtype, layout, _log_int(rng, 1, 128), kv_heads, group * kv_heads, head_dim, page, max_len, max_len)
    if kind == "tree":
        drafts = _log_int(rng, 1, 64)
        # no more logits than the largest listed tree has
        most = min(16384, (1 << 27) // (seqs * kv_heads * group * drafts))
        more = {"drafts": drafts}
    else:
        most = min(65536, (1 << 21) // (seqs * kv_heads))
        more = {"pages": _log_int(rng, 1, 512), "bounds": rng.choice(("none", "recent", "all"))} if kind == "sparse" else {}
    max_len = _log_int(rng, 1, max(1, most))
    # (an empty cache is one of the lengths: a sequence that has just begun)
    min_len = 0 if rng.random() < 0.2 else rng.randint(1, max_len)
    return _unnamed(kind, dtype, layout, seqs, kv_heads, group * kv_heads, head_dim, page, min_len, max_len, **more)


# ---- inputs ------------------------------------------------------------------------------------------------------
def _lens(case):
    """Evenly spread; the seed gives only their order, so that all seeds have the same work."""
    S, lo, hi = case["seqs"], case["min_len"], case["max_len"]
    if case["kind"] == "commit":   # sequences stand at different places of their newest page
        return [hi - 1 - (5 * s) % (case["page"] - 1) for s in range(S)]
    return [hi - (hi - lo) * s // max(1, S - 1) for s in range(S)]


def _rows(shape, g, dtype):
    """Rows of D elements ~ N(0,1) with a lognormal scale per row (token, head)."""
    x = torch.randn(shape, generator=g, device=DEVICE, dtype=torch.float32)
    x *= torch.exp(0.5 * torch.randn(shape[:-1] + (1,), generator=g, device=DEVICE, dtype=torch.float32))
    return x.to(dtype)


def _fill(pool, g):
    step = max(1, (1 << 26) // pool[0].numel())
    for i in range(0, pool.shape[0], step):
        part = pool[i:i + step]
        part.copy_(_rows(tuple(part.shape), g, pool.dtype))


def _trees(S, T, r):
    """Masks of random trees: draft i descends from an earlier one or from the cache's last token, and attends to its
    ancestors and to itself."""
    words = np.zeros((S, T), np.uint64)
    for s in range(S):
        for i in range(T):
            parent = int(r.integers(-1, i)) if i else -1
            words[s, i] = np.uint64(1 << i) | (words[s, parent] if parent >= 0 else np.uint64(0))
    return torch.from_numpy(words.view(np.int64)).to(DEVICE)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    r = np.random.default_rng(int(seed))
    dtype, B, D = DTYPES[case["dtype"]], case["page"], case["head_dim"]
    S, Hk, Hq, shared = case["seqs"], case["kv_heads"], case["q_heads"], case["layout"] == "shared"
    lens = np.array(_lens(case), np.int64)
    r.shuffle(lens)
    rows = 1 if shared else Hk
    need = -(-lens // B)
    if case["kind"] == "commit":
        need = np.full(S, case["max_len"] // B)
    width = int(need.max())
    used = np.broadcast_to(np.arange(width)[None, None, :] < need[:, None, None], (S, rows, width))
    pages = int(used.sum())
    table = np.full((S, rows, width), -1, np.int32)
    table[used] = r.permutation(pages).astype(np.int32)
    if shared:
        table = table[:, 0]
    pool = (pages, B) + ((Hk, D) if shared else (D,))
    state = {"case": case, "k_pool": torch.empty(pool, dtype=dtype, device=DEVICE), "v_pool": torch.empty(pool, dtype=dtype, device=DEVICE),
             "table": torch.from_numpy(np.ascontiguousarray(table)).to(DEVICE),
             "seq_lens": torch.from_numpy(lens.astype(np.int32)).to(DEVICE), "scale": D ** -0.5}
    _fill(state["k_pool"], g)
    _fill(state["v_pool"], g)
    more = {"tree": _prepare_tree, "commit": _prepare_commit, "weights": _prepare_weights, "sparse": _prepare_sparse}
    more[case["kind"]](state, case, dtype, g, r)
    return state


def _desc(state, width=None):
    from paper_2509_04377_amd import binding as pe
    c = state["case"]
    return pe.make_desc(DTYPES[c["dtype"]], c["seqs"], c["kv_heads"], c["q_heads"], c["head_dim"], c["page"],
                        state["table"].shape[-1] if width is None else width, state["k_pool"].shape[0],
                        pe.PE_LAYOUT_SHARED if c["layout"] == "shared" else pe.PE_LAYOUT_PER_HEAD)


def _prepare_tree(state, case, dtype, g, r):
    S, T, Hk, Hq, D = case["seqs"], case["drafts"], case["kv_heads"], case["q_heads"], case["head_dim"]
    state["k_draft"], state["v_draft"] = _rows((S, T, Hk, D), g, dtype), _rows((S, T, Hk, D), g, dtype)
    state["q"] = torch.randn((S, T, Hq, D), generator=g, device=DEVICE).to(dtype)
    state["mask"] = _trees(S, T, r)
    # sequences whose trees are smaller leave their last rows as they were
    counts = np.where(np.arange(S) % 4 == 3, np.maximum(1, T - T // 4), T).astype(np.int32)
    state["draft_lens"] = torch.from_numpy(counts).to(DEVICE)
    state["out"] = torch.zeros_like(state["q"])
    state["lib"] = {}


def _prepare_commit(state, case, dtype, g, r):
    S, Hk, D, B = case["seqs"], case["kv_heads"], case["head_dim"], case["page"]
    T = min(64, 2 * B)
    state["k_draft"], state["v_draft"] = _rows((S, T, Hk, D), g, dtype), _rows((S, T, Hk, D), g, dtype)
    # a page's worth of tokens: up to 64 drafts, some of a page of 128 twice
    state["path"] = torch.from_numpy(np.sort(r.integers(0, T, (S, B)), axis=1).astype(np.int32)).to(DEVICE)
    state["path_lens"] = torch.full((S,), B, dtype=torch.int32, device=DEVICE)
    state["path_done"] = torch.zeros(S, dtype=torch.int32, device=DEVICE)
    per_row = tuple(state["table"].shape[:-1])
    state["spare"] = torch.zeros(per_row + (1,), dtype=torch.int32, device=DEVICE)
    state["spare_used"] = torch.zeros(per_row, dtype=torch.int32, device=DEVICE)
    state["freed"] = torch.full(per_row, -1, dtype=torch.int32, device=DEVICE)
    state["evicted"] = torch.full(per_row, -1, dtype=torch.int32, device=DEVICE)
    state["lib"] = {}


def _prepare_weights(state, case, dtype, g, r):
    S, Hk, Hq, D = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"]
    state["q"] = torch.randn((S, Hq, D), generator=g, device=DEVICE).to(dtype)
    # what earlier steps left: some weight for each page, +inf behind a row's last one
    w = torch.rand((S, Hk, state["table"].shape[-1]), generator=g, device=DEVICE) * 4.0
    n = (state["seq_lens"] + case["page"] - 1) // case["page"]
    w.masked_fill_(torch.arange(w.shape[-1], device=DEVICE) >= n[:, None, None], INF)
    state["before"], state["weights"] = w, torch.empty_like(w)
    state["out"] = torch.zeros_like(state["q"])
    state["lib"] = {}


def _prepare_sparse(state, case, dtype, g, r):
    S, Hk, Hq, D, B = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"], case["page"]
    state["q"] = torch.randn((S, Hq, D), generator=g, device=DEVICE).to(dtype)
    k = state["k_pool"]
    bounds = torch.zeros((k.shape[0], 2) + tuple(k.shape[2:]), dtype=dtype, device=DEVICE)
    if case["bounds"] != "all":   # kept from the steps before (those of an unfinished page are never read)
        bounds[:, 0], bounds[:, 1] = k.amin(1), k.amax(1)
    state["bounds"] = bounds
    shape = tuple(state["table"].shape[:-1]) + (case["pages"],)
    state["sel_table"] = torch.full(shape, -1, dtype=torch.int32, device=DEVICE)
    state["sel_idx"] = torch.full(shape, -1, dtype=torch.int32, device=DEVICE)
    state["sel_lens"] = torch.zeros(S, dtype=torch.int32, device=DEVICE)
    state["out"] = torch.zeros_like(state["q"])
    state["lib"] = {}


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"tree": _own_tree, "commit": _own_commit, "weights": _own_weights, "sparse": _own_sparse}[kind](state)
    return {"tree": _plain_tree, "commit": _plain_commit, "weights": _plain_weights, "sparse": _plain_sparse}[kind](state)


# The library's calls. A program that decodes keeps the descriptor and the workspace; they are made with the first pass.
def _own_tree(s):
    from paper_2509_04377_amd import binding as pe
    lib, T = s["lib"], s["case"]["drafts"]
    if not lib:
        lib["desc"] = _desc(s)
        lib["ws"] = pe.alloc_workspace(pe.PE_OP_TREE_DECODE, lib["desc"], T, device=DEVICE)
    pe.pe_tree_decode(lib["desc"], T, s["q"], s["k_draft"], s["v_draft"], s["draft_lens"], s["mask"], s["k_pool"], s["v_pool"],
                      s["table"], s["seq_lens"], s["scale"], s["out"], lib["ws"])
    return {"out": s["out"]}


def _own_commit(s):
    from paper_2509_04377_amd import binding as pe
    lib, c = s["lib"], s["case"]
    if not lib:
        lib["desc"] = _desc(s)
        lib["opts"] = pe.pe_evict_opts(pe.PE_POLICY_OLDEST, 0, 0, 0, 0)
    s["path_done"].zero_()
    for fills in (True, False):
        pe.pe_append_path(lib["desc"], s["k_draft"], s["v_draft"], s["path"], s["path_lens"], s["path_done"], s["k_pool"], s["v_pool"],
                          s["table"], s["seq_lens"], s["freed"], s["spare"], s["spare_used"])
        if fills:
            pe.pe_evict_blocks_ex(lib["desc"], lib["opts"], None, s["table"], s["seq_lens"], c["max_len"], s["evicted"], s["freed"])
    return {n: s[n] for n in ("k_pool", "v_pool", "table", "seq_lens", "path_done")}


def _own_weights(s):
    from paper_2509_04377_amd import binding as pe
    lib = s["lib"]
    if not lib:
        lib["desc"] = _desc(s)
        lib["ws"] = pe.alloc_workspace(pe.PE_OP_DECODE_WEIGHTS, lib["desc"], device=DEVICE)
    pe.pe_paged_decode_weights(lib["desc"], s["q"], s["k_pool"], s["v_pool"], s["table"], s["seq_lens"], s["scale"], DECAY, s["before"],
                               s["weights"], s["out"], lib["ws"])
    return {"out": s["out"], "weights": s["weights"]}


def _own_sparse(s):
    from paper_2509_04377_amd import binding as pe
    lib, c = s["lib"], s["case"]
    if not lib:
        lib["desc"], lib["sel"] = _desc(s), _desc(s, c["pages"])
        lib["ws"] = pe.alloc_workspace(pe.PE_OP_SELECT_PAGES, lib["desc"], device=DEVICE)
        lib["attend"] = pe.alloc_workspace(pe.PE_OP_PAGED_DECODE, lib["sel"], device=DEVICE)
    if c["bounds"] != "none":
        pe.pe_page_bounds(lib["desc"], s["k_pool"], s["table"], s["seq_lens"], 1 if c["bounds"] == "recent" else 0, s["bounds"])
    pe.pe_select_pages(lib["desc"], s["q"], s["bounds"], s["table"], s["seq_lens"], c["pages"], s["sel_table"], s["sel_lens"],
                       s["sel_idx"], lib["ws"])
    pe.pe_paged_decode(lib["sel"], s["q"], s["k_pool"], s["v_pool"], s["sel_table"], s["sel_lens"], s["scale"], s["out"],
                       lib["attend"])
    return {n: s[n] for n in ("out", "sel_table", "sel_lens", "sel_idx", "bounds")}


# The same in elementary operations.
def _tokens(pool, table, shared):
    """fp32 [S, Hk, tokens, D] of the pages of `table`; unused entries read page 0."""
    pages = pool[table.clamp(min=0).long()].float()
    if shared:
        return pages.flatten(1, 2).transpose(1, 2).contiguous()
    return pages.flatten(2, 3)


def _softmax(x):
    """Weights of the last axis; a row in which every logit is -inf gets none."""
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - torch.where(top == -INF, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    return p / torch.where(total == 0, torch.ones_like(total), total)


def _plain_tree(s):
    c = s["case"]
    S, T, Hk, Hq, D = c["seqs"], c["drafts"], c["kv_heads"], c["q_heads"], c["head_dim"]
    k, v = (_tokens(s[n], s["table"], c["layout"] == "shared") for n in ("k_pool", "v_pool"))
    kd, vd = (s[n].float().transpose(1, 2) for n in ("k_draft", "v_draft"))
    q = s["q"].float().view(S, T, Hk, Hq // Hk, D).permute(0, 2, 3, 1, 4).reshape(S, Hk, -1, D)
    cached = torch.arange(k.shape[2], device=DEVICE) < s["seq_lens"][:, None]
    j = torch.arange(T, device=DEVICE)
    drafted = ((s["mask"][:, :, None] >> j) & 1).bool() & (j < s["draft_lens"][:, None])[:, None, :]
    x = q @ k.transpose(2, 3) * s["scale"]
    x = x.masked_fill_(~cached[:, None, None, :], -INF)
    xd = (q @ kd.transpose(2, 3) * s["scale"]).view(S, Hk, -1, T, T).masked_fill(~drafted[:, None, None], -INF).view(S, Hk, -1, T)
    p = _softmax(torch.cat((x, xd), -1))
    out = p[..., :k.shape[2]] @ v + p[..., k.shape[2]:] @ vd
    out = out.view(S, Hk, -1, T, D).permute(0, 3, 1, 2, 4).reshape(S, T, Hq, D).to(s["q"].dtype)
    real = (j < s["draft_lens"][:, None])[:, :, None, None]
    return {"out": torch.where(real, out, s["out"])}


def _plain_append(s):
    """What is left of the paths joins the cache, up to the end of the newest page."""
    c = s["case"]
    B, shared, table, lens, done = c["page"], c["layout"] == "shared", s["table"], s["seq_lens"], s["path_done"]
    S, Hk = c["seqs"], c["kv_heads"]
    slot, logical = lens % B, lens // B
    count = torch.minimum(s["path_lens"] - done, B - slot)
    # a new page, where the newest is full: the one that was freed
    link = ((slot == 0) & (count > 0)).view((S,) + (1,) * (table.dim() - 1))
    at = logical.clamp(max=table.shape[-1] - 1).long().view(link.shape).expand(table.shape[:-1] + (1,))
    page = torch.where(link, s["freed"][..., None], table.gather(-1, at))
    table.scatter_(-1, at, page)
    s["freed"].copy_(torch.where(link[..., 0], torch.full_like(s["freed"], -1), s["freed"]))
    i = torch.arange(B, device=DEVICE)
    takes = i < count[:, None]
    draft = s["path"].gather(1, (done[:, None] + i).clamp(max=B - 1).long())
    sq = torch.arange(S, device=DEVICE)[:, None].expand(S, B)[takes]
    to_slot, of_draft = (slot[:, None] + i)[takes].long(), draft[takes].long()
    to = (page[sq, 0].long(), to_slot) if shared else (page[sq, :, 0].long(), to_slot[:, None].expand(-1, Hk))
    s["k_pool"][to] = s["k_draft"][sq, of_draft]                      # [n, Hk, D]
    s["v_pool"][to] = s["v_draft"][sq, of_draft]
    lens += count
    done += count


def _plain_evict_oldest(s):
    c = s["case"]
    table, lens, B = s["table"], s["seq_lens"], c["page"]
    goes = ((lens > 0) & (lens % B == 0) & (lens >= c["max_len"])).view((c["seqs"],) + (1,) * (table.dim() - 1))
    n = (lens // B).view(goes.shape)
    shifted = torch.cat((table[..., 1:], torch.full_like(table[..., :1], -1)), -1)
    s["freed"].copy_(torch.where(goes[..., 0], table[..., 0], torch.full_like(s["freed"], -1)))
    inside = torch.arange(table.shape[-1], device=DEVICE) < n
    table.copy_(torch.where(goes & inside, shifted, table))
    lens -= torch.where(goes.flatten(), torch.full_like(lens, B), torch.zeros_like(lens))


def _plain_commit(s):
    s["path_done"].zero_()
    _plain_append(s)
    _plain_evict_oldest(s)
    _plain_append(s)
    return {n: s[n] for n in ("k_pool", "v_pool", "table", "seq_lens", "path_done")}


def _plain_attend(s, table, lens):
    """The output and each token's weight, [S, Hk, G, tokens]."""
    c = s["case"]
    S, Hk, Hq, D = c["seqs"], c["kv_heads"], c["q_heads"], c["head_dim"]
    k, v = (_tokens(s[n], table, c["layout"] == "shared") for n in ("k_pool", "v_pool"))
    x = s["q"].float().view(S, Hk, Hq // Hk, D) @ k.transpose(2, 3) * s["scale"]
    x = x.masked_fill_((torch.arange(k.shape[2], device=DEVICE) >= lens[:, None])[:, None, None, :], -INF)
    p = _softmax(x)
    return (p @ v).view(S, Hq, D).to(s["q"].dtype), p


def _plain_weights(s):
    c = s["case"]
    out, p = _plain_attend(s, s["table"], s["seq_lens"])
    got = p.view(c["seqs"], c["kv_heads"], -1, s["table"].shape[-1], c["page"]).sum((2, 4))
    before = torch.where(torch.isfinite(s["before"]), s["before"], torch.zeros_like(s["before"]))
    n = (s["seq_lens"] + c["page"] - 1) // c["page"]
    behind = torch.arange(got.shape[-1], device=DEVICE) >= n[:, None, None]
    return {"out": out, "weights": (before * DECAY + got).masked_fill(behind, INF)}


def _plain_sparse(s):
    c = s["case"]
    S, Hk, Hq, D, B, k = c["seqs"], c["kv_heads"], c["q_heads"], c["head_dim"], c["page"], c["pages"]
    table, lens, shared = s["table"], s["seq_lens"], c["layout"] == "shared"
    full = (lens // B).view((S,) + (1,) * (table.dim() - 1))
    j = torch.arange(table.shape[-1], device=DEVICE)
    if c["bounds"] != "none":
        which = j < full
        if c["bounds"] == "recent":
            which = which & (j >= full - 1)
        fresh = table[which.expand(table.shape)].long()
        s["bounds"][fresh, 0], s["bounds"][fresh, 1] = s["k_pool"][fresh].amin(1), s["k_pool"][fresh].amax(1)
    # the sum over the heads of max(q lo, q hi), in 64 bits: the order of pages next to the border depends on it
    q = s["q"].double().view(S, Hk, Hq // Hk, D)
    up, down = q.clamp(min=0).sum(2), q.clamp(max=0).sum(2)           # [S, Hk, D]
    b = s["bounds"][table.clamp(min=0).long()]                         # [S, Hk, n, 2, D]; shared: [S, n, 2, Hk, D]
    if shared:
        up, down = up.reshape(S, -1), down.reshape(S, -1)
        b = b.flatten(-2)
    score = ((b[..., 1, :].double() @ up[..., None]) + (b[..., 0, :].double() @ down[..., None]))[..., 0].float()
    n = ((lens + B - 1) // B).view(full.shape)
    # the newest page before all others, what is no page behind them; equal scores in the pages' order
    order = torch.where(j >= n, torch.full_like(j, 2), torch.where(j == n - 1, torch.full_like(j, 0), torch.full_like(j, 1)))
    by_score = torch.sort(score, dim=-1, descending=True, stable=True).indices
    by_kind = torch.sort(order.expand(table.shape).gather(-1, by_score), dim=-1, stable=True).indices
    best = by_score.gather(-1, by_kind)[..., :k]
    idx = torch.where(order.expand(table.shape).gather(-1, best) == 2, torch.full_like(best, table.shape[-1]), best).sort(-1).values
    taken = idx < table.shape[-1]
    sel = torch.where(taken, table.gather(-1, idx.clamp(max=table.shape[-1] - 1)), torch.full_like(table[..., :1], -1))
    idx = torch.where(taken, idx, torch.full_like(idx, -1)).int()
    pad = tuple(table.shape[:-1]) + (k - idx.shape[-1],)
    idx, sel = (torch.cat((x, torch.full(pad, -1, dtype=torch.int32, device=DEVICE)), -1) for x in (idx, sel))
    count = torch.clamp((lens + B - 1) // B, max=k)
    sel_lens = torch.where(lens > 0, (count - 1) * B + (lens - 1) % B + 1, torch.zeros_like(lens)).int()
    out, _ = _plain_attend(s, sel, sel_lens)
    return {"out": out, "sel_table": sel, "sel_lens": sel_lens, "sel_idx": idx, "bounds": s["bounds"]}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    S, Hk, Hq, D, B = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"], case["page"]
    rows = 1 if case["layout"] == "shared" else Hk
    lens = _lens(case)
    kv, token = Hk * D * e * 2, Hq * D * e
    tables = sum(4 * rows * -(-n // B) for n in lens)
    if case["kind"] == "tree":
        T = case["drafts"]
        counts = [max(1, T - T // 4) if i % 4 == 3 else T for i in range(S)]
        mean = sum(counts) / S
        return {"bytes": sum(lens) * kv + tables + sum(counts) * (2 * token + kv + 8),
                "flops": 4 * Hq * D * (mean * sum(lens) + sum(n * n for n in counts) / 2)}
    if case["kind"] == "commit":
        return {"bytes": 2 * S * B * kv + 2 * tables + 4 * S * B, "flops": 0}
    if case["kind"] == "weights":
        return {"bytes": sum(lens) * kv + tables + 2 * S * token + sum(8 * Hk * -(-n // B) for n in lens), "flops": 4 * sum(lens) * Hq * D}
    full = sum(n // B for n in lens)
    scored = (full + (full if case["bounds"] == "all" else S if case["bounds"] == "recent" else 0)) * kv   # min and max of the pages' keys
    made = {"none": 0, "recent": S, "all": full}[case["bounds"]] * B * kv // 2                            # the keys they are made from
    read = sum(min(n, case["pages"] * B) for n in lens)
    return {"bytes": scored + made + read * kv + tables + 2 * S * token + 8 * rows * S * case["pages"],
            "flops": 4 * read * Hq * D + 4 * full * Hk * D}


# ---- the same in 64 bits, sequence by sequence -------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "commit":
        return None   # copies and whole numbers: no computed values
    s = prepare(case, seed)
    return {"tree": _exact_tree, "weights": _exact_weights, "sparse": _exact_sparse}[case["kind"]](s, case)


def _row64(s, case, table, i, h, n, pool):
    """The n tokens of one row in 64 bits, read through the table."""
    B = case["page"]
    t = torch.arange(n, device=DEVICE)
    if case["layout"] == "shared":
        return s[pool][table[i][t // B].long(), t % B, h].double()
    return s[pool][table[i, h][t // B].long(), t % B].double()


def _exact_tree(s, case):
    T, Hk, G = case["drafts"], case["kv_heads"], case["q_heads"] // case["kv_heads"]
    out = s["out"].double()
    lens, counts, words = (s[n].tolist() for n in ("seq_lens", "draft_lens", "mask"))
    for i, (n, m) in enumerate(zip(lens, counts)):
        sees = torch.tensor([[(w >> j) & 1 for j in range(m)] for w in words[i][:m]], dtype=torch.bool, device=DEVICE)
        sees = torch.cat((torch.ones((m, n), dtype=torch.bool, device=DEVICE), sees), 1)
        for h in range(Hk):
            k = torch.cat((_row64(s, case, s["table"], i, h, n, "k_pool"), s["k_draft"][i, :m, h].double()))
            v = torch.cat((_row64(s, case, s["table"], i, h, n, "v_pool"), s["v_draft"][i, :m, h].double()))
            for x in range(h * G, h * G + G):
                logits = (s["q"][i, :m, x].double() @ k.t().contiguous() * s["scale"]).masked_fill(~sees, -INF)
                w = torch.exp(logits - logits.max(1, keepdim=True).values)
                out[i, :m, x] = (w @ v) / w.sum(1, keepdim=True)
    return {"out": out}


def _exact_attend(s, case, table, lens, per_token=None):
    G = case["q_heads"] // case["kv_heads"]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    for i, n in enumerate(lens):
        for h in range(case["kv_heads"] if n else 0):
            k, v = (_row64(s, case, table, i, h, n, p) for p in ("k_pool", "v_pool"))
            logits = s["q"][i, h * G:h * G + G].double() @ k.t().contiguous() * s["scale"]
            w = torch.exp(logits - logits.max(1, keepdim=True).values)
            w /= w.sum(1, keepdim=True)
            out[i, h * G:h * G + G] = w @ v
            if per_token is not None:
                per_token(i, h, w.sum(0))
    return out


def _exact_weights(s, case):
    B = case["page"]
    weights = torch.full(s["before"].shape, INF, dtype=torch.float64, device=DEVICE)

    def add(i, h, w):
        n = -(-w.numel() // B)
        by_page = torch.zeros(n * B, dtype=torch.float64, device=DEVICE)
        by_page[:w.numel()] = w
        weights[i, h, :n] = s["before"][i, h, :n].double() * DECAY + by_page.view(n, B).sum(1)

    out = _exact_attend(s, case, s["table"], s["seq_lens"].tolist(), add)
    return {"out": out, "weights": weights}


def _exact_sparse(s, case):
    """Which pages: the largest sums of max(q lo, q hi) over heads and elements, straight from the keys."""
    B, k, G, Hk = case["page"], case["pages"], case["q_heads"] // case["kv_heads"], case["kv_heads"]
    shared = case["layout"] == "shared"
    lens = s["seq_lens"].tolist()
    sel = torch.full(s["sel_table"].shape, -1, dtype=torch.int32, device=DEVICE)
    sel_lens = []
    for i, n in enumerate(lens):
        pages = -(-n // B)
        sel_lens.append(n if pages <= k else (k - 1) * B + n - (pages - 1) * B)
        total = torch.zeros(max(0, pages - 1), dtype=torch.float64, device=DEVICE)
        for h in range(Hk):
            if pages > k and pages > 1:
                key = _row64(s, case, s["table"], i, h, (pages - 1) * B, "k_pool").view(pages - 1, B, -1)
                lo, hi = key.amin(1), key.amax(1)
                one = sum(torch.maximum(x * lo, x * hi).sum(1) for x in s["q"][i, h * G:h * G + G].double())
                total = total + one if shared else one
            if shared and h < Hk - 1:
                continue
            if pages <= k:
                idx = torch.arange(pages, device=DEVICE)
            else:
                best = torch.sort(total.float(), descending=True, stable=True).indices[:k - 1]
                idx = torch.cat((best, torch.tensor([pages - 1], device=DEVICE))).sort().values
            at = (i,) if shared else (i, h)
            sel[at][:idx.numel()] = s["table"][at][idx]
    return {"out": _exact_attend(s, case, sel, sel_lens), "sel_table": None, "sel_lens": None, "sel_idx": None, "bounds": None}
