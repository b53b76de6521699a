"""From request lengths to attention over an 8-bit cache, as cases that can be timed and checked.

  plan    pe_plan_tokens: block tables, slots and positions of the tokens that requests bring, from their lengths and a
          list of free pages.
  rotate  pe_rotate: rotary positions of queries and keys, and where the case stores, the rotated keys and the values
          into their pages by the slots.
  pages   pe_quant_pages: the full pages of a cache rounded to e4m3 with one scale for K and one for V of each page and
          head, their scores, and the unfinished pages put aside as they are.
  append  pe_quant_append: the new token of every sequence, rotated, joins the 8-bit cache; pages that fill are rounded.
  decode  pe_quant_decode: one query a sequence over the 8-bit pages and the unfinished one.

A case is a dict of plain values: `kind`; `dtype`, `layout`, `seqs`, `kv_heads`, `q_heads`, `head_dim`, `page`, `min_len`,
`max_len` everywhere (lengths of prompts or caches, spread evenly between the two, in an order that the seed gives; what
rotate turns are the tokens of one batch of such prompts); `new` for plan (tokens a sequence brings to a cache of that length,
or 0: the lengths are the requests' own, of new sequences); `rotary` (turned elements of a head), `pairs` ("half" or
"interleaved") and `scaling` ("none", "linear", "parts") for rotate and append; `store`, `packed` (q, k and v are parts of
one row a token) and `transpose` for rotate.
"""
import math

import numpy as np
import torch

own = False   # True: run() calls the library; False: the same in plain torch operations, in 32 bits and more

DEVICE = "cuda"
DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
E4M3 = torch.float8_e4m3fn
INF = float("inf")
# long contexts: 8 times an original one of 8192, frequencies of less than one turn in it slowed down, of more than four not
BASE, FACTOR, LOW, HIGH, ORIGINAL = 500000.0, 8.0, 1.0, 4.0, 8192.0


def _case(name, kind, dtype, layout, seqs, kv_heads, q_heads, head_dim, page, min_len, max_len, **more):
    return dict({"name": name, "kind": kind, "dtype": dtype, "layout": layout, "seqs": seqs, "kv_heads": kv_heads,
                 "q_heads": q_heads, "head_dim": head_dim, "page": page, "min_len": min_len, "max_len": max_len}, **more)


def _unnamed(*args, **more):
    case = _case("", *args, **more)
    del case["name"]
    return case


def _turn(rotary, pairs="half", scaling="none"):
    return {"rotary": rotary, "pairs": pairs, "scaling": scaling}


def listed():
    return [
        # a step of a serving batch of the 8B shape: one token each, now and then a page; a launch, nothing else
        _case("plan_8b_step", "plan", "bf16", "per_head", 32, 8, 32, 128, 16, 1009, 2048, new=1),
        # a batch of ragged prompts is let in: tables of eight heads, a slot for each token and head
        _case("plan_8b_prompts", "plan", "bf16", "per_head", 32, 8, 32, 128, 16, 17, 16384, new=0),
        # the new tokens of a small batch, into their pages: bound by latency
        _case("rotate_1b_step", "rotate", "bf16", "per_head", 8, 8, 32, 64, 16, 1, 1, store=True, packed=False, transpose=False, **_turn(64)),
        # a batch of prompts of the 8B shape as the projection leaves it, scaled for long contexts, into the cache
        _case("rotate_8b_prompts", "rotate", "bf16", "per_head", 8, 8, 32, 128, 16, 2001, 6000, store=True, packed=True, transpose=False,
              **_turn(128, "half", "parts")),
        # a gradient in 32 bits: half of each head turned, neighbours as pairs, an odd number of tokens
        _case("rotate_f32_gradient", "rotate", "f32", "shared", 3, 4, 12, 64, 32, 901, 2047, store=False, packed=False, transpose=True,
              **_turn(32, "interleaved", "linear")),
        # a layer of the 8B shape behind its prune: every page at the budget
        _case("pages_8b_layer", "pages", "bf16", "per_head", 32, 8, 32, 128, 16, 2033, 2048),
        # fp32, head-shared, ragged, larger pages
        _case("pages_f32_ragged", "pages", "f32", "shared", 6, 4, 12, 64, 32, 1, 2999),
        # one layer of the 1B shape, no page fills: a launch
        _case("append_1b_layer", "append", "bf16", "per_head", 8, 8, 32, 64, 16, 1001, 1006, **_turn(64)),
        # all layers of the 8B shape at once, layers folded into the sequences: some pages fill, some begin
        _case("append_8b_model", "append", "bf16", "per_head", 1024, 8, 32, 128, 16, 1, 256, **_turn(128, "half", "parts")),
        # one layer of the 1B shape: bound by the chain of a launch
        _case("decode_1b_layer", "decode", "bf16", "per_head", 8, 8, 32, 64, 16, 1013, 1024),
        # the 8B shape at full batch and budget: bound by the cache's traffic
        _case("decode_8b_batch", "decode", "bf16", "per_head", 32, 8, 32, 128, 16, 2033, 2048),
        # few long caches
        _case("decode_8b_long", "decode", "bf16", "per_head", 4, 8, 32, 128, 16, 60001, 65536),
    ]


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """A case of the ranges above: any supported type, layout, head size, page size and number of query heads a KV head;
    lengths from none or one token on, odd ones among them; none costs more than the largest listed ones."""
    kind = rng.choice(("plan", "rotate", "rotate", "pages", "append", "decode", "decode", "decode"))
    dtype = rng.choice(("bf16", "bf16", "f32"))
    layout = rng.choice(("per_head", "shared"))
    group = rng.choice((1, 2, 3, 4, 4, 5, 7, 8))
    kv_heads = rng.choice((1, 2, 3, 4, 8))
    head_dim = rng.choice((64, 128))
    page = rng.choice((16, 16, 32, 64, 128))
    seqs = _log_int(rng, 1, 64)
    heads = kv_heads * (group + 2 if kind == "rotate" else 1)
    most = {"plan": 1 << 21, "rotate": 1 << 19, "pages": 1 << 18, "append": 1 << 18, "decode": 1 << 20}[kind]   # tokens x heads
    per = max(1, most // (seqs * heads))
    max_len = _log_int(rng, 1, min(65536, per))
    min_len = 0 if kind != "rotate" and rng.random() < 0.2 else rng.randint(1, max_len)
    more = {}
    if kind == "plan":
        more["new"] = rng.choice((0, 0, 1, _log_int(rng, 1, 300)))
    if kind in ("rotate", "append"):
        rotary = head_dim if rng.random() < 0.6 else 2 * rng.randint(1, head_dim // 2)
        more = _turn(rotary, rng.choice(("half", "interleaved")), rng.choice(("none", "linear", "parts")))
    if kind == "rotate":
        more.update(store=rng.random() < 0.5, packed=rng.random() < 0.5, transpose=rng.random() < 0.3)
    return _unnamed(kind, dtype, layout, seqs, kv_heads, group * kv_heads, head_dim, page, min_len, max_len, **more)


# ---- inputs ------------------------------------------------------------------------------------------------------
def _lens(case):
    """Evenly spread; the seed gives only their order, so that all seeds have the same work."""
    S, lo, hi = case["seqs"], case["min_len"], case["max_len"]
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


def _on(x):
    return torch.from_numpy(np.ascontiguousarray(x)).to(DEVICE)


def _table(case, tokens, r, extra=0):
    """Shuffled pages of so many tokens a sequence, [S, rows, width] (-1 behind a row's last), and how many there are; `extra` columns more."""
    need = -(-np.asarray(tokens, np.int64) // case["page"])
    rows, width = 1 if case["layout"] == "shared" else case["kv_heads"], max(1, int(need.max()) + extra)
    used = np.broadcast_to(np.arange(width)[None, None, :] < need[:, None, None], (case["seqs"], rows, width))
    table = np.full((case["seqs"], rows, width), -1, np.int32)
    table[used] = r.permutation(int(used.sum())).astype(np.int32)
    return table, int(used.sum())


def _per_row(case, x):
    """Head-shared: arrays of rows lose their head dimension."""
    return _on(x[:, 0] if case["layout"] == "shared" else x)


def _pool_shape(case, pages):
    return (max(1, pages), case["page"]) + ((case["kv_heads"],) if case["layout"] == "shared" else ()) + (case["head_dim"],)


def prepare(case, seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(int(seed))
    r = np.random.default_rng(int(seed))
    lens = np.array(_lens(case), np.int64)
    r.shuffle(lens)
    state = {"case": case, "lib": {}}
    {"plan": _prepare_plan, "rotate": _prepare_rotate, "pages": _prepare_pages, "append": _prepare_append,
     "decode": _prepare_decode}[case["kind"]](state, case, lens, DTYPES[case["dtype"]], g, r)
    return state


def _prepare_plan(s, case, lens, dtype, g, r):
    S, B, new = case["seqs"], case["page"], case["new"]
    rows = 1 if case["layout"] == "shared" else case["kv_heads"]
    have, add = (lens, np.full(S, new)) if new else (np.zeros(S, np.int64), lens)
    table, used = _table(case, have, r)
    width = max(1, int((-(-(have + add) // B)).max()))
    table = np.concatenate((table, np.full((S, rows, max(0, width - table.shape[2])), -1, np.int32)), 2)[:, :, :max(width, 1)]
    need = int((-(-(have + add) // B) - -(-have // B)).sum()) * rows
    free = used + r.permutation(need + 7).astype(np.int32)     # some are left over
    s["table"], s["free"] = _per_row(case, table), _on(free.astype(np.int32))
    s["pages"] = used + need + 7
    s["free_used"] = torch.full((1,), 3, dtype=torch.int32, device=DEVICE)
    s["seq_lens"], s["new_lens"] = _on(have.astype(np.int32)), _on(add.astype(np.int32))
    s["total"] = int(add.sum())
    i32 = dict(dtype=torch.int32, device=DEVICE)
    s["lens_out"], s["used_out"], s["cu"] = torch.zeros(S, **i32), torch.zeros(1, **i32), torch.zeros(S + 1, **i32)
    s["positions"] = torch.zeros(s["total"], **i32)
    s["slots"] = torch.zeros((s["total"],) + (() if case["layout"] == "shared" else (rows,)), dtype=torch.int64, device=DEVICE)


def _prepare_rotate(s, case, lens, dtype, g, r):
    Hk, Hq, D, B = case["kv_heads"], case["q_heads"], case["head_dim"], case["page"]
    T = int(lens.sum())
    if case["packed"]:
        x = torch.randn((T, Hq + 2 * Hk, D), generator=g, device=DEVICE).to(dtype)
        s["q"], s["k"], s["v"] = x[:, :Hq], x[:, Hq:Hq + Hk], x[:, Hq + Hk:]
    else:
        s["q"], s["k"], s["v"] = (torch.randn((T, h, D), generator=g, device=DEVICE).to(dtype) for h in (Hq, Hk, Hk))
    # prompts begin at 0; where contexts are scaled, some go on from far behind the original one
    first = r.integers(0, 100000 if case["scaling"] != "none" else 2, case["seqs"])
    s["positions"] = _on(np.concatenate([f + np.arange(n) for f, n in zip(first, lens)]).astype(np.int32))
    s["q_out"], s["k_out"] = (torch.zeros((T, h, D), dtype=dtype, device=DEVICE) for h in (Hq, Hk))
    if case["store"]:
        table, pages = _table(case, lens, r)
        at = [table[i][:, np.arange(n) // B].T.astype(np.int64) * B + (np.arange(n) % B)[:, None] for i, n in enumerate(lens)]
        slots = np.concatenate(at)
        s["slots"] = _on(slots[:, 0] if case["layout"] == "shared" else slots)
        s["k_pool"], s["v_pool"] = (torch.zeros(_pool_shape(case, pages), dtype=dtype, device=DEVICE) for _ in range(2))


def _quant_state(s, case, pages, dtype):
    """An empty 8-bit cache of so many pages."""
    shape = _pool_shape(case, pages)
    s["k8"], s["v8"] = (torch.zeros(shape, dtype=torch.uint8, device=DEVICE).view(E4M3) for _ in range(2))
    s["scales"] = torch.ones((shape[0],) + ((case["kv_heads"],) if case["layout"] == "shared" else ()) + (2,), device=DEVICE)
    tail = (case["seqs"], case["kv_heads"], case["page"], case["head_dim"])
    s["k_tail"], s["v_tail"] = (torch.zeros(tail, dtype=dtype, device=DEVICE) for _ in range(2))


def _prepare_pages(s, case, lens, dtype, g, r):
    table, pages = _table(case, lens, r)
    s["src_table"], s["seq_lens"] = _per_row(case, table), _on(lens.astype(np.int32))
    moved = r.permutation(max(1, pages)).astype(np.int32)
    s["table"] = _per_row(case, np.where(table < 0, -1, moved[np.maximum(table, 0)]).astype(np.int32))
    s["k_pool"], s["v_pool"] = (torch.empty(_pool_shape(case, pages), dtype=dtype, device=DEVICE) for _ in range(2))
    _fill(s["k_pool"], g)
    _fill(s["v_pool"], g)
    _quant_state(s, case, pages, dtype)
    s["scores"] = torch.zeros((case["seqs"], case["kv_heads"], table.shape[2]), device=DEVICE)


def _prepare_append(s, case, lens, dtype, g, r):
    S, Hk, Hq, D = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"]
    table, pages = _table(case, lens, r, extra=1)
    rows = table.shape[1]
    s["table"], s["seq_lens"] = _per_row(case, table), _on(lens.astype(np.int32))
    s["lens_out"] = torch.zeros_like(s["seq_lens"])
    _quant_state(s, case, pages + S * rows, dtype)
    _fill(s["k_tail"], g)
    _fill(s["v_tail"], g)
    # the page that an eviction has freed a moment ago, or none: then the next spare one
    extra = (pages + r.permutation(S * rows)).astype(np.int32).reshape(S, rows)
    some = r.random((S, 1)) < 0.5
    s["freed_before"] = _per_row(case, np.where(some, extra, -1).astype(np.int32))
    s["spare"] = _per_row(case, extra[:, :, None])
    s["freed"], s["spare_used"] = s["freed_before"].clone(), torch.zeros_like(s["freed_before"])
    s["links"] = bool((lens % case["page"] == 0).any())
    s["k_new"], s["v_new"] = _rows((S, Hk, D), g, dtype), _rows((S, Hk, D), g, dtype)
    s["q"] = torch.randn((S, Hq, D), generator=g, device=DEVICE).to(dtype)
    s["q_out"] = torch.zeros_like(s["q"])
    # pages have gone before: tokens stand further behind than the cache is long
    s["positions"] = _on((lens + r.integers(0, 100000 if case["scaling"] != "none" else 8192, S)).astype(np.int32))
    s["scores"] = torch.rand((S, Hk, table.shape[2]), generator=g, device=DEVICE)


def _prepare_decode(s, case, lens, dtype, g, r):
    S, Hk, Hq, D = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"]
    table, pages = _table(case, lens, r)
    s["table"], s["seq_lens"] = _per_row(case, table), _on(lens.astype(np.int32))
    _quant_state(s, case, pages, dtype)
    step = max(1, (1 << 26) // s["k8"][0].numel())
    for i in range(0, s["k8"].shape[0], step):
        for n, name in enumerate(("k8", "v8")):
            part = s[name][i:i + step]
            held, scale = _round(_rows(tuple(part.shape), g, torch.float32))
            part.copy_(held)
            s["scales"][i:i + step][..., n] = scale
    _fill(s["k_tail"], g)
    _fill(s["v_tail"], g)
    s["q"] = torch.randn((S, Hq, D), generator=g, device=DEVICE).to(dtype)
    s["out"] = torch.zeros_like(s["q"])


# ---- one pass ----------------------------------------------------------------------------------------------------
def run(state):
    kind = state["case"]["kind"]
    if own:
        return {"plan": _own_plan, "rotate": _own_rotate, "pages": _own_pages, "append": _own_append, "decode": _own_decode}[kind](state)
    return {"plan": _plain_plan, "rotate": _plain_rotate, "pages": _plain_pages, "append": _plain_append, "decode": _plain_decode}[kind](state)


# The library's calls. A program keeps the descriptor, the frequencies and the workspace; they are made with the first pass.
def _desc(pe, s, width, pages):
    c = s["case"]
    return pe.make_desc(DTYPES[c["dtype"]], c["seqs"], c["kv_heads"], c["q_heads"], c["head_dim"], c["page"], width, pages,
                        pe.PE_LAYOUT_SHARED if c["layout"] == "shared" else pe.PE_LAYOUT_PER_HEAD)


def _rope(pe, c):
    how = {"none": pe.PE_ROPE_PLAIN, "linear": pe.PE_ROPE_LINEAR, "parts": pe.PE_ROPE_BY_PARTS}[c["scaling"]]
    return pe.make_rope(c["rotary"], BASE, interleaved=c["pairs"] == "interleaved", scaling=how, factor=FACTOR, low=LOW, high=HIGH,
                        original=ORIGINAL, magnitude=_magnitude(c))


def _cache(pe, s, desc):
    return pe.make_quant_cache(desc, s["k8"], s["v8"], s["scales"], s["k_tail"], s["v_tail"])


def _own_plan(s):
    from paper_2509_04377_amd import binding as pe
    lib = s["lib"]
    if not lib:
        lib["desc"] = _desc(pe, s, s["table"].shape[-1], s["pages"])
    pe.pe_plan_tokens(lib["desc"], s["seq_lens"], s["new_lens"], None, s["total"], 0, s["free"], s["free_used"], s["table"], None,
                      s["lens_out"], s["used_out"], s["cu"], s["positions"], s["slots"])
    return {n: s[n] for n in ("table", "lens_out", "used_out", "cu", "positions", "slots")}


def _own_rotate(s):
    from paper_2509_04377_amd import binding as pe
    lib, c = s["lib"], s["case"]
    if not lib:
        lib["desc"] = _desc(pe, s, 1, s["k_pool"].shape[0] if c["store"] else 1)
        lib["rope"] = _rope(pe, c)
    pe.pe_rotate(lib["desc"], lib["rope"], c["transpose"], s["positions"], s["q"], s["k"], s["v"] if c["store"] else None, s["q_out"], s["k_out"],
                 s.get("slots"), s.get("k_pool"), s.get("v_pool"))
    return {n: s[n] for n in ("q_out", "k_out") + (("k_pool", "v_pool") if c["store"] else ())}


def _own_pages(s):
    from paper_2509_04377_amd import binding as pe
    lib = s["lib"]
    if not lib:
        lib["desc"] = _desc(pe, s, s["table"].shape[-1], s["k8"].shape[0])
        lib["cache"] = _cache(pe, s, lib["desc"])
    pe.pe_quant_pages(lib["desc"], lib["cache"], s["k_pool"], s["v_pool"], s["src_table"], s["seq_lens"], s["table"], s["scores"])
    return {n: s[n] for n in ("k8", "v8", "scales", "k_tail", "v_tail", "scores")}


def _own_append(s):
    from paper_2509_04377_amd import binding as pe
    lib = s["lib"]
    if not lib:
        lib["desc"] = _desc(pe, s, s["table"].shape[-1], s["k8"].shape[0])
        lib["cache"] = _cache(pe, s, lib["desc"])
        lib["rope"] = _rope(pe, s["case"])
    if s["links"]:
        s["freed"].copy_(s["freed_before"])
        s["spare_used"].zero_()
    pe.pe_quant_append(lib["desc"], lib["cache"], lib["rope"], s["positions"], s["q"], s["q_out"], s["k_new"], s["v_new"], s["table"],
                       s["seq_lens"], s["lens_out"], s["freed"], s["spare"], s["spare_used"], s["scores"])
    return {n: s[n] for n in ("q_out", "k8", "v8", "scales", "k_tail", "v_tail", "scores", "table", "lens_out", "freed", "spare_used")}


def _own_decode(s):
    from paper_2509_04377_amd import binding as pe
    lib = s["lib"]
    if not lib:
        lib["desc"] = _desc(pe, s, s["table"].shape[-1], s["k8"].shape[0])
        lib["cache"] = _cache(pe, s, lib["desc"])
        lib["ws"] = pe.alloc_workspace(pe.PE_OP_QUANT_DECODE, lib["desc"], device=DEVICE)
    pe.pe_quant_decode(lib["desc"], lib["cache"], s["q"], s["table"], s["seq_lens"], s["case"]["head_dim"] ** -0.5, s["out"], lib["ws"])
    return {"out": s["out"]}


# The same in elementary operations.
def _plain_plan(s):
    c = s["case"]
    B, shared, table, lens, new = c["page"], c["layout"] == "shared", s["table"], s["seq_lens"], s["new_lens"]
    S = c["seqs"]
    rows = 1 if shared else c["kv_heads"]
    t3 = table.view(S, rows, -1)
    have, after = (lens + B - 1) // B, lens + new
    need = (after + B - 1) // B - have                               # pages a row
    total = need * rows
    off = s["free_used"] + torch.cumsum(total, 0) - total
    serves = (off + total <= s["free"].shape[0]) & (have + need <= t3.shape[2])
    j = torch.arange(t3.shape[2], device=DEVICE)
    h = torch.arange(rows, device=DEVICE)[:, None]
    nth = (off[:, None, None] + h * need[:, None, None] + (j - have[:, None])[:, None, :]).long()
    fresh = ((j >= have[:, None]) & (j < (have + need)[:, None]) & serves[:, None])[:, None, :]
    page = s["free"][nth.clamp(0, s["free"].shape[0] - 1)]
    t3.copy_(torch.where(fresh, page, t3))
    s["lens_out"].copy_(torch.where(serves, after, lens))
    s["used_out"].copy_(torch.where(serves, off + total, s["free_used"]).amax().view(1))
    cu = torch.cumsum(new, 0)
    s["cu"][0], s["cu"][1:] = 0, cu
    t = torch.arange(s["total"], device=DEVICE)
    of = torch.searchsorted(cu, t.to(cu.dtype), right=True)
    at = lens[of] + (t - (cu - new)[of])
    s["positions"].copy_(at)
    held = t3[of[:, None], torch.arange(rows, device=DEVICE)[None], (at // B).clamp(max=t3.shape[2] - 1)[:, None]].long()   # [T, rows]
    slot = torch.where((held >= 0) & serves[of][:, None], held * B + (at % B)[:, None], torch.full_like(held, -1))
    s["slots"].copy_(slot[:, 0] if shared else slot)
    return {n: s[n] for n in ("table", "lens_out", "used_out", "cu", "positions", "slots")}


def _magnitude(c):
    """Queries and keys of scaled contexts a little larger: softmax over more tokens."""
    return 0.1 * math.log(FACTOR) + 1.0 if c["scaling"] == "parts" else 1.0


def _angles(c, positions):
    """cos and sin of every token's angles, [T, rotary / 2], times the magnitude: angles of far positions take 64 bits."""
    f = BASE ** (-torch.arange(0, c["rotary"], 2, dtype=torch.float64, device=DEVICE) / c["rotary"])
    if c["scaling"] == "linear":
        f = f / FACTOR
    elif c["scaling"] == "parts":
        turns = ORIGINAL * f / (2 * math.pi)
        keep = ((turns - LOW) / (HIGH - LOW)).clamp(0, 1)
        f = f * ((1 - keep) / FACTOR + keep)
    a = positions.double()[:, None] * f
    m = _magnitude(c)
    return (torch.cos(a) * m).float(), (torch.sin(a) * m).float()


def _turned(c, x, cos, sin):
    """x [T, heads, D] fp32, its first `rotary` elements turned."""
    n = c["rotary"]
    cos, sin = cos[:, None], sin[:, None]
    out = x.clone()
    if c["pairs"] == "half":
        a, b = x[..., :n // 2], x[..., n // 2:n]
        out[..., :n // 2], out[..., n // 2:n] = a * cos - b * sin, b * cos + a * sin
    else:
        a, b = x[..., 0:n:2], x[..., 1:n:2]
        out[..., 0:n:2], out[..., 1:n:2] = a * cos - b * sin, b * cos + a * sin
    return out


def _plain_rotate(s):
    c = s["case"]
    cos, sin = _angles(c, s["positions"])
    if c["transpose"]:
        sin = -sin
    s["q_out"].copy_(_turned(c, s["q"].float(), cos, sin))
    s["k_out"].copy_(_turned(c, s["k"].float(), cos, sin))
    if c["store"]:
        for pool, x in ((s["k_pool"], s["k_out"]), (s["v_pool"], s["v"])):
            flat = pool.flatten(0, 1)
            if c["layout"] == "shared":
                flat[s["slots"]] = x
            else:
                flat[s["slots"].flatten()] = x.reshape(-1, c["head_dim"])
    return {n: s[n] for n in ("q_out", "k_out") + (("k_pool", "v_pool") if c["store"] else ())}


def _round(x):
    """Pages [n, B, (Hk,) D] in fp32 -> the e4m3 numbers and the scale of each page (and head): the least power of two that
    leaves nothing above 448."""
    top = x.abs().amax(-1).amax(1)                                   # [n(, Hk)]
    m, e = torch.frexp(top)                                          # 448 is 0.875 times 2^9
    e = torch.where(m > 0.875, e - 8, e - 9).clamp(-126, 127)
    scale = torch.where(top == 0, torch.ones_like(top), ((e + 127) << 23).to(torch.int32).view(torch.float32))
    return (x / (scale[:, None, ..., None] if x.dim() == 4 else scale[:, None, None])).to(E4M3), scale


def _page_scores(k, v):
    """Pages [n, B, (Hk,) D] -> the mean over a page's tokens of ||V|| / ||K||, in 64 bits, rounded once."""
    nk, nv = k.double().square().sum(-1).sqrt(), v.double().square().sum(-1).sqrt()
    return torch.where(nv == 0, torch.zeros_like(nv), nv / nk).mean(1).float()


def _plain_pages(s):
    c = s["case"]
    S, Hk, B, D, shared = c["seqs"], c["kv_heads"], c["page"], c["head_dim"], c["layout"] == "shared"
    src, dst, lens = s["src_table"], s["table"], s["seq_lens"]
    full = (lens // B).view((S,) + (1,) * (src.dim() - 1))
    which = torch.arange(src.shape[-1], device=DEVICE) < full
    which = which.expand(src.shape)
    a, b = src[which].long(), dst[which].long()
    k, v = s["k_pool"][a].float(), s["v_pool"][a].float()
    s["scores"].fill_(INF)
    for n, (x, name) in enumerate(((k, "k8"), (v, "v8"))):
        held, scale = _round(x)
        s[name].view(torch.uint8)[b] = held.view(torch.uint8)
        s["scales"][..., n][b] = scale
    got = _page_scores(k, v)                                         # [n(, Hk)]
    if shared:
        i, j = which.nonzero(as_tuple=True)
        s["scores"][i, :, j] = got
    else:
        s["scores"][which] = got
    # unfinished pages stay as they are
    last = full.clamp(max=src.shape[-1] - 1).long().expand(src.shape[:-1] + (1,))
    page = src.gather(-1, last)[..., 0].clamp(min=0).long()
    real = (torch.arange(B, device=DEVICE) < (lens % B)[:, None])[:, None, :, None]
    for pool, tail in (("k_pool", "k_tail"), ("v_pool", "v_tail")):
        x = s[pool][page]                                            # [S, Hk, B, D], or [S, B, Hk, D]
        s[tail].copy_(torch.where(real, x.transpose(1, 2) if shared else x, s[tail]))
    return {n: s[n] for n in ("k8", "v8", "scales", "k_tail", "v_tail", "scores")}


def _plain_append(s):
    c = s["case"]
    S, B, shared, lens, table = c["seqs"], c["page"], c["layout"] == "shared", s["seq_lens"], s["table"]
    if s["links"]:
        s["freed"].copy_(s["freed_before"])
        s["spare_used"].zero_()
    cos, sin = _angles(c, s["positions"])
    s["q_out"].copy_(_turned(c, s["q"].float(), cos, sin))
    slot, logical = (lens % B).long(), (lens // B).long()
    i = torch.arange(S, device=DEVICE)
    s["k_tail"][i, :, slot] = _turned(c, s["k_new"].float(), cos, sin).to(s["k_tail"].dtype)
    s["v_tail"][i, :, slot] = s["v_new"]
    # a new page where one begins: the freed one, else the next spare one
    per = (S,) + (1,) * (table.dim() - 1)
    begins = (slot == 0).view(per)
    at = logical.view(per).expand(table.shape[:-1] + (1,))
    freed = s["freed"][..., None]
    spare = s["spare"].gather(-1, s["spare_used"][..., None].clamp(max=s["spare"].shape[-1] - 1).long())
    page = torch.where(begins, torch.where(freed >= 0, freed, spare), table.gather(-1, at))
    table.scatter_(-1, at, page)
    s["spare_used"] += (begins & (freed < 0))[..., 0].int()
    s["freed"].copy_(torch.where(begins & (freed >= 0), torch.full_like(freed, -1), freed)[..., 0])
    s["lens_out"].copy_(lens + 1)
    # a page that has filled is rounded
    full = slot == B - 1
    k, v = s["k_tail"][full].float(), s["v_tail"][full].float()      # [n, Hk, B, D]
    s["scores"][full, :, logical[full]] = _page_scores(k.flatten(0, 1), v.flatten(0, 1)).view(-1, c["kv_heads"])
    to = page[full].flatten().long()
    for n, (x, name) in enumerate(((k, "k8"), (v, "v8"))):
        held, scale = _round(x.flatten(0, 1))
        held, scale = held.view(torch.uint8).view(x.shape), scale.view(x.shape[:2])
        s[name].view(torch.uint8)[to] = held.transpose(1, 2) if shared else held.flatten(0, 1)
        s["scales"][..., n][to] = scale if shared else scale.flatten()
    return {n: s[n] for n in ("q_out", "k8", "v8", "scales", "k_tail", "v_tail", "scores", "table", "lens_out", "freed", "spare_used")}


def _plain_decode(s):
    c = s["case"]
    S, Hk, Hq, D, B, shared = c["seqs"], c["kv_heads"], c["q_heads"], c["head_dim"], c["page"], c["layout"] == "shared"
    page, lens = s["table"].clamp(min=0).long(), s["seq_lens"]
    both = []
    for n, (name, tail) in enumerate((("k8", "k_tail"), ("v8", "v_tail"))):
        x, scale = s[name].view(torch.uint8)[page].view(E4M3).float(), s["scales"][page][..., n]
        x = x * (scale[:, :, None, :, None] if shared else scale[..., None, None])
        x = x.flatten(1, 2).transpose(1, 2) if shared else x.flatten(2, 3)
        both.append(torch.cat((x, s[tail].float()), 2))              # [S, Hk, tokens, D], the unfinished page behind the others
    t = torch.arange(both[0].shape[2], device=DEVICE)
    old = both[0].shape[2] - B
    real = torch.where(t < old, t < (lens // B * B)[:, None], t - old < (lens % B)[:, None])[:, None, None, :]
    logits = s["q"].float().view(S, Hk, Hq // Hk, D) @ both[0].transpose(2, 3) * D ** -0.5
    logits = logits.masked_fill_(~real, -INF)
    top = logits.amax(-1, keepdim=True)
    p = torch.exp(logits - torch.where(top == -INF, torch.zeros_like(top), top))
    total = p.sum(-1, keepdim=True)
    v = torch.where(real.transpose(2, 3), both[1], torch.zeros_like(both[1]))
    out = p @ v / torch.where(total == 0, torch.ones_like(total), total)
    s["out"].copy_(out.view(S, Hq, D))
    return {"out": s["out"]}


# ---- what a pass cannot do without ---------------------------------------------------------------------------------
def work(case):
    e = 2 if case["dtype"] == "bf16" else 4
    S, Hk, Hq, D, B = case["seqs"], case["kv_heads"], case["q_heads"], case["head_dim"], case["page"]
    rows = 1 if case["layout"] == "shared" else Hk
    lens = _lens(case)
    total = sum(lens)
    if case["kind"] == "plan":
        new = case["new"]
        fresh = sum(-(-(n + new) // B) - -(-n // B) for n in lens) if new else sum(-(-n // B) for n in lens)
        tokens = S * new if new else total
        return {"bytes": 8 * rows * fresh + 16 * S + tokens * (4 + 8 * rows), "flops": 0}
    if case["kind"] == "rotate":
        once = total * (Hq + Hk) * D * e
        store = total * (3 * Hk * D * e + 8 * rows) if case["store"] else 0     # V read, K and V into the pages
        return {"bytes": 2 * once + 4 * total + store, "flops": 3 * total * (Hq + Hk) * case["rotary"]}
    if case["kind"] == "pages":
        pages = sum(n // B for n in lens) * Hk
        left = sum(n % B for n in lens) * Hk * D * e * 4
        return {"bytes": pages * (2 * B * D * (e + 1) + 12) + 8 * rows * sum(n // B for n in lens) + left, "flops": pages * B * D * 6}
    if case["kind"] == "append":
        fills = sum(1 for n in lens if n % B == B - 1) * Hk
        return {"bytes": S * (Hq * 2 + Hk * 4) * D * e + fills * (2 * (B - 1) * D * e + 2 * B * D + 12) + 12 * S, "flops": 3 * S * (Hq + Hk) * case["rotary"]}
    pages = sum(n // B for n in lens)
    left = sum(n % B for n in lens)
    return {"bytes": pages * Hk * (2 * B * D + 8) + 4 * rows * pages + left * Hk * 2 * D * e + 2 * S * Hq * D * e, "flops": 4 * total * Hq * D}


# ---- the same in 64 bits, sequence by sequence -------------------------------------------------------------------------
def exact(case, seed):
    if case["kind"] == "plan":
        return None   # whole numbers
    s = prepare(case, seed)
    return {"rotate": _exact_rotate, "pages": _exact_pages, "append": _exact_append, "decode": _exact_decode}[case["kind"]](s, case)


def _exact_turn(case, x, positions, back=False):
    """Pairs as complex numbers, turned by exp(i angle)."""
    n = case["rotary"]
    theta = np.power(BASE, -np.arange(n // 2, dtype=np.float64) * 2.0 / n)
    if case["scaling"] == "linear":
        theta = theta / FACTOR
    if case["scaling"] == "parts":
        wave = 2.0 * np.pi / theta
        blend = np.clip((ORIGINAL / wave - LOW) / (HIGH - LOW), 0.0, 1.0)
        theta = blend * theta + (1.0 - blend) * theta / FACTOR
    angle = positions.double()[:, None] * torch.from_numpy(theta).to(DEVICE)
    turn = torch.polar(torch.full_like(angle, _magnitude(case)), -angle if back else angle)[:, None]
    x = x.double()
    half = case["pairs"] == "half"
    pair = torch.stack((x[..., :n // 2], x[..., n // 2:n]), -1) if half else x[..., :n].unflatten(-1, (n // 2, 2))
    y = torch.view_as_real(torch.view_as_complex(pair.contiguous()) * turn)
    y = torch.cat((y[..., 0], y[..., 1]), -1) if half else y.flatten(-2)
    return torch.cat((y, x[..., n:]), -1)


def _exact_rotate(s, case):
    q, k = (_exact_turn(case, s[n], s["positions"], case["transpose"]) for n in ("q", "k"))
    got = {"q_out": q, "k_out": k}
    if case["store"]:
        for name, x in (("k_pool", k), ("v_pool", s["v"].double())):
            pool = s[name].double()
            if case["layout"] == "shared":
                pool.view(-1, *pool.shape[2:]).index_copy_(0, s["slots"], x)
            else:
                pool.view(-1, pool.shape[2]).index_copy_(0, s["slots"].reshape(-1), x.reshape(-1, x.shape[-1]))
            got[name] = pool
    return got


def _exact_page(x):
    """A head's page [B, D] in 64 bits: the values before their rounding, relative to the scale, and the scale."""
    top = float(x.abs().max())
    scale = 1.0 if top == 0 else 2.0 ** max(-126, math.ceil(math.log2(top / 448.0)))
    return x / scale, scale


def _exact_ratio(k, v):
    return float((torch.linalg.vector_norm(v, dim=1) / torch.linalg.vector_norm(k, dim=1)).mean())


def _exact_pages(s, case):
    # one by one: not where there are many
    if sum(n // case["page"] for n in _lens(case)) * case["kv_heads"] > 2000:
        return None
    B, Hk, shared = case["page"], case["kv_heads"], case["layout"] == "shared"
    got = {n: s[n].double() for n in ("k8", "v8", "scales", "k_tail", "v_tail")}
    got["scores"] = torch.full(s["scores"].shape, INF, dtype=torch.float64, device=DEVICE)
    for i, n in enumerate(s["seq_lens"].tolist()):
        for h in range(Hk):
            at = (i,) if shared else (i, h)
            src, dst = s["src_table"][at].tolist(), s["table"][at].tolist()
            part = (slice(None), h) if shared else (slice(None),)
            for j in range(n // B):
                k, v = (s[p][src[j]][part].double() for p in ("k_pool", "v_pool"))
                for c, (x, name) in enumerate(((k, "k8"), (v, "v8"))):
                    held, scale = _exact_page(x)
                    got[name][dst[j]][part] = held
                    got["scales"][(dst[j], h, c) if shared else (dst[j], c)] = scale
                got["scores"][i, h, j] = _exact_ratio(k, v)
            if n % B:
                for p, name in (("k_pool", "k_tail"), ("v_pool", "v_tail")):
                    got[name][i, h, :n % B] = s[p][src[n // B]][part].double()[:n % B]
    return got


def _exact_append(s, case):
    B, Hk, shared = case["page"], case["kv_heads"], case["layout"] == "shared"
    lens = s["seq_lens"].tolist()
    if sum(1 for n in lens if n % B == B - 1) * Hk > 2000:
        return None
    got = {n: s[n].double() for n in ("k8", "v8", "scales", "k_tail", "v_tail", "scores")}
    got["q_out"] = _exact_turn(case, s["q"], s["positions"])
    k_new = _exact_turn(case, s["k_new"], s["positions"])
    for i, n in enumerate(lens):
        got["k_tail"][i, :, n % B], got["v_tail"][i, :, n % B] = k_new[i], s["v_new"][i].double()
        for h in range(Hk if n % B == B - 1 else 0):
            table = s["table"][i] if shared else s["table"][i, h]
            begins = s["freed"][i] if shared else s["freed"][i, h]
            spare = s["spare"][i] if shared else s["spare"][i, h]
            page = int(table[n // B]) if B > 1 and n % B else int(begins if begins >= 0 else spare[0])
            k, v = got["k_tail"][i, h], got["v_tail"][i, h]
            part = (slice(None), h) if shared else (slice(None),)
            for c, (x, name) in enumerate(((k, "k8"), (v, "v8"))):
                held, scale = _exact_page(x)
                got[name][page][part] = held
                got["scales"][(page, h, c) if shared else (page, c)] = scale
            got["scores"][i, h, n // B] = _exact_ratio(k, v)
    return {n: got.get(n) for n in ("q_out", "k8", "v8", "scales", "k_tail", "v_tail", "scores", "table", "lens_out", "freed", "spare_used")}


def _exact_decode(s, case):
    B, Hk, G, shared = case["page"], case["kv_heads"], case["q_heads"] // case["kv_heads"], case["layout"] == "shared"
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device=DEVICE)
    k8, v8 = (s[n].view(torch.uint8) for n in ("k8", "v8"))
    for i, n in enumerate(s["seq_lens"].tolist()):
        full, left = n // B, n % B
        for h in range(Hk if n else 0):
            page = (s["table"][i] if shared else s["table"][i, h])[:full].long()
            rows = []
            for c, (pool, tail) in enumerate(((k8, s["k_tail"]), (v8, s["v_tail"]))):
                x = (pool[page][:, :, h] if shared else pool[page]).view(E4M3).to(torch.float32).double()
                scale = (s["scales"][page, h, c] if shared else s["scales"][page, c]).double()
                rows.append(torch.cat(((x * scale[:, None, None]).flatten(0, 1), tail[i, h, :left].double())))
            x = s["q"][i, h * G:h * G + G].double() @ rows[0].t().contiguous() * case["head_dim"] ** -0.5
            w = torch.exp(x - x.max(1, keepdim=True).values)
            out[i, h * G:h * G + G] = (w @ rows[1]) / w.sum(1, keepdim=True)
    return {"out": out}
