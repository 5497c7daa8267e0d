"""The operators of a paged beam search, as measurable cases.

Five kinds of call, in the order in which one decoding step makes them:

  plan     mtp_page_plan: pages, block tables and slot maps of the tokens that each slot gets
  append   mtp_cache_append: the new keys and values into the cache, by slot map
  attend   mtp_chunk_attention: a chunk of new tokens per slot against everything cached
  select   mtp_beam_select: the best continuations over all beams and the vocabulary
  reorder  mtp_beam_reorder: block tables, lengths and page counts of the kept beams, with the
           copies of their last, partly filled pages

`own` chooses between the plain form (elementary torch operations in 32 bits) and the package.
Sizes are the repository's own (16 heads of 64, 12 layers, pages of 16 to 128, codec vocabulary 1025,
prompts of 182 to 578 positions, contexts of 180 to 2000 keys, prefill passes of 14592 rows) and, for
programs with another model around the same cache, head groups, 128-wide heads, longer contexts and
larger vocabularies.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = {"f32": F32, "bf16": BF16, "f16": F16}
INF = float("inf")


def listed():
    return [
        # one decoding step of 32 utterances, one token each: the smallest call, all latency
        {"name": "plan step 32", "kind": "plan", "slots": 32, "len_lo": 180, "len_hi": 2000, "new_lo": 1, "new_hi": 1,
         "page": 64, "pages": 2048},
        # admission of a large mixed batch: some slots get a prompt, some a token, some nothing
        {"name": "plan mixed 1000", "kind": "plan", "slots": 1000, "len_lo": 0, "len_hi": 900, "new_lo": 0,
         "new_hi": 300, "page": 16, "pages": 90001},
        # keys and values of one decoding step of 128 utterances, out of the fused fp32 projection
        {"name": "append step 128", "kind": "append", "rows": 128, "heads": 16, "kv_heads": 16, "dim": 64, "page": 64,
         "src": "f32", "type": "bf16", "fused": True},
        # those of a whole prefill pass
        {"name": "append pass 14592", "kind": "append", "rows": 14592, "heads": 16, "kv_heads": 16, "dim": 64,
         "page": 64, "src": "bf16", "type": "bf16", "fused": True},
        # one layer of a decoding step of 32 utterances: one new token each, ragged contexts
        {"name": "attend step 32", "kind": "attend", "slots": 32, "new_lo": 1, "new_hi": 1, "ctx_lo": 180,
         "ctx_hi": 2000, "heads": 16, "kv_heads": 16, "dim": 64, "page": 64, "type": "bf16", "window": 0, "fused": True},
        # verification of 4 drafts against long contexts, four query heads to a key head
        {"name": "attend drafts 8", "kind": "attend", "slots": 8, "new_lo": 4, "new_hi": 4, "ctx_lo": 4000,
         "ctx_hi": 30000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "type": "f16", "window": 0, "fused": False},
        # packed prompts from nothing, every position of each
        {"name": "attend prompts 25", "kind": "attend", "slots": 25, "new_lo": 182, "new_hi": 578, "ctx_lo": 0,
         "ctx_hi": 0, "heads": 16, "kv_heads": 16, "dim": 64, "page": 64, "type": "bf16", "window": 0, "fused": True},
        # chunked prefill of two long requests: the next few thousand tokens of each
        {"name": "attend chunk 2", "kind": "attend", "slots": 2, "new_lo": 2000, "new_hi": 4000, "ctx_lo": 6000,
         "ctx_hi": 9000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 64, "type": "bf16", "window": 0, "fused": True},
        # beam search of one utterance over the codec vocabulary, straight from the logits
        {"name": "select codec 1x5", "kind": "select", "batch": 1, "beams": 5, "vocab": 1025, "k": 10, "type": "f32",
         "lse": False},
        # a served batch over a large vocabulary of another model, with the heads' log-sum-exp
        {"name": "select 32x4 large", "kind": "select", "batch": 32, "beams": 4, "vocab": 48001, "k": 8,
         "type": "bf16", "lse": True},
        # the cache after a step of one utterance's 4 beams
        {"name": "reorder 1x4", "kind": "reorder", "batch": 1, "beams": 4, "len_lo": 300, "len_hi": 900, "page": 64,
         "layers": 12, "kv_heads": 16, "dim": 64, "type": "bf16"},
        # after a step of 12 utterances with 8 beams each
        {"name": "reorder 12x8", "kind": "reorder", "batch": 12, "beams": 8, "len_lo": 200, "len_hi": 800, "page": 64,
         "layers": 12, "kv_heads": 16, "dim": 64, "type": "bf16"},
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "attend", "select", "select", "reorder"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "plan":
        slots = _log_int(rng, 1, 1000)
        lo, new = rng.randint(0, 300), rng.choice([1, 4, rng.randint(2, 300)])
        hi = lo + rng.randint(0, 600)
        return {"kind": kind, "slots": slots, "len_lo": lo, "len_hi": hi, "new_lo": rng.randint(0, 1), "new_hi": new,
                "page": page, "pages": slots * (-(-(hi + new) // page) + 1) + rng.randint(0, 20000)}
    dim, group = rng.choice([64, 128]), rng.choice([1, 2, 4, 5, 8])
    kv_heads = rng.choice([1, 2, 4, 8] if dim == 128 else [2, 4, 8, 16])
    while kv_heads * group > 32:
        group = rng.choice([1, 2, 4])
        kv_heads = max(1, kv_heads // 2)
    shape = {"heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "page": page}
    if kind == "append":
        return {"kind": kind, "rows": _log_int(rng, 1, 14592), **shape, "src": rng.choice(["f32", "bf16"]),
                "type": "bf16", "fused": rng.random() < 0.7}
    if kind == "attend":
        type_ = rng.choice(["bf16", "f16"])
        window = rng.choice([0, 0, 0, rng.randint(100, 2000)])
        form = rng.choice(["step", "drafts", "prompts", "chunk"])
        if form in ("step", "drafts"):
            lo = _log_int(rng, 30, 16000)
            hi = min(32000, lo * rng.randint(1, 3))
            slots = _log_int(rng, 1, max(1, min(128, 250000 // hi)))
            new = 1 if form == "step" else rng.randint(2, 9)
            return {"kind": kind, "slots": slots, "new_lo": new, "new_hi": new, "ctx_lo": lo, "ctx_hi": hi, **shape,
                    "type": type_, "window": window, "fused": rng.random() < 0.5}
        if form == "prompts":
            return {"kind": kind, "slots": _log_int(rng, 1, 48), "new_lo": rng.randint(20, 200),
                    "new_hi": rng.randint(200, 600), "ctx_lo": 0, "ctx_hi": 0, **shape, "type": type_,
                    "window": window, "fused": True}
        ctx = rng.randint(500, 6000)
        return {"kind": kind, "slots": rng.randint(1, 2), "new_lo": rng.randint(150, 900),
                "new_hi": rng.randint(900, 3000), "ctx_lo": ctx, "ctx_hi": ctx + rng.randint(0, 2000), **shape,
                "type": type_, "window": window, "fused": rng.random() < 0.5}
    if kind == "select":
        vocab = rng.choice([1025, _log_int(rng, 64, 48001)])
        batch, beams = _log_int(rng, 1, 64 if vocab < 9000 else 32), rng.choice([1, 2, 3, 4, 5, 8])
        if vocab > 9000:
            beams = min(beams, 4)
        return {"kind": kind, "batch": batch, "beams": beams, "vocab": vocab,
                "k": min(rng.choice([1, 2]) * beams, vocab), "type": rng.choice(["f32", "bf16", "f16"]),
                # orders are compared between forms that sum in another order: log-sum-exps of many requests are given
                "lse": batch > 3 or rng.random() < 0.5}
    lo = rng.randint(20, 500)
    return {"kind": kind, "batch": _log_int(rng, 1, 12), "beams": rng.choice([2, 3, 4, 5, 8]), "len_lo": lo,
            "len_hi": lo + rng.randint(0, 300), "page": page, "layers": rng.choice([2, 6, 12]),
            "kv_heads": kv_heads, "dim": dim, "type": rng.choice(["bf16", "f16"])}


# ---- inputs ----


def _host(case, seed):
    return random.Random("%d %s" % (seed, case["kind"]))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + 12345) % (1 << 61))


def _ints(values):
    return torch.tensor(values, dtype=torch.int32).cuda()


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, device="cuda", generator=gen) * scale).to(dtype)


def _tables(rng, counts, n_pages, stride):
    """Block tables of slots with `counts` pages each, the pages in no order, -1 past them; and the pages' counts."""
    pages = torch.randperm(n_pages, generator=torch.Generator().manual_seed(rng.randrange(1 << 30)))
    table = torch.full((len(counts), stride), -1, dtype=torch.int32)
    inside = torch.arange(stride)[None, :] < torch.tensor(counts)[:, None]
    used = pages[:sum(counts)]
    table[inside] = used.int()
    refs = torch.zeros(n_pages, dtype=torch.int32)
    refs[used] = 1
    return table.cuda(), refs.cuda()


def _lengths(case, seed):
    """Tokens that each slot of an attention case gets, and its length with them."""
    rng = _host(case, seed)
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["slots"])]
    ctx = [rng.randint(case["ctx_lo"], case["ctx_hi"]) for _ in range(case["slots"])]
    return new, [c + n for c, n in zip(ctx, new)]


def prepare(case, seed):
    st = SimpleNamespace(case=case, kind=case["kind"], stream=torch.cuda.current_stream().cuda_stream)
    _PREPARE[case["kind"]](st, case, seed)
    if own:  # a program makes the same step again and again: it keeps its argument blocks and its scratch
        _KEEP[case["kind"]](st)
    return st


def _prepare_plan(st, c, seed):
    rng = _host(c, seed)
    slots, page = c["slots"], c["page"]
    lens = [rng.randint(c["len_lo"], c["len_hi"]) for _ in range(slots)]
    new = [rng.randint(c["new_lo"], c["new_hi"]) for _ in range(slots)]
    new[rng.randrange(slots)] = c["new_hi"]
    stride = -(-(c["len_hi"] + c["new_hi"]) // page) + 2
    st.table, st.refs = _tables(rng, [-(-n // page) for n in lens], c["pages"], stride)
    st.lens, st.new = _ints(lens), _ints(new)
    st.max_rows = slots * c["new_hi"]  # what the program's buffers hold
    st.stride = stride
    i32 = dict(dtype=torch.int32, device="cuda")
    st.out_lens, st.out_refs = torch.empty(slots, **i32), torch.empty(c["pages"], **i32)
    st.slot_map = torch.empty(st.max_rows, dtype=torch.int64, device="cuda")
    st.row_seq, st.row_pos = torch.empty(st.max_rows, **i32), torch.empty(st.max_rows, **i32)
    st.cu_rows, st.status = torch.empty(slots + 1, **i32), torch.empty(4, **i32)


def _keys(st, c, n_pages, gen):
    """One layer of two in a cache pool, and a fused q | k | v row buffer or three of its own."""
    rows, h, hk, d = st.rows, c["heads"], c["kv_heads"], c["dim"]
    st.layers, st.layer = 2, 1
    st.pool = _normal(gen, (n_pages, 2, 2, hk, c["page"], d), TYPES[c["type"]])
    src = TYPES[c.get("src", c["type"])]
    if c["fused"]:
        x = _normal(gen, (rows, h + 2 * hk, d), src)
        st.q, st.k, st.v = x[:, :h], x[:, h:h + hk], x[:, h + hk:]
    else:
        st.q = _normal(gen, (rows, h, d), src)
        st.k, st.v = _normal(gen, (rows, hk, d), src), _normal(gen, (rows, hk, d), src)


def _prepare_append(st, c, seed):
    gen, rows, page = _gen(seed), c["rows"], c["page"]
    n_pages = -(-rows // page) * 2 + 8
    st.rows = rows
    _keys(st, c, n_pages, gen)
    # runs of positions inside pages, the pages in no order; a few rows of a padded batch have no place
    at = torch.arange(rows, device="cuda")
    order = torch.randperm(n_pages, device="cuda", generator=gen)
    off = int(torch.randint(0, page, (1,), generator=torch.Generator().manual_seed(seed)))
    st.slot_map = order[(at + off) // page] * page + (at + off) % page
    if rows > 16:
        st.slot_map[torch.randint(0, rows, (rows // 16,), device="cuda", generator=gen)] = -1


def _prepare_attend(st, c, seed):
    gen, page = _gen(seed), c["page"]
    new, lens = _lengths(c, seed)
    st.rows = c["slots"] * c["new_hi"]  # what the program's row buffers hold
    st.live, st.max_new, st.max_keys = sum(new), max(new), max(lens)
    counts = [-(-n // page) for n in lens]
    st.stride = max(counts) + 1
    st.table, _ = _tables(_host(c, seed), counts, sum(counts) + 3, st.stride)
    st.lens = _ints(lens)
    st.cu_rows = _ints([sum(new[:i]) for i in range(len(new) + 1)])
    _keys(st, c, sum(counts) + 3, gen)
    st.q *= 2.0  # scores that spread as a trained model's do
    st.scale = c["dim"] ** -0.5
    st.out = torch.zeros(st.rows, c["heads"], c["dim"], dtype=TYPES[c["type"]], device="cuda")
    st.lse = torch.zeros(st.rows, c["heads"], device="cuda")


def _prepare_select(st, c, seed):
    gen, b, w, v = _gen(seed), c["batch"], c["beams"], c["vocab"]
    x = 2.0 * torch.randn(b, w, v, device="cuda", generator=gen)
    # some codes are likely after every prefix, and a constrained decoder's masks leave a few out
    x += 2.0 * torch.randn(1, 1, v, device="cuda", generator=gen)
    x[:, :, torch.randint(0, v - 1, (max(1, v // 50),), device="cuda", generator=gen)] = -INF
    st.logits = x.to(TYPES[c["type"]])
    st.given = torch.logsumexp(st.logits.float(), -1) if c["lse"] else None
    st.scores = -4.0 * torch.rand(b, w, device="cuda", generator=gen).cumsum(1)
    st.done = (torch.rand(b, w, device="cuda", generator=gen) < 0.1).int()
    st.eos = v - 1
    i32 = dict(dtype=torch.int32, device="cuda")
    st.out_scores, st.lse = torch.empty(b, c["k"], device="cuda"), torch.empty(b, w, device="cuda")
    st.parent, st.token, st.out_done = (torch.empty(b, c["k"], **i32) for _ in range(3))


def _prepare_reorder(st, c, seed):
    rng, gen = _host(c, seed), _gen(seed)
    b, w, page = c["batch"], c["beams"], c["page"]
    lens = [rng.randint(c["len_lo"], c["len_hi"]) for _ in range(b)]
    # full pages that an utterance's beams have in common: its prompt's, and those of a common beginning
    shared = [rng.randint(n // page // 2, n // page) for n in lens]
    st.stride = -(-(c["len_hi"] + 1) // page) + 1
    own_pages = sum(w * (-(-n // page) - s) + s for n, s in zip(lens, shared))
    most = c["len_hi"] // page
    st.n_pages = b * (w * (most + 1 - most // 2) + most // 2 + w)
    order = iter(rng.sample(range(st.n_pages), own_pages))
    refs, table = [0] * st.n_pages, []
    for n, s in zip(lens, shared):
        common = [next(order) for _ in range(s)]
        for _ in range(w):
            pages = common + [next(order) for _ in range(-(-n // page) - s)]
            for p in pages:
                refs[p] += 1
            table.append(pages + [-1] * (st.stride - len(pages)))
    st.table, st.refs = _ints(table), _ints(refs)
    st.lens = _ints([n for n in lens for _ in range(w)])
    # a few beams have most of the children
    st.parent = _ints([[min(rng.randrange(w), rng.randrange(w)) for _ in range(w)] for _ in range(b)])
    st.pool = _normal(gen, (st.n_pages, c["layers"], 2, c["kv_heads"], page, c["dim"]), TYPES[c["type"]])
    i32 = dict(dtype=torch.int32, device="cuda")
    st.out_table, st.out_lens = torch.empty(b * w, st.stride, **i32), torch.empty(b * w, **i32)
    st.out_refs, st.status = torch.empty(st.n_pages, **i32), torch.empty(4, **i32)


_PREPARE = {"plan": _prepare_plan, "append": _prepare_append, "attend": _prepare_attend, "select": _prepare_select,
            "reorder": _prepare_reorder}


# ---- the package's operators ----


def _scratch(nbytes):
    return torch.zeros(max(16, nbytes), dtype=torch.uint8, device="cuda"), nbytes


def _keep_plan(st):
    from paper_2410_13839_gb300 import mtp
    c = st.case
    st.mtp, st.args = mtp, mtp.page_plan_args(
        slots=c["slots"], page_size=c["page"], n_pages=c["pages"], bt_stride=st.stride, max_rows=st.max_rows,
        kv_lens=st.lens, new_lens=st.new, block_table=st.table, page_refs=st.refs, out_kv_lens=st.out_lens,
        out_page_refs=st.out_refs, out_slot_map=st.slot_map, out_row_seq=st.row_seq, out_row_pos=st.row_pos,
        out_cu_rows=st.cu_rows, out_status=st.status)


def _keep_append(st):
    from paper_2410_13839_gb300 import mtp
    st.mtp, st.args = mtp, mtp.cache_append_args(k=st.k, v=st.v, slot_map=st.slot_map, kv_pool=st.pool, layer=st.layer)


def _keep_attend(st):
    from paper_2410_13839_gb300 import mtp
    st.mtp, st.args = mtp, mtp.chunk_attention_args(
        q=st.q, kv_pool=st.pool, layer=st.layer, block_table=st.table, cu_rows=st.cu_rows, kv_lens=st.lens, out=st.out,
        out_lse=st.lse, scale=st.scale, window=st.case["window"], max_new=st.max_new, max_keys=st.max_keys)
    st.scratch = _scratch(mtp.mtp_chunk_attention_workspace_bytes(st.args))


def _keep_select(st):
    from paper_2410_13839_gb300 import mtp
    st.mtp, st.args = mtp, mtp.beam_select_args(
        logits=st.logits, lse=st.given, scores=st.scores, done=st.done, k=st.case["k"], eos_id=st.eos,
        out_scores=st.out_scores, out_parent=st.parent, out_token=st.token, out_done=st.out_done, out_lse=st.lse)
    st.scratch = _scratch(mtp.mtp_beam_select_workspace_bytes(st.args))


def _keep_reorder(st):
    from paper_2410_13839_gb300 import mtp
    st.mtp, st.args = mtp, mtp.beam_reorder_args(
        parent=st.parent, block_table=st.table, kv_lens=st.lens, page_refs=st.refs, kv_pool=st.pool,
        out_block_table=st.out_table, out_kv_lens=st.out_lens, out_page_refs=st.out_refs, out_status=st.status)
    st.scratch = _scratch(mtp.mtp_beam_reorder_workspace_bytes(st.args))


_KEEP = {"plan": _keep_plan, "append": _keep_append, "attend": _keep_attend, "select": _keep_select,
         "reorder": _keep_reorder}


def run(st):
    return (_OWN if own else _PLAIN)[st.kind](st)


def _own_plan(st):
    st.mtp.mtp_page_plan(st.args, st.stream)
    return {"table": st.table, "lens": st.out_lens, "refs": st.out_refs, "slot_map": st.slot_map,
            "row_seq": st.row_seq, "row_pos": st.row_pos, "cu_rows": st.cu_rows, "status": st.status}


def _own_append(st):
    st.mtp.mtp_cache_append(st.args, st.stream)
    return {"pool": st.pool}


def _own_attend(st):
    st.mtp.mtp_chunk_attention(st.args, st.scratch[0], st.scratch[1], st.stream)
    return {"out": st.out, "lse": st.lse}


def _own_select(st):
    st.mtp.mtp_beam_select(st.args, st.scratch[0], st.scratch[1], st.stream)
    return {"scores": st.out_scores, "parent": st.parent, "token": st.token, "done": st.out_done, "lse": st.lse}


def _own_reorder(st):
    st.mtp.mtp_beam_reorder(st.args, st.scratch[0], st.scratch[1], st.stream)
    return {"table": st.out_table, "lens": st.out_lens, "refs": st.out_refs, "status": st.status, "pool": st.pool}


_OWN = {"plan": _own_plan, "append": _own_append, "attend": _own_attend, "select": _own_select,
        "reorder": _own_reorder}


# ---- the plain forms ----


def _plain_plan(st):
    page, pages = st.case["page"], st.case["pages"]
    lens, new = st.lens.long(), st.new.long()
    slots = lens.numel()
    after = lens + new
    had, want = (lens + page - 1) // page, (after + page - 1) // page
    free = torch.sort(torch.where(st.refs == 0, torch.arange(pages, device="cuda"), pages))[0]  # lowest first
    first = torch.cumsum(want - had, 0) - (want - had)
    col = torch.arange(st.stride, device="cuda")[None, :]
    fresh = (col >= had[:, None]) & (col < want[:, None])
    rank = (first[:, None] + col - had[:, None]).clamp(0, pages - 1)
    st.table.copy_(torch.where(fresh, free[rank].int(), st.table))
    refs = torch.cat([st.refs, st.refs[:1]])
    refs[torch.where(fresh, free[rank], pages)] = 1
    cu = torch.cumsum(torch.cat([new[:1] * 0, new]), 0)
    at = torch.arange(st.max_rows, device="cuda")
    seq = torch.searchsorted(cu[1:], at, right=True)
    live = seq < slots
    seq = seq.clamp(max=slots - 1)
    pos = lens[seq] + at - cu[seq]
    where = st.table[seq, (pos // page).clamp(0, st.stride - 1)].long() * page + pos % page
    none = torch.full_like(where, -1)
    taken = (want - had).sum()
    status = torch.stack([taken * 0, cu[-1], taken, (st.refs == 0).sum() - taken]).int()
    return {"table": st.table, "lens": after.int(), "refs": refs[:pages], "slot_map": torch.where(live, where, none),
            "row_seq": torch.where(live, seq, none).int(), "row_pos": torch.where(live, pos, none).int(),
            "cu_rows": cu.int(), "status": status}


def _plain_append(st):
    page = st.case["page"]
    live = torch.nonzero(st.slot_map >= 0)[:, 0]
    at = st.slot_map[live]
    st.pool[at // page, st.layer, 0, :, at % page] = st.k[live].to(st.pool.dtype)
    st.pool[at // page, st.layer, 1, :, at % page] = st.v[live].to(st.pool.dtype)
    return {"pool": st.pool}


def _plain_attend(st):
    c = st.case
    page, h, hk, d = c["page"], c["heads"], c["kv_heads"], c["dim"]
    slots, new = st.lens.numel(), st.cu_rows.long().diff()
    lens = st.lens.long()
    key = torch.arange(st.max_keys, device="cuda")
    pages = st.table[:, key // page].long().clamp(min=0)
    k, v = (st.pool[pages, st.layer, i, :, key % page].float() for i in (0, 1))  # [slots, keys, kv heads, dim]
    i = torch.arange(st.max_new, device="cuda")
    row = (st.cu_rows[:-1].long()[:, None] + i).clamp(max=st.rows - 1)
    q = st.q[row].float().reshape(slots, st.max_new, hk, h // hk, d).permute(0, 2, 3, 1, 4)
    s = torch.matmul(q.reshape(slots, hk, -1, d), k.permute(0, 2, 3, 1)) * st.scale
    s = s.view(slots, hk, h // hk, st.max_new, st.max_keys)
    pos = (lens - new)[:, None] + i
    hidden = key > pos[:, :, None]
    if c["window"]:
        hidden |= key <= pos[:, :, None] - c["window"]
    s.masked_fill_(hidden[:, None, None], -INF)
    m = s.amax(-1, keepdim=True)
    m = torch.where(m == -INF, torch.zeros_like(m), m)
    p = s.sub_(m).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.view(slots, hk, -1, st.max_keys), v.permute(0, 2, 1, 3)).view(slots, hk, h // hk, st.max_new, d)
    o = o / torch.where(total == 0, torch.ones_like(total), total)
    lse = (m + total.log())[..., 0]
    live = i < new[:, None]
    st.out[:st.live] = o.permute(0, 3, 1, 2, 4).reshape(slots, st.max_new, h, d)[live].to(st.out.dtype)
    st.lse[:st.live] = lse.permute(0, 3, 1, 2).reshape(slots, st.max_new, h)[live]
    return {"out": st.out, "lse": st.lse}


def _plain_select(st):
    b, w, v = st.logits.shape
    x = st.logits.float()
    lse = st.given
    if lse is None:
        m = x.amax(-1, keepdim=True)
        lse = (m + (x - m).exp().sum(-1, keepdim=True).log())[..., 0]
    s = st.scores[..., None] + (x - lse[..., None])
    s = torch.where(s.isnan(), torch.full_like(s, -INF), s)
    done = st.done[..., None] != 0
    eos = torch.arange(v, device="cuda") == st.eos
    s = torch.where(done, torch.where(eos, st.scores[..., None], -INF), s)
    best, at = torch.sort(s.view(b, w * v), dim=-1, descending=True, stable=True)
    best, at = best[:, :st.case["k"]], at[:, :st.case["k"]]
    token = (at % v).int()
    parent = at // v
    ended = ((token == st.eos) | (st.done.gather(1, parent) != 0)).int()
    return {"scores": best, "parent": parent.int(), "token": token, "done": ended, "lse": lse}


def _plain_reorder(st):
    b, w = st.parent.shape
    page, n, rows = st.case["page"], st.n_pages, st.parent.numel()
    lens = st.lens.long()
    from_ = (torch.arange(b, device="cuda")[:, None] * w + st.parent.long()).view(-1)
    earlier = torch.arange(w, device="cuda")[None, :] < torch.arange(w, device="cuda")[:, None]
    again = ((st.parent[:, :, None] == st.parent[:, None, :]) & earlier).any(-1).view(-1)
    new = lens[from_]
    copy = again & (new % page != 0)
    col = torch.arange(st.stride, device="cuda")[None, :]
    old_used, used = col < ((lens + page - 1) // page)[:, None], col < ((new + page - 1) // page)[:, None]
    table = torch.where(used, st.table[from_], -1)
    free = torch.sort(torch.where(st.refs == 0, torch.arange(n, device="cuda"), n))[0]
    fresh = free[(torch.cumsum(copy.long(), 0) - 1).clamp(0, n - 1)]
    last = (new // page).clamp(max=st.stride - 1)
    each = torch.arange(rows, device="cuda")
    src = table[each, last].long()
    table[each, last] = torch.where(copy, fresh.int(), table[each, last])
    ones = torch.ones_like(table)
    count = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    count.index_add_(0, torch.where(used, table, n).view(-1).long(), ones.view(-1))
    count.index_add_(0, torch.where(old_used, st.table, n).view(-1).long(), -ones.view(-1))
    taken = copy.sum()
    refs = st.refs + count[:n]
    at = torch.nonzero(copy)[:, 0]
    cached = (torch.arange(page, device="cuda") < (new % page)[at][:, None])[:, None, None, None, :, None]
    st.pool[fresh[at]] = torch.where(cached, st.pool[src[at]], st.pool[fresh[at]])
    status = torch.stack([taken * 0, taken, (refs == 0).sum(), taken * 0]).int()
    return {"table": table, "lens": new.int(), "refs": refs, "status": status, "pool": st.pool}


_PLAIN = {"plan": _plain_plan, "append": _plain_append, "attend": _plain_attend, "select": _plain_select,
          "reorder": _plain_reorder}


# ---- what a pass cannot do without ----


def _seen(new, length, window):
    """Keys that a slot's new rows see, summed, and the cached keys that any of them sees."""
    first = length - new + 1
    if not window:
        return new * first + new * (new - 1) // 2, length
    return sum(min(window, first + i) for i in range(new)), min(length, window + new - 1)


def work(case):
    c, kind = case, case["kind"]
    size = 2 if c.get("type") in ("bf16", "f16") else 4
    if kind == "plan":
        # lengths in and out, row plan out, the pages' counts in and out
        return {"bytes": c["slots"] * 16 + c["slots"] * (c["new_lo"] + c["new_hi"]) // 2 * 16 + c["pages"] * 8,
                "flops": 0}
    if kind == "append":
        n = c["rows"] * c["kv_heads"] * c["dim"] * 2
        return {"bytes": n * (size + (4 if c["src"] == "f32" else 2)) + c["rows"] * 8, "flops": 0}
    if kind == "attend":
        new, lens = _lengths(c, 1)
        pairs, keys = (sum(x) for x in zip(*(_seen(n, t, c["window"]) for n, t in zip(new, lens))))
        rows = sum(new) * c["heads"]
        return {"bytes": (keys * c["kv_heads"] * 2 + rows * 2) * c["dim"] * size + rows * 4,
                "flops": 4 * pairs * c["heads"] * c["dim"]}
    if kind == "select":
        n = c["batch"] * c["beams"]
        return {"bytes": n * c["vocab"] * size + n * 16 + c["batch"] * c["k"] * 16, "flops": 0}
    # about a third of the beams share their parent with an earlier one, and a last page is half full
    rows, token = c["batch"] * c["beams"], c["layers"] * 2 * c["kv_heads"] * c["dim"] * size
    pages = rows * (c["len_lo"] + c["len_hi"]) // 2 // c["page"]
    return {"bytes": rows // 2 * c["page"] // 2 * token * 2 + pages * 8, "flops": 0}


# ---- the definition in 64 bits ----


def exact(case, seed):
    kind = case["kind"]
    if kind == "plan":
        return None  # whole numbers only
    st = SimpleNamespace(case=case)
    _PREPARE[kind](st, case, seed)
    return _EXACT[kind](st, case)


def _exact_append(st, c):
    pool = st.pool.double()
    for r, at in enumerate(st.slot_map.tolist()):
        if at >= 0:
            pool[at // c["page"], st.layer, 0, :, at % c["page"]] = st.k[r].double()
            pool[at // c["page"], st.layer, 1, :, at % c["page"]] = st.v[r].double()
    return {"pool": pool}


def _exact_attend(st, c):
    """Slot by slot and head by head, a block of rows at a time."""
    group = c["heads"] // c["kv_heads"]
    out = torch.zeros(st.rows, c["heads"], c["dim"], dtype=torch.float64, device="cuda")
    lse = torch.zeros(st.rows, c["heads"], dtype=torch.float64, device="cuda")
    cu = st.cu_rows.tolist()
    for b, length in enumerate(st.lens.tolist()):
        pages = st.table[b, :-(-length // c["page"])].long()
        kv = st.pool[pages, st.layer].transpose(0, 1)  # 2, pages, kv heads, page, dim
        for g in range(c["kv_heads"]):
            k, v = (x[:, g].reshape(-1, c["dim"])[:length].double() for x in kv)
            for r0 in range(cu[b], cu[b + 1], 512):
                r1 = min(cu[b + 1], r0 + 512)
                pos = length - cu[b + 1] + torch.arange(r0, r1, device="cuda")
                t = torch.arange(length, device="cuda")
                sees = t <= pos[:, None]
                if c["window"]:
                    sees &= t > pos[:, None] - c["window"]
                q = st.q[r0:r1, g * group:(g + 1) * group].double()
                s = torch.einsum("rgd,td->rgt", q, k) * st.scale
                s = s.masked_fill(~sees[:, None], -INF)
                out[r0:r1, g * group:(g + 1) * group] = torch.einsum("rgt,td->rgd", torch.softmax(s, -1), v)
                lse[r0:r1, g * group:(g + 1) * group] = torch.logsumexp(s, -1)
    return {"out": out, "lse": lse}


def _exact_select(st, c):
    x = st.logits.double()
    lse = torch.logsumexp(x, -1) if st.given is None else st.given.double()
    s = torch.log_softmax(x, -1) if st.given is None else x - lse[..., None]
    s = s + st.scores.double()[..., None]
    for b, w in torch.nonzero(st.done).tolist():
        s[b, w] = -INF
        s[b, w, st.eos] = st.scores[b, w].double()
    return {"scores": torch.topk(s.flatten(1), c["k"]).values, "parent": None, "token": None, "done": None, "lse": lse}


def _exact_reorder(st, c):
    """Only copies: the pool after them, in 64 bits; the rest is whole numbers."""
    pool, page, w = st.pool.double(), c["page"], c["beams"]
    lens, table = st.lens.tolist(), st.table.tolist()
    free = [p for p, n in enumerate(st.refs.tolist()) if n == 0]
    for b, parents in enumerate(st.parent.tolist()):
        for j, p in enumerate(parents):
            n = lens[b * w + p]
            if p in parents[:j] and n % page:
                to = free.pop(0)
                pool[to, :, :, :, :n % page] = pool[table[b * w + p][n // page], :, :, :, :n % page]
    return {"table": None, "lens": None, "refs": None, "status": None, "pool": pool}


_EXACT = {"append": _exact_append, "attend": _exact_attend, "select": _exact_select, "reorder": _exact_reorder}
