"""The operators of speculative decoding over long contexts in a paged cache, as measurable cases.

Four kinds of call, in the order in which a decoding step makes them:

  rotary   mtp_rotary_append: rotary positions of a step's queries and keys, keys and values into the cache
  weights  mtp_key_weights: the attention weight that each cached key gets from a step's tokens, added up
  verify   mtp_draft_verify: which drafted tokens the target's distribution keeps, and the token after them
  evict    mtp_cache_evict: the keys of largest weight stay, in their order, and pages become free

`own` chooses between the plain form (elementary torch operations in 32 bits, in 64 for angles of far positions
and for sums whose borders decide about a token) and the package.  Sizes are the repository's own (16 heads
of 64, 12 layers, pages of 16 to 128, codec vocabulary 1025, contexts of 180 to 2000 keys, prefill passes of 14592
rows) and, for programs with another model around the same cache, head groups, 128-wide heads, longer contexts
and larger vocabularies.
"""
import math
import random
from types import SimpleNamespace

import torch

own = False

F32, F64, BF16, F16 = torch.float32, torch.float64, torch.bfloat16, torch.float16
TYPES = {"f32": F32, "bf16": BF16, "f16": F16}
INF = float("inf")


def listed():
    return [
        # queries, keys and values of one decoding step of 32 utterances, out of the fused fp32 projection: the smallest
        # call, all latency
        {"name": "rotary step 32", "kind": "rotary", "rows": 32, "heads": 16, "kv_heads": 16, "dim": 64, "rot": 64,
         "layout": "halves", "scaling": "plain", "far": 2000, "page": 64, "src": "f32", "type": "bf16", "fused": True},
        # a prefill pass of 14592 rows
        {"name": "rotary prefill 14592", "kind": "rotary", "rows": 14592, "heads": 16, "kv_heads": 16, "dim": 64,
         "rot": 64, "layout": "halves", "scaling": "linear", "far": 2000, "page": 64, "src": "f32", "type": "bf16",
         "fused": True},
        # a chunk far into a long text, neighbouring pairs, half of every head, frequencies scaled by bands
        {"name": "rotary chunk 3501 at 200k", "kind": "rotary", "rows": 3501, "heads": 32, "kv_heads": 8, "dim": 128,
         "rot": 64, "layout": "pairs", "scaling": "bands", "far": 200000, "page": 16, "src": "f16", "type": "f16",
         "fused": False},
        # one decoding step of 32 utterances of ragged lengths
        {"name": "weights step 32", "kind": "weights", "slots": 32, "new_lo": 1, "new_hi": 1, "ctx_lo": 180,
         "ctx_hi": 2000, "heads": 16, "kv_heads": 16, "dim": 64, "page": 64, "type": "bf16", "window": 0},
        # drafts to verify on long contexts, four query heads to a key head
        {"name": "weights drafts 8 long", "kind": "weights", "slots": 8, "new_lo": 4, "new_hi": 4, "ctx_lo": 4000,
         "ctx_hi": 30000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 16, "type": "f16", "window": 0},
        # two long prompts in chunks
        {"name": "weights chunk 2", "kind": "weights", "slots": 2, "new_lo": 2000, "new_hi": 4000, "ctx_lo": 6000,
         "ctx_hi": 9000, "heads": 32, "kv_heads": 8, "dim": 128, "page": 128, "type": "bf16", "window": 0},
        # the drafts of one step of 32 utterances, single paths of the codec's vocabulary
        {"name": "verify codec 32", "kind": "verify", "slots": 32, "new_lo": 4, "new_hi": 4, "vocab": 1025,
         "type": "f32", "drafter": False, "page": 64},
        # one request with drafts that another model drew
        {"name": "verify 1 x 5 of 32003", "kind": "verify", "slots": 1, "new_lo": 5, "new_hi": 5, "vocab": 32003,
         "type": "f16", "drafter": True, "page": 64},
        # 32 requests with up to 8 drafts each over a large vocabulary
        {"name": "verify 32 of 48001", "kind": "verify", "slots": 32, "new_lo": 1, "new_hi": 9, "vocab": 48001,
         "type": "bf16", "drafter": True, "page": 16},
        # one utterance that has grown past its budget by a page
        {"name": "evict 1", "kind": "evict", "slots": 1, "len_lo": 1088, "len_hi": 1088, "keep": 1024, "sinks": 4,
         "recent": 256, "layers": 12, "kv_heads": 16, "dim": 64, "page": 64, "type": "bf16"},
        # a batch of which some contexts are over their budget, and are halved
        {"name": "evict 16 of 12 layers", "kind": "evict", "slots": 16, "len_lo": 180, "len_hi": 2000, "keep": 700,
         "sinks": 4, "recent": 128, "layers": 12, "kv_heads": 16, "dim": 64, "page": 64, "type": "bf16"},
        # long contexts after their prefill
        {"name": "evict 4 long", "kind": "evict", "slots": 4, "len_lo": 20000, "len_hi": 30000, "keep": 8192,
         "sinks": 64, "recent": 2000, "layers": 4, "kv_heads": 8, "dim": 128, "page": 16, "type": "f16"},
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["rotary", "weights", "weights", "verify", "verify", "evict"])
    page = rng.choice([16, 32, 64, 128])
    if kind == "verify":
        vocab = rng.choice([1025, _log_int(rng, 64, 48001)])
        lo = rng.randint(1, 4)
        return {"kind": kind, "slots": _log_int(rng, 1, 64 if vocab < 9000 else 32), "new_lo": lo,
                "new_hi": min(9, lo + rng.randint(0, 5)), "vocab": vocab, "type": rng.choice(["f32", "bf16", "f16"]),
                "drafter": rng.random() < 0.6, "page": page}
    dim, group = rng.choice([64, 128]), rng.choice([1, 2, 4, 5, 8])
    kv_heads = rng.choice([1, 2, 4, 8] if dim == 128 else [2, 4, 8, 16])
    while kv_heads * group > 32:
        group = rng.choice([1, 2, 4])
        kv_heads = max(1, kv_heads // 2)
    shape = {"heads": kv_heads * group, "kv_heads": kv_heads, "dim": dim, "page": page,
             "type": rng.choice(["bf16", "f16"])}
    if kind == "rotary":
        return {"kind": kind, "rows": _log_int(rng, 1, 14592), **shape,
                "rot": rng.choice([dim, dim, dim // 2, 2 * rng.randint(4, dim // 2)]),
                "layout": rng.choice(["halves", "pairs"]), "scaling": rng.choice(["plain", "linear", "base", "bands"]),
                "far": _log_int(rng, 20, 1000000), "src": rng.choice(["f32", shape["type"]]),
                "fused": rng.random() < 0.7}
    if kind == "weights":
        window = rng.choice([0, 0, 0, rng.randint(100, 2000)])
        form = rng.choice(["step", "drafts", "prompts", "chunk"])
        if form in ("step", "drafts"):
            lo = _log_int(rng, 30, 16000)
            hi = min(32000, lo * rng.randint(1, 3))
            new = 1 if form == "step" else rng.randint(2, 9)
            return {"kind": kind, "slots": _log_int(rng, 1, max(1, min(128, 250000 // hi))), "new_lo": new, "new_hi": new,
                    "ctx_lo": lo, "ctx_hi": hi, **shape, "window": window}
        if form == "prompts":
            return {"kind": kind, "slots": _log_int(rng, 1, 48), "new_lo": rng.randint(20, 200),
                    "new_hi": rng.randint(200, 600), "ctx_lo": 0, "ctx_hi": 0, **shape, "window": window}
        ctx = rng.randint(500, 6000)
        return {"kind": kind, "slots": rng.randint(1, 2), "new_lo": rng.randint(150, 900),
                "new_hi": rng.randint(900, 2900), "ctx_lo": ctx, "ctx_hi": ctx + rng.randint(0, 2000), **shape,
                "window": window}
    hi = _log_int(rng, 40, 20000)
    lo = rng.randint(max(1, hi // 4), hi)
    keep = rng.randint(max(1, lo // 4), hi)
    layers = rng.choice([1, 2, 6, 12])
    while layers > 1 and hi * layers * kv_heads * dim // 64 > 3000000:
        layers //= 2
    slots = _log_int(rng, 1, max(1, min(16, 3000000 * 64 // (hi * layers * kv_heads * dim))))
    return {"kind": kind, "slots": slots, "len_lo": lo, "len_hi": hi, "keep": keep, "sinks": rng.randint(0, min(64, keep)),
            "recent": rng.randint(0, keep // 2), "layers": layers, "kv_heads": kv_heads, "dim": dim, "page": page,
            "type": shape["type"]}


# ---- inputs ----


def _host(case, seed):
    return random.Random("%d %s" % (seed, case["kind"]))


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed((seed * 1000003 + 54321) % (1 << 61))


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
    """Tokens that each slot gets, and its length with them."""
    rng = _host(case, seed)
    new = [rng.randint(case["new_lo"], case["new_hi"]) for _ in range(case["slots"])]
    lo, hi = _context(case)
    return new, [rng.randint(lo, hi) + n for n in new]


def _context(case):
    return (case["ctx_lo"], case["ctx_hi"]) if "ctx_lo" in case else (180, 2000)


def _most_pages(case):
    """Pages that a slot can have: what tables and pools are made for, whatever the lengths are."""
    return -(-(case["len_hi"] if "len_hi" in case else _context(case)[1] + case["new_hi"]) // case["page"])


def prepare(case, seed):
    st = SimpleNamespace(case=case, kind=case["kind"], stream=torch.cuda.current_stream().cuda_stream)
    _PREPARE[case["kind"]](st, case, seed)
    if own:  # a program makes the same step again and again: it keeps its argument blocks and its scratch
        _KEEP[case["kind"]](st)
    return st


# how far apart frequencies are, and how each form of scaling for long contexts changes them
ROTARY = {"base": 10000.0, "factor": 8.0, "context": 8192.0, "low": 1.0, "high": 4.0}


def _frequencies(rot, scaling):
    """Radians per position of each rotated pair."""
    r, base = ROTARY, ROTARY["base"]
    if scaling == "base":  # the slowest pair turns `factor` times slower, the fastest as before
        base *= r["factor"] ** (rot / (rot - 2.0))
    f = base ** (-torch.arange(0, rot, 2, dtype=F64) / rot)
    if scaling == "linear":
        f = f / r["factor"]
    if scaling == "bands":  # pairs that turn less than `low` times in the trained context are slowed down, from `high` on none
        kept = ((r["context"] * f / (2 * math.pi) - r["low"]) / (r["high"] - r["low"])).clamp(0, 1)
        f = kept * f + (1 - kept) * f / r["factor"]
    return f.cuda()


def _prepare_rotary(st, c, seed):
    gen, rows, page = _gen(seed), c["rows"], c["page"]
    h, hk, d = c["heads"], c["kv_heads"], c["dim"]
    src = TYPES[c["src"]]
    if c["fused"]:
        x = _normal(gen, (rows, h + 2 * hk, d), src)
        st.q, st.k, st.v = x[:, :h], x[:, h:h + hk], x[:, h + hk:]
    else:
        st.q = _normal(gen, (rows, h, d), src)
        st.k, st.v = _normal(gen, (rows, hk, d), src), _normal(gen, (rows, hk, d), src)
    n_pages = -(-rows // page) * 2 + 8
    st.layers, st.layer = 2, 1
    st.pool = _normal(gen, (n_pages, 2, 2, hk, page, d), TYPES[c["type"]])
    # runs of positions inside pages, the pages in no order; a decoding step's rows are of utterances of their own
    at = torch.arange(rows, device="cuda")
    order = torch.randperm(n_pages, device="cuda", generator=gen)
    off = int(torch.randint(0, page, (1,), generator=torch.Generator().manual_seed(seed)))
    st.slot_map = order[(at + off) // page] * page + (at + off) % page
    start = torch.randint(0, c["far"], (rows // 200 + 1,), device="cuda", generator=gen)
    st.positions = (start[at // 200] + at % 200).int()
    st.out_q = torch.zeros(rows, h, d, dtype=TYPES[c["type"]], device="cuda")
    st.freq, st.gain = _frequencies(c["rot"], c["scaling"]), 1.1 if c["scaling"] == "bands" else 1.0


def _prepare_weights(st, c, seed):
    gen, page, h, hk, d = _gen(seed), c["page"], c["heads"], c["kv_heads"], c["dim"]
    new, lens = _lengths(c, seed)
    st.rows = sum(new)
    st.max_new, st.max_keys = max(new), max(lens)
    counts = [-(-n // page) for n in lens]
    st.stride = _most_pages(c) + 1
    st.table, _ = _tables(_host(c, seed), counts, sum(counts) + 3, st.stride)
    st.lens, st.layers, st.layer = _ints(lens), 2, 1
    st.cu_rows = _ints([sum(new[:i]) for i in range(len(new) + 1)])
    st.pool = _normal(gen, (sum(counts) + 3, 2, 2, hk, page, d), TYPES[c["type"]])
    st.q = _normal(gen, (st.rows, h, d), TYPES[c["type"]], 2.0)  # scores that spread as a trained model's do
    st.scale = d ** -0.5
    # what earlier steps have given to the keys; the buffer is as wide as the tables
    st.weights = 0.02 * torch.rand((c["slots"], 2, hk, st.stride * page), device="cuda", generator=gen)
    # the log-sum-exps that the step's attention left, slot by slot
    st.lse = torch.empty(st.rows, h, device="cuda")
    for b, (n, length) in enumerate(zip(new, lens)):
        r0 = int(sum(new[:b]))
        s, _ = _scores(st, c, b, r0, n, length, F32)
        st.lse[r0:r0 + n] = torch.logsumexp(s, -1).permute(1, 0, 2).reshape(n, h)


def _scores(st, c, b, r0, n, length, dtype):
    """Scaled products of slot b's rows with its keys, [key head, row, query head of it, key]; and which are seen."""
    pages = st.table[b, :-(-length // c["page"])].long()
    k = st.pool[pages, st.layer, 0].transpose(0, 1).reshape(c["kv_heads"], -1, c["dim"])[:, :length].to(dtype)
    g = c["heads"] // c["kv_heads"]
    q = st.q[r0:r0 + n].to(dtype).view(n, c["kv_heads"], g, c["dim"]).transpose(0, 1)
    s = torch.matmul(q.reshape(c["kv_heads"], n * g, c["dim"]), k.transpose(1, 2)).view(c["kv_heads"], n, g, length) * st.scale
    t = torch.arange(length, device="cuda")
    pos = (length - n + torch.arange(n, device="cuda"))[:, None]
    sees = t <= pos
    if c["window"]:
        sees &= t > pos - c["window"]
    return s.masked_fill_(~sees[:, None], -INF), sees


def _prepare_verify(st, c, seed):
    gen, v = _gen(seed), c["vocab"]
    new, lens = _lengths(c, seed)
    rows, page = sum(new), c["page"]
    st.max_new, st.eos = c["new_hi"], v - 1
    x = 2.0 * torch.randn(rows, v, device="cuda", generator=gen)
    x += 2.0 * torch.randn(1, v, device="cuda", generator=gen)  # some tokens are likely everywhere
    st.logits = x.to(TYPES[c["type"]])
    st.temperature = torch.tensor([0.0, 0.7, 1.0], device="cuda")[
        torch.randint(0, 3, (c["slots"],), device="cuda", generator=gen)]
    slot = torch.repeat_interleave(torch.arange(c["slots"], device="cuda"), _ints(new).long())
    st.cu_rows, st.lens = _ints([sum(new[:i]) for i in range(len(new) + 1)]), _ints(lens)
    # a drafter that is near the target; its drafts are drawn from it, or are its best
    y = (x + 0.8 * torch.randn(rows, v, device="cuda", generator=gen)).to(TYPES[c["type"]])
    st.draft = y if c["drafter"] else None
    noise = -torch.log(-torch.log(torch.rand(rows, v, device="cuda", generator=gen).clamp(1e-7, 1 - 1e-6)))
    drawn = (y.float() + (st.temperature[slot][:, None] * noise if c["drafter"] else 0)).argmax(-1).int()
    st.tokens = torch.cat([drawn[:1] * 0, drawn[:-1]])  # the token fed at a row was drafted at the row before it
    st.uniforms = torch.rand(rows, 2, device="cuda", generator=gen)
    counts = [-(-n // page) for n in lens]
    st.table, st.refs = _tables(_host(c, seed), counts, c["slots"] * _most_pages(c), _most_pages(c) + 1)
    i32 = dict(dtype=torch.int32, device="cuda")
    st.out_tokens, st.counts = torch.empty(c["slots"], st.max_new, **i32), torch.empty(c["slots"], **i32)
    st.out_lens, st.done = torch.empty(c["slots"], **i32), torch.empty(c["slots"], **i32)


def _prepare_evict(st, c, seed):
    rng, gen, page = _host(c, seed), _gen(seed), c["page"]
    lens = [rng.randint(c["len_lo"], c["len_hi"]) for _ in range(c["slots"])]
    lens[rng.randrange(len(lens))] = c["len_hi"]
    counts = [-(-n // page) for n in lens]
    st.stride, n_pages = _most_pages(c) + 1, c["slots"] * _most_pages(c)
    st.table, st.refs = _tables(rng, counts, n_pages, st.stride)
    st.lens, st.keep = _ints(lens), _ints([c["keep"]] * len(lens))
    # a few keys have most of the weight, many almost the same, and some none at all
    w = torch.randn((c["slots"], c["layers"], c["kv_heads"], st.stride * page), device="cuda", generator=gen)
    st.weights = torch.where(w < -1.2, torch.zeros_like(w), (2.0 * w).exp())
    st.pool = torch.empty((n_pages, c["layers"], 2, c["kv_heads"], page, c["dim"]), dtype=TYPES[c["type"]],
                          device="cuda").normal_(generator=gen)
    st.out_table, st.out_lens = torch.empty_like(st.table), torch.empty_like(st.lens)
    st.out_refs, st.out_weights = torch.empty_like(st.refs), torch.zeros_like(st.weights)
    st.status = torch.empty_like(st.lens)


_PREPARE = {"rotary": _prepare_rotary, "weights": _prepare_weights, "verify": _prepare_verify, "evict": _prepare_evict}


# ---- the package's operators ----


def _scratch(nbytes):
    return torch.zeros(max(16, nbytes), dtype=torch.uint8, device="cuda"), nbytes


def _keep_rotary(st):
    from paper_2410_13839_gb300 import mtp
    c, r = st.case, ROTARY
    layout = {"halves": mtp.MTP_ROTARY_HALVES, "pairs": mtp.MTP_ROTARY_PAIRS}[c["layout"]]
    scaling = {"plain": mtp.MTP_ROTARY_PLAIN, "linear": mtp.MTP_ROTARY_LINEAR, "base": mtp.MTP_ROTARY_BASE,
               "bands": mtp.MTP_ROTARY_BANDS}[c["scaling"]]
    st.turns = mtp.mtp_rotary_turns(c["rot"], base=r["base"], scaling=scaling, factor=r["factor"], context=r["context"],
                                    low=r["low"], high=r["high"])
    st.mtp, st.args = mtp, mtp.rotary_append_args(
        q=st.q, k=st.k, v=st.v, positions=st.positions, slot_map=st.slot_map, turns=st.turns, kv_pool=st.pool,
        layer=st.layer, out_q=st.out_q, layout=layout, gain=st.gain)


def _keep_weights(st):
    from paper_2410_13839_gb300 import mtp
    st.mtp, st.args = mtp, mtp.key_weights_args(
        q=st.q, kv_pool=st.pool, layer=st.layer, block_table=st.table, cu_rows=st.cu_rows, kv_lens=st.lens, lse=st.lse,
        weights=st.weights, scale=st.scale, window=st.case["window"], max_new=st.max_new, max_keys=st.max_keys)
    st.scratch = _scratch(mtp.mtp_key_weights_workspace_bytes(st.args))


def _keep_verify(st):
    from paper_2410_13839_gb300 import mtp
    st.mtp, st.args = mtp, mtp.draft_verify_args(
        logits=st.logits, tokens=st.tokens, uniforms=st.uniforms, cu_rows=st.cu_rows, kv_lens=st.lens,
        out_tokens=st.out_tokens, out_counts=st.counts, out_kv_lens=st.out_lens, max_new=st.max_new,
        draft_logits=st.draft, temperature=st.temperature, eos_id=st.eos, out_done=st.done, block_table=st.table,
        page_refs=st.refs, page_size=st.case["page"])


def _keep_evict(st):
    from paper_2410_13839_gb300 import mtp
    c = st.case
    st.mtp, st.args = mtp, mtp.cache_evict_args(
        kv_lens=st.lens, keep=st.keep, block_table=st.table, page_refs=st.refs, weights=st.weights, kv_pool=st.pool,
        out_kv_lens=st.out_lens, out_block_table=st.out_table, out_page_refs=st.out_refs, out_weights=st.out_weights,
        out_status=st.status, sinks=c["sinks"], recent=c["recent"])
    st.scratch = _scratch(mtp.mtp_cache_evict_workspace_bytes(st.args))


_KEEP = {"rotary": _keep_rotary, "weights": _keep_weights, "verify": _keep_verify, "evict": _keep_evict}


def run(st):
    return (_OWN if own else _PLAIN)[st.kind](st)


def _own_rotary(st):
    st.mtp.mtp_rotary_append(st.args, st.stream)
    return {"q": st.out_q, "pool": st.pool}


def _own_weights(st):
    st.mtp.mtp_key_weights(st.args, st.scratch[0], st.scratch[1], st.stream)
    return {"weights": st.weights}


def _own_verify(st):
    st.mtp.mtp_draft_verify(st.args, st.stream)
    return {"tokens": st.out_tokens, "counts": st.counts, "lens": st.out_lens, "done": st.done, "table": st.table,
            "refs": st.refs}


def _own_evict(st):
    st.mtp.mtp_cache_evict(st.args, st.scratch[0], st.scratch[1], st.stream)
    return {"lens": st.out_lens, "table": st.out_table, "refs": st.out_refs, "weights": st.out_weights,
            "status": st.status, "pool": st.pool}


_OWN = {"rotary": _own_rotary, "weights": _own_weights, "verify": _own_verify, "evict": _own_evict}


# ---- the plain forms ----


def _plain_rotary(st):
    c, rot, page = st.case, st.case["rot"], st.case["page"]
    angle = st.positions.double()[:, None] * st.freq
    cos, sin = (st.gain * angle.cos()).float()[:, None], (st.gain * angle.sin()).float()[:, None]

    def turn(x):
        x = x.float()
        if c["layout"] == "halves":
            a, b = x[..., :rot // 2], x[..., rot // 2:rot]
            return torch.cat([a * cos - b * sin, a * sin + b * cos, x[..., rot:]], -1)
        a, b = x[..., 0:rot:2], x[..., 1:rot:2]
        return torch.cat([torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2), x[..., rot:]], -1)
    st.out_q.copy_(turn(st.q))
    at = st.slot_map
    st.pool[at // page, st.layer, 0, :, at % page] = turn(st.k).to(st.pool.dtype)
    st.pool[at // page, st.layer, 1, :, at % page] = st.v.to(st.pool.dtype)
    return {"q": st.out_q, "pool": st.pool}


def _plain_weights(st):
    c = st.case
    page, h, hk, d = c["page"], c["heads"], c["kv_heads"], c["dim"]
    slots, new, lens = st.lens.numel(), st.cu_rows.long().diff(), st.lens.long()
    key = torch.arange(st.max_keys, device="cuda")
    pages = st.table[:, key // page].long().clamp(min=0)
    k = st.pool[pages, st.layer, 0, :, key % page].float()  # [slots, keys, kv heads, dim]
    i = torch.arange(st.max_new, device="cuda")
    row = (st.cu_rows[:-1].long()[:, None] + i).clamp(max=st.rows - 1)
    q = st.q[row].float().reshape(slots, st.max_new, hk, h // hk, d).permute(0, 2, 3, 1, 4)
    lse = st.lse[row].reshape(slots, st.max_new, hk, h // hk).permute(0, 2, 3, 1)
    s = torch.matmul(q.reshape(slots, hk, -1, d), k.permute(0, 2, 3, 1)) * st.scale
    s = s.view(slots, hk, h // hk, st.max_new, st.max_keys)
    pos = (lens - new)[:, None] + i
    hidden = (key > pos[:, :, None]) | (i >= new[:, None])[:, :, None]
    if c["window"]:
        hidden |= key <= pos[:, :, None] - c["window"]
    p = s.sub_(lse[..., None]).exp_().masked_fill_(hidden[:, None, None], 0.0)
    got = p.sum((2, 3))
    before = st.weights[:, st.layer, :, :st.max_keys]
    # the keys of the step's own tokens begin at nothing
    total = torch.where(key >= (lens - new)[:, None, None], got, before + got)
    st.weights[:, st.layer, :, :st.max_keys] = torch.where(key < lens[:, None, None], total, before)
    return {"weights": st.weights}


def _plain_verify(st):
    v, page = st.case["vocab"], st.case["page"]
    slots, new, lens = st.lens.numel(), st.cu_rows.long().diff(), st.lens.long()
    i = torch.arange(st.max_new, device="cuda")
    row = (st.cu_rows[:-1].long()[:, None] + i).clamp(max=st.logits.shape[0] - 1)
    t = st.temperature.double()[:, None, None]
    greedy = t <= 0
    number = torch.arange(v, device="cuda")

    def shares(x):
        x = x[row].double()
        top = x.amax(-1, keepdim=True)
        e = ((x - top) / torch.where(greedy, 1.0, t)).exp()
        best = torch.where(x == top, number, v).amin(-1, keepdim=True)
        return torch.where(greedy, (number == best).double(), e / e.sum(-1, keepdim=True))
    p = shares(st.logits)
    drafted = st.tokens[(row + 1).clamp(max=st.logits.shape[0] - 1)].long()
    if st.draft is None:
        q = (number == drafted[..., None]).double()
    else:
        q = shares(st.draft)
    at = drafted[..., None]
    u = st.uniforms[row].double()
    pd, qd = p.gather(-1, at)[..., 0], q.gather(-1, at)[..., 0]
    keeps = torch.where(greedy[..., 0], pd > 0, u[..., 0] * qd < pd) & (i < (new - 1)[:, None])
    kept = keeps.long().cumprod(-1).sum(-1)
    # a kept draft that ends the text is the last
    ends = (drafted == st.eos) & (i < kept[:, None])
    cut = ends.any(-1)
    kept = torch.where(cut, ends.long().argmax(-1) + 1, kept)
    last = kept.clamp(max=st.max_new - 1)[:, None, None].expand(slots, 1, v)
    pr, qr = p.gather(1, last)[:, 0], q.gather(1, last)[:, 0]
    w = torch.where((greedy[:, 0] | (kept >= new - 1)[:, None]), pr, (pr - qr).clamp(min=0))
    w = torch.where(w.sum(-1, keepdim=True) > 0, w, pr)
    before = w.cumsum(-1)
    draw = u[..., 1].gather(1, last[:, :, 0])
    token = (before <= draw * before[:, -1:]).sum(-1)
    token = torch.minimum(token, torch.where(w > 0, number, 0).amax(-1))
    counts = torch.where(cut, kept, kept + 1)
    out = torch.where(i < kept[:, None], drafted, torch.where((i == kept[:, None]) & ~cut[:, None], token[:, None], -1))
    after = lens - (new - 1 - kept)
    col = torch.arange(st.table.shape[1], device="cuda")
    gone = (col >= ((after + page - 1) // page)[:, None]) & (col < ((lens + page - 1) // page)[:, None]) & (st.table >= 0)
    count = torch.zeros(st.refs.numel() + 1, dtype=torch.int32, device="cuda")
    count.index_add_(0, torch.where(gone, st.table, st.refs.numel()).view(-1).long(), torch.ones_like(st.table).view(-1))
    st.refs -= count[:-1]
    st.table.masked_fill_(gone, -1)
    return {"tokens": out.int(), "counts": counts.int(), "lens": after.int(),
            "done": (cut | (token == st.eos)).int(), "table": st.table, "refs": st.refs}


def _plain_evict(st):
    c, page = st.case, st.case["page"]
    lens = st.lens.long()
    after = torch.minimum(lens, st.keep.long())
    n = st.stride * page
    key = torch.arange(n, device="cuda")
    inside = key < lens[:, None]
    sinks = torch.minimum(after, torch.full_like(after, c["sinks"]))
    recent = torch.minimum(after - sinks, torch.full_like(after, c["recent"]))
    # first the keys that stay whatever their weight, then by weight, then those that do not exist; equal ones in their order
    forced = (key < sinks[:, None]) | (key >= (lens - recent)[:, None])
    rank = torch.where(inside, torch.where(forced, 0, 1), 2)[:, None, None].expand_as(st.weights)
    order = torch.sort(st.weights, dim=-1, descending=True, stable=True)[1]
    order = order.gather(-1, torch.sort(rank.gather(-1, order), dim=-1, stable=True)[1])
    most = int(min(c["keep"], c["len_hi"]))
    place = torch.arange(most, device="cuda")
    there = (place < after[:, None])[:, None, None].expand(*st.weights.shape[:3], most)
    kept = torch.sort(torch.where(there, order[..., :most], n), dim=-1)[0].clamp(max=n - 1)
    st.out_weights[..., :most] = torch.where(there, st.weights.gather(-1, kept), st.out_weights[..., :most])
    # slots that stay as they are keep all of their weights
    st.out_weights.copy_(torch.where((inside & (after == lens)[:, None])[:, None, None], st.weights, st.out_weights))
    moves = (there & (after < lens)[:, None, None, None]).nonzero(as_tuple=True)
    s, layer, head, to = moves
    old, now = kept[moves], to
    fp, tp = st.table[s, old // page].long(), st.table[s, now // page].long()
    st.pool[tp, layer, :, head, now % page] = st.pool[fp, layer, :, head, old % page]
    col = torch.arange(st.stride, device="cuda")
    held, left = (col < ((x + page - 1) // page)[:, None] for x in (lens, after))
    count = torch.zeros(st.refs.numel() + 1, dtype=torch.int32, device="cuda")
    count.index_add_(0, torch.where(held & ~left, st.table, st.refs.numel()).view(-1).long(),
                     torch.ones_like(st.table).view(-1))
    return {"lens": after.int(), "table": torch.where(left, st.table, -1), "refs": st.refs - count[:-1],
            "weights": st.out_weights, "status": torch.zeros_like(st.lens), "pool": st.pool}


_PLAIN = {"rotary": _plain_rotary, "weights": _plain_weights, "verify": _plain_verify, "evict": _plain_evict}


# ---- what a pass cannot do without ----


def _seen(new, length, window):
    """Keys that a slot's new rows see, summed, and the cached keys that any of them sees."""
    first = length - new + 1
    if not window:
        return new * first + new * (new - 1) // 2, length
    return sum(min(window, first + i) for i in range(new)), min(length, window + new - 1)


def work(case):
    c, kind = case, case["kind"]
    size = 2 if c["type"] in ("bf16", "f16") else 4
    if kind == "rotary":
        n = c["rows"] * (c["heads"] + 2 * c["kv_heads"]) * c["dim"]
        return {"bytes": n * (size + (4 if c["src"] == "f32" else 2)) + c["rows"] * 12, "flops": 0}
    if kind == "weights":
        new, lens = _lengths(c, 1)
        pairs, keys = (sum(x) for x in zip(*(_seen(n, t, c["window"]) for n, t in zip(new, lens))))
        rows = sum(new) * c["heads"]
        # keys, queries, log-sum-exps; the keys' weights are read and written
        return {"bytes": (keys * c["kv_heads"] + rows) * c["dim"] * size + rows * 4 + keys * c["kv_heads"] * 8,
                "flops": 2 * pairs * c["heads"] * c["dim"]}
    if kind == "verify":
        new, _ = _lengths(c, 1)
        # of the drafter's last row nothing is needed
        rows = sum(new) + (sum(new) - len(new) if c["drafter"] else 0)
        return {"bytes": rows * c["vocab"] * size + sum(new) * 12, "flops": 0}
    rng = _host(c, 1)
    lens = [rng.randint(c["len_lo"], c["len_hi"]) for _ in range(c["slots"])]
    moved = sum(max(0, c["keep"] - c["sinks"]) for n in lens if n > c["keep"])
    heads = c["layers"] * c["kv_heads"]
    # the weights, and the kept ones; the keys and values behind the first that goes are read and written
    return {"bytes": (sum(lens) + sum(min(n, c["keep"]) for n in lens)) * heads * 4 + moved * heads * c["dim"] * size * 4,
            "flops": 0}


# ---- the definition in 64 bits ----


def exact(case, seed):
    kind = case["kind"]
    if kind == "verify":
        return None  # whole numbers only
    st = SimpleNamespace(case=case)
    _PREPARE[kind](st, case, seed)
    return _EXACT[kind](st, case)


def _exact_rotary(st, c):
    """Pairs as complex numbers, turned by the angle's point on the unit circle."""
    page, rot = c["page"], c["rot"]
    unit = st.gain * torch.polar(torch.ones_like(st.freq), st.positions.double()[:, None] * st.freq)[:, None]

    def turn(x):
        x = x.double().clone()
        first, second = (slice(0, rot // 2), slice(rot // 2, rot)) if c["layout"] == "halves" else (
            slice(0, rot, 2), slice(1, rot, 2))
        z = torch.complex(x[..., first], x[..., second]) * unit
        x[..., first], x[..., second] = z.real, z.imag
        return x
    k, v, pool, at = turn(st.k), st.v.double(), st.pool.double(), st.slot_map
    for half, x in enumerate((k, v)):
        pool[at // page, st.layer, half, :, at % page] = x
    return {"q": turn(st.q), "pool": pool}


def _exact_weights(st, c):
    """Slot by slot, a block of rows at a time."""
    total = st.weights.double()
    cu, g = st.cu_rows.tolist(), c["heads"] // c["kv_heads"]
    for b, length in enumerate(st.lens.tolist()):
        n = cu[b + 1] - cu[b]
        total[b, st.layer, :, length - n:length] = 0
        pages = st.table[b, :-(-length // c["page"])].long()
        k = st.pool[pages, st.layer, 0].transpose(0, 1).reshape(c["kv_heads"], -1, c["dim"])[:, :length].double()
        t = torch.arange(length, device="cuda")
        for r0 in range(cu[b], cu[b + 1], 512):
            r1 = min(cu[b + 1], r0 + 512)
            pos = length - cu[b + 1] + torch.arange(r0, r1, device="cuda")
            sees = t <= pos[:, None]
            if c["window"]:
                sees &= t > pos[:, None] - c["window"]
            q = st.q[r0:r1].double().view(r1 - r0, c["kv_heads"], g, c["dim"])
            s = torch.einsum("rhgd,htd->hrgt", q, k) * st.scale
            s -= st.lse[r0:r1].double().view(r1 - r0, c["kv_heads"], g).transpose(0, 1)[..., None]
            total[b, st.layer, :, :length] += s.exp().mul_(sees[:, None]).sum((1, 2))
    return {"weights": total}


def _exact_evict(st, c):
    """Only copies, slot by slot and head by head."""
    page, pool, out = c["page"], st.pool.double(), st.out_weights.double()
    for b, length in enumerate(st.lens.tolist()):
        keep = min(length, c["keep"])
        w = st.weights[b].flatten(0, 1)[:, :length].double()
        if keep == length:
            out[b, ..., :length] = st.weights[b, ..., :length].double()
            continue
        w[:, :c["sinks"]] = INF
        if c["recent"]:
            w[:, max(0, length - min(c["recent"], keep - min(keep, c["sinks"]))):] = INF
        kept = torch.argsort(-w, dim=-1, stable=True)[:, :keep].sort(-1)[0]
        out[b, ..., :keep] = st.weights[b].flatten(0, 1).double().gather(-1, kept).view(c["layers"], -1, keep)
        table, to = st.table[b].long(), torch.arange(keep, device="cuda")
        for row, old in enumerate(kept):
            layer, head = divmod(row, c["kv_heads"])
            pool[table[to // page], layer, :, head, to % page] = st.pool[table[old // page], layer, :, head, old % page].double()
    return {"lens": None, "table": None, "refs": None, "weights": out, "status": None, "pool": pool}


_EXACT = {"rotary": _exact_rotary, "weights": _exact_weights, "evict": _exact_evict}
