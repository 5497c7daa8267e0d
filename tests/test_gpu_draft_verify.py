"""mtp_draft_verify against the rule in 64 bits, one slot at a time: whole numbers, all equal.

The kernel's sums are exact to about 2^-36 of the whole, numpy's to 2^-50; a number in [0, 1) that falls between the two
is met with a chance of 2^-35 per border between tokens, below one in a million for all cases here together."""
import numpy as np
import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu

HUGE = float(np.float32(1e38))


def _tame(x):
    return np.clip(np.where(np.isnan(x), -HUGE, x), -HUGE, HUGE)


def _unit(u):
    return min(float(u), 1.0) if u > 0 else 0.0


def _shares(x, t):
    x = _tame(x)
    if not t > 0:
        p = np.zeros(len(x))
        p[np.argmax(x)] = 1.0
        return p
    e = np.exp((x - x.max()) / min(max(float(t), 1e-30), 1e30))
    return e / e.sum()


def _oracle(c):
    """(tokens, counts, lens, done, table, refs) as lists."""
    slots, max_new, v, page = len(c["new"]), c["max_new"], c["logits"].shape[1], c["page"]
    out = [[-1] * max_new for _ in range(slots)]
    counts, lens, done = [0] * slots, list(c["lens"]), [0] * slots
    table, refs = [list(r) for r in c["table"]], list(c["refs"])
    row = 0
    for s, n in enumerate(c["new"]):
        if n == 0:
            continue
        t = c["temperature"][s] if c["temperature"] is not None else 1.0
        kept, cut, drafts = 0, False, c["tokens"][row + 1:row + n]
        p, q = None, None
        for i in range(n):
            p = _shares(c["logits"][row + i], t)
            if i == n - 1:
                break
            d = drafts[i]
            if c["draft"] is not None:
                q = _shares(c["draft"][row + i], t)
            else:
                q = np.zeros(v)
                if 0 <= d < v:
                    q[d] = 1.0
            ok = 0 <= d < v and (p[d] > 0 if not t > 0 else _unit(c["uniforms"][row + i][0]) * q[d] < p[d])
            if not ok:
                break
            kept += 1
            if d == c["eos"]:
                cut = True
                break
        out[s][:kept] = drafts[:kept]
        if not cut:
            w = p if kept == n - 1 or not t > 0 else np.maximum(p - q, 0)
            if not w.sum() > 0:
                w = p
            u = _unit(c["uniforms"][row + kept][1])
            cum = np.cumsum(w)
            token = int(np.searchsorted(cum, u * cum[-1], side="right"))
            out[s][kept] = min(token, int(np.flatnonzero(w)[-1]))
            done[s] = int(out[s][kept] == c["eos"])
        else:
            done[s] = 1
        counts[s] = kept + (not cut)
        lens[s] = c["lens"][s] - (n - 1 - kept)
        for col in range(-(-lens[s] // page), -(-c["lens"][s] // page)):
            if table[s][col] >= 0:
                if table[s][col] < len(refs):
                    refs[table[s][col]] -= 1
                table[s][col] = -1
        row += n
    return out, counts, lens, done, table, refs


def _case(seed, new, vocab, dtype, drafter, temps, page=16, near=0.5, eos=None):
    """Logits of random rows, a drafter near them, drafts from it, in numpy as the values that the types hold."""
    import torch
    rng = np.random.default_rng(seed)
    rows = sum(new)

    def held(x):
        return torch.from_numpy(x).to(getattr(torch, dtype)).double().numpy()
    x = held(rng.normal(0, 2, (rows, vocab)))
    y = held(x + rng.normal(0, near, (rows, vocab)))
    temperature = None if temps is None else [float(np.float32(temps[i % len(temps)])) for i in range(len(new))]
    tokens, row = [0] * rows, 0
    for s, n in enumerate(new):
        t = 1.0 if temperature is None else temperature[s]
        for i in range(n - 1):
            tokens[row + i + 1] = int(rng.choice(vocab, p=_shares(y[row + i], t)))
        row += n
    lens = [n + int(rng.integers(0, 90)) for n in new]
    counts = [-(-n // page) for n in lens]
    stride = max(counts) + 2
    n_pages = sum(counts) + 2
    order = iter(rng.permutation(n_pages).tolist())
    table = [[next(order) for _ in range(k)] + [-1] * (stride - k) for k in counts]
    refs = [0] * n_pages
    for r in table:
        for p in r:
            if p >= 0:
                refs[p] += 1 + int(rng.integers(0, 2))
    return dict(new=list(new), logits=x, draft=y if drafter else None, temperature=temperature, tokens=tokens,
                uniforms=rng.random((rows, 2), dtype=np.float32).tolist(), lens=lens, table=table, refs=refs, page=page,
                max_new=max(max(new), 1) + 1, eos=vocab - 1 if eos is None else eos, dtype=dtype)


def _args(torch, mtp, c, pad=0, paged=True, in_place=False):
    """The call's arguments, and its outputs."""
    dt = getattr(torch, c["dtype"])

    def put(x):
        buf = torch.zeros(x.shape[0], x.shape[1] + pad, dtype=dt, device="cuda")
        buf[:, :x.shape[1]] = torch.from_numpy(x).to(dt).cuda()
        return buf[:, :x.shape[1]]

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    slots = len(c["new"])
    cu = [sum(c["new"][:i]) for i in range(slots + 1)]
    o = dict(tokens=torch.full((slots, c["max_new"]), 7, dtype=torch.int32, device="cuda"), counts=ints([7] * slots), lens=ints([7] * slots),
             done=ints([7] * slots), table=ints(c["table"]), refs=ints(c["refs"]), err=ints([0]))
    lens = ints(c["lens"])
    if in_place:
        o["lens"] = lens
    keep = [put(c["logits"]), None if c["draft"] is None else put(c["draft"]), ints(c["tokens"]), ints(cu), lens,
            torch.tensor(c["uniforms"], dtype=torch.float32, device="cuda").view(-1, 2),
            None if c["temperature"] is None else torch.tensor(c["temperature"], dtype=torch.float32, device="cuda")]
    args = mtp.draft_verify_args(
        logits=keep[0], draft_logits=keep[1], tokens=keep[2], cu_rows=keep[3], kv_lens=lens, uniforms=keep[5],
        temperature=keep[6], out_tokens=o["tokens"], out_counts=o["counts"], out_kv_lens=o["lens"], out_done=o["done"],
        max_new=c["max_new"], eos_id=c["eos"], block_table=o["table"] if paged else None,
        page_refs=o["refs"] if paged else None, page_size=c["page"] if paged else 0, err_word=o["err"])
    return args, o, keep


def _got(o):
    return tuple(o[k].tolist() for k in ("tokens", "counts", "lens", "done", "table", "refs"))


def _check(c, **kw):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    args, o, keep = _args(torch, mtp, c, **kw)
    mtp.mtp_draft_verify(args, torch.cuda.current_stream())
    want = _oracle(c)
    for name, a, b in zip(("tokens", "counts", "lens", "done", "table", "refs"), _got(o), want):
        assert a == b, name
    assert int(o["err"]) == 0
    return want


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("drafter", [False, True])
@pytest.mark.parametrize("new,vocab,pad,temps", [
    ([1], 1, 0, None), ([3, 1, 4], 2, 1, [0.7, 0.0]), ([2, 0, 5, 1], 7, 0, [1.0]), ([4] * 40, 255, 0, [0.0, 0.7, 1.0]),
    ([5, 9, 1, 2], 256, 8, [0.3, 2.0]), ([4, 4, 3], 257, 0, None), ([4] * 33, 1025, 0, [0.0, 0.7, 1.0]),
    ([3] * 200, 1025, 7, [0.7]), ([5], 32003, 0, [1.0]), ([2, 7, 3], 8191, 0, [1.5, 0.5]), ([64, 30], 3001, 1, [1.0, 0.0]),
    ([2, 3], 131071, 0, [1.0, 5.0]), ([3, 2], 48001, 3, [0.9])])
def test_drafts_are_kept_and_a_token_is_drawn(dtype, drafter, new, vocab, pad, temps):
    c = _case(len(new) * 1000 + vocab, new, vocab, dtype, drafter, temps)
    c["max_new"] = min(64, c["max_new"])
    want = _check(c, pad=pad)
    if len(new) >= 33 and temps == [0.0, 0.7, 1.0]:  # the case has drafts of every fate
        kept = {k - 1 for k in want[1]}
        assert 0 in kept and max(kept) == max(new) - 1


def test_many_slots_take_one_cta_each():
    _check(_case(5, [2] * 700, 300, "bfloat16", True, [1.0, 0.0]))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("slots,new,vocab", [(160, 1, 8193), (160, 2, 8192), (153, 2, 9001), (40, 2, 9001), (17, 3, 9001), (14, 3, 9001), (9, 2, 40001),
                                             (8, 2, 33001), (7, 3, 33001), (76, 2, 4100), (77, 2, 4100)])
def test_slots_at_the_bounds_of_the_launches_forms(dtype, slots, new, vocab):
    _check(_case(slots + vocab, [new] * slots, vocab, dtype, slots % 2 == 0, [0.8, 0.0, 1.2]), pad=slots % 3)


def test_the_end_cuts():
    """eos among the drafts: kept, and nothing after it; eos drawn: done."""
    c = _case(9, [5, 5, 3, 1], 40, "float32", False, [0.0], eos=11)
    for row in range(14):
        c["logits"][row, (row * 7) % 40] = 30.0  # the likeliest token of every row
    best = [(r * 7) % 40 for r in range(14)]
    for s, r0 in enumerate((0, 5, 10)):
        for i in range(c["new"][s] - 1):
            c["tokens"][r0 + i + 1] = best[r0 + i]
    c["logits"][2, :], c["logits"][2, 11] = 0.0, 30.0
    c["tokens"][3] = 11  # slot 0: the third draft ends it
    c["logits"][13, :], c["logits"][13, 11] = 0.0, 30.0  # slot 3: the end is drawn
    want = _check(c)
    assert want[1] == [3, 5, 3, 1] and want[3] == [1, 0, 0, 1] and want[0][0][:3][2] == 11


def test_no_end_and_no_tables():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = _case(10, [3, 4], 100, "float16", True, [1.0])
    c["eos"] = -1
    args, o, keep = _args(torch, mtp, c, paged=False, in_place=True)
    args.out_done = None
    mtp.mtp_draft_verify(args)
    want = _oracle(c)
    assert _got(o)[:3] == want[:3] and o["done"].tolist() == [7, 7]
    assert o["table"].tolist() == c["table"] and o["refs"].tolist() == c["refs"]


@pytest.mark.parametrize("drafter", [False, True])
def test_numbers_at_their_limits(drafter):
    """0, the largest below 1, 1 and beyond, NaN; drafts as likely as the target has them, to the last bit."""
    values = [0.0, 1.0 - 2.0 ** -24, 1.0, 5.0, -3.0, float("nan"), 2.0 ** -24, 0.5]
    c = _case(12, [2] * 64, 50, "float32", drafter, [1.0])
    for r in range(128):
        c["uniforms"][r] = [values[(r // 2) % 8] if r % 2 == 0 else 0.5, values[(r // 16) % 8]]
    if drafter:
        c["draft"][:] = c["logits"]  # u q(d) < p(d) is u < 1, exactly
    _check(c)


def test_near_comparisons_are_made_in_64_bits():
    """Numbers a few 2^-24 to either side of p / q: fp32 sums cannot tell them apart."""
    c = _case(13, [2] * 96, 3000, "float32", True, [1.0], near=1.0)
    for s in range(96):
        r, d = 2 * s, c["tokens"][2 * s + 1]
        p, q = _shares(c["logits"][r], 1.0)[d], _shares(c["draft"][r], 1.0)[d]
        ratio = np.float32(min(p / q, 0.99))
        for _ in range(abs(s % 7 - 3)):
            ratio = np.nextafter(ratio, np.float32(2.0 if s % 7 > 3 else 0.0))
        c["uniforms"][r][0] = float(ratio)
    want = _check(c)
    assert 10 < sum(k == 2 for k in want[1]) < 90


def test_logits_that_are_not_finite():
    inf, nan = float("inf"), float("nan")
    for dtype in ("float32", "bfloat16", "float16"):
        for drafter in (False, True):
            c = _case(14, [3] * 12, 600, dtype, drafter, [1.0, 0.0, 0.4])
            for r in range(0, 36, 2):
                c["logits"][r, ::3] = -inf
                c["logits"][r, 5:9] = nan
            c["logits"][4, :] = -inf      # a row of nothing: all tokens alike
            c["logits"][10, 300:303] = inf
            c["logits"][13, :] = nan
            c["logits"][17, :] = -inf
            c["logits"][17, 599] = 1.0
            if drafter:
                c["draft"][1, 7] = inf
                c["draft"][6, :] = -inf
                c["draft"][18, 100:] = nan
            _check(c)


def test_extreme_temperatures_and_logits():
    c = _case(15, [3] * 10, 500, "float32", True, [1e-3, 1e-38, 1e38, float("inf"), float("nan"), -1.0, 0.0, 30.0, 1e-6, 0.01])
    c["logits"][::2] *= 1e4
    c["draft"][::2] *= 1e4
    c["logits"][3] += 1e10
    c["logits"][5] = 3e38
    c["logits"], c["draft"] = (x.astype(np.float32).astype(np.float64) for x in (c["logits"], c["draft"]))
    for i in range(10):  # no draft of these is a matter of 64 bits
        c["uniforms"][3 * i][0] = c["uniforms"][3 * i + 1][0] = 0.5
    _check(c)


def test_drafts_outside_the_vocabulary():
    for drafter in (False, True):
        c = _case(16, [3] * 6, 90, "float32", drafter, [1.0, 0.0])
        for s, bad in enumerate((-1, 90, 2 ** 31 - 1, -2 ** 31, 89, 0)):
            c["tokens"][3 * s + 1 + s % 2] = bad
        _check(c)


def test_slots_that_do_not_fit_stay_as_they_are_and_are_reported():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    for what in ("rows", "max_new", "length", "table", "order"):
        c = _case(17, [3, 4, 2], 70, "bfloat16", True, [1.0])
        want = _oracle(c)
        args, o, keep = _args(torch, mtp, c)
        cu, lens = keep[3], keep[4]
        if what == "rows":
            cu[3], bad = 10, {2}
        elif what == "max_new":
            args.max_new, bad = 3, {1}
            o["tokens"] = o["tokens"].flatten()[:9].view(3, 3)
        elif what == "length":
            lens[0], bad = 2, {0}
        elif what == "table":
            lens[1], bad = c["page"] * len(c["table"][0]) + 1, {1}
        else:
            cu[2], bad = 2, {1, 2}
            args.max_new = 5
        given = lens.tolist()
        mtp.mtp_draft_verify(args)
        assert int(o["err"]) == 2, what
        for s in range(3):
            if s not in bad:
                k = min(args.max_new, c["max_new"])
                assert o["tokens"][s, :k].tolist() == want[0][s][:k] and int(o["lens"][s]) == want[2][s], what
                assert o["table"][s].tolist() == want[4][s], what
            elif what != "order":
                assert set(o["tokens"][s].tolist()) == {-1} and int(o["counts"][s]) == 0 and int(o["done"][s]) == 0
                assert int(o["lens"][s]) == given[s] and o["table"][s].tolist() == c["table"][s]


def test_pages_that_were_free_already_are_reported():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = _case(18, [9], 30, "float32", False, [0.0])
    c["lens"], c["table"], c["refs"] = [33], [[2, 1, 5, -1, -1]], [0, 1, 1, 0, 0, 0, 0]
    c["tokens"] = [-1] * 9
    for third, refs in ((5, [0, 1, 1, 0, 0, 0, 0]), (7, [0, 1, 1, 0, 0, 0, 0]), (1 << 30, [0, 1, 1, 0, 0, 0, 0])):
        c["table"][0][2] = third
        args, o, keep = _args(torch, mtp, c)
        mtp.mtp_draft_verify(args)
        assert int(o["err"]) == 2 and o["refs"].tolist() == refs and o["table"].tolist() == [[2, 1, -1, -1, -1]]


@pytest.mark.parametrize("vocab", [2000, 40000])
def test_shared_pages_of_several_slots_and_a_graph(vocab):
    """Slots that give back the same page drop its count once each; a replay takes what the buffers hold then."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = _case(19, [4, 4, 4], vocab, "float16", True, [1.0, 0.0])
    c["lens"] = [50, 50, 50]
    c["table"] = [[0, 1, 2, 3, -1], [0, 1, 4, 3, -1], [0, 1, 5, 3, -1]]
    c["refs"] = [3, 3, 1, 3, 1, 1, 0]
    args, o, keep = _args(torch, mtp, c)
    mtp.mtp_draft_verify(args)
    want = _oracle(c)
    assert _got(o) == want
    stream, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        mtp.mtp_draft_verify(args, torch.cuda.current_stream())
    for seed in (1, 2):
        keep[5].copy_(torch.rand(12, 2, generator=torch.Generator().manual_seed(seed)))
        c["uniforms"] = keep[5].tolist()
        o["table"].copy_(torch.tensor(c["table"]))
        o["refs"].copy_(torch.tensor(c["refs"]))
        graph.replay()
        torch.cuda.synchronize()
        assert _got(o) == _oracle(c)


def test_drawn_tokens_are_distributed_as_the_targets():
    """Drafts in the drafter's shares and numbers spread evenly: the first token's shares are p's, to the grid's spacing."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    p, q = np.array([0.5, 0.25, 0.125, 0.125]), np.array([0.125, 0.5, 0.125, 0.25])
    grid, slots, found = 64, 4096, np.zeros(4)
    uu = np.stack(np.meshgrid((np.arange(grid) + 0.5) / grid, (np.arange(grid) + 0.5) / grid, indexing="ij"), -1).reshape(-1, 2)
    for d in range(4):
        c = dict(new=[2] * slots, logits=np.tile(np.log(p), (2 * slots, 1)), draft=np.tile(np.log(q), (2 * slots, 1)),
                 temperature=None, tokens=[d] * (2 * slots), lens=[9] * slots, table=[[0]] * slots, refs=[slots], page=16,
                 max_new=2, eos=-1, dtype="float32", uniforms=np.repeat(uu, 2, 0).tolist())
        args, o, keep = _args(torch, mtp, c)
        mtp.mtp_draft_verify(args)
        assert torch.equal(o["lens"], 9 - (o["counts"] == 1).int())  # a draft that is not kept leaves the cache
        found += q[d] * np.bincount(o["tokens"][:, 0].cpu().numpy(), minlength=4) / slots
    # acceptance p / q and the residual's borders: off by one of 64 rows or columns of the grid at most
    assert np.abs(found - p).max() <= 2 / grid


def test_the_largest_vocabulary_of_equal_logits():
    """2^18 tokens alike: the largest sum there is; token t's border is t / 2^18 exactly."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    v, slots = 1 << 18, 6
    numbers = [0.0, 0.5, 1.0 - 2.0 ** -24, 1.0, 123456.0 / v, (123457.0 - 2.0 ** -6) / v]
    for value in (0.0, -3.0, float("-inf")):
        c = dict(new=[1] * slots, logits=np.full((slots, v), value), draft=None, temperature=[0.7] * slots, tokens=[0] * slots,
                 lens=[1] * slots, table=[[i] for i in range(slots)], refs=[1] * slots, page=16, max_new=1, eos=-1, dtype="float32",
                 uniforms=[[0.0, u] for u in numbers])
        args, o, keep = _args(torch, mtp, c)
        mtp.mtp_draft_verify(args)
        assert o["tokens"][:, 0].tolist() == [0, v // 2, v - 1, v - 1, 123456, 123456]


def test_no_rows_at_all():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = dict(new=[0, 0, 0], logits=np.zeros((0, 50)), draft=None, temperature=None, tokens=[], lens=[5, 0, 17],
             table=[[0, -1], [-1, -1], [1, 2]], refs=[1, 1, 1], page=16, max_new=4, eos=3, dtype="bfloat16", uniforms=[])
    args, o, keep = _args(torch, mtp, c)
    mtp.mtp_draft_verify(args)
    assert _got(o) == ([[-1] * 4] * 3, [0, 0, 0], [5, 0, 17], [0, 0, 0], c["table"], c["refs"]) and int(o["err"]) == 0


def test_two_streams_at_once():
    """Calls that overlap share nothing."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    cases = [_case(60 + i, [5, 3, 7], 30000, "bfloat16", True, [1.0, 0.6]) for i in range(2)]
    calls = [_args(torch, mtp, c) for c in cases]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    for (args, o, keep), s in zip(calls, streams):
        mtp.mtp_draft_verify(args, s)
    torch.cuda.synchronize()
    for c, (args, o, keep) in zip(cases, calls):
        assert _got(o) == _oracle(c)


def test_places_without_a_page_are_reported():
    """An entry below 0 where a page is to be given back is no page of the pool."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = _case(18, [9], 30, "float32", False, [0.0])
    c["lens"], c["refs"] = [50], [0, 1, 1, 1, 0, 0, 0]
    c["tokens"] = [-1] * 9
    for entry in (-1, -2, -2 ** 31):
        c["table"] = [[2, 1, 3, entry, -1]]
        args, o, keep = _args(torch, mtp, c)
        mtp.mtp_draft_verify(args)
        assert int(o["err"]) == 2 and o["refs"].tolist() == c["refs"] and o["table"].tolist() == [[2, 1, 3, -1, -1]]


def _without_draft(c):
    """Every slot's draft outside the vocabulary: a token is drawn behind its first row."""
    for s in range(len(c["new"])):
        c["tokens"][2 * s + 1] = -1 - s
    return c


@pytest.mark.parametrize("vocab,scale", [(50, 2.0), (1025, 2.0), (9000, 0.0), (9000, 5.0), (48001, 1.0), (48001, 8.0), (70001, 2.0)])
def test_a_drafter_that_is_the_target_leaves_only_rounding(vocab, scale):
    """q = p, its logits a constant away: nothing is left of p - q but the rounding of both, and the token is drawn from p."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    slots = 24
    c = _without_draft(_case(vocab, [2] * slots, vocab, "float32", True, [1.0, 0.7, 1.3]))
    rng = np.random.default_rng(vocab)
    # multiples of 2^-10, and sums that fp32 holds
    c["logits"] = np.round(rng.normal(0, scale, c["logits"].shape) * 1024) / 1024
    c["draft"] = c["logits"] + np.array([3.0, -1.0, 0.625, 17.5])[np.arange(2 * slots) % 4][:, None]
    args, o, keep = _args(torch, mtp, c)
    mtp.mtp_draft_verify(args)
    want = []
    for s in range(slots):
        cum = np.cumsum(_shares(c["logits"][2 * s], c["temperature"][s]))
        want.append(int(np.searchsorted(cum, c["uniforms"][2 * s][1] * cum[-1], side="right")))
    assert o["counts"].tolist() == [1] * slots and o["tokens"][:, 0].tolist() == want


@pytest.mark.parametrize("vocab,near", [(1025, 1e-3), (9000, 1e-4), (48001, 1e-3), (48001, 1e-5)])
def test_a_drafter_very_near_the_target(vocab, near):
    """What is left of p - q is small: the borders of its draw are as exact as p and q are.  A weight errs by 2^-32 of itself at
    most (its exponent's rest, below 2^-10, and the power of that are in fp32: three sums, three roundings each of 2^-35),
    a share by twice that, p - q by four times, a border and the whole so much each; and every weight by 3 units of 2^-44 of the
    row's largest."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    slots = 48
    c = _case(vocab, [2] * slots, vocab, "float32", True, [1.0, 0.8], near=near)
    rng = np.random.default_rng(vocab)
    for s in range(slots):
        t = c["temperature"][s]
        p, q = _shares(c["logits"][2 * s], t), _shares(c["draft"][2 * s], t)
        c["tokens"][2 * s + 1] = int(rng.choice(np.flatnonzero(p < q * (1 - near / 8))))  # not kept by the largest number
        c["uniforms"][2 * s][0] = 1.0 - 2.0 ** -24
    args, o, keep = _args(torch, mtp, c)
    mtp.mtp_draft_verify(args)
    assert o["counts"].tolist() == [1] * slots
    for s, token in enumerate(o["tokens"][:, 0].tolist()):
        t = c["temperature"][s]
        p = _shares(c["logits"][2 * s], t)
        w = np.maximum(p - _shares(c["draft"][2 * s], t), 0)
        cum, v = np.cumsum(w) / w.sum(), c["uniforms"][2 * s][1]
        tol = (2.0 ** -29 + 6 * vocab * 2.0 ** -44 * p.max()) / w.sum()
        assert (token == 0 or cum[token - 1] <= v + tol) and v < cum[token] + tol and tol < 1e-2, (s, token)


def test_a_small_rest_of_a_sharp_target_is_drawn_from():
    """Two rare tokens changed about, 2^-25 of the whole: the rest is the one that the target likes better."""
    slots = 8
    c = _case(3, [2] * slots, 3000, "float32", True, [1.0])
    for r in range(2 * slots):
        c["logits"][r], c["draft"][r] = -60.0, -60.0
        c["logits"][r, 100] = c["draft"][r, 100] = 0.0
        c["logits"][r, 7], c["draft"][r, 7] = -17.0, -18.0
        c["logits"][r, 2000 + r], c["draft"][r, 2000 + r] = -18.0, -17.0
    for s in range(slots):
        c["tokens"][2 * s + 1] = 2000 + 2 * s
        c["uniforms"][2 * s] = [0.9, (s + 0.5) / slots]
    assert [t[0] for t in _check(c)[0]] == [7] * slots


def _nearest_numbers(x):
    """Of each row the number in fp32 that is nearest to a border between tokens, relative to it."""
    e = np.exp(x - x.max(-1, keepdims=True))
    borders = np.cumsum(e, -1)[:, :-1] / e.sum(-1, keepdims=True)
    near = borders.astype(np.float32)
    best = np.argmin(np.abs(near.astype(np.float64) / borders - 1.0), -1)[:, None]
    return np.take_along_axis(near, best, -1)[:, 0]


@pytest.mark.parametrize("slots,padded", [(3000, 2048), (3000, 2560), (150, 4096), (40, 16385), (10, 50257), (1, 32768)])
def test_masked_tokens_behind_a_row_change_nothing(slots, padded):
    """Tokens of -infinity have no part in a draw, to the last bit of its borders, wherever the row is cut: the numbers are
    the ones next to a border."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    vocab, many = 1025, 3000
    x = np.random.default_rng(padded).normal(0, 2, (many, vocab)).astype(np.float32).astype(np.float64)
    numbers = _nearest_numbers(x)

    def drawn(first, logits):
        n = len(logits)
        c = dict(new=[1] * n, logits=logits, draft=None, temperature=None, tokens=[0] * n, lens=[1] * n, table=[[0]] * n,
                 refs=[n], page=16, max_new=1, eos=-1, dtype="float32", uniforms=[[0.0, float(u)] for u in numbers[first:first + n]])
        args, o, keep = _args(torch, mtp, c)
        mtp.mtp_draft_verify(args)
        return o["tokens"][:, 0].tolist()
    want = drawn(0, x)
    for first in range(0, min(many, 60 * slots), slots):
        masked = np.full((slots, padded), -np.inf)
        masked[:, :vocab] = x[first:first + slots]
        assert drawn(first, masked) == want[first:first + slots]


@pytest.mark.parametrize("slots,vocab", [(2, 1024), (32, 1024), (1, 4096), (32, 4096), (3, 16384), (1, 16385), (32, 16384), (1, 32768),
                                         (2, 50257), (32, 50257), (1, 128256)])
def test_vocabularies_that_leave_parts_without_tokens(slots, vocab):
    c = _case(slots + vocab, [2 + slots % 2] * slots, vocab, "bfloat16", slots < 3, [0.8, 1.2, 0.0])
    if slots > 2:
        c["logits"][::2, vocab // 3:vocab // 2] = -np.inf
        c["logits"][1::4, 7] = np.inf
    _check(c)


@pytest.mark.parametrize("vocab", [1024, 16385, 50257])
def test_parts_without_tokens_at_extreme_temperatures(vocab):
    """Temperatures whose exponents overflow where a part has no token, and where it has only -infinity."""
    for dtype in ("float32", "float16"):
        c = _case(vocab, [2] * 6, vocab, dtype, True, [1e-38, 0.01, 0.3, 1e30, float("inf"), 2.0])
        c["logits"][1::2, 600:] = -np.inf
        for s in range(6):  # no draft is a matter of 64 bits
            c["uniforms"][2 * s][0] = 0.5
        _check(c)
