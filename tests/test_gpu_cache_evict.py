"""mtp_cache_evict against sorting, one slot, layer and head at a time: copies and whole numbers, all equal."""
import math
import random

import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu


def _state(torch, seed, lens, page, layers, kv_heads, dim, dtype, weights="random", spare=2, stride=None):
    rng, gen = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
    counts = [-(-n // page) for n in lens]
    stride = max(counts) + spare if stride is None else stride
    n_pages = sum(counts) + 3
    order = iter(rng.sample(range(n_pages), sum(counts)))
    table = [[next(order) for _ in range(c)] + [rng.randint(-3, n_pages + 3) for _ in range(stride - c)] for c in counts]
    refs = [0] * n_pages
    for r, c in zip(table, counts):
        for p in r[:c]:
            refs[p] = 1
    shape = (len(lens), layers, kv_heads, stride * page)
    w = torch.randn(shape, device="cuda", generator=gen)
    if weights == "ties":
        w = (w * 2).round() * 0.5
    elif weights == "zeros":
        w = torch.where(w < 1.0, torch.zeros_like(w), w)
        w[..., ::3] *= -0.0
    elif weights == "same":
        w = torch.full_like(w, 0.25)
    elif weights == "special":
        pick = torch.randint(0, 12, shape, device="cuda", generator=gen)
        for i, v in enumerate((math.nan, math.inf, -math.inf, 0.0, -0.0, 1e-42, -1e-42, 3e38)):
            w[pick == i] = v
    elif weights == "positive":
        w = torch.where(w < -1.2, torch.zeros_like(w), (2 * w).exp())
    pool = torch.randn(n_pages, layers, 2, kv_heads, page, dim, device="cuda", generator=gen).to(dtype)
    return dict(table=torch.tensor(table, dtype=torch.int32), refs=refs, lens=lens, weights=w, pool=pool, page=page)


def _oracle(torch, st, keep, sinks, recent):
    """(lens, table, refs, weights, pool, places that are kept) after the call."""
    page, pool, w = st["page"], st["pool"].clone(), st["weights"]
    out_w, table, refs, lens = torch.full_like(w, 9.0), st["table"].clone(), list(st["refs"]), list(st["lens"])
    for s, n in enumerate(st["lens"]):
        m = min(n, keep[s])
        lens[s] = m
        held = st["table"][s].long().cuda()
        table[s, -(-m // page):] = -1
        for p in st["table"][s, -(-m // page):-(-n // page)].tolist():
            refs[p] -= 1
        if m == n:
            out_w[s, ..., :n] = w[s, ..., :n]
            continue
        a = min(m, sinks)
        b = min(m - a, recent)
        x = w[s, ..., :n].double()
        x = torch.where(x.isnan(), torch.full_like(x, math.inf), x)
        # NaN above infinity, the forced ones above all
        rank = w[s, ..., :n].isnan().double()
        rank[..., :a] = 2.0
        if b:
            rank[..., n - b:] = 2.0
        order = torch.argsort(-x, dim=-1, stable=True)
        order = order.gather(-1, torch.argsort(-rank.gather(-1, order), dim=-1, stable=True))
        kept = order[..., :m].sort(-1)[0]
        out_w[s, ..., :m] = w[s].gather(-1, kept)
        to = torch.arange(m, device="cuda")
        for layer in range(w.shape[1]):
            for head in range(w.shape[2]):
                k = kept[layer, head]
                pool[held[to // page], layer, :, head, to % page] = st["pool"][held[k // page], layer, :, head, k % page]
    return lens, table.tolist(), refs, out_w, pool


def _call(torch, mtp, st, keep, sinks, recent, in_place=False):
    slots = len(st["lens"])

    def ints(x):
        return torch.tensor(x, dtype=torch.int32, device="cuda")
    refs, table = ints(st["refs"]), st["table"].cuda()
    o = dict(lens=ints([7] * slots), table=torch.full_like(table, 7), refs=refs if in_place else torch.full_like(refs, 7),
             weights=torch.full_like(st["weights"], 9.0), status=ints([7] * slots), pool=st["pool"].clone())
    keep_alive = [ints(st["lens"]), ints(keep), table, refs]
    args = mtp.cache_evict_args(kv_lens=keep_alive[0], keep=keep_alive[1], block_table=table, page_refs=refs, weights=st["weights"],
                                kv_pool=o["pool"], out_kv_lens=o["lens"], out_block_table=o["table"], out_page_refs=o["refs"],
                                out_weights=o["weights"], out_status=o["status"], sinks=sinks, recent=recent)
    nbytes = mtp.mtp_cache_evict_workspace_bytes(args)
    ws = torch.full((max(nbytes, 16),), 255, dtype=torch.uint8, device="cuda")
    mtp.mtp_cache_evict(args, ws, nbytes, torch.cuda.current_stream())
    return o, args, (ws, nbytes), keep_alive


def _bits(torch, x):
    return x.view(torch.int16 if x.element_size() == 2 else torch.int32)


def _check(torch, o, want):
    lens, table, refs, w, pool = want
    assert o["lens"].tolist() == lens and o["table"].tolist() == table and o["refs"].tolist() == refs
    assert torch.equal(_bits(torch, o["weights"]), _bits(torch, w))
    assert torch.equal(_bits(torch, o["pool"]), _bits(torch, pool))
    assert set(o["status"].tolist()) == {0}


@pytest.mark.parametrize("weights", ["random", "ties", "zeros", "same", "special", "positive"])
@pytest.mark.parametrize("lens,keep,sinks,recent,page,layers,kv_heads,dim", [
    ([1, 0, 5], [1, 3, 0], 0, 0, 16, 1, 1, 64), ([40, 33, 100, 7], [16, 32, 99, 7], 4, 8, 16, 2, 2, 64),
    ([300, 180], [64, 170], 64, 0, 32, 1, 3, 128), ([200, 130], [10, 130], 50, 50, 64, 2, 1, 8),
    ([1088], [1024], 4, 256, 64, 2, 4, 64), ([2000, 700, 701], [700] * 3, 4, 128, 64, 2, 2, 64),
    ([500, 400], [399, 1], 0, 399, 128, 1, 2, 256), ([2500, 100], [1300, 99], 3, 7, 16, 1, 2, 128),
    ([9000], [4097], 64, 1000, 128, 1, 2, 24), ([20000, 300], [5000, 299], 64, 700, 64, 1, 2, 64)])
def test_the_keys_of_largest_weight_stay(weights, lens, keep, sinks, recent, page, layers, kv_heads, dim):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    dtype = torch.bfloat16 if len(lens) % 2 else torch.float16
    st = _state(torch, len(weights) + lens[0], lens, page, layers, kv_heads, dim, dtype, weights)
    _check(torch, _call(torch, mtp, st, keep, sinks, recent, in_place=len(lens) > 1)[0], _oracle(torch, st, keep, sinks, recent))


@pytest.mark.parametrize("values", [1, 3, 50, 2000])
@pytest.mark.parametrize("alike", [2, 255, 256, 257, 600])
@pytest.mark.parametrize("lens,page,layers,kv_heads", [
    ([700, 701], 16, 1, 2), ([700, 701, 900, 650], 16, 4, 16), ([3000, 700], 64, 1, 2), ([4100, 2700, 650], 16, 4, 20), ([13000, 800], 128, 1, 2)])
def test_borders_among_weights_that_are_nearly_alike(lens, page, layers, kv_heads, alike, values):
    """A border between weights whose first bits are the same: few of them, more, and equal ones among them."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, alike + values, lens, page, layers, kv_heads, 8, torch.bfloat16, "positive")
    gen = torch.Generator(device="cuda").manual_seed(alike * values)
    w = st["weights"]
    for s, n in enumerate(lens):
        x = 4.0 + torch.rand(w.shape[1:3] + (n,), device="cuda", generator=gen)
        x[..., n // 2:] -= 3.0
        where = torch.rand(x.shape, device="cuda", generator=gen).argsort(-1)[..., :alike]
        near = 2.0 + torch.randint(0, values, where.shape, device="cuda", generator=gen) * 2.0 ** -22
        w[s, ..., :n] = x.scatter(-1, where, near)
    # kept: the large ones, and about half of those that are alike
    above = int((w[0, 0, 0, : lens[0]] > 3.0).sum())
    keep = [min(n, above * n // lens[0] + alike // 2) for n in lens]
    _check(torch, _call(torch, mtp, st, keep, 0, 0)[0], _oracle(torch, st, keep, 0, 0))


@pytest.mark.parametrize("weights", ["random", "ties"])
@pytest.mark.parametrize("lens,page,layers,kv_heads", [
    ([2816, 900, 30, 1], 16, 4, 20), ([2817, 2000, 64], 16, 4, 20), ([2800, 2000, 64], 16, 4, 20), ([4096, 300], 128, 6, 20), ([4097, 300], 16, 1, 2), ([4080, 300], 16, 1, 2),
    ([12288], 16, 1, 200), ([12289], 16, 1, 90), ([32768], 128, 1, 3)])
def test_widths_at_the_bounds_of_the_launches_forms(lens, page, layers, kv_heads, weights):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, lens[0], lens, page, layers, kv_heads, 8, torch.float16, weights)
    keep = [max(1, n * 2 // 3) for n in lens]
    _check(torch, _call(torch, mtp, st, keep, 4, 9)[0], _oracle(torch, st, keep, 4, 9))


@pytest.mark.parametrize("weights", ["ties", "same", "positive"])
def test_more_keys_than_a_cta_holds(weights):
    """Rows of weights that are read again for every bit."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, 3, [70001, 32769, 100], 128, 1, 1, 64, torch.float16, weights)
    keep = [40000, 32768, 50]
    _check(torch, _call(torch, mtp, st, keep, 5, 300)[0], _oracle(torch, st, keep, 5, 300))


def test_a_pool_past_32_bits():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, 4, [300, 290], 64, 2, 2, 128, torch.bfloat16)
    keep = [100, 130]
    want = _oracle(torch, st, keep, 4, 50)
    shift = 66000
    big = torch.zeros(shift + st["pool"].shape[0], 2, 2, 2, 64, 128, dtype=torch.bfloat16, device="cuda")
    assert big.numel() > 1 << 32
    big[shift:] = st["pool"]
    moved = dict(st, pool=big, refs=[0] * shift + st["refs"], table=torch.where(st["table"] >= 0, st["table"] + shift, st["table"]))
    o = _call(torch, mtp, moved, keep, 4, 50)[0]
    assert torch.equal(o["pool"][shift:], want[4]) and torch.equal(o["weights"], want[3])
    assert int(o["pool"][:shift].count_nonzero()) == 0 and o["refs"].tolist()[shift:] == want[2]


def test_slots_that_cannot_be_evicted_stay_and_are_reported():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, 6, [100, 90, 80, 70, 60, 64], 16, 1, 2, 64, torch.bfloat16, spare=0)
    keep = [50, 40, 30, -1, 20, 48]
    good = _state(torch, 6, [100, 90, 80, 70, 60, 64], 16, 1, 2, 64, torch.bfloat16, spare=0)
    st["table"][0, 5] = st["pool"].shape[0]        # a held page outside the pool
    st["refs"][st["table"][1, 4].item()] = 0       # one that is free
    st["refs"][st["table"][2, 1].item()] = 2       # one that would be written and another slot holds
    st["lens"] = [100, 90, 80, 70, 1000, 64]       # a length outside the table
    st["refs"][st["table"][5, 0].item()] = 2       # shared, but within the sinks
    st["refs"][st["table"][5, 3].item()] = 3       # shared, and given back
    o = _call(torch, mtp, st, keep, 17, 5)[0]
    assert o["status"].tolist() == [-1, -1, -1, -1, -1, 0]
    assert o["lens"].tolist() == [100, 90, 80, 70, 1000, 48]
    assert o["table"][:5].tolist() == st["table"][:5].tolist() and o["table"][5].tolist() == st["table"][5, :3].tolist() + [-1] * 4
    refs = list(st["refs"])
    refs[st["table"][5, 3].item()] -= 1
    assert o["refs"].tolist() == refs
    for s, n in enumerate([100, 90, 80, 70]):
        assert torch.equal(o["weights"][s, ..., :n], st["weights"][s, ..., :n])
        pages = [p for p in st["table"][s, :-(-n // 16)].tolist() if p < st["pool"].shape[0]]
        assert torch.equal(o["pool"][pages], st["pool"][pages])
    alone = dict(good, lens=[0, 0, 0, 0, 0, 64])
    want = _oracle(torch, alone, [0, 0, 0, 0, 0, 48], 17, 5)
    pages = st["table"][5].tolist()[:4]
    assert torch.equal(o["pool"][pages], want[4][pages]) and torch.equal(o["weights"][5, ..., :48], want[3][5, ..., :48])


def test_a_graph_on_another_stream_and_two_of_one_workspace():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    states = [_state(torch, 40 + i, [333, 1500, 20], 32, 2, 2, 64, torch.float16, "positive") for i in range(2)]
    keep = [200, 800, 64]
    calls = [_call(torch, mtp, st, keep, 4, 32) for st in states]
    wants = [_oracle(torch, st, keep, 4, 32) for st in states]
    for (o, *_), want in zip(calls, wants):
        _check(torch, o, want)
    stream, graphs = torch.cuda.Stream(), []
    ws, nbytes = calls[0][2]
    for o, args, *_ in calls:
        graphs.append(torch.cuda.CUDAGraph())
        with torch.cuda.graph(graphs[-1], stream=stream):
            mtp.mtp_cache_evict(args, ws, nbytes, torch.cuda.current_stream())
    for _ in range(2):
        for (o, *_), st in zip(calls, states):
            o["pool"].copy_(st["pool"])
            for k in ("lens", "table", "refs", "status"):
                o[k].fill_(7)
            o["weights"].fill_(9.0)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for (o, *_), want in zip(calls, wants):
            _check(torch, o, want)


def test_evicted_again_and_again():
    """A context that grows and is cut down several times: the outputs of a call are the inputs of the next."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, 50, [500], 16, 1, 2, 64, torch.bfloat16, "positive")
    for keep in (400, 399, 200, 64, 1, 0):
        want = _oracle(torch, st, [keep], 4, 30)
        o = _call(torch, mtp, st, [keep], 4, 30)[0]
        _check(torch, o, want)
        st = dict(st, lens=o["lens"].tolist(), table=o["table"].cpu(), refs=o["refs"].tolist(), weights=o["weights"], pool=o["pool"])
    assert sum(st["refs"]) == 0


def test_weights_off_the_16_byte_boundary():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    for lens, keep in (([300, 77], [100, 77]), ([5000], [1234])):
        st = _state(torch, 70, lens, 16, 1, 2, 64, torch.float16, "special")
        buf = torch.empty(st["weights"].numel() + 1, device="cuda")
        moved = buf[1:].view(st["weights"].shape)
        moved.copy_(st["weights"])
        st["weights"] = moved
        assert moved.data_ptr() % 16 == 4
        _check(torch, _call(torch, mtp, st, keep, 3, 20)[0], _oracle(torch, st, keep, 3, 20))


def test_two_streams_at_once():
    """Calls on pools of their own, which overlap: wide tables in workspaces of their own."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    for lens, keep in (([900, 1200], [400, 700]), ([40000], [9000])):
        states = [_state(torch, 80 + i, lens, 64, 1, 2, 64, torch.bfloat16, "positive") for i in range(2)]
        calls = [_call(torch, mtp, st, keep, 4, 64) for st in states]
        streams = [torch.cuda.Stream() for _ in states]
        torch.cuda.synchronize()
        for (o, *_), st in zip(calls, states):
            o["pool"].copy_(st["pool"])
        torch.cuda.synchronize()
        for (o, args, (ws, nbytes), _), s in zip(calls, streams):
            mtp.mtp_cache_evict(args, ws, nbytes, s)
        torch.cuda.synchronize()
        for (o, *_), st in zip(calls, states):
            _check(torch, o, _oracle(torch, st, keep, 4, 64))


@pytest.mark.parametrize("sinks,keep", [(20, 20), (20, 19), (20, 17), (17, 5), (64, 33), (40, 40)])
def test_budgets_within_the_sinks_write_nothing(sinks, keep):
    """A budget that the sinks fill: no row moves, so shared pages are no hindrance, whole or not; the others are given back."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, sinks * keep, [64, 70], 16, 2, 2, 64, torch.bfloat16, "positive")
    for s in range(2):
        for c in range(-(-st["lens"][s] // 16)):
            st["refs"][st["table"][s, c].item()] = 1 + (c + s) % 3
    _check(torch, _call(torch, mtp, st, [keep] * 2, sinks, 3)[0], _oracle(torch, st, [keep] * 2, sinks, 3))


def test_one_key_behind_the_sinks_is_written():
    """The page that the sinks end in is written where a key follows them: a shared one is refused."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    st = _state(torch, 91, [64, 64], 16, 1, 2, 64, torch.float16)
    for s, keep in ((0, 20), (1, 21)):
        st["refs"][st["table"][s, 1].item()] = 2
    o = _call(torch, mtp, st, [20, 21], 20, 0)[0]
    assert o["status"].tolist() == [0, -1] and o["lens"].tolist() == [20, 64]
