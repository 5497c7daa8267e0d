"""mtp_key_weights against the sums in 64 bits.

Tolerance, per pair: a score is a sum of dim exact products in fp32 whose additions err by 2^-23 of the sum of magnitudes
each at most (tensor cores may cut off); scale log2 e, the log-sum-exp in log2 units, and their difference are rounded to 2^-24
relatively each; the exponential errs by 2^-22.  The sum over rows adds 2^-24 of itself per addition (at most 64 in a row
without compensation), and so does the addition to the weight before."""
import math
import random

import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu

NAN = float("nan")


def _case(torch, seed, new, lens, heads, kv_heads, dim, page, dtype, layers=2, spare=2, q_pad=0):
    rng, gen = random.Random(seed), torch.Generator(device="cuda").manual_seed(seed)
    slots, rows = len(new), sum(new)
    counts = [-(-max(n, 0) // page) for n in lens]
    stride = max(counts) + spare
    n_pages = sum(counts) + 2
    order = iter(rng.sample(range(n_pages), sum(counts)))
    table = [[next(order) for _ in range(c)] + [rng.randint(-3, n_pages + 3) for _ in range(stride - c)] for c in counts]
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(n_pages, layers, 2, kv_heads, page, dim, device="cuda", generator=gen).to(dtype)
    for b, (n, c) in enumerate(zip(lens, counts)):  # behind a length: anything
        if c and n % page:
            pool[table[b][c - 1], :, :, :, n % page:] = NAN
    buf = (2.0 * torch.randn(rows, heads * dim + q_pad, device="cuda", generator=gen)).to(dtype)
    q = buf[:, q_pad:].unflatten(1, (heads, dim))
    cu = [0]
    for n in new:
        cu.append(cu[-1] + n)
    return dict(q=q, pool=pool, table=torch.tensor(table, **i32), cu=torch.tensor(cu, **i32), lens=torch.tensor(lens, **i32),
                weights=0.1 * torch.rand(slots, layers, kv_heads, stride * page, device="cuda", generator=gen),
                scale=dim ** -0.5, page=page, new=new, lengths=lens, heads=heads, kv_heads=kv_heads, dim=dim)


def _oracle(torch, c, layer, window, lse=None):
    """(weights, tolerance, lse) in 64 bits."""
    want, tol = c["weights"].double().clone(), torch.zeros_like(c["weights"], dtype=torch.float64)
    out_lse = torch.full((c["q"].shape[0], c["heads"]), -math.inf, dtype=torch.float64, device="cuda")
    g, row = c["heads"] // c["kv_heads"], 0
    for b, (n, length) in enumerate(zip(c["new"], c["lengths"])):
        q = c["q"][row:row + n].double().view(n, c["kv_heads"], g, c["dim"])
        pages = c["table"][b, :-(-length // c["page"])].long()
        k = c["pool"][pages, layer, 0].transpose(0, 1).reshape(c["kv_heads"], -1, c["dim"])[:, :length].double()
        if n and length:
            s = torch.einsum("nhgd,htd->nhgt", q, k) * c["scale"]
            size = torch.einsum("nhgd,htd->nhgt", q.abs(), k.abs()) * c["scale"]
            pos = length - n + torch.arange(n, device="cuda")[:, None]
            t = torch.arange(length, device="cuda")
            sees = t <= pos
            if window:
                sees &= t > pos - window
            l = torch.logsumexp(s.masked_fill(~sees[:, None, None], -math.inf), -1)
            out_lse[row:row + n] = l.reshape(n, -1)
            if lse is not None:
                l = lse[row:row + n].double().view(n, c["kv_heads"], g)
            p = (s - l[..., None]).exp().masked_fill(~sees[:, None, None], 0.0)
            e = c["dim"] * size * 2.0 ** -23 + (s.abs() + l.abs()[..., None] + 1) * 2.0 ** -21
            got, seen = p.sum((0, 2)), sees.any(0)
            fresh = t >= length - n
            old = want[b, layer, :, :length]
            want[b, layer, :, :length] = torch.where(seen, torch.where(fresh, got, old + got), old)
            slip = (p * e).masked_fill(~sees[:, None, None], 0.0).sum((0, 2)) + got * 70 * 2.0 ** -24 + (old + got) * 2.0 ** -23
            tol[b, layer, :, :length] = torch.where(seen, slip, torch.zeros_like(slip))
        row += n
    return want, tol, out_lse


def _run(torch, mtp, c, layer, window, lse, stream=None, max_new=None, max_keys=None, err=None):
    args = mtp.key_weights_args(q=c["q"], kv_pool=c["pool"], layer=layer, block_table=c["table"], cu_rows=c["cu"],
                                kv_lens=c["lens"], lse=lse, weights=c["weights"], scale=c["scale"], window=window,
                                max_new=max(c["new"]) if max_new is None else max_new,
                                max_keys=max(c["lengths"]) if max_keys is None else max_keys, err_word=err)
    nbytes = mtp.mtp_key_weights_workspace_bytes(args)
    ws = torch.full((max(nbytes, 16),), 255, dtype=torch.uint8, device="cuda")
    mtp.mtp_key_weights(args, ws, nbytes, stream or torch.cuda.current_stream())
    return args, ws, nbytes


def _check(torch, c, want, tol):
    err = (c["weights"].double() - want).abs()
    assert bool((err <= tol).all()), (float((err - tol).max()), float(err.max()))


CASES = [  # new, lens, heads, kv_heads, dim, page
    ([1], [1], 1, 1, 64, 16), ([1], [1], 4, 1, 128, 128), ([1, 1, 1], [5, 180, 333], 16, 16, 64, 64),
    ([1, 0, 1], [129, 77, 1], 8, 2, 128, 16), ([4, 2, 0, 3], [260, 2, 50, 31], 16, 4, 128, 16),
    ([9, 5], [300, 9], 12, 4, 64, 32), ([3], [700], 32, 4, 64, 128), ([32, 1], [40, 500], 5, 5, 128, 32),
    # more than 32 rows of a key head: tensor-core tiles, tails, groups that do not divide 128
    ([33, 0, 1], [33, 20, 400], 4, 4, 64, 16), ([40, 129, 7], [400, 129, 300], 8, 2, 128, 64),
    ([30, 77], [30, 205], 10, 2, 64, 32), ([200, 3], [200, 640], 20, 4, 128, 128), ([300], [301], 1, 1, 64, 16),
    ([65, 64], [65, 1000], 16, 2, 64, 16), ([10], [2000], 64, 1, 128, 64),
    # few keys and many rows: the rows are cut into segments
    ([1200], [1300], 4, 1, 64, 64), ([700, 1500], [700, 1600], 8, 1, 128, 16),
    # long contexts with work for every SM: four key tiles of a CTA
    ([40, 3, 60, 33, 50, 1, 0, 70], [2100, 1900, 60, 1500, 2048, 2, 500, 2000], 16, 16, 64, 64),
    ([20, 9, 130, 1, 8, 30, 7, 0, 40, 25], [2300, 2000, 1990, 1, 800, 30, 513, 700, 640, 1025], 40, 8, 128, 16),
    # 17 to 64 rows on work for every SM: in registers, in shared memory
    ([8, 0, 1, 5] * 5, [1100, 90, 700, 5] * 5, 32, 8, 128, 16), ([16, 9, 0, 1] * 5, [1100, 200, 640, 33] * 5, 32, 8, 128, 64),
    ([16, 1, 13, 0] * 5, [1100, 1, 512, 600] * 5, 16, 8, 64, 128), ([31, 2, 25, 0] * 5, [1500, 2, 500, 1025] * 5, 16, 8, 64, 16)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("window", [0, 1, 90])
@pytest.mark.parametrize("case", range(len(CASES)))
def test_weights_add_up(case, window, dtype):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    new, lens, heads, kv_heads, dim, page = CASES[case]
    c = _case(torch, case, new, lens, heads, kv_heads, dim, page, getattr(torch, dtype), q_pad=(0, 8, 3)[case % 3])
    layer = case % 2
    _, _, lse = _oracle(torch, c, layer, window)
    lse = lse.float()
    want, tol, _ = _oracle(torch, c, layer, window, lse)
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    _run(torch, mtp, c, layer, window, lse, err=err)
    _check(torch, c, want, tol)
    assert int(err) == 0
    again = _case(torch, case, new, lens, heads, kv_heads, dim, page, getattr(torch, dtype), q_pad=(0, 8, 3)[case % 3])
    _run(torch, mtp, again, layer, window, lse)
    assert torch.equal(again["weights"], c["weights"])  # the same sums in every call


def test_a_length_shorter_than_its_rows():
    """Rows of positions below 0 see no key."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    for new, heads in (([6], 2), ([90], 2)):
        c = _case(torch, 3, new, [4], heads, 1, 64, 16, torch.bfloat16)
        _, _, lse = _oracle(torch, c, 0, 0)
        lse = lse.float()
        want, tol, _ = _oracle(torch, c, 0, 0, lse)
        _run(torch, mtp, c, 0, 0, lse)
        _check(torch, c, want, tol)


@pytest.mark.parametrize("new", [[3, 2], [60, 50]])
def test_what_is_not_finite_stays_by_itself(new):
    """NaN in one slot's rows, and in a key: other slots' weights, and other keys', are as without."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c, d = (_case(torch, 11, new, [200, 150], 4, 2, 64, 16, torch.float16) for _ in range(2))
    _, _, lse = _oracle(torch, c, 1, 0)
    lse = lse.float()
    _run(torch, mtp, c, 1, 0, lse)
    d["q"][:new[0]] = NAN
    _run(torch, mtp, d, 1, 0, lse)
    assert torch.equal(c["weights"][1], d["weights"][1])
    e = _case(torch, 11, new, [200, 150], 4, 2, 64, 16, torch.float16)
    e["pool"][e["table"][1, 2].item(), 1, 0, 0, 5] = NAN
    _run(torch, mtp, e, 1, 0, lse)
    same = torch.ones_like(c["weights"], dtype=torch.bool)
    same[1, 1, 0, 37] = False
    assert torch.equal(c["weights"][same], e["weights"][same]) and bool(e["weights"][1, 1, 0, 37].isnan())


def test_pages_outside_the_pool_count_as_zeros():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    for new in ([2, 1], [70, 40]):
        c = _case(torch, 5, new, [100, 90], 2, 2, 128, 16, torch.bfloat16)
        _, _, lse = _oracle(torch, c, 0, 0)
        lse = lse.float()
        bad = c["table"][0, 1].item()
        c["pool"][bad, 0, 0] = 0
        want, tol, _ = _oracle(torch, c, 0, 0, lse)
        for page in (-1, c["pool"].shape[0], 1 << 30):
            w = c["weights"].clone()
            c["table"][0, 1] = page
            _run(torch, mtp, c, 0, 0, lse)
            _check(torch, c, want, tol)
            c["weights"].copy_(w)


@pytest.mark.parametrize("what", ["max_new", "max_keys", "rows", "length", "order"])
@pytest.mark.parametrize("new", [[2, 5, 1], [60, 45, 50]])
def test_what_does_not_fit_is_left_out_and_reported(what, new):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    lens = [120, 200, 90]
    c = _case(torch, 21, new, lens, 2, 1, 64, 16, torch.bfloat16)
    _, _, lse = _oracle(torch, c, 1, 0)
    lse = lse.float()
    want, tol, _ = _oracle(torch, c, 1, 0, lse)
    before = c["weights"].clone()
    err = torch.zeros(1, dtype=torch.int32, device="cuda")
    kw = dict(err=err)
    sound = [0, 2]  # slots whose weights are right
    if what == "max_new":
        kw["max_new"] = max(new) - 1 if new[0] < 10 else 50
        sound = [2] if new[0] > 10 else [0, 2]
    if what == "max_keys":
        kw["max_keys"] = 128
    if what == "rows":
        c["cu"][3] = sum(new) + 7
        sound = [0, 1]
    if what == "length":
        c["lens"][1] = c["weights"].shape[3] + 1
    if what == "order":
        c["cu"][2] = c["cu"][1] - 1
        sound = [0]
    _run(torch, mtp, c, 1, 0, lse, **kw)
    assert int(err) == 2
    for s in sound:
        assert bool(((c["weights"][s].double() - want[s]).abs() <= tol[s]).all())
    assert torch.equal(c["weights"][:, 0], before[:, 0]) and bool(c["weights"].isfinite().all())
    for s, n in enumerate(lens):
        assert torch.equal(c["weights"][s, :, :, n:], before[s, :, :, n:])
    if what == "max_keys":
        assert torch.equal(c["weights"][1, :, :, 128:], before[1, :, :, 128:])


def test_offsets_past_32_bits():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    for new in ([2], [80]):
        c = _case(torch, 8, new, [150], 2, 2, 128, 128, torch.bfloat16, layers=2)
        _, _, lse = _oracle(torch, c, 1, 0)
        lse = lse.float()
        want, tol, _ = _oracle(torch, c, 1, 0, lse)
        small = c["pool"]
        big = torch.zeros(33000, 2, 2, 2, 128, 128, dtype=torch.bfloat16, device="cuda")
        assert big.numel() > 1 << 32
        for i, p in enumerate(c["table"][0, :2].tolist()):
            big[32990 + i] = small[p]
            c["table"][0, i] = 32990 + i
        c["pool"] = big
        _run(torch, mtp, c, 1, 0, lse)
        _check(torch, c, want, tol)


@pytest.mark.parametrize("new", [[1, 1], [90, 30], [600, 400]])
def test_two_graphs_share_a_workspace_and_another_stream(new):
    """Two captured calls on one workspace, replayed in turn, and their sums against calls of their own."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    stream = torch.cuda.Stream()
    cases = [_case(torch, 31 + i, new, [620, 450], 2, 1, 64, 64, torch.bfloat16) for i in range(2)]
    lses = [_oracle(torch, c, 0, 0)[2].float() for c in cases]
    wants = [_oracle(torch, c, 0, 0, l)[:2] for c, l in zip(cases, lses)]
    start = [c["weights"].clone() for c in cases]
    calls = [_run(torch, mtp, c, 0, 0, l) for c, l in zip(cases, lses)]
    ws = calls[0][1]
    graphs = []
    for (args, _, nbytes) in calls:
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph, stream=stream):
            mtp.mtp_key_weights(args, ws, nbytes, torch.cuda.current_stream())
        graphs.append(graph)
    for _ in range(2):
        for c, w in zip(cases, start):
            c["weights"].copy_(w)
        ws.fill_(255)
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        for c, (want, tol) in zip(cases, wants):
            _check(torch, c, want, tol)


def test_nothing_to_do():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = _case(torch, 2, [0, 0], [30, 0], 2, 1, 64, 16, torch.bfloat16)
    before = c["weights"].clone()
    lse = torch.zeros(0, 2, device="cuda")
    _run(torch, mtp, c, 0, 0, lse, max_new=4)
    assert torch.equal(before, c["weights"])


@pytest.mark.parametrize("new", [[1, 3], [90, 30], [600, 400]])
def test_two_streams_at_once(new):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    cases = [_case(torch, 41 + i, new, [700, 450], 4, 1, 64, 32, torch.float16) for i in range(2)]
    lses = [_oracle(torch, c, 1, 0)[2].float() for c in cases]
    wants = [_oracle(torch, c, 1, 0, l)[:2] for c, l in zip(cases, lses)]
    streams = [torch.cuda.Stream() for _ in cases]
    torch.cuda.synchronize()
    held = [_run(torch, mtp, c, 1, 0, l, stream=s) for c, l, s in zip(cases, lses, streams)]
    torch.cuda.synchronize()
    assert len(held) == 2
    for c, (want, tol) in zip(cases, wants):
        _check(torch, c, want, tol)


def test_attention_and_weights_follow_each_other_on_one_stream():
    """Kernels that hold tensor memory, launched behind each other without a wait of the host: each layer's weights come out
    as alone."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    c = _case(torch, 51, [300, 150, 70], [2100, 1500, 70], 16, 16, 64, 64, torch.bfloat16, layers=4)
    i32 = dict(dtype=torch.int32, device="cuda")
    err = torch.zeros(1, **i32)
    out, lse = torch.zeros_like(c["q"]).contiguous(), torch.zeros(c["q"].shape[0], 16, device="cuda")
    lses = []
    start = c["weights"].clone()
    for rounds in range(3):
        c["weights"].copy_(start)
        for layer in range(4):
            shared = dict(q=c["q"], kv_pool=c["pool"], layer=layer, block_table=c["table"], cu_rows=c["cu"], kv_lens=c["lens"],
                          scale=c["scale"], max_new=300, max_keys=2100, err_word=err)
            attend = mtp.chunk_attention_args(out=out, out_lse=lse, **shared)
            n = mtp.mtp_chunk_attention_workspace_bytes(attend)
            ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
            weigh = mtp.key_weights_args(lse=lse, weights=c["weights"], **shared)
            m = mtp.mtp_key_weights_workspace_bytes(weigh)
            ws2 = torch.zeros(max(m, 16), dtype=torch.uint8, device="cuda")
            mtp.mtp_chunk_attention(attend, ws, n, torch.cuda.current_stream())
            mtp.mtp_key_weights(weigh, ws2, m, torch.cuda.current_stream())
            if rounds == 2:
                lses.append(lse.clone())
    assert int(err) == 0
    got = c["weights"].clone()
    c["weights"].copy_(start)
    for layer in range(4):
        want, tol, _ = _oracle(torch, c, layer, 0, lses[layer])
        assert bool(((got[:, layer].double() - want[:, layer]).abs() <= tol[:, layer]).all())
