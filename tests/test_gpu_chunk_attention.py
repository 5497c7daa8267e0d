"""mtp_chunk_attention against 64 bits.

Bounds, element by element, with u the type's unit roundoff (2^-8 bf16, 2^-11 fp16: test_unit_roundoff), p a row's
weights and A = sum_j p_j |v_j|: the output's rounding gives u |out|; weights rounded once to the type, as the kernel of
many rows has them, give u A at most (that of up to 32 rows per slot and key head keeps their residues: nothing); scores
of up to 128 products summed in fp32, exp2's approximation and sums in fp32 stay below 2^-14 A; fp16 weights below 2^-14
of the largest are rounded to multiples of 2^-24, which gives 2^-25 sum_j |v_j| over the keys.  The log-sum-exp errs as
one score does, and by its own rounding: 4e-5 + 2^-22 |lse|."""
import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu

NAN = float("nan")


def reference(torch, q, pool, layer, table, new, lens, scale, window):
    """(out, lse, A, sum |v|) in 64 bits, rows packed; rows without a key 0 and -inf."""
    rows, heads, dim = q.shape
    page, kv_heads = pool.shape[4], pool.shape[3]
    out = torch.zeros(rows, heads, dim, dtype=torch.float64, device="cuda")
    size, total = out.clone(), out.clone()
    lse = torch.full((rows, heads), -float("inf"), dtype=torch.float64, device="cuda")
    row = 0
    for s, (n, length) in enumerate(zip(new, lens)):
        pos = length - n + torch.arange(n, device="cuda")
        key = torch.arange(length, device="cuda")
        if n and length:
            pages = torch.tensor([p if 0 <= p < len(pool) else 0 for p in table[s][:-(-length // page)]], device="cuda")
            k, v = (pool[pages, layer, i].transpose(1, 2).flatten(0, 1)[:length].double().repeat_interleave(heads // kv_heads, 1)
                    for i in (0, 1))
            sees = key <= pos[:, None]
            if window:
                sees &= key > pos[:, None] - window
            unseen = ~sees.any(0)
            k[unseen], v[unseen] = 0.0, 0.0
            for h in range(heads):
                x = (q[row:row + n, h].double() @ k[:, h].T * scale).masked_fill(~sees, -float("inf"))
                some = sees.any(1)
                p = torch.where(some[:, None], torch.softmax(x, -1), 0.0).nan_to_num(0.0)
                out[row:row + n, h] = p @ v[:, h]
                size[row:row + n, h] = p @ v[:, h].abs()
                total[row:row + n, h] = sees.double() @ v[:, h].abs()
                lse[row:row + n, h] = torch.logsumexp(x, -1)
        row += n
    return out, lse, size, total


def check(new, lens, heads, kv_heads, dim, page, dtype="bfloat16", window=0, layout="own", layers=2, layer=1, seed=0,
          spread=2.0, rows_past=3, stream=None, workspace=None, hints=None, scale=None):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    dt = getattr(torch, dtype)
    gen = torch.Generator(device="cuda").manual_seed(seed + sum(lens))
    counts = [-(-n // page) for n in lens]
    n_pages, stride = sum(counts) + 2, max(counts + [1]) + 1
    order = torch.randperm(n_pages, device="cuda", generator=gen).tolist()
    bad = order.pop()  # a page of NaN, which no slot holds
    pool = torch.randn(n_pages, layers, 2, kv_heads, page, dim, device="cuda", generator=gen).to(dt)
    pool[bad] = NAN
    table, it = [], iter(order)
    for n, c in zip(lens, counts):
        mine = [next(it) for _ in range(c)]
        if n % page:
            pool[mine[-1], :, :, :, n % page:] = NAN  # past the length: anything
        table.append(mine + [bad] * (stride - c))
    if window:  # what lies before every row's window: NaN, or pages given away
        for s, (n, length) in enumerate(zip(new, lens)):
            first = max(0, length - n - window + 1)
            for c in range(first // page):
                pool[table[s][c]] = NAN
                table[s][c] = [bad, -1, 1 << 30][c % 3]
            if first % page and first < length:
                pool[table[s][first // page], :, :, :, :first % page] = NAN
    pool[:, [i for i in range(layers) if i != layer]] = NAN
    live, rows = sum(new), sum(new) + rows_past
    pad = {"own": 0, "fused": 2 * kv_heads * dim, "odd": 1, "shifted": 3}[layout]
    at = 1 if layout == "shifted" else 0

    def buffer():
        return torch.full((rows, heads * dim + pad), -7.0, device="cuda").to(dt)[:, at:at + heads * dim].unflatten(1, (heads, dim))
    q, out = buffer(), buffer()
    q.copy_((spread * torch.randn(rows, heads, dim, device="cuda", generator=gen)).to(dt))
    lse = torch.full((rows, heads), -7.0, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    d_table, cu, d_lens, err = ints(table), ints([sum(new[:i]) for i in range(len(new) + 1)]), ints(lens), ints([0])
    scale = dim ** -0.5 if scale is None else scale
    max_new, max_keys = hints or (max(new), max(lens))
    args = mtp.chunk_attention_args(q=q, kv_pool=pool, layer=layer, block_table=d_table, cu_rows=cu, kv_lens=d_lens, out=out,
                                    out_lse=lse, scale=scale, window=window, max_new=max_new, max_keys=max_keys, err_word=err)
    nbytes = mtp.mtp_chunk_attention_workspace_bytes(args)
    if workspace is None:
        workspace = torch.full((max(16, nbytes),), 255, dtype=torch.uint8, device="cuda")  # any content (here NaN)
    torch.cuda.synchronize()
    mtp.mtp_chunk_attention(args, workspace, nbytes, stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert int(err) == 0
    ref, want_lse, size, total = reference(torch, q[:live], pool, layer, table, new, lens, scale, window)
    u = 2.0 ** -8 if dtype == "bfloat16" else 2.0 ** -11
    once = u if max_new * (heads // kv_heads) > 32 else 0.0  # (the header: max_new chooses the kernel)
    bound = u * ref.abs() + (once + 2.0 ** -14) * size + (2.0 ** -25 * total + 2.0 ** -25 if dtype == "float16" else 1e-30)
    off = (out[:live].double() - ref).abs()
    assert bool(out[:live].isfinite().all())
    assert bool((off <= bound).all()), f"{(off - bound).max().item()} over its bound, {int((off > bound).sum())} values"
    none = want_lse == -float("inf")
    assert torch.equal(lse[:live] == -float("inf"), none)
    assert bool((out[:live][none] == 0).all())
    off = (lse[:live].double() - want_lse)[~none].abs()
    assert bool((off <= 4e-5 + 2.0 ** -22 * want_lse[~none].abs()).all()), off.max().item()
    assert bool((out[live:] == -7).all()) and bool((lse[live:] == -7).all())
    return out, lse


@pytest.mark.parametrize("dtype,u", [("bfloat16", 2.0 ** -8), ("float16", 2.0 ** -11)])
def test_unit_roundoff(dtype, u):
    """The largest relative error of rounding to the type is u, just above a power of two."""
    torch = pytest.importorskip("torch")
    x = torch.linspace(1.0, 2.0, 100001, dtype=torch.float64)
    worst = ((x.to(getattr(torch, dtype)).double() - x).abs() / x).max().item()
    assert 0.95 * u < worst <= u


SHAPES = [(1, 1, 64), (16, 16, 64), (4, 1, 128), (8, 2, 64), (5, 1, 128), (32, 8, 128), (16, 1, 64)]


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,kv_heads,dim", SHAPES)
@pytest.mark.parametrize("page", [16, 32, 64, 128])
def test_decoding_steps(heads, kv_heads, dim, page, dtype):
    """One token a slot: lengths of one, around pages and units, and long ones."""
    check([1] * 12, [1, 2, 15, 16, 17, 63, 64, 65, 127, 129, 1000, 5000], heads, kv_heads, dim, page, dtype)


@pytest.mark.parametrize("new", [1, 2, 3, 5, 8, 17])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 64), (8, 2, 128), (6, 2, 64)])
def test_drafts(heads, kv_heads, dim, new):
    """A few new tokens a slot: the causal edge inside a unit, slots without tokens, a slot that holds nothing else."""
    for lens in ([new, 64 + new, 63 + new, 129, 700, 64], [new] * 6):
        tokens = [new, new, 0, max(1, new - 1), new, new] if new <= 64 else [new] * 6
        check(tokens, lens, heads, kv_heads, dim, 16, seed=new)


@pytest.mark.parametrize("dtype", ["bfloat16", "float16"])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 64), (4, 1, 128), (16, 2, 64), (3, 1, 128)])
@pytest.mark.parametrize("page", [16, 64, 128])
def test_chunks(heads, kv_heads, dim, page, dtype):
    """Prompts from nothing and chunks behind cached tokens, of ragged sizes around tiles and units."""
    check([33, 1, 127, 128, 129, 256, 257, 0, 500], [33, 300, 127, 700, 129, 256, 1257, 40, 513], heads, kv_heads, dim, page, dtype)


def test_a_long_chunk_and_a_long_context():
    check([2500], [2500], 4, 2, 128, 64)
    check([700, 1, 90], [9000, 12000, 90], 8, 2, 64, 32, "float16")


@pytest.mark.parametrize("window", [1, 2, 16, 63, 64, 65, 200, 4000])
@pytest.mark.parametrize("new,lens", [([1, 1, 1, 4], [1, 300, 64, 2000]), ([300, 40, 1], [300, 500, 1500])])
def test_windows(window, new, lens):
    check(new, lens, 4, 2, 64, 16, window=window)
    check(new, lens, 4, 1, 128, 64, "float16", window=window)


def test_rows_that_see_no_key():
    """More rows than the slot has tokens: the first of them are at positions below 0."""
    check([5, 3, 1], [2, 3, 0], 4, 2, 64, 16)
    check([300, 5], [100, 0], 2, 1, 128, 16)


@pytest.mark.parametrize("layout", ["fused", "odd", "shifted"])
@pytest.mark.parametrize("new", [1, 4, 150])
def test_rows_at_any_stride_and_alignment(layout, new):
    check([new, new], [200, 333], 4, 2, 64, 16, layout=layout)
    check([new, new], [200, 333], 4, 4, 128, 32, layout=layout, dtype="float16")


@pytest.mark.parametrize("new", [1, 200])
def test_peaked_and_flat_scores(new):
    for spread in (0.0, 30.0):
        check([new], [1500], 4, 4, 64, 64, spread=spread)
    check([new], [1500], 4, 4, 64, 64, scale=1e-3)


def test_many_slots():
    check([1] * 700, [1 + 7 * i % 400 for i in range(700)], 2, 1, 64, 16)
    check([1 + i % 9 for i in range(300)], [10 + 13 * i % 300 for i in range(300)], 4, 1, 64, 32)


def test_hints_may_be_generous():
    for hints in ((1, 100000), (8, 300), (64, 20000), (1000, 1 << 20)):
        check([1, 1, 1], [300, 20, 299], 4, 2, 64, 16, hints=hints, rows_past=1200)


@pytest.mark.parametrize("new", [1, 300])
def test_the_same_call_gives_the_same_bits(new):
    torch = pytest.importorskip("torch")
    a = check([new] * 5, [3000, 2500, 400, 1000, 301], 8, 2, 64, 16)
    for _ in range(3):
        b = check([new] * 5, [3000, 2500, 400, 1000, 301], 8, 2, 64, 16)
        assert torch.equal(a[0], b[0]) and torch.equal(a[1], b[1])


def test_another_stream_and_one_workspace():
    torch = pytest.importorskip("torch")
    stream = torch.cuda.Stream()
    ws = torch.full((128 << 20,), 255, dtype=torch.uint8, device="cuda")
    for new, lens in (([1, 1], [900, 4000]), ([400], [600]), ([3] * 40, [500] * 40), ([1], [1])):
        check(new, lens, 8, 2, 128, 64, stream=stream, workspace=ws)


@pytest.mark.parametrize("new", [1, 140])
def test_a_cache_past_32_bits(new):
    """Element offsets above 2^32: a pool of 8 GB whose last pages are used."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    pool = torch.zeros(4200, 8, 2, 8, 128, 64, dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 1 << 32
    torch.manual_seed(1)
    kv = torch.randn(3, 2, 8, 128, 64, device="cuda").bfloat16()
    pages = [4199, 4100, 4198]
    pool[pages, 7] = kv
    q = torch.randn(new, 8, 64, device="cuda").bfloat16()
    out, lse = torch.zeros_like(q), torch.zeros(new, 8, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    table, cu, lens = ints([pages]), ints([0, new]), ints([300])
    args = mtp.chunk_attention_args(q=q, kv_pool=pool, layer=7, block_table=table, cu_rows=cu, kv_lens=lens, out=out,
                                    out_lse=lse, scale=0.125, max_new=new, max_keys=300)
    n = mtp.mtp_chunk_attention_workspace_bytes(args)
    mtp.mtp_chunk_attention(args, torch.empty(n, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream())
    k, v = (kv[:, i].transpose(0, 1).flatten(1, 2)[:, :300].double() for i in (0, 1))
    x = torch.einsum("rhd,hkd->hrk", q.double(), k) * 0.125
    x = x.masked_fill(torch.arange(300, device="cuda") > 300 - new + torch.arange(new, device="cuda")[:, None], -float("inf"))
    ref = torch.einsum("hrk,hkd->rhd", torch.softmax(x, -1), v)
    assert bool(((out.double() - ref).abs() <= 2.0 ** -9 * ref.abs() + (2.0 ** -9 + 2.0 ** -14) * 5).all())
    assert bool(((lse.double() - torch.logsumexp(x, -1).T).abs() <= 4e-5).all())
    assert float((out.double() - ref).norm() / ref.norm()) < 2.0 ** -8


@pytest.mark.parametrize("kw", [dict(q=None), dict(kv_pool=None), dict(block_table=None), dict(cu_rows=None), dict(kv_lens=None),
                                dict(out=None), dict(kv_pool=(1 << 20) + 8), dict(q=(1 << 20) + 1), dict(out=(1 << 20) + 1),
                                dict(q_stride=255), dict(out_stride=0), dict(slots=4000, rows=1 << 20, max_new=300)])
def test_refusals_behind_the_device_query(kw):
    """Checked once the number of SMs is known; the addresses are never followed."""
    from test_paged_refusals import A, _chunk, _refused
    lib_module()
    _refused(lambda mtp: mtp.mtp_chunk_attention(_chunk(**kw), A, 1 << 40))


def test_workspace_and_empty_calls():
    from test_paged_refusals import A, _chunk, _refused
    mtp = lib_module()
    need = mtp.mtp_chunk_attention_workspace_bytes(_chunk())
    assert need > 0
    for ws, n in ((None, need), (A, need - 1), (A + 8, need)):
        _refused(lambda m: m.mtp_chunk_attention(_chunk(), ws, n))
    mtp.mtp_chunk_attention(_chunk(rows=0), None, 0)
    mtp.mtp_chunk_attention(_chunk(max_new=0), None, 0)


@pytest.mark.parametrize("new,lens", [([1, 3], [700, 900]), ([150, 40], [300, 2000])])
def test_captured_in_a_graph(new, lens):
    """A plan, an append and the attention of a step as one graph: replays follow the buffers' contents."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    heads, kv_heads, dim, page, slots = 4, 2, 64, 16, len(new)
    gen = torch.Generator(device="cuda").manual_seed(3)
    stride, rows = -(-max(lens) // page), sum(new)
    n_pages = slots * stride + 5
    i32 = dict(dtype=torch.int32, device="cuda")
    pool = torch.randn(n_pages, 1, 2, kv_heads, page, dim, device="cuda", generator=gen).bfloat16()
    before = [n - a for n, a in zip(lens, new)]
    pages = torch.randperm(n_pages).tolist()
    table = [[pages.pop() for _ in range(-(-n // page))] for n in before]
    refs = torch.zeros(n_pages, **i32)
    refs[[p for t in table for p in t]] = 1
    d_table = torch.tensor([t + [-1] * (stride - len(t)) for t in table], **i32)
    d_new, d_before = torch.tensor(new, **i32), torch.tensor(before, **i32)
    cu, d_lens, out_refs, status = torch.zeros(slots + 1, **i32), torch.zeros(slots, **i32), torch.zeros(n_pages, **i32), torch.zeros(4, **i32)
    seq, pos, places = torch.zeros(rows, **i32), torch.zeros(rows, **i32), torch.zeros(rows, dtype=torch.int64, device="cuda")
    x = torch.randn(rows, heads + 2 * kv_heads, dim, device="cuda", generator=gen).bfloat16()
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    out, lse = torch.zeros(rows, heads, dim, dtype=torch.bfloat16, device="cuda"), torch.zeros(rows, heads, device="cuda")
    plan = mtp.page_plan_args(kv_lens=d_before, new_lens=d_new, block_table=d_table, page_refs=refs, out_kv_lens=d_lens,
                              out_page_refs=out_refs, out_cu_rows=cu, out_slot_map=places, out_row_seq=seq, out_row_pos=pos,
                              out_status=status, page_size=page)
    append = mtp.cache_append_args(k=k, v=v, slot_map=places, kv_pool=pool, layer=0)
    attend = mtp.chunk_attention_args(q=q, kv_pool=pool, layer=0, block_table=d_table, cu_rows=cu, kv_lens=d_lens, out=out,
                                      out_lse=lse, scale=0.125, max_new=max(new), max_keys=max(lens))
    n = mtp.mtp_chunk_attention_workspace_bytes(attend)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")

    def step():
        stream = torch.cuda.current_stream()
        mtp.mtp_page_plan(plan, stream)
        mtp.mtp_cache_append(append, stream)
        mtp.mtp_chunk_attention(attend, ws, n, stream)
    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for _ in range(3):
        x.normal_(generator=gen)
        graph.replay()
        torch.cuda.synchronize()
        assert status[0] == 0 and d_lens.tolist() == lens
        ref, want, size, total = reference(torch, q, pool, 0, d_table.tolist(), new, lens, 0.125, 0)
        assert bool(((out.double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -14) * size).all())
        assert bool(((lse.double() - want).abs() <= 4e-5 + 2.0 ** -22 * want.abs()).all())


@pytest.mark.parametrize("heads,kv_heads,dim", [(4, 2, 64), (5, 1, 128), (8, 2, 128)])
def test_query_rows_past_the_last_may_be_anything(heads, kv_heads, dim):
    """Rows of the buffer that belong to no slot, NaN here, share tiles with the last slot's: they leave no trace."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    page, n, length, rows = 16, 70, 200, 90
    i32 = dict(dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(5)
    pool = torch.randn(20, 1, 2, kv_heads, page, dim, device="cuda", generator=gen).bfloat16()
    q = torch.randn(rows, heads, dim, device="cuda", generator=gen).bfloat16()
    q[n:] = NAN
    out, lse = torch.full_like(q, -7.0), torch.full((rows, heads), -7.0, device="cuda")
    args = mtp.chunk_attention_args(q=q, kv_pool=pool, layer=0, block_table=torch.arange(13, **i32)[None].contiguous(),
                                    cu_rows=torch.tensor([0, n], **i32), kv_lens=torch.tensor([length], **i32), out=out,
                                    out_lse=lse, scale=dim ** -0.5, max_new=n, max_keys=length)
    nbytes = mtp.mtp_chunk_attention_workspace_bytes(args)
    mtp.mtp_chunk_attention(args, torch.zeros(nbytes, dtype=torch.uint8, device="cuda"), nbytes, torch.cuda.current_stream())
    ref, want, size, _ = reference(torch, q[:n], pool, 0, [list(range(13))], [n], [length], dim ** -0.5, 0)
    assert bool(((out[:n].double() - ref).abs() <= 2.0 ** -8 * ref.abs() + (2.0 ** -8 + 2.0 ** -14) * size).all())
    assert bool(((lse[:n].double() - want).abs() <= 4e-5 + 2.0 ** -22 * want.abs()).all())
    assert bool((out[n:] == -7).all()) and bool((lse[n:] == -7).all())


def test_tokens_of_one_slot_in_every_size():
    """One to 300 tokens behind a short context: every filling of a tile, both kernels, both tiles of a CTA."""
    for n in list(range(1, 40)) + list(range(60, 70)) + list(range(120, 136)) + list(range(250, 262)) + [300]:
        check([n], [n + 5], 2, 1, 128 if n % 2 else 64, 16, seed=n)


@pytest.mark.parametrize("window", [(1 << 24) + 1, (1 << 30), (1 << 31) - 3, (1 << 31) - 1])
def test_windows_longer_than_any_table(window):
    """Such a window leaves nothing out, at positions below 0 too."""
    for new, lens in (([5, 3, 1], [2, 3, 0]), ([4, 1], [300, 64]), ([300, 5, 40], [100, 0, 700])):
        check(new, lens, 4, 2, 64, 16, window=window)
        check(new, lens, 4, 1, 128, 16, "float16", window=window)


def _call(torch, mtp, heads, kv_heads, dim, page, new, lens, rows, stride, max_new, window=0, claimed=None):
    """Attention of `rows` buffer rows of slots with `new` tokens each, whose lengths are given as `claimed`; the inputs, out,
    lse and the error word."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    counts = [-(-n // page) for n in lens]
    pages = torch.randperm(sum(counts) + 1).tolist()
    table = [[pages.pop() for _ in range(c)] + [-1] * (stride - c) for c in counts]
    pool = torch.randn(sum(counts) + 1, 1, 2, kv_heads, page, dim, device="cuda", generator=gen).bfloat16()
    q = torch.randn(rows, heads, dim, device="cuda", generator=gen).bfloat16()
    out, lse = torch.full_like(q, -7.0), torch.full((rows, heads), -7.0, device="cuda")
    ints = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    err, cu, d_lens, d_table = ints([0]), ints([sum(new[:i]) for i in range(len(new) + 1)]), ints(claimed or lens), ints(table)
    args = mtp.chunk_attention_args(q=q, kv_pool=pool, layer=0, block_table=d_table, cu_rows=cu, kv_lens=d_lens, out=out, out_lse=lse,
                                    scale=dim ** -0.5, window=window, max_new=max_new, max_keys=max(lens), err_word=err)
    n = mtp.mtp_chunk_attention_workspace_bytes(args)
    mtp.mtp_chunk_attention(args, torch.full((n,), 255, dtype=torch.uint8, device="cuda"), n, torch.cuda.current_stream())
    torch.cuda.synchronize()
    return q, pool, table, out, lse, int(err)


def _right(torch, out, lse, ref):
    """Within the bounds above, weights rounded once."""
    want, want_lse, size, _ = ref
    assert bool(((out.double() - want).abs() <= 2.0 ** -8 * want.abs() + (2.0 ** -8 + 2.0 ** -14) * size).all())
    none = want_lse == -float("inf")
    assert torch.equal(lse == -float("inf"), none)
    assert bool(((lse.double() - want_lse)[~none].abs() <= 4e-5 + 2.0 ** -22 * want_lse[~none].abs()).all())


BOUNDS = 2  # MTP_DEVICE_ERR_BOUNDS


@pytest.mark.parametrize("window", [0, 9])
@pytest.mark.parametrize("heads,kv_heads,dim", [(2, 2, 64), (4, 2, 128)])
@pytest.mark.parametrize("new,lens,rows", [([3, 6], [20, 50], 5), ([3, 6, 4], [20, 50, 4], 5), ([40, 300], [60, 900], 200),
                                           ([1] * 150 + [7], [5] * 150 + [90], 153),
                                           ([1] * 200, [9] * 200, 40), ([130] * 5, [200] * 5, 131)])
def test_rows_past_the_buffers(new, lens, rows, heads, kv_heads, dim, window):
    """Row starts that pass the buffers' rows: what lies in the buffers keeps its position, and the error word says that
    rows are missing."""
    torch = pytest.importorskip("torch")
    q, pool, table, out, lse, err = _call(torch, lib_module(), heads, kv_heads, dim, 16, new, lens, rows, 60, max(new), window)
    all_q = torch.cat([q, torch.zeros(sum(new) - rows, heads, dim, device="cuda", dtype=q.dtype)])
    _right(torch, out, lse, [x[:rows] for x in reference(torch, all_q, pool, 0, table, new, lens, dim ** -0.5, window)])
    assert err == BOUNDS


@pytest.mark.parametrize("new", [2, 90])
@pytest.mark.parametrize("wrong", [-1, -(1 << 31), 4 * 16 + 1, (1 << 31) - 1])
def test_lengths_outside_the_table(wrong, new):
    """A slot whose length is negative or longer than its table sees no key, and the error word says so; the others are
    computed."""
    torch = pytest.importorskip("torch")
    stride = 4 if new < 60 else 8
    wrong = wrong + 64 if stride == 8 and wrong == 65 else wrong
    lens = [stride * 16, stride * 16 - 3, new]
    q, pool, table, out, lse, err = _call(torch, lib_module(), 2, 1, 64, 16, [new] * 3, lens, 3 * new, stride, new,
                                          claimed=[lens[0], wrong, lens[2]])
    ref = reference(torch, q, pool, 0, table, [new] * 3, lens, 0.125, 0)
    for x in ref[:1] + ref[2:]:
        x[new:2 * new] = 0.0
    ref[1][new:2 * new] = -float("inf")
    _right(torch, out, lse, ref)
    assert bool((out[new:2 * new] == 0).all()) and err == BOUNDS


def test_the_length_of_a_slot_without_new_tokens_may_be_anything():
    torch = pytest.importorskip("torch")
    for new in ([3, 0, 2], [2, 0, 90], [1, 0] * 100):
        lens = [max(1, 3 * n) for n in new]
        q, pool, table, out, lse, err = _call(torch, lib_module(), 2, 1, 64, 16, new, lens, sum(new), 20, max(new),
                                              claimed=[n if a else (-5 if i % 4 == 1 else 1 << 30) for i, (n, a) in enumerate(zip(lens, new))])
        _right(torch, out, lse, reference(torch, q, pool, 0, table, new, lens, 0.125, 0))
        assert err == 0


def test_row_starts_that_descend():
    torch = pytest.importorskip("torch")
    q, pool, table, out, lse, err = _call(torch, lib_module(), 2, 1, 64, 16, [4, -2], [30, 20], 4, 4, 4)
    _right(torch, out, lse, reference(torch, q, pool, 0, table, [4], [30], 0.125, 0))
    assert err == BOUNDS


@pytest.mark.parametrize("new,max_new,slots", [(20, 1, 3), (20, 8, 200), (300, 17, 2)])
def test_more_tokens_than_the_bound(new, max_new, slots):
    """Rows that a wrong max_new leaves out are reported."""
    torch = pytest.importorskip("torch")
    assert _call(torch, lib_module(), 2, 2, 64, 16, [new] * slots, [new + 1] * slots, new * slots, 20, max_new)[5] == BOUNDS
