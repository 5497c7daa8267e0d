"""mtp_page_plan against a plain allocator that takes one request at a time: whole numbers, equal exactly."""
import random

import pytest

import paged_util
from gpu_util import lib_module

pytestmark = pytest.mark.gpu


def _run(lens, new, table, refs, page, max_rows, in_place=False):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    i32 = lambda *n: torch.full(n, -77, dtype=torch.int32, device="cuda")  # noqa: E731
    d = dict(kv_lens=t(lens), new_lens=t(new), block_table=t(table), page_refs=t(refs))
    out = dict(out_kv_lens=d["kv_lens"] if in_place else i32(len(lens)),
               out_page_refs=d["page_refs"] if in_place else i32(len(refs)), out_cu_rows=i32(len(lens) + 1),
               out_slot_map=torch.full((max_rows,), -77, dtype=torch.int64, device="cuda"),
               out_row_seq=i32(max_rows), out_row_pos=i32(max_rows), out_status=i32(4))
    mtp.mtp_page_plan(mtp.page_plan_args(**d, **out, page_size=page), torch.cuda.current_stream())
    if not in_place:
        assert d["kv_lens"].tolist() == lens and d["page_refs"].tolist() == refs
    assert d["new_lens"].tolist() == new
    return (out["out_kv_lens"].tolist(), d["block_table"].tolist(), out["out_page_refs"].tolist(),
            out["out_cu_rows"].tolist(), out["out_slot_map"].tolist(), out["out_row_seq"].tolist(),
            out["out_row_pos"].tolist(), out["out_status"].tolist())


def _state(seed, slots, page, len_hi, new_hi, n_pages):
    rng = random.Random(seed)
    lens = [rng.choice([0, page, rng.randint(0, len_hi)]) if len_hi >= page else rng.randint(0, len_hi)
            for _ in range(slots)]
    new = [rng.choice([0, new_hi, rng.randint(0, new_hi)]) for _ in range(slots)]
    stride = -(-(max(page, len_hi) + new_hi) // page) + 1
    counts = [-(-n // page) for n in lens]
    order = iter(rng.sample(range(n_pages), sum(counts)))
    table = [[next(order) for _ in range(c)] + [-1] * (stride - c) for c in counts]
    refs = [0] * n_pages
    for r in table:
        for p in r:
            if p >= 0:
                refs[p] = rng.randint(1, 3)
    return lens, new, table, refs


def _same(got, want):
    for name, g, w in zip(("lens", "table", "refs", "cu_rows", "slot_map", "row_seq", "row_pos", "status"), got, want):
        assert g == w, name


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("slots,page,len_hi,new_hi,n_pages", [
    (1, 16, 0, 1, 1), (1, 64, 0, 700, 40), (2, 16, 40, 0, 9), (7, 128, 300, 130, 64), (32, 64, 2000, 1, 1100),
    (33, 32, 100, 33, 257), (1000, 16, 50, 9, 6000), (1024, 64, 64, 2, 4096), (1025, 16, 16, 17, 4999),
    (3000, 16, 31, 1, 33000), (8192, 128, 10, 1, 20001), (5, 16, 100, 3000, 300007)])
def test_plan_equals_the_plain_allocator(slots, page, len_hi, new_hi, n_pages, in_place):
    lens, new, table, refs = _state(slots * 7 + page, slots, page, len_hi, new_hi, n_pages)
    rows = sum(new)
    for max_rows in (rows, rows + 777):
        _same(_run(lens, new, table, refs, page, max_rows, in_place),
              paged_util.plan(lens, new, table, refs, page, max_rows))


def test_rows_past_one_launch():
    lens, new, table, refs = _state(5, 900, 16, 200, 400, 60000)
    _same(_run(lens, new, table, refs, 16, 900 * 400), paged_util.plan(lens, new, table, refs, 16, 900 * 400))


def test_all_or_nothing_when_pages_run_out():
    lens, new, table, refs = _state(3, 40, 16, 100, 50, 700)
    want = paged_util.plan(lens, new, table, refs, 16, 4000)
    need, spare = want[7][2], want[7][3]
    assert need > 1
    for keep in (need, need - 1, 0):  # as many free pages as needed, one fewer, none
        less = list(refs)
        for p in paged_util.free_pages(refs)[keep:]:
            less[p] = 1
        got = _run(lens, new, table, less, 16, 4000)
        _same(got, paged_util.plan(lens, new, table, less, 16, 4000))
        assert got[7][0] == (0 if keep == need else -2)
    assert spare > 0


@pytest.mark.parametrize("what", ["negative length", "negative count", "table too narrow", "too many rows", "far too many rows"])
def test_invalid_requests_change_nothing(what):
    lens, new, table, refs = _state(4, 20, 32, 90, 40, 400)
    max_rows = 20 * 40
    if what == "negative length":
        lens[7] = -1
    elif what == "negative count":
        new[19] = -3
    elif what == "table too narrow":
        new[0] = len(table[0]) * 32 - lens[0] + 1
        max_rows += new[0]
    elif what == "too many rows":
        max_rows = sum(new) - 1
    else:
        table, lens, new = [[-1] * (1 << 12)] * 8192, [0] * 8192, [1 << 17] * 8192  # 2^30 rows
        max_rows = 100
    got = _run(lens, new, table, refs, 32, max_rows)
    _same(got, paged_util.plan(lens, new, table, refs, 32, max_rows))
    assert got[7][0] == -1 and got[0] == lens


def test_a_foreign_page_has_no_place():
    """Positions on table entries outside the pool, which the caller left there, get no place."""
    got = _run([20, 5], [3, 2], [[0, -1, -1], [99, -1, -1]], [1, 0, 0, 0], 16, 6)
    _same(got, paged_util.plan([20, 5], [3, 2], [[0, -1, -1], [99, -1, -1]], [1, 0, 0, 0], 16, 6))
    assert got[4][:3] == [-1] * 3 and got[4][3:] == [-1, -1, -1]
