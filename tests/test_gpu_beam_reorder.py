"""mtp_beam_reorder against a plain reordering, one beam at a time: whole numbers and copied rows, equal exactly."""
import random

import pytest

import paged_util
from gpu_util import lib_module

pytestmark = pytest.mark.gpu


def _check(parent, table, lens, refs, page, layers=2, heads=3, dim=64, dtype="bfloat16", in_place=False, seed=1):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    t = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")  # noqa: E731
    gen = torch.Generator(device="cuda").manual_seed(seed)
    pool = torch.randn(len(refs), layers, 2, heads, page, dim, device="cuda", generator=gen).to(getattr(torch, dtype))
    if len(refs) > 2:
        pool[1].fill_(float("nan"))  # whatever a page holds is copied or left
    before = pool.clone()
    d_table, d_lens, d_refs = t(table), t(lens), t(refs)
    out_table, out_lens, status = t(table) * 0 - 9, t(lens) * 0 - 9, t([-9] * 4)
    out_refs = d_refs if in_place else t(refs) * 0 - 9
    args = mtp.beam_reorder_args(parent=t(parent), block_table=d_table, kv_lens=d_lens, page_refs=d_refs, kv_pool=pool,
                                 out_block_table=out_table, out_kv_lens=out_lens, out_page_refs=out_refs,
                                 out_status=status)
    nbytes = mtp.mtp_beam_reorder_workspace_bytes(args)
    mtp.mtp_beam_reorder(args, torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes, torch.cuda.current_stream())
    new_table, new_lens, new_refs, copies, want_status = paged_util.reorder(parent, table, lens, refs, page)
    assert status.tolist() == want_status
    assert out_table.tolist() == new_table
    assert out_lens.tolist() == new_lens
    assert out_refs.tolist() == new_refs
    assert d_table.tolist() == table and d_lens.tolist() == lens
    for a, b, n in copies:
        before[b, :, :, :, :n] = before[a, :, :, :, :n]
    assert torch.equal(pool.view(torch.int16), before.view(torch.int16))
    return want_status


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("batch,beams,page,lo,hi", [
    (1, 1, 16, 5, 5), (1, 2, 16, 0, 40), (1, 4, 64, 64, 64), (3, 5, 32, 1, 200), (12, 8, 64, 200, 800),
    (40, 8, 16, 0, 33), (200, 6, 128, 1, 300), (128, 64, 16, 0, 20), (2, 64, 64, 100, 400)])
def test_kept_beams(batch, beams, page, lo, hi, in_place):
    table, lens, refs = paged_util.beams_state(batch + beams, batch, beams, page, lo, hi, batch * beams + 3)
    rng = random.Random(batch)
    for kind in ("any", "first", "itself", "some end"):
        parent = [[{"any": rng.randrange(beams), "first": 0, "itself": j,
                    "some end": rng.choice([-1, rng.randrange(beams)])}[kind] for j in range(beams)] for _ in range(batch)]
        assert _check(parent, table, lens, refs, page, in_place=in_place)[0] == 0


@pytest.mark.parametrize("heads,dim,layers,dtype", [(1, 8, 1, "float16"), (16, 64, 12, "bfloat16"), (8, 128, 3, "float16"),
                                                    (2, 256, 1, "bfloat16")])
def test_copied_rows_of_every_shape(heads, dim, layers, dtype):
    table, lens, refs = paged_util.beams_state(9, 3, 4, 32, 10, 90, 13)
    _check([[1, 1, 1, 0]] * 3, table, lens, refs, 32, layers, heads, dim, dtype)


def test_lengths_differ_between_the_beams_of_an_item():
    table, lens, refs = paged_util.beams_state(2, 4, 4, 16, 17, 60, 20)
    for r in range(1, 16, 4):  # a shorter beam gives its pages back first
        cut = 3 if lens[r] > 3 else 0
        for p in table[r][-(-cut // 16):-(-lens[r] // 16)]:
            refs[p] -= 1
        lens[r] = cut
    _check([[1, 1, 0, 3]] * 4, table, lens, refs, 16)


def test_all_or_nothing_when_pages_run_out():
    table, lens, refs = paged_util.beams_state(3, 5, 4, 32, 33, 63, 12)  # every copy needed: 15
    assert _check([[2] * 4] * 5, table, lens, refs, 32)[0] == -2
    table, lens, refs = paged_util.beams_state(3, 5, 4, 32, 33, 63, 15)
    assert _check([[2] * 4] * 5, table, lens, refs, 32)[:2] == [0, 15]


@pytest.mark.parametrize("what", ["parent", "length", "negative length", "page", "count"])
def test_invalid_states_change_nothing(what):
    table, lens, refs = paged_util.beams_state(6, 6, 3, 16, 20, 90, 30)
    parent = [[0, 0, 2] for _ in range(6)]
    if what == "parent":
        parent[5][2] = 3
    elif what == "length":
        lens[4] = len(table[0]) * 16 + 1
    elif what == "negative length":
        lens[17] = -1
    elif what == "page":
        table[3][0] = len(refs)
    else:
        refs[table[7][1]] = 0
    assert _check(parent, table, lens, refs, 16)[0] == -1


def test_steps_in_turn_keep_the_counts():
    """Ten reorderings in a row: a page's count stays the number of tables that hold it."""
    rng = random.Random(4)
    table, lens, refs = paged_util.beams_state(4, 5, 4, 16, 20, 100, 40)
    for _ in range(10):
        parent = [[rng.randrange(4) for _ in range(4)] for _ in range(5)]
        assert _check(parent, table, lens, refs, 16)[0] == 0
        table, lens, refs, _, _ = paged_util.reorder(parent, table, lens, refs, 16)
        held = [0] * len(refs)
        for r in table:
            for p in r:
                if p >= 0:
                    held[p] += 1
        assert held == refs


def test_steps_in_turn_by_eight_ctas():
    """The same where eight CTAs share the tables, and beams of uneven lengths, some of which end, free their pages."""
    rng = random.Random(8)
    batch, beams = 60, 5
    table, lens, refs = paged_util.beams_state(8, batch, beams, 16, 1, 150, 400)
    for _ in range(4):
        parent = [[rng.choice([-1, rng.randrange(beams), rng.randrange(beams), 0]) for _ in range(beams)] for _ in range(batch)]
        assert _check(parent, table, lens, refs, 16, layers=1, heads=1, dim=8)[0] == 0
        table, lens, refs, _, _ = paged_util.reorder(parent, table, lens, refs, 16)
        held = [0] * len(refs)
        for r in table:
            for p in r:
                if p >= 0:
                    held[p] += 1
        assert held == refs
