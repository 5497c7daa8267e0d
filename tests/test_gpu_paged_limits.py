"""The paged operators at sizes where a launch's shared memory or a limit of theirs is at its edge."""
import os
import random
import subprocess
import sys

import pytest

import paged_util
import test_gpu_beam_reorder as reorder
import test_gpu_page_plan as plan
from gpu_util import lib_module

pytestmark = pytest.mark.gpu


def _alone(call):
    """`call`, a function of this file by name, in a process of its own: what a larger call of the same kernel set up
    before would hide a launch that is refused."""
    lib_module()
    here = os.path.dirname(os.path.abspath(__file__))
    run = subprocess.run([sys.executable, "-c", f"import test_gpu_paged_limits as t; t.{call}"], cwd=here, capture_output=True,
                         text=True, timeout=300, env={**os.environ, "PYTHONPATH": os.pathsep.join([here, os.path.dirname(here)])})
    assert run.returncode == 0, run.stderr[-2000:]


def plan_case(slots, n_pages, page=16, len_hi=40, new_hi=2):
    lens, new, table, refs = plan._state(slots, slots, page, len_hi, new_hi, n_pages)
    max_rows = sum(new) + 5
    plan._same(plan._run(lens, new, table, refs, page, max_rows), paged_util.plan(lens, new, table, refs, page, max_rows))


def reorder_case(batch, beams, n_pages, **kw):
    table, lens, refs = paged_util.beams_state(batch, batch, beams, 16, 1, 20, 0)
    refs += [0] * (n_pages - len(refs))
    rng = random.Random(beams)
    parent = [[rng.randrange(beams) for _ in range(beams)] for _ in range(batch)]
    assert len(refs) == n_pages
    assert reorder._check(parent, table, lens, refs, 16, layers=1, heads=1, dim=8, **kw)[0] == 0


# dynamic shared memory at most 48 KB, with the kernel's static part more: 48952, 49032, 48856, 48832 bytes and 528
@pytest.mark.parametrize("slots,n_pages", [(4000, 30000), (4000, 32768), (3900, 65536), (32, 1550000)])
def test_plan_just_below_48_kb(slots, n_pages):
    _alone(f"plan_case({slots}, {n_pages})")


# 49044, 49092 and 49148 bytes and 144
@pytest.mark.parametrize("batch,beams,n_pages", [(500, 8, 33280), (480, 8, 96256), (512, 7, 196352)])
def test_reorder_just_below_48_kb(batch, beams, n_pages):
    _alone(f"reorder_case({batch}, {beams}, {n_pages})")


def test_plan_of_the_most_pages_and_slots():
    plan_case(8192, 1 << 22)


def test_reorder_of_the_most_pages_and_beams():
    reorder_case(128, 64, 1 << 22)


def test_reorder_of_the_most_table_entries():
    """8192 tables of 131072 entries, one item's beams full to the last: equal to the same in torch."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    batch, beams, page, stride = 128, 64, 16, 1 << 17
    rows = batch * beams
    i32 = dict(dtype=torch.int32, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(2)
    used = torch.randint(0, 4, (batch,), generator=torch.Generator().manual_seed(1))  # full pages: nothing is copied
    used[-1] = stride
    n_pages = stride + 3 * (batch - 1) * beams + 7
    order = torch.randperm(n_pages, device="cuda", generator=gen)
    table = torch.full((rows, stride), 1 << 30, **i32)
    at = stride
    for r in range(rows - beams):
        n = int(used[r // beams])
        table[r, :n] = order[at:at + n].int()
        at += n
    table[-beams:] = order[:stride].int()  # a context that the last item's beams share
    lens = (used.repeat_interleave(beams) * page).int().cuda()
    refs = torch.zeros(n_pages, **i32)
    refs[order[stride:at]] = 1
    refs[order[:stride]] = beams
    parent = torch.randint(-1, beams, (batch, beams), device="cuda", generator=gen).int()
    src = torch.arange(batch, device="cuda")[:, None] * beams + parent
    gone = (parent < 0).flatten()
    pool = torch.zeros(n_pages, 1, 2, 1, page, 8, dtype=torch.bfloat16, device="cuda")
    out_table, out_lens, out_refs, status = torch.full_like(table, -9), torch.empty_like(lens), torch.empty_like(refs), torch.empty(4, **i32)
    args = mtp.beam_reorder_args(parent=parent, block_table=table, kv_lens=lens, page_refs=refs, kv_pool=pool,
                                 out_block_table=out_table, out_kv_lens=out_lens, out_page_refs=out_refs, out_status=status)
    nbytes = mtp.mtp_beam_reorder_workspace_bytes(args)
    mtp.mtp_beam_reorder(args, torch.empty(nbytes, dtype=torch.uint8, device="cuda"), nbytes, torch.cuda.current_stream())
    want_lens = torch.where(gone, 0, lens[src.flatten().clamp(min=0)])
    assert torch.equal(out_lens, want_lens)
    want_refs = torch.zeros(n_pages, dtype=torch.int64, device="cuda")
    one = torch.ones(stride, dtype=torch.int64, device="cuda")
    for r in range(rows):
        n = int(want_lens[r]) // page
        if n < stride:
            assert bool((out_table[r, n:] == -1).all())
        if n:
            held = table[int(src.flatten()[r]), :n]
            assert torch.equal(out_table[r, :n], held)
            want_refs.index_add_(0, held.long(), one[:n])
    assert torch.equal(out_refs.long(), want_refs)
    assert status.tolist() == [0, 0, int((want_refs == 0).sum()), 0]
