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
