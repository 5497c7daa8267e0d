"""mtp_beam_select against a stable sort of the same fp32 scores: beams, tokens, scores and ends are equal exactly.
A computed log-sum-exp is compared with 64 bits, and the selection then checked on the log-sum-exp that it gives."""
import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu


def _expected(torch, logits, lse, scores, done, eos, k):
    """On the CPU: one fp32 subtraction and one addition, then a stable sort."""
    x, lse, scores = logits.float().cpu(), lse.cpu(), scores.cpu()
    b, w, v = x.shape
    s = scores[..., None] + (x - lse[..., None])
    s = torch.where(s.isnan(), torch.tensor(-float("inf")), s)
    ended = torch.zeros(b, w, dtype=torch.bool) if done is None else done.cpu() != 0
    only = torch.full_like(s, -float("inf"))
    if eos >= 0:
        only[..., eos] = scores
    s = torch.where(ended[..., None], only, s)
    best, at = torch.sort(s.view(b, -1), dim=-1, descending=True, stable=True)
    parent, token = at[:, :k] // v, at[:, :k] % v
    return best[:, :k], parent.int(), token.int(), ((token == eos) | ended.gather(1, parent)).int()


def _run(torch, mtp, logits, lse, scores, done, eos, k, workspace=None, out_lse=True):
    b, w, _ = logits.shape
    dev = dict(device="cuda")
    out = dict(out_scores=torch.zeros(b, k, **dev), out_parent=torch.zeros(b, k, dtype=torch.int32, **dev),
               out_token=torch.zeros(b, k, dtype=torch.int32, **dev), out_done=torch.zeros(b, k, dtype=torch.int32, **dev),
               out_lse=torch.full((b, w), 77.0, **dev) if out_lse else None)
    args = mtp.beam_select_args(logits=logits, lse=lse, scores=scores, done=done, eos_id=eos, k=k, **out)
    nbytes = mtp.mtp_beam_select_workspace_bytes(args)
    if workspace is None:
        workspace = torch.zeros(max(1, nbytes), dtype=torch.uint8, device="cuda")
    assert workspace.numel() >= nbytes
    mtp.mtp_beam_select(args, workspace, nbytes, torch.cuda.current_stream())
    return out


def _equal(torch, out, want):
    for name, w in zip(("out_scores", "out_parent", "out_token", "out_done"), want):
        assert torch.equal(out[name].cpu(), w), name


def _lse_error(torch, got, logits):
    """exp's approximation errs by 2^-21 relative at most; a thread adds up to vocab / 32 terms in turn, then 10 levels;
    the logarithm turns relative into absolute error, and the last sum rounds once."""
    x = logits.double().cpu()
    want = torch.logsumexp(x, -1)
    bound = 2.0 ** -21 + (x.shape[-1] / 32 + 10) * 2.0 ** -24 + 2.0 ** -22 * want.abs()
    assert bool(((got.double().cpu() - want).abs() <= bound).all())


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("given", [True, False])
@pytest.mark.parametrize("batch,beams,vocab,k", [
    (1, 1, 1, 1), (1, 5, 1025, 10), (3, 8, 1025, 16), (128, 4, 1025, 8), (2, 64, 300, 64), (1, 1, 20000, 64), (5, 3, 7, 21),
    (2, 2, 8192, 4), (2, 2, 8193, 4), (1, 4, 48001, 8), (7, 5, 16385, 33), (1, 2, 262144, 64), (1, 64, 20001, 2)])
def test_equals_a_stable_sort(dtype, given, batch, beams, vocab, k):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    gen = torch.Generator(device="cuda").manual_seed(vocab + k)
    logits = (3 * torch.randn(batch, beams, vocab, device="cuda", generator=gen)).to(getattr(torch, dtype))
    scores = -5 * torch.rand(batch, beams, device="cuda", generator=gen)
    done = (torch.rand(batch, beams, device="cuda", generator=gen) < 0.3).int()
    lse = torch.logsumexp(logits.float(), -1) if given else None
    for d, eos in ((None, -1), (done, vocab - 1), (done, 0)):
        out = _run(torch, mtp, logits, lse, scores, d, eos, k)
        if not given:
            _lse_error(torch, out["out_lse"], logits)
        else:
            assert torch.equal(out["out_lse"], lse)
        _equal(torch, out, _expected(torch, logits, out["out_lse"], scores, d, eos, k))
    hidden = _run(torch, mtp, logits, lse, scores, done, 0, k, out_lse=False)
    for name in ("out_scores", "out_parent", "out_token", "out_done"):
        assert torch.equal(hidden[name], out[name])


@pytest.mark.parametrize("batch,beams,vocab,k", [(2, 4, 1025, 64), (1, 3, 30011, 40), (1, 1, 16384, 64)])
@pytest.mark.parametrize("what", ["all equal", "two values", "all masked", "few allowed", "lowest value", "zeros of both signs",
                                  "one thread's", "nan"])
def test_ties_and_masks(what, batch, beams, vocab, k):
    """Equal scores go by beam and token, -inf ones too; a NaN counts as -inf."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    gen = torch.Generator(device="cuda").manual_seed(3)
    x = torch.zeros(batch, beams, vocab, device="cuda")
    scores, lse = torch.zeros(batch, beams, device="cuda"), torch.zeros(batch, beams, device="cuda")
    if what == "two values":
        x[torch.rand(x.shape, device="cuda", generator=gen) < 0.5] = 1.0
    elif what == "all masked":
        x.fill_(-float("inf"))
    elif what == "few allowed":
        x.fill_(-float("inf"))
        x[:, -1, torch.randint(0, vocab, (5,), device="cuda", generator=gen)] = 2.0
    elif what == "lowest value":
        x = torch.where(torch.rand(x.shape, device="cuda", generator=gen) < 0.999, torch.finfo(torch.float32).min, x)
    elif what == "zeros of both signs":
        x[torch.rand(x.shape, device="cuda", generator=gen) < 0.5] = -0.0
    elif what == "one thread's":  # the largest all in places of one thread group
        x[..., ::512] = 1.0
    elif what == "nan":
        x.normal_(generator=gen)
        x[torch.rand(x.shape, device="cuda", generator=gen) < 0.9] = float("nan")
    out = _run(torch, mtp, x, lse, scores, None, -1, k)
    _equal(torch, out, _expected(torch, x, lse, scores, None, -1, k))


def test_beams_that_are_left_out():
    """At a search's start only the first beam counts; items without any beam give -inf in order."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    x = torch.randn(3, 4, 1025, device="cuda")
    scores = torch.full((3, 4), -float("inf"), device="cuda")
    scores[:2, 0] = 0.0
    out = _run(torch, mtp, x, None, scores, None, 7, 8)
    _equal(torch, out, _expected(torch, x, out["out_lse"], scores, None, 7, 8))
    assert out["out_parent"][:2].tolist() == [[0] * 8] * 2
    assert out["out_token"][2].tolist() == list(range(8))


@pytest.mark.parametrize("vocab", [1025, 40001])
def test_rows_without_a_log_sum_exp(vocab):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    x = torch.randn(2, 3, vocab, device="cuda")
    x[0, 0, 5], x[0, 1, 9], x[1, 2] = float("nan"), float("inf"), -float("inf")
    scores = torch.zeros(2, 3, device="cuda")
    out = _run(torch, mtp, x, None, scores, None, -1, 6)
    lse = out["out_lse"].cpu()
    assert bool(lse[0, :2].isnan().all()) and float(lse[1, 2]) == -float("inf")
    assert bool((out["out_parent"][0] == 2).all()) and bool((out["out_parent"][1] < 2).all())
    _equal(torch, out, _expected(torch, x, lse, scores, None, -1, 6))


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("shift,stride", [(0, 1032), (1, 1027), (3, 1025), (5, 2000)])
def test_rows_at_any_stride_and_alignment(dtype, shift, stride):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    buf = torch.randn(shift + 12 * stride, device="cuda").to(getattr(torch, dtype))
    x = buf[shift:].view(3, 4, stride)[..., :1025]
    scores, lse = -torch.rand(3, 4, device="cuda"), torch.logsumexp(x.float(), -1)
    _equal(torch, _run(torch, mtp, x, lse, scores, None, 3, 9), _expected(torch, x, lse, scores, None, 3, 9))


def test_one_workspace_for_calls_of_all_sizes():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    ws = torch.zeros(8 << 20, dtype=torch.uint8, device="cuda")
    for batch, beams, vocab, k in ((1, 2, 60000, 64), (64, 4, 20000, 3), (3, 5, 1025, 5), (2, 8, 131072, 16), (1, 1, 17000, 1)):
        x = torch.randn(batch, beams, vocab, device="cuda")
        scores = torch.zeros(batch, beams, device="cuda")
        for given in (True, False):
            lse = torch.logsumexp(x, -1) if given else None
            out = _run(torch, mtp, x, lse, scores, None, -1, k, ws)
            _equal(torch, out, _expected(torch, x, out["out_lse"], scores, None, -1, k))


def test_captured_in_a_graph():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    x, scores = torch.randn(2, 3, 50000, device="cuda"), torch.zeros(2, 3, device="cuda")
    i32 = lambda: torch.zeros(2, 6, dtype=torch.int32, device="cuda")  # noqa: E731
    out = dict(out_scores=torch.zeros(2, 6, device="cuda"), out_parent=i32(), out_token=i32(), out_lse=torch.zeros(2, 3, device="cuda"))
    args = mtp.beam_select_args(logits=x, scores=scores, k=6, **out)
    n = mtp.mtp_beam_select_workspace_bytes(args)
    ws = torch.zeros(n, dtype=torch.uint8, device="cuda")
    mtp.mtp_beam_select(args, ws, n, torch.cuda.current_stream())
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        mtp.mtp_beam_select(args, ws, n, torch.cuda.current_stream())
    for _ in range(3):
        x.normal_()
        graph.replay()
        want = _expected(torch, x, out["out_lse"], scores, None, -1, 6)
        assert torch.equal(out["out_scores"].cpu(), want[0]) and torch.equal(out["out_token"].cpu(), want[2])


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("batch,beams,vocab", [(64, 8, 1025), (512, 1, 20001), (1, 16, 40001), (1, 16, 5000), (1, 1, 16385)])
def test_a_nan_in_a_masked_row(dtype, batch, beams, vocab):
    """Wherever the NaN of a row stands that is masked but for one logit: its log-sum-exp is NaN, none of its
    continuations counts.  (Held items, rows by a CTA each, rows by clusters.)"""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    rows = batch * beams
    g = torch.Generator().manual_seed(vocab)
    # places of a first load's every lane, the last ones, and any others
    near = list(range(min(vocab, 512))) + list(range(vocab - 40, vocab))
    for start in range(0, min(len(near), max(4 * rows, 64)), rows):
        at = torch.tensor((near[start:start + rows] + torch.randint(0, vocab, (rows,), generator=g).tolist())[:rows])
        allowed = torch.where(at == vocab // 2, at // 2, torch.full_like(at, vocab // 2))
        x = torch.full((rows, vocab), -float("inf"))
        x[torch.arange(rows), allowed] = 1.5
        clean = x.clone()
        x[torch.arange(rows), at] = float("nan")
        x[rows // 2] = clean[rows // 2] if rows > 1 else x[0]  # one row without a NaN
        x = x.view(batch, beams, vocab).cuda().to(getattr(torch, dtype))
        scores = torch.zeros(batch, beams, device="cuda")
        out = _run(torch, mtp, x, None, scores, None, -1, 1)
        lse = out["out_lse"].flatten().cpu()
        want = torch.full((rows,), float("nan"))
        if rows > 1:
            want[rows // 2] = 1.5
        assert torch.equal(lse.isnan(), want.isnan()), torch.nonzero(lse.isnan() != want.isnan())[:5].tolist()
        _equal(torch, out, _expected(torch, x, out["out_lse"], scores, None, -1, 1))


def _one_large(torch, vocab):
    """Places whose logit a summing kernel may miss: the row's ends, both sides of every 16-byte border near them (of
    any row start) and of parts of 1 to 8 CTAs."""
    places = set(range(min(vocab, 24))) | set(range(max(0, vocab - 24), vocab))
    for ctas in range(1, 9):
        seg = (-(-vocab // ctas) + 7) // 8 * 8
        for edge in range(0, vocab + 1, seg):
            places |= set(range(edge - 10, edge + 10))
    for step in (32 * 4, 32 * 8, 32 * 4 * 4, 32 * 4 * 8, 512 * 4, 512 * 8, 512 * 4 * 4, 512 * 4 * 8):
        places |= set(range(step - 9, step + 9)) | set(range(2 * step - 9, 2 * step + 9))
    return sorted(p for p in places if 0 <= p < vocab)


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float16"])
@pytest.mark.parametrize("vocab,rows,shift", [(1025, 64, 0), (1025, 13, 3), (16385, 320, 0), (16385, 16, 1), (48001, 8, 0), (48001, 16, 5),
                                              (20003, 320, 7), (33333, 1, 2)])
def test_every_logit_is_summed(dtype, vocab, rows, shift):
    """One logit of 20 among zeros, at places that a sum's heads, tails and cuts could miss: without it the log-sum-exp
    would be log(vocab - 1), with it counted twice 0.69 more."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    places = _one_large(torch, vocab)
    if rows < 16:
        places = places[::3] + places[1::7]
    stride = vocab + shift % 4
    value = 20.0
    want = torch.tensor([value], dtype=torch.float64).exp().add(vocab - 1).log().item()
    for start in range(0, len(places), rows):
        at = torch.tensor([places[(start + i) % len(places)] for i in range(rows)], device="cuda")
        buf = torch.zeros(shift + rows * stride, device="cuda").to(getattr(torch, dtype))
        x = buf[shift:].view(1, rows, stride)[..., :vocab] if rows <= 64 else buf[shift:].view(rows, 1, stride)[..., :vocab]
        x.scatter_(2, at.view(x.shape[0], x.shape[1], 1), value)
        out = _run(torch, mtp, x, None, torch.zeros(x.shape[:2], device="cuda"), None, -1, 1)
        # (20 + log(1 + 48000 e^-20): a rounding of the sum and of the last addition, exp of 0 exactly 1)
        assert float((out["out_lse"].double() - want).abs().max()) <= 2.0 ** -18


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("batch,beams,vocab", [(1, 4, 48001), (32, 4, 48001), (7, 5, 16385), (1, 2, 262144), (3, 2, 30003)])
def test_log_sum_exp_of_long_rows(dtype, batch, beams, vocab):
    """Rows of more than one item's scores in shared memory, of which a thread of 512 adds few terms.  __expf errs by
    2 + 1.173 |x| units of 2^-23 at most; over a term's way to the sum these |x| add up to the distance to the row's maximum,
    and there is one exponential per 16 bytes that a thread reads and one per join (13 levels at most); an addition
    rounds by 2^-24, as many of them and the 8 of a piece.  Then the logarithm and the last sum."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    gen = torch.Generator(device="cuda").manual_seed(vocab)
    x = (3 * torch.randn(batch, beams, vocab, device="cuda", generator=gen)).to(getattr(torch, dtype))
    out = _run(torch, mtp, x, None, torch.zeros(batch, beams, device="cuda"), None, -1, 4)
    y = x.double()
    want = torch.logsumexp(y, -1)
    depth = (torch.softmax(y, -1) * (y.amax(-1, keepdim=True) - y)).sum(-1)  # mean distance to the maximum
    sms = torch.cuda.get_device_properties(0).multi_processor_count
    ctas = 1
    while ctas < 8 and batch * beams * ctas <= sms and vocab // (ctas * 2) >= 4096:
        ctas *= 2
    vecs = -(-vocab // ctas) // (4 if dtype == "float32" else 8) + 1
    pieces = 4 * -(-vecs // 2048) + 2  # four to a stretch of 128 pieces, a stretch per warp in turn; a head's and a tail's element
    bound = 2.0 ** -23 * (2 * (pieces + 14) + 1.173 * depth) + 2.0 ** -24 * (pieces + 21) + 2.0 ** -22 * want.abs()
    assert bool(((out["out_lse"].double() - want).abs() <= bound).all()), ((out["out_lse"].double() - want).abs() / bound).max()
