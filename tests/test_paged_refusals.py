"""What the paged operators refuse on the host, before anything is queued: no GPU is needed.  The addresses are
never followed."""
import pytest

from test_lib_cpu import libpath  # noqa: F401

A = 1 << 20  # an aligned address that nothing follows


def _plan(**kw):
    from paper_2410_13839_gb300._lib import MtpPagePlanArgs
    d = dict(slots=4, page_size=16, n_pages=8, bt_stride=4, max_rows=9)
    d.update({n: A for n, t in MtpPagePlanArgs._fields_[5:]})
    return MtpPagePlanArgs(**{**d, **kw})


def _append(**kw):
    from paper_2410_13839_gb300._lib import MtpCacheAppendArgs
    d = dict(rows=4, n_kv_heads=2, head_dim=64, page_size=16, layers=2, layer=1, n_pages=8, src_dtype=0, pool_dtype=1,
             k_stride=128, v_stride=128, k=A, v=A, slot_map=A, kv_pool=A)
    return MtpCacheAppendArgs(**{**d, **kw})


def _reorder(**kw):
    from paper_2410_13839_gb300._lib import MtpBeamReorderArgs
    d = dict(batch=2, beams=4, page_size=16, n_pages=8, bt_stride=4, layers=2, n_kv_heads=2, head_dim=64, pool_dtype=1)
    d.update({n: A * (i + 1) for i, (n, t) in enumerate(MtpBeamReorderArgs._fields_[9:])})
    return MtpBeamReorderArgs(**{**d, **kw})


def _select(**kw):
    from paper_2410_13839_gb300._lib import MtpBeamSelectArgs
    d = dict(batch=2, beams=4, vocab=1025, k=8, eos_id=1024, logits_dtype=0, logits_stride=1025)
    d.update({n: A * (i + 1) for i, (n, t) in enumerate(MtpBeamSelectArgs._fields_[7:])})
    return MtpBeamSelectArgs(**{**d, **kw})


def _chunk(**kw):
    from paper_2410_13839_gb300._lib import MtpChunkAttentionArgs
    d = dict(slots=2, rows=4, n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, layers=2, layer=1, n_pages=8, bt_stride=4,
             dtype=1, window=0, max_new=2, max_keys=64, scale=0.125, q_stride=256, out_stride=256, q=A, kv_pool=A, block_table=A,
             cu_rows=A, kv_lens=A, out=A, out_lse=A)
    return MtpChunkAttentionArgs(**{**d, **kw})


def _refused(call):
    from paper_2410_13839_gb300 import mtp
    with pytest.raises(mtp.MTPError) as e:
        call(mtp)
    assert e.value.code == -1 and str(e.value)


@pytest.mark.parametrize("kw", [dict(slots=0), dict(slots=8193), dict(page_size=24), dict(page_size=256), dict(n_pages=0),
                                dict(n_pages=(1 << 22) + 1), dict(bt_stride=0), dict(bt_stride=(1 << 26) + 1),
                                dict(max_rows=-1), dict(max_rows=(1 << 24) + 1), dict(kv_lens=None),
                                dict(block_table=None), dict(out_slot_map=None), dict(out_status=None)])
def test_page_plan(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_page_plan(_plan(**kw)))


@pytest.mark.parametrize("kw", [dict(rows=-1), dict(rows=1 << 28), dict(n_kv_heads=0), dict(head_dim=60),
                                dict(head_dim=264), dict(page_size=8), dict(layer=2), dict(layer=-1), dict(n_pages=0),
                                dict(src_dtype=2), dict(src_dtype=7), dict(pool_dtype=0), dict(k_stride=127),
                                dict(v_stride=0), dict(k=None), dict(v=None), dict(slot_map=None), dict(kv_pool=None),
                                dict(kv_pool=A + 8), dict(k=A + 2)])
def test_cache_append(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_cache_append(_append(**kw)))


@pytest.mark.parametrize("kw", [dict(batch=0), dict(beams=0), dict(beams=65), dict(batch=4096), dict(page_size=20),
                                dict(n_pages=0), dict(bt_stride=0), dict(layers=0), dict(n_kv_heads=0),
                                dict(head_dim=12), dict(pool_dtype=0), dict(parent=None), dict(kv_pool=None),
                                dict(out_status=None), dict(kv_pool=A + 4), dict(out_block_table=A * 2),
                                dict(out_kv_lens=A * 3)])
def test_beam_reorder(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_beam_reorder(_reorder(**kw), A, 1 << 20))


def test_beam_reorder_workspace(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    need = mtp.mtp_beam_reorder_workspace_bytes(_reorder())
    assert need > 0
    for ws, n in ((None, need), (A, need - 1), (A + 8, need)):
        _refused(lambda m: m.mtp_beam_reorder(_reorder(), ws, n))


@pytest.mark.parametrize("kw", [dict(slots=0), dict(slots=4097), dict(rows=-1), dict(n_heads=3), dict(n_kv_heads=0),
                                dict(n_heads=130), dict(n_heads=1026), dict(head_dim=96), dict(page_size=48), dict(layer=2),
                                dict(layers=0), dict(n_pages=0), dict(n_pages=1 << 29), dict(bt_stride=0),
                                dict(bt_stride=(1 << 20) + 1), dict(dtype=0), dict(window=-1), dict(max_new=-1),
                                dict(max_keys=-1), dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan"))])
def test_chunk_attention(libpath, kw):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    _refused(lambda m: m.mtp_chunk_attention(_chunk(**kw), A, 1 << 40))
    assert mtp.mtp_chunk_attention_workspace_bytes(_chunk(**kw)) == 0


@pytest.mark.parametrize("kw", [dict(batch=0), dict(batch=4097), dict(beams=0), dict(beams=65), dict(vocab=0), dict(k=0),
                                dict(k=65), dict(vocab=1, logits_stride=1, k=5, eos_id=0), dict(vocab=1 << 29),
                                dict(eos_id=1025), dict(eos_id=-1), dict(logits_dtype=3), dict(logits_stride=1024),
                                dict(logits=None), dict(scores=None), dict(out_scores=None), dict(out_parent=None),
                                dict(out_token=None), dict(logits=A + 2)])
def test_beam_select(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_beam_select(_select(**kw), A, 1 << 30))


def test_beam_select_workspace(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    assert mtp.mtp_beam_select_workspace_bytes(_select()) == 0  # an item of one segment needs none
    big = dict(vocab=100000, logits_stride=100000, eos_id=5)
    need = mtp.mtp_beam_select_workspace_bytes(_select(**big))
    assert need > 0 and mtp.mtp_beam_select_workspace_bytes(_select(vocab=-1)) == 0
    for ws, n in ((None, need), (A, need - 1), (A + 8, need)):
        _refused(lambda m: m.mtp_beam_select(_select(**big), ws, n))


def test_null_argument_blocks(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import _lib
    for call in (lambda: _lib.lib.mtp_page_plan(None, None), lambda: _lib.lib.mtp_cache_append(None, None),
                 lambda: _lib.lib.mtp_chunk_attention(None, None, 0, None),
                 lambda: _lib.lib.mtp_beam_select(None, None, 0, None), lambda: _lib.lib.mtp_beam_reorder(None, None, 0, None)):
        assert call() == -1
    assert _lib.lib.mtp_beam_reorder_workspace_bytes(None) == 0


def test_argument_blocks_refuse_tensors_they_cannot_describe(libpath):  # noqa: F811
    torch = pytest.importorskip("torch")
    from paper_2410_13839_gb300 import mtp
    pool = torch.zeros(2, 1, 2, 2, 16, 64, dtype=torch.bfloat16)
    k, places = torch.zeros(3, 2, 64, dtype=torch.bfloat16), torch.zeros(3, dtype=torch.int64)
    with pytest.raises(ValueError):  # host memory
        mtp.cache_append_args(k=k, v=k, slot_map=places, kv_pool=pool, layer=0)
    with pytest.raises(TypeError):
        mtp.cache_append_args(k=k, v=k, slot_map=places, kv_pool=pool.float(), layer=0)


class _OnGpu:
    """A CPU tensor that says it is on the GPU: argument blocks are built from it, nothing is launched."""
    is_cuda = True

    def __init__(self, x):
        self._x = x

    def __getattr__(self, name):
        return getattr(self._x, name)


@pytest.mark.parametrize("rows,stride", [(1000, 0), (2, 0), (3, 64), (3, 127)])
@pytest.mark.parametrize("which", ["k", "v", "q", "out"])
def test_rows_that_overlap(libpath, which, rows, stride):  # noqa: F811
    """Expanded or overlapping rows of 128 elements are refused: read at a stride of a row's width, as if they were
    packed, they would end past their buffer."""
    torch = pytest.importorskip("torch")
    from paper_2410_13839_gb300 import mtp
    i32 = dict(dtype=torch.int32)
    pool = _OnGpu(torch.zeros(2, 1, 2, 2, 16, 64, dtype=torch.bfloat16))
    overlapping = _OnGpu(torch.zeros((rows - 1) * stride + 128, dtype=torch.bfloat16).as_strided((rows, 2, 64), (stride, 64, 1)))
    good = _OnGpu(torch.zeros(rows, 2, 64, dtype=torch.bfloat16))
    x = {n: overlapping if n == which else good for n in ("k", "v", "q", "out")}

    def append():
        return mtp.cache_append_args(k=x["k"], v=x["v"], slot_map=_OnGpu(torch.zeros(rows, dtype=torch.int64)), kv_pool=pool,
                                     layer=0)

    def attend():
        return mtp.chunk_attention_args(q=x["q"], kv_pool=pool, layer=0, block_table=_OnGpu(torch.zeros(1, 2, **i32)),
                                        cu_rows=_OnGpu(torch.zeros(2, **i32)), kv_lens=_OnGpu(torch.zeros(1, **i32)),
                                        out=x["out"], scale=0.125, max_new=rows, max_keys=32)
    wrong, right = (append, attend) if which in "kv" else (attend, append)
    with pytest.raises(ValueError, match=which):
        wrong()
    right()


@pytest.mark.parametrize("rows,stride", [(0, 0), (1, 0), (1, 128), (1, 500), (4, 128), (4, 200)])
def test_row_strides_that_are_taken(libpath, rows, stride):  # noqa: F811
    """The stride of several rows is the tensor's; of one row, whatever the tensor says, it is at least a row's width."""
    torch = pytest.importorskip("torch")
    from paper_2410_13839_gb300 import mtp
    pool = _OnGpu(torch.zeros(2, 1, 2, 2, 16, 64, dtype=torch.bfloat16))
    k = _OnGpu(torch.zeros(4 * 512, dtype=torch.bfloat16).as_strided((rows, 2, 64), (stride, 64, 1)))
    args = mtp.cache_append_args(k=k, v=k, slot_map=_OnGpu(torch.zeros(rows, dtype=torch.int64)), kv_pool=pool, layer=0)
    assert args.rows == rows and args.k_stride == args.v_stride == max(stride, 128)
