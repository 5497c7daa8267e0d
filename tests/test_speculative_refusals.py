"""What the operators of speculative decoding over long contexts refuse on the host, before anything is queued: no GPU
is needed.  The addresses are never followed."""
import pytest

from test_lib_cpu import libpath  # noqa: F401
from test_paged_refusals import A, _refused


def _args(name, **kw):
    """An argument block, every pointer that is not given an address of its own."""
    from paper_2410_13839_gb300 import _lib
    import ctypes
    cls = getattr(_lib, name)
    pointers = [n for n, t in cls._fields_ if t is ctypes.c_void_p]
    return cls(**{**{n: A * (i + 1) for i, n in enumerate(pointers)}, **kw})


def _rotary(**kw):
    return _args("MtpRotaryAppendArgs", **{**dict(
        rows=4, n_heads=4, n_kv_heads=2, head_dim=64, rot_dim=64, layout=0, page_size=16, layers=2, layer=1, n_pages=8,
        src_dtype=0, pool_dtype=1, gain=1.0, q_stride=256, k_stride=128, v_stride=128, out_stride=256), **kw})


def _weights(**kw):
    return _args("MtpKeyWeightsArgs", **{**dict(
        slots=2, rows=4, n_heads=4, n_kv_heads=2, head_dim=64, page_size=16, layers=2, layer=1, n_pages=8, bt_stride=4,
        dtype=1, window=0, max_new=2, max_keys=64, scale=0.125, q_stride=256), **kw})


def _verify(**kw):
    return _args("MtpDraftVerifyArgs", **{**dict(
        slots=2, rows=4, vocab=1025, max_new=4, eos_id=1024, logits_dtype=0, page_size=16, bt_stride=4, n_pages=8,
        logits_stride=1025, draft_stride=1025), **kw})


def _evict(**kw):
    return _args("MtpCacheEvictArgs", **{**dict(
        slots=2, page_size=16, n_pages=8, bt_stride=4, layers=2, n_kv_heads=2, head_dim=64, pool_dtype=1, sinks=4,
        recent=8), **kw})


@pytest.mark.parametrize("kw", [
    dict(rows=-1), dict(rows=1 << 28), dict(n_heads=0), dict(n_heads=1025), dict(n_kv_heads=0), dict(head_dim=60),
    dict(head_dim=264), dict(rot_dim=0), dict(rot_dim=63), dict(rot_dim=66), dict(rot_dim=-2), dict(layout=2), dict(layout=-1),
    dict(page_size=8), dict(layer=2), dict(layer=-1), dict(n_pages=0), dict(src_dtype=2), dict(src_dtype=7),
    dict(pool_dtype=0), dict(gain=float("nan")), dict(gain=float("inf")), dict(q_stride=255), dict(k_stride=127),
    dict(v_stride=0), dict(out_stride=255), dict(q=None), dict(k=None), dict(v=None), dict(positions=None),
    dict(slot_map=None), dict(turns=None), dict(kv_pool=None), dict(out_q=None), dict(kv_pool=A + 8), dict(q=A + 2),
    dict(out_q=A), dict(out_q=A + 1), dict(slot_map=A + 4), dict(turns=A + 4)])
def test_rotary_append(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_rotary_append(_rotary(**kw)))


@pytest.mark.parametrize("kw", [
    dict(slots=0), dict(slots=4097), dict(rows=-1), dict(n_heads=3), dict(n_kv_heads=0), dict(n_heads=130), dict(n_heads=1026),
    dict(head_dim=96), dict(page_size=48), dict(layer=2), dict(layers=0), dict(n_pages=0), dict(n_pages=1 << 29),
    dict(bt_stride=0), dict(bt_stride=(1 << 20) + 1), dict(dtype=0), dict(window=-1), dict(max_new=-1), dict(max_keys=-1),
    dict(scale=0.0), dict(scale=-1.0), dict(scale=float("nan")), dict(rows=1 << 20)])
def test_key_weights(libpath, kw):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    _refused(lambda m: m.mtp_key_weights(_weights(**kw), A, 1 << 40))
    assert mtp.mtp_key_weights_workspace_bytes(_weights(**kw)) == 0


@pytest.mark.parametrize("kw", [
    dict(slots=0), dict(slots=8193), dict(rows=-1), dict(vocab=0), dict(vocab=(1 << 18) + 1, logits_stride=1 << 19, draft_stride=1 << 19),
    dict(max_new=0), dict(max_new=65), dict(eos_id=1025), dict(eos_id=-2), dict(logits_dtype=3), dict(logits_stride=1024),
    dict(draft_stride=1024), dict(logits=None), dict(tokens=None), dict(uniforms=None), dict(cu_rows=None), dict(kv_lens=None),
    dict(out_tokens=None), dict(out_counts=None), dict(out_kv_lens=None), dict(block_table=None), dict(page_refs=None),
    dict(page_size=24), dict(n_pages=0), dict(bt_stride=0), dict(bt_stride=(1 << 26) + 1), dict(logits=A + 2),
    dict(draft_logits=A + 2), dict(uniforms=A + 2)])
def test_draft_verify(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_draft_verify(_verify(**kw)))


@pytest.mark.parametrize("kw", [
    dict(slots=0), dict(slots=8193), dict(page_size=20), dict(n_pages=0), dict(bt_stride=0), dict(bt_stride=(1 << 20) + 1),
    dict(layers=0), dict(n_kv_heads=0), dict(head_dim=12), dict(pool_dtype=0), dict(sinks=-1), dict(recent=-1),
    dict(kv_lens=None), dict(keep=None), dict(block_table=None), dict(page_refs=None), dict(weights=None), dict(kv_pool=None),
    dict(out_kv_lens=None), dict(out_block_table=None), dict(out_page_refs=None), dict(out_weights=None),
    dict(out_status=None), dict(kv_pool=A + 4), dict(out_kv_lens=A), dict(out_kv_lens=A * 2), dict(out_block_table=A * 3),
    dict(out_weights=A * 5)])
def test_cache_evict(libpath, kw):  # noqa: F811
    _refused(lambda mtp: mtp.mtp_cache_evict(_evict(**kw), A, 1 << 40))


def test_cache_evict_workspace(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    assert mtp.mtp_cache_evict_workspace_bytes(_evict()) == 0  # tables of 64 keys need none
    wide = dict(bt_stride=4096)
    need = mtp.mtp_cache_evict_workspace_bytes(_evict(**wide))
    assert need > 0
    for ws, n in ((None, need), (A, need - 1), (A + 8, need)):
        _refused(lambda m: m.mtp_cache_evict(_evict(**wide), ws, n))


def test_null_arguments(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    from paper_2410_13839_gb300._lib import lib
    assert lib.mtp_rotary_append(None, None) == -1 and lib.mtp_key_weights(None, None, 0, None) == -1
    assert lib.mtp_draft_verify(None, None) == -1 and lib.mtp_cache_evict(None, None, 0, None) == -1
    assert lib.mtp_key_weights_workspace_bytes(None) == 0 and lib.mtp_cache_evict_workspace_bytes(None) == 0
    assert lib.mtp_rotary_turns(64, 0, 1e4, 1.0, 0.0, 0.0, 0.0, None) == -1
    assert mtp.mtp_last_error()


def test_no_work_needs_nothing(libpath):  # noqa: F811
    from paper_2410_13839_gb300 import mtp
    mtp.mtp_rotary_append(_rotary(rows=0, q=None, k=None, v=None))
