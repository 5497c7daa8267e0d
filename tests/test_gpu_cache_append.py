"""mtp_cache_append against indexing, bit by bit: copies of the pool's own type are exact, and fp32 values are
rounded to nearest even as torch rounds them."""
import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("src,dst", [("float32", "bfloat16"), ("float32", "float16"), ("bfloat16", "bfloat16"),
                                     ("float16", "float16")])
@pytest.mark.parametrize("rows,heads,dim,page,layers,layer,layout", [
    (1, 1, 8, 16, 1, 0, "own"), (3, 16, 64, 64, 3, 1, "fused"), (130, 2, 128, 32, 2, 1, "fused"),
    (77, 5, 24, 16, 1, 0, "odd"), (1000, 8, 128, 128, 2, 0, "own"), (33, 4, 256, 64, 1, 0, "shifted")])
def test_rows_land_at_their_places(src, dst, rows, heads, dim, page, layers, layer, layout):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    src, dst = getattr(torch, src), getattr(torch, dst)
    gen = torch.Generator(device="cuda").manual_seed(rows + dim)
    n_pages = rows // page * 2 + 3
    pool = torch.randn(n_pages, layers, 2, heads, page, dim, device="cuda", generator=gen).to(dst)
    width = heads * dim

    def part():
        x = torch.randn(rows, width, device="cuda", generator=gen).to(src)
        x[0, :6] = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 70000.0], device="cuda").to(src)
        return x
    k, v = part(), part()
    if layout == "own":
        kk, vv = k.view(rows, heads, dim), v.view(rows, heads, dim)
    else:  # rows of a wider buffer; "odd": a row stride that is no multiple of 16 bytes; "shifted": nor is the base
        pad, at = {"fused": (32 * width, 16 * width), "odd": (1, 0), "shifted": (9, 1)}[layout]
        buf = torch.zeros(rows, 2 * width + pad, device="cuda", dtype=src)
        kk, vv = buf[:, at:at + width], buf[:, at + width:at + 2 * width]
        kk.copy_(k)
        vv.copy_(v)
        kk, vv = kk.unflatten(1, (heads, dim)), vv.unflatten(1, (heads, dim))
    places = torch.randperm(n_pages * page, device="cuda", generator=gen)[:rows]
    places[rows // 2] = -1
    if rows > 5:
        places[4], places[5] = n_pages * page, 1 << 40  # outside the pool
    want = pool.clone()
    for r, at in enumerate(places.tolist()):
        if 0 <= at < n_pages * page:
            want[at // page, layer, 0, :, at % page] = k[r].to(dst).view(heads, dim)
            want[at // page, layer, 1, :, at % page] = v[r].to(dst).view(heads, dim)
    mtp.mtp_cache_append(mtp.cache_append_args(k=kk, v=vv, slot_map=places, kv_pool=pool, layer=layer),
                         torch.cuda.current_stream())
    nan = pool.isnan()
    assert torch.equal(nan, want.isnan())
    assert torch.equal(pool.view(torch.int16)[~nan], want.view(torch.int16)[~nan])


def test_a_pool_past_32_bits_and_another_stream():
    """Element offsets above 2^32, enqueued on a stream of the caller's."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    pool = torch.zeros(4200, 8, 2, 8, 128, 64, dtype=torch.bfloat16, device="cuda")  # 2^32 elements and more
    assert pool.numel() > 1 << 32
    k = torch.randn(4, 8, 64, device="cuda").bfloat16()
    places = torch.tensor([4199 * 128 + 127, 4100 * 128, 0, 4199 * 128], device="cuda")
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    mtp.mtp_cache_append(mtp.cache_append_args(k=k, v=k, slot_map=places, kv_pool=pool, layer=7), stream)
    stream.synchronize()
    assert torch.equal(pool[places // 128, 7, 0, :, places % 128], k)
    assert torch.equal(pool[places // 128, 7, 1, :, places % 128], k)
    assert int(pool.count_nonzero()) == int(k.count_nonzero()) * 2


def test_no_rows():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    pool = torch.ones(1, 1, 2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    k = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    mtp.mtp_cache_append(mtp.cache_append_args(k=k, v=k, slot_map=torch.zeros(0, dtype=torch.int64, device="cuda"),
                                               kv_pool=pool, layer=0))
    assert bool((pool == 1).all())
