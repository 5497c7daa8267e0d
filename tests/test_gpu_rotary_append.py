"""mtp_rotary_append against the rotation in 64 bits, every element within its own rounding and the error of a sine.

Tolerance: sine and cosine err by 2^-22 g at most (the angle's 32 bits in fp32: 2^-25 half turns = 2^-23.3 radians; the
functions and the product with g: half a unit of 2^-24 each, some), each of the two products and their sum by 2^-24 of
(|a| + |b|) g; then the rounding to 16 bits, half a step of the value (of 2^-14 below fp16's normal range)."""
import math

import pytest

from gpu_util import lib_module

pytestmark = pytest.mark.gpu

FAR = [0, 1, -1, 7, 1999, 65535, 1000000, 123456789, 2 ** 31 - 1, -2 ** 31]


def _turned(torch, x, pos, freq, gain, layout):
    """(turned, |a| + |b| of each element's pair) in 64 bits; x [rows, heads, dim]."""
    rot = 2 * freq.numel()
    x = x.double()
    # turns of the exact fractions, whole ones taken out by integers: position * freq in 64 bits is off by 1e-7 at 2^31
    angle = torch.tensor([[(int(p) * int(f)) % (1 << 64) / 2.0 ** 64 * 2 * math.pi for f in freq.tolist()] for p in pos],
                         dtype=torch.float64, device=x.device)
    cos, sin = gain * angle.cos()[:, None], gain * angle.sin()[:, None]
    y, size = x.clone(), x.abs().clone()
    a, b = (slice(0, rot // 2), slice(rot // 2, rot)) if layout == "halves" else (slice(0, rot, 2), slice(1, rot, 2))
    y[..., a], y[..., b] = x[..., a] * cos - x[..., b] * sin, x[..., a] * sin + x[..., b] * cos
    size[..., a] = size[..., b] = abs(gain) * (x[..., a].abs() + x[..., b].abs())
    return y, size


def _close(torch, got, want, size, rot):
    eps, tiny = torch.finfo(got.dtype).eps, 2.0 ** -25 if got.dtype == torch.float16 else 0.0
    err, slip = (got.double() - want).abs(), size * 2.0 ** -21
    bad = err > slip + torch.maximum(eps / 2 * (want.abs() + slip), torch.full_like(want, tiny))
    assert not bool(bad[..., :rot].any()), float(err[bad].max())


@pytest.mark.parametrize("src,dst", [("float32", "bfloat16"), ("float32", "float16"), ("bfloat16", "bfloat16"),
                                     ("float16", "float16")])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("rows,heads,kv_heads,dim,rot,page,layers,layer,memory", [
    (1, 1, 1, 8, 2, 16, 1, 0, "own"), (3, 16, 16, 64, 64, 64, 3, 1, "fused"), (130, 4, 2, 128, 64, 32, 2, 1, "fused"),
    (77, 10, 5, 24, 24, 16, 1, 0, "odd"), (1000, 8, 1, 128, 22, 128, 2, 0, "own"), (33, 4, 4, 256, 256, 64, 1, 0, "shifted"),
    (700, 5, 1, 64, 50, 16, 1, 0, "fused"), (65, 32, 8, 128, 128, 16, 2, 1, "odd")])
def test_rows_are_turned_and_land(src, dst, layout, rows, heads, kv_heads, dim, rot, page, layers, layer, memory):
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    src, dst = getattr(torch, src), getattr(torch, dst)
    gen = torch.Generator(device="cuda").manual_seed(rows + dim + rot)
    n_pages = rows // page * 2 + 3
    pool = torch.randn(n_pages, layers, 2, kv_heads, page, dim, device="cuda", generator=gen).to(dst)
    total = heads + 2 * kv_heads
    pad, at = {"own": (0, 0), "fused": (0, 0), "odd": (1, 0), "shifted": (9, 1)}[memory]
    buf = torch.randn(rows, total * dim + pad, device="cuda", generator=gen).to(src)
    x = buf[:, at:at + total * dim].unflatten(1, (total, dim))
    q, k, v = x[:, :heads], x[:, heads:heads + kv_heads], x[:, heads + kv_heads:]
    special = torch.tensor([float("inf"), -float("inf"), float("nan"), 0.0, -0.0, 70000.0], device="cuda").to(src)
    v[0, 0, :6] = special  # values, and what is behind rot, may be anything
    if dim - rot >= 6:
        q[0, 0, rot:rot + 6], k[0, 0, rot:rot + 6] = special, special
    if memory == "own":
        q, k, v = q.contiguous(), k.contiguous(), v.contiguous()
    places = torch.randperm(n_pages * page, device="cuda", generator=gen)[:rows]
    if rows > 2:
        places[rows // 2] = -1
    if rows > 5:
        places[4], places[5] = n_pages * page, 1 << 40  # outside the pool
    positions = torch.tensor([FAR[i % len(FAR)] + (i // len(FAR) if FAR[i % len(FAR)] < 2 ** 30 else 0) for i in range(rows)],
                             dtype=torch.int32, device="cuda")
    turns = mtp.mtp_rotary_turns(rot)
    gain = 1.25 if layout == "pairs" else 1.0
    wide = torch.full((rows, heads * dim + (8 if memory == "own" else 3)), 5.0, dtype=dst, device="cuda")
    out_q = wide[:, :heads * dim].unflatten(1, (heads, dim))
    before = pool.clone()
    mtp.mtp_rotary_append(mtp.rotary_append_args(
        q=q, k=k, v=v, positions=positions, slot_map=places, turns=turns, kv_pool=pool, layer=layer, out_q=out_q,
        layout=getattr(mtp, "MTP_ROTARY_" + layout.upper()), gain=gain), torch.cuda.current_stream())
    assert bool((wide[:, heads * dim:] == 5.0).all())
    pos, freq = positions.tolist(), turns.cpu()

    def same(a, b):
        return torch.equal(a.isnan(), b.isnan()) and torch.equal(a.nan_to_num(7.0), b.nan_to_num(7.0))
    want, size = _turned(torch, q, pos, freq, gain, layout)
    _close(torch, out_q, want, size, rot)
    assert same(out_q[..., rot:], q[..., rot:].to(dst))
    there = (places >= 0) & (places < n_pages * page)
    p = places[there]
    keys, values = pool[p // page, layer, 0, :, p % page], pool[p // page, layer, 1, :, p % page]
    want, size = _turned(torch, k, pos, freq, gain, layout)
    _close(torch, keys, want[there], size[there], rot)
    assert same(keys[..., rot:], k[there][..., rot:].to(dst)) and same(values, v[there].to(dst))
    for half in (0, 1):  # nothing else of the pool
        pool[p // page, layer, half, :, p % page] = before[p // page, layer, half, :, p % page]
    assert torch.equal(pool, before)


def test_scalings_reach_the_rows():
    """One far position, each scaling: the turned unit vector is the angle's point on the circle."""
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    x = torch.zeros(1, 1, 64, device="cuda")
    x[..., :32] = 1.0
    seen = []
    for scaling in range(4):
        turns = mtp.mtp_rotary_turns(64, scaling, factor=8.0, context=8192.0)
        pool = torch.zeros(1, 1, 2, 1, 16, 64, dtype=torch.float16, device="cuda")
        out = torch.zeros(1, 1, 64, dtype=torch.float16, device="cuda")
        mtp.mtp_rotary_append(mtp.rotary_append_args(
            q=x, k=x, v=x, positions=torch.tensor([100000], dtype=torch.int32, device="cuda"),
            slot_map=torch.zeros(1, dtype=torch.int64, device="cuda"), turns=turns, kv_pool=pool, layer=0, out_q=out))
        want, size = _turned(torch, x, [100000], turns.cpu(), 1.0, "halves")
        _close(torch, out, want, size, 64)
        seen.append(out.clone())
    assert all(not torch.equal(seen[0], y) for y in seen[1:])


def test_a_pool_past_32_bits_another_stream_and_a_replayed_graph():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    pool = torch.zeros(4200, 8, 2, 8, 128, 64, dtype=torch.bfloat16, device="cuda")
    assert pool.numel() > 1 << 32
    x = torch.randn(4, 24, 64, device="cuda").bfloat16()
    places = torch.tensor([4199 * 128 + 127, 4100 * 128, 0, 4199 * 128], device="cuda")
    positions = torch.tensor([0, 5, 1000, 99], dtype=torch.int32, device="cuda")
    out = torch.zeros(4, 8, 64, dtype=torch.bfloat16, device="cuda")
    turns = mtp.mtp_rotary_turns(64)  # (an argument block holds addresses: the tensor has to live as long)
    args = mtp.rotary_append_args(q=x[:, :8], k=x[:, 8:16], v=x[:, 16:], positions=positions, slot_map=places,
                                  turns=turns, kv_pool=pool, layer=7, out_q=out)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    mtp.mtp_rotary_append(args, stream)
    stream.synchronize()
    assert torch.equal(pool[places // 128, 7, 1, :, places % 128], x[:, 16:])
    assert torch.equal(pool[0, 7, 0, :, 0], pool[places[2:3] // 128, 7, 0, :, places[2:3] % 128][0])
    assert int(pool[..., 1, :, :, :].count_nonzero()) == int(x[:, 16:].count_nonzero())
    first, keys = out.clone(), pool[places // 128, 7, 0, :, places % 128].clone()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=stream):
        mtp.mtp_rotary_append(args, torch.cuda.current_stream())
    out.zero_()
    pool[places // 128, 7] = 0
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, first) and torch.equal(pool[places // 128, 7, 0, :, places % 128], keys)
    x.mul_(0.5)  # a replay takes what the buffers hold then
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(out, (first.float() * 0.5).bfloat16())


def test_no_rows():
    torch = pytest.importorskip("torch")
    mtp = lib_module()
    pool = torch.ones(1, 1, 2, 1, 16, 64, dtype=torch.bfloat16, device="cuda")
    x = torch.zeros(0, 1, 64, dtype=torch.bfloat16, device="cuda")
    turns = mtp.mtp_rotary_turns(64)
    mtp.mtp_rotary_append(mtp.rotary_append_args(
        q=x, k=x, v=x, positions=torch.zeros(0, dtype=torch.int32, device="cuda"),
        slot_map=torch.zeros(0, dtype=torch.int64, device="cuda"), turns=turns, kv_pool=pool, layer=0,
        out_q=torch.empty_like(x)))
    assert bool((pool == 1).all())
