"""Microscaled 4-bit rows and products on the GPU against their definitions in 64 bits.

Codes and scales of values as they are given are exact: a quotient by a power of two is. A gated value is off by
(1.5 |g| + 8) 2^-24 of itself, so its code may be that of either end of that interval. In a product the sum over a block of
32 is exact; adding n of them rounds each by at most 2^-23 of the sizes added so far (a matrix instruction may cut
off what an addition would round), and joining up to 16 parts of a sum rounds those: (n + 16) 2^-23 of the sum of sizes. Then
one rounding to the result's type, which keeps order.
"""
import numpy as np
import pytest
import torch

import mx_reference as mx
import paper_2608_00358_amd as H
from gpu_helpers import SideStream
from test_zz_gpu_moe import DEV, F32, INF, TYPES, Room, host, place, rand, rounded

pytestmark = pytest.mark.gpu
U8 = torch.uint8


@pytest.fixture(scope="module")
def comm():
    with H.Comm(4, device=0) as c:
        yield c


def bytes_of(n):
    return (n + 1) // 2


def quantize(comm, x, cols, gated=False, pad=0, shift=0):
    codes, scale = Room(x.shape[0], bytes_of(cols), U8, pad, shift), Room(x.shape[0], mx.blocks(cols), U8, pad, shift)
    comm.moe_quantize_mx(x, codes.view, scale.view, gated=gated)
    torch.cuda.synchronize()
    codes.check(), scale.check()
    return host(codes.view), host(scale.view)


# ------------------------------------------------------------------------------------------- rows

@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,cols", [
    (1, 1), (1, 2), (3, 3), (2, 7), (5, 8), (9, 9), (300, 17), (4, 31), (17, 32), (33, 33), (5, 63), (6, 64), (100, 65), (7, 255), (19, 480), (3, 511),
    (70, 513), (1, 4096), (40, 1001), (2050, 321), (130, 4099)])
def test_quantize(comm, rows, cols, dt):
    rng = np.random.default_rng(rows + cols)
    for pad, shift in ((0, 0), (3, 1)):
        x = rand(rng, rows, cols, dt, pad, 1.0, shift)
        x *= torch.exp2(torch.randint(-9, 9, x.shape, device=DEV)).to(x.dtype)
        codes, scale = quantize(comm, x, cols, pad=pad, shift=shift)
        want = mx.quantize(host(x))
        assert np.array_equal(scale, want[1]) and np.array_equal(codes, want[0])


@pytest.mark.parametrize("dt", TYPES)
def test_quantize_where_values_lie_between_codes(comm, dt):
    """Ties and the neighbours of ties, the borders where the scale changes, signs of zeros."""
    eps = torch.finfo(TYPES[dt]).eps
    ties = np.array([0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 6.5])
    x = []
    for k in (-20, -3, 0, 5, 12) if dt != "fp16" else (-10, -3, 0, 5):
        for top in (4.0, 6.0, 7.0 * (1 - eps), 3.5, 7.0, 6.0 * (1 + eps)):
            for near in (ties, ties * (1 + eps), ties * (1 - eps / 2)):
                row = np.zeros(32)
                row[0] = top
                row[1:9] = np.minimum(near, top)
                row[9:17] = -row[1:9]
                row[17] = -0.0
                x.append(row * 2.0 ** k)
    x = torch.from_numpy(np.array(x)).to(TYPES[dt]).to(DEV)
    codes, scale = quantize(comm, x, 32)
    want = mx.quantize(host(x))
    assert np.array_equal(scale, want[1]) and np.array_equal(codes, want[0])


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_quantize_at_the_ends_of_the_range(comm, dt):
    """Magnitudes from the least subnormal number to the greatest there is."""
    big = torch.finfo(TYPES[dt]).max
    rows = [2.0 ** k * np.linspace(-1, 1, 32) for k in (-149, -133, -130, -127, -126, -125, -124, -123, -100, 100, 126)] + [np.full(32, big), np.zeros(32)]
    x = torch.from_numpy(np.array(rows)).to(TYPES[dt]).to(DEV)
    codes, scale = quantize(comm, x, 32)
    want = mx.quantize(host(x))
    assert np.array_equal(scale, want[1]) and np.array_equal(codes, want[0])
    assert scale[-2] == 253 and scale[-1] == 0


@pytest.mark.parametrize("dt", TYPES)
def test_blocks_that_are_no_numbers(comm, dt):
    """An infinity or NaN takes its block of 32 and no other."""
    rng = np.random.default_rng(0)
    x = rand(rng, 5, 100, dt)
    x[0, 5], x[1, 40], x[2, 99], x[3, 64] = INF, float("nan"), -INF, float("nan")
    codes, scale = quantize(comm, x, 100)
    want = mx.quantize(host(x))
    assert np.array_equal(scale, want[1]) and np.array_equal(codes, want[0])
    assert [(r, b) for r, b in np.argwhere(scale == 255).tolist()] == [(0, 0), (1, 1), (2, 3), (3, 2)]
    out = torch.empty(5, 100, dtype=TYPES[dt], device=DEV)
    comm.moe_dequantize_mx(torch.from_numpy(codes).to(DEV), torch.from_numpy(scale).to(DEV), out)
    assert np.array_equal(np.isnan(host(out)), np.repeat(scale == 255, 32, 1)[:, :100])


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 2048), (3, 1407), (2049, 72), (5, 33)])
def test_quantize_of_a_gate(comm, rows, cols, dt):
    rng = np.random.default_rng(rows)
    for pad, shift in ((0, 0), (5, 1)):
        x = rand(rng, rows, 2 * cols, dt, pad, 2.0, shift)
        codes, scale = quantize(comm, x, cols, gated=True, pad=pad, shift=shift)
        v = host(x)
        z = mx.silu(v[:, :cols]) * v[:, cols:]
        off = (1.5 * np.abs(v[:, :cols]) + 8) * F32 * np.abs(z) + 1e-37
        got = mx.values(codes, scale, cols)
        lo, hi = (z - off).astype(float), (z + off).astype(float)
        # a block's scale is that of its greatest magnitude, at either end of the interval
        small, great = (mx.scales(np.sign(z) * np.maximum(np.abs(z) + s * off, 0)) for s in (-1, 1))
        assert ((small <= scale) & (scale <= great)).all()
        ends = [np.where(np.signbit(e), -1, 1) * mx.VALUES[mx.codes(e, scale) & 7] * 2.0 ** (np.repeat(scale.astype(float), 32, 1)[:, :cols] - 127) for e in (lo, hi)]
        assert ((ends[0] <= got) & (got <= ends[1])).all()


def test_quantize_up_to_a_limit_on_the_device(comm):
    rng = np.random.default_rng(0)
    x = rand(rng, 30, 100, "bf16")
    want, want_scale = mx.quantize(host(x))
    back = mx.values(want, want_scale, 100)
    for n in (0, 1, 17, 30, 99, -4):
        limit = torch.tensor([n], device=DEV)
        codes, scale, out = torch.full((30, 50), 77, dtype=U8, device=DEV), torch.full((30, 4), 77, dtype=U8, device=DEV), torch.full((30, 100), 77.0, device=DEV)
        comm.moe_quantize_mx(x, codes, scale, limit=limit)
        comm.moe_dequantize_mx(codes, scale, out, limit=limit)
        k = min(max(n, 0), 30)
        assert np.array_equal(host(codes)[:k], want[:k]) and bool((codes[k:] == 77).all())
        assert np.array_equal(host(scale)[:k], want_scale[:k]) and bool((scale[k:] == 77).all())
        assert np.array_equal(host(out)[:k], back[:k]) and bool((out[k:] == 77).all())


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("tokens,top_k,cols", [(1, 1, 1), (1, 4, 4096), (37, 4, 1001), (100, 8, 64), (3, 32, 33), (2050, 2, 255), (600, 3, 2048)])
def test_dispatch(comm, tokens, top_k, cols, dt):
    """Routes without a row, rows beyond the capacity, rows that nobody names."""
    rng = np.random.default_rng(tokens + cols)
    x = rand(rng, tokens, cols, dt, 2, 1.0, 1)
    want, want_scale = mx.quantize(host(x))
    capacity = tokens * top_k + 3
    row = rng.permutation(capacity + 5)[:tokens * top_k].reshape(tokens, top_k).astype(np.int32)
    row[rng.random(row.shape) < 0.2] = -1
    codes, scale = Room(capacity, bytes_of(cols), U8, 1, 1), Room(capacity, mx.blocks(cols), U8, 2)
    comm.moe_dispatch_mx(x, torch.from_numpy(row).to(DEV), codes.view, scale.view)
    torch.cuda.synchronize()
    codes.check(), scale.check()
    all_codes, all_scale = np.full((capacity, bytes_of(cols)), 77, np.uint8), np.full((capacity, mx.blocks(cols)), 77, np.uint8)
    for t in range(tokens):
        for r in row[t]:
            if 0 <= r < capacity:
                all_codes[r], all_scale[r] = want[t], want_scale[t]
    assert np.array_equal(host(codes.view), all_codes) and np.array_equal(host(scale.view), all_scale)


@pytest.mark.parametrize("dt", TYPES)
def test_dequantize_every_code_and_scale(comm, dt):
    codes = np.tile(np.arange(256, dtype=np.uint8), (256, 1))
    scale = np.repeat(np.arange(256, dtype=np.uint8)[:, None], 16, 1)
    out = torch.empty(256, 512, dtype=TYPES[dt], device=DEV)
    comm.moe_dequantize_mx(torch.from_numpy(codes).to(DEV), torch.from_numpy(scale).to(DEV), out)
    want = torch.from_numpy(mx.values(codes, scale, 512)).float().to(TYPES[dt])
    assert torch.equal(torch.nan_to_num(out.cpu(), nan=77.0), torch.nan_to_num(want, nan=77.0))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,cols", [(1, 1), (2, 3), (3, 7), (5, 9), (300, 17), (33, 33), (70, 513), (40, 1001), (2050, 321)])
def test_dequantize(comm, rows, cols, dt):
    rng = np.random.default_rng(rows + cols)
    codes = place(torch.from_numpy(rng.integers(0, 256, (rows, bytes_of(cols) + 1), dtype=np.uint8)), 1)[:, :bytes_of(cols)]
    scale = place(torch.from_numpy(rng.integers(117, 137, (rows, mx.blocks(cols) + 2), dtype=np.uint8)), 3)[:, :mx.blocks(cols)]
    out = Room(rows, cols, TYPES[dt], 5, 1)
    comm.moe_dequantize_mx(codes, scale, out.view)
    torch.cuda.synchronize()
    out.check()
    want = torch.from_numpy(mx.values(host(codes), host(scale), cols)).to(TYPES[dt])
    assert torch.equal(out.view.cpu(), want)


def test_large_rows(comm):
    """More blocks than a launch of few has, in rows to several places, against the same rows in small calls."""
    g = torch.Generator(device=DEV).manual_seed(0)
    x = torch.randn(40000, 1003, generator=g, device=DEV).to(torch.bfloat16)
    row = torch.randperm(80000, generator=g, device=DEV).to(torch.int32).view(40000, 2)
    codes, scale = torch.zeros(80000, 502, dtype=U8, device=DEV), torch.zeros(80000, 32, dtype=U8, device=DEV)
    comm.moe_dispatch_mx(x, row, codes, scale)
    out = torch.empty(80000, 1003, device=DEV, dtype=torch.bfloat16)
    comm.moe_dequantize_mx(codes, scale, out)
    part = torch.arange(0, 40000, 997, device=DEV)
    want = mx.quantize(host(x[part]))
    back = torch.from_numpy(mx.values(*want, 1003)).to(torch.bfloat16)
    for k in range(2):
        at = row[part, k].long()
        assert np.array_equal(host(codes[at]), want[0]) and np.array_equal(host(scale[at]), want[1]) and torch.equal(out[at].cpu(), back)


# ---------------------------------------------------------------------------------------- product

def random_mx(rng, *shape, pad=0, spad=0, shift=0, lo=117, hi=130):
    """Random codes and scales (..., inner) and their values."""
    *lead, n = shape
    codes = place(torch.from_numpy(rng.integers(0, 256, (*lead, bytes_of(n) + pad), dtype=np.uint8)), shift)[..., :bytes_of(n)]
    scale = place(torch.from_numpy(rng.integers(lo, hi, (*lead, mx.blocks(n) + spad), dtype=np.uint8)), shift)[..., :mx.blocks(n)]
    return codes, scale


def on_gpu(a, b, ends, out):
    """The product of values and of their sizes in 64 bits, segment by segment."""
    size = torch.zeros_like(out)
    for s, (first, last) in enumerate(zip(ends[:-1], ends[1:])):
        e = s % b.shape[0]
        if last > first:
            out[first:last] = torch.mm(a[first:last], b[e].t().contiguous())
            size[first:last] = torch.mm(a[first:last].abs(), b[e].abs().t().contiguous())
    return out, size


def values(codes, scale, cols):
    """mx.values on the GPU."""
    table = torch.from_numpy(np.concatenate([mx.VALUES, -mx.VALUES])).to(DEV)
    code = torch.stack([codes & 15, codes >> 4], -1).flatten(-2)[..., :cols]
    power = torch.ldexp(torch.ones((), device=DEV, dtype=torch.float64), scale.int() - 127)
    return table[code.int()] * power.repeat_interleave(32, -1)[..., :cols]


def check_product(comm, a, b, inner, ends, dt, pad=0, shift=0, stream=None):
    rows, (experts, cols) = a[0].shape[0], b[0].shape[:2]
    out = Room(rows, cols, TYPES[dt], pad, shift)
    offsets = None if ends is None else torch.tensor(ends, dtype=torch.int64, device=DEV)
    comm.moe_product_mx(*a, *b, out.view, inner, offsets=offsets, stream=stream)
    torch.cuda.synchronize()
    out.check()
    clipped = [0, rows] if ends is None else [min(max(e, 0), rows) for e in ends]
    base = torch.full((rows, cols), 77.0, dtype=torch.float64, device=DEV)
    want, size = on_gpu(values(*a, inner), values(*b, inner), clipped, base)
    bound = (mx.blocks(inner) + 16) * 2 * F32 * size + F32 * want.abs() + 1e-37
    lo, hi = ((want + s * bound).float().to(TYPES[dt]).double() for s in (-1, 1))
    got = out.view.double()
    bad = ~((lo <= got) & (got <= hi))
    assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}: {got[bad][0]} for {want[bad][0]}"


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("rows,inner,cols", [
    (1, 1, 1), (1, 4096, 4096), (1, 127, 65), (2, 129, 30), (3, 31, 20), (5, 33, 17), (15, 64, 16), (16, 128, 64), (17, 1000, 100), (33, 2048, 48),
    (64, 512, 255), (100, 16, 300), (128, 256, 128), (129, 1407, 257), (255, 96, 512), (300, 640, 1000), (513, 320, 768), (1000, 2049, 70), (40, 0, 33)])
def test_product_of_one_expert(comm, rows, inner, cols, dt):
    rng = np.random.default_rng(rows + inner)
    for pad, spad, shift, ends in ((0, 0, 0, None), (16, 3, 0, [0, rows]), (5, 1, 1, None)):
        a, b = random_mx(rng, rows, inner, pad=pad, spad=spad, shift=shift), random_mx(rng, 1, cols, inner, pad=pad, spad=spad, shift=shift)
        check_product(comm, a, b, inner, ends, dt, pad, shift)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,inner,cols,experts,sources", [
    (1, 256, 64, 4, 1), (7, 100, 40, 16, 1), (64, 512, 200, 8, 1), (256, 384, 130, 64, 1), (300, 130, 64, 100, 1), (1500, 256, 300, 5, 1),
    (900, 272, 256, 3, 4), (4000, 128, 520, 8, 1), (200, 64, 32, 70, 2)])
def test_product_of_segments(comm, rows, inner, cols, experts, sources, dt):
    """Segments of all lengths, some empty, some rows in none; several sources that use the same experts."""
    rng = np.random.default_rng(rows + experts)
    n = experts * sources
    a, b = random_mx(rng, rows, inner), random_mx(rng, experts, cols, inner)
    for skew in (0.0, 3.0):
        p = np.exp(skew * rng.normal(size=n + 1))
        ends = np.concatenate([[0], np.cumsum(rng.multinomial(rows, p / p.sum())[:n])])
        check_product(comm, a, b, inner, ends.tolist(), dt)
    check_product(comm, a, b, inner, [0] * (n + 1), dt)
    check_product(comm, a, b, inner, [0] * n + [rows], dt, pad=3)
    check_product(comm, a, b, inner, [rows // 3] + [rows] * n, dt, pad=16)
    # offsets beyond the rows move nothing beyond them
    check_product(comm, a, b, inner, [0] + [rows + 1000] * n, dt)


# (rows, columns, experts): sizes for each of the tiles that a product chooses among on 256 CUs
TILES = {"256x256": (6000, 2100, 8), "256x256 dense": (3000, 4100, 1), "128x128": (3000, 1500, 12), "64x128": (1000, 2000, 40), "64x64": (300, 3000, 1),
         "few 16x64": (100, 4096, 30), "few 16x32": (3, 8200, 1), "few 16x16": (9, 300, 1), "few 32x64": (512, 2050, 40), "few 32x32": (48, 4100, 1),
         "few 32x16": (505, 185, 1)}


@pytest.mark.parametrize("inner", [16, 32, 33, 64, 128, 129, 255, 256, 384, 511, 512, 640, 896, 1000, 1024, 1151, 1280, 1999, 2048])
@pytest.mark.parametrize("tile", TILES)
def test_product_of_every_tile_and_length(comm, tile, inner):
    rows, cols, experts = TILES[tile]
    rng = np.random.default_rng(rows + inner)
    ends = np.concatenate([[0], np.cumsum(rng.multinomial(rows, rng.dirichlet(np.full(experts, 8.0))))]).tolist() if experts > 1 else None
    dt = ("bf16", "fp16", "fp32")[inner % 3]
    whole = -bytes_of(inner) % 16
    for pa, pb in ((whole, whole), (1 + whole, whole), (whole, 1 + whole), (3, 3)):
        check_product(comm, random_mx(rng, rows, inner, pad=pa, spad=pa % 4), random_mx(rng, experts, cols, inner, pad=pb, spad=pb % 3), inner, ends, dt, pa)


# more of them: tiles that only many columns, or a block for every CU, lead to
MORE_TILES = {"64x64": (400, 3000, 1), "few 16x64": (90, 24000, 8), "few 32x64": (104, 24000, 8)}


@pytest.mark.parametrize("inner", [31, 33, 256, 513, 1000, 1024, 1280])
@pytest.mark.parametrize("tile", MORE_TILES)
def test_product_of_more_tiles_and_lengths(comm, tile, inner):
    rows, cols, experts = MORE_TILES[tile]
    rng = np.random.default_rng(rows + inner)
    ends = np.concatenate([[0], np.cumsum(rng.multinomial(rows, rng.dirichlet(np.full(experts, 8.0))))]).tolist() if experts > 1 else None
    whole = -bytes_of(inner) % 16
    for pad in (whole, 1 + whole):
        check_product(comm, random_mx(rng, rows, inner, pad=pad, spad=pad % 4), random_mx(rng, experts, cols, inner, pad=pad, spad=pad % 3), inner, ends, "bf16", pad)


def test_product_of_many_segments(comm):
    """More segments than a wave has lanes, in one-row tiles and in large ones, some of them empty."""
    for rows, cols, experts, sources in ((700, 512, 100, 3), (9000, 1024, 70, 2), (20000, 300, 33, 8)):
        n = experts * sources
        rng = np.random.default_rng(n)
        ends = np.concatenate([[0], np.cumsum(rng.multinomial(rows, rng.dirichlet(np.full(n, 0.7))))]).tolist()
        check_product(comm, random_mx(rng, rows, 192), random_mx(rng, experts, cols, 192), 192, ends, "fp32")


@pytest.mark.parametrize("rows,cols", [(6, 40), (700, 3000)])
def test_product_of_rows_and_columns_that_are_no_numbers(comm, rows, cols):
    rng = np.random.default_rng(0)
    (a, sa), (b, sb) = random_mx(rng, rows, 320), random_mx(rng, 1, cols, 320)
    sa[1, 3], sa[rows - 1, 9], sb[0, 7, 0] = 255, 255, 255
    a[1, 48:64] = 0
    out = torch.empty(rows, cols, device=DEV)
    comm.moe_product_mx(a, sa, b, sb, out, 320)
    want = torch.zeros(rows, cols, dtype=torch.bool)
    want[1], want[rows - 1], want[:, 7] = True, True, True
    assert torch.equal(torch.isnan(out).cpu(), want)


def test_product_of_far_scales(comm):
    """Scales whose product leaves 32 bits on neither side, though either is far from 1."""
    rng = np.random.default_rng(1)
    a, b = random_mx(rng, 20, 160, lo=1, hi=40), random_mx(rng, 1, 50, 160, lo=200, hi=240)
    check_product(comm, a, b, 160, None, "fp32")


def test_the_upper_half_of_an_odd_rows_last_byte_never_counts(comm):
    rng = np.random.default_rng(2)
    for rows, cols in ((4, 40), (600, 3000)):
        for inner in (31, 97, 225, 513):
            (a, sa), (b, sb) = random_mx(rng, rows, inner), random_mx(rng, 1, cols, inner)
            got = []
            for fill in (0, 0xf0):
                for t in (a, b):
                    t[..., -1] = t[..., -1] & 0x0f | fill
                out = torch.empty(rows, cols, device=DEV)
                comm.moe_product_mx(a, sa, b, sb, out, inner)
                got.append(out)
            assert torch.equal(*got)


# ------------------------------------------------------------------- offsets, streams, graphs, order

def test_nothing_to_do(comm):
    u8, f32 = dict(dtype=U8, device=DEV), dict(device=DEV)
    comm.moe_quantize_mx(torch.empty(0, 8, **f32), torch.empty(0, 4, **u8), torch.empty(0, 1, **u8))
    comm.moe_quantize_mx(torch.empty(3, 0, **f32), torch.empty(3, 0, **u8), torch.empty(3, 0, **u8))
    comm.moe_dispatch_mx(torch.empty(0, 8, **f32), torch.empty(0, 2, dtype=torch.int32, device=DEV), torch.empty(5, 4, **u8), torch.empty(5, 1, **u8))
    comm.moe_dequantize_mx(torch.empty(0, 4, **u8), torch.empty(0, 1, **u8), torch.empty(0, 8, **f32))
    comm.moe_product_mx(torch.empty(0, 4, **u8), torch.empty(0, 1, **u8), torch.zeros(2, 4, 4, **u8), torch.zeros(2, 4, 1, **u8), torch.empty(0, 4, **f32), 8,
                        offsets=torch.zeros(3, dtype=torch.int64, device=DEV))
    torch.cuda.synchronize()


def test_rows_far_apart(comm):
    """Byte offsets beyond 32 bits in every array of rows."""
    step = (1 << 32) + 16
    rng = np.random.default_rng(0)
    big = torch.empty(2 * step + 4096, dtype=U8, device=DEV)
    far_codes, far_scale = big.as_strided((3, 32), (step, 1)), big.as_strided((3, 2), (step, 1), 1024)
    near = rand(rng, 3, 64, "bf16")
    want = mx.quantize(host(near))
    row = torch.tensor([[2], [0], [1]], dtype=torch.int32, device=DEV)
    comm.moe_dispatch_mx(near, row, far_codes, far_scale)
    assert np.array_equal(host(far_codes[[2, 0, 1]]), want[0]) and np.array_equal(host(far_scale[[2, 0, 1]]), want[1])
    far = big.view(torch.bfloat16).as_strided((3, 64), (step // 2, 1), 1024)
    comm.moe_dequantize_mx(far_codes, far_scale, far)
    back = mx.values(*want, 64)
    assert np.array_equal(host(far[[2, 0, 1]]), back)
    codes, scale = torch.empty(3, 32, dtype=U8, device=DEV), torch.empty(3, 2, dtype=U8, device=DEV)
    comm.moe_quantize_mx(far, codes, scale)
    again = mx.quantize(host(far))
    assert np.array_equal(host(codes), again[0]) and np.array_equal(host(scale), again[1])
    b = random_mx(rng, 1, 40, 64)
    same, got = torch.empty(3, 40, device=DEV), torch.empty(3, 40, device=DEV)
    comm.moe_product_mx(far_codes.clone(), far_scale.clone(), *b, same, 64)
    comm.moe_product_mx(far_codes, far_scale, *b, got, 64)
    assert torch.equal(got, same)
    far_w, far_ws = big.as_strided((1, 3, 32), (3 * step, step, 1), 256), big.as_strided((1, 3, 2), (3 * step, step, 1), 512)
    far_w.copy_(b[0][:, :3]), far_ws.copy_(b[1][:, :3])
    comm.moe_product_mx(far_codes, far_scale, far_w, far_ws, got[:, :3], 64)
    assert torch.equal(got[:, :3], same[:, :3])
    far_out = big.view(torch.bfloat16).as_strided((3, 40), (step // 2, 1), 1024)
    comm.moe_product_mx(far_codes, far_scale, *b, far_out, 64)
    assert torch.equal(far_out, same.to(torch.bfloat16))


class Experts:
    """Tokens through experts in 4 bits: routing, order, dispatch, product, gate, product, combination."""

    def __init__(self, comm, T=300, E=16, K=4, C=256, F=96, seed=1):
        g = torch.Generator(device=DEV).manual_seed(seed)
        self.comm = comm
        self.x = torch.randn(T, C, generator=g, device=DEV).to(torch.bfloat16)
        self.logits = torch.randn(T, E, generator=g, device=DEV)

        def weights(n, d):
            codes, scale = torch.empty(E * n, d // 2, dtype=U8, device=DEV), torch.empty(E * n, d // 32, dtype=U8, device=DEV)
            comm.moe_quantize_mx(torch.randn(E * n, d, generator=g, device=DEV) * d ** -0.5, codes, scale)
            return codes.view(E, n, -1), scale.view(E, n, -1)

        self.w_in, self.w_out = weights(2 * F, C), weights(C, F)
        new = lambda *s, dtype=U8: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
        index, weight, row = new(T, K, dtype=torch.int32), new(T, K, dtype=torch.float32), new(T, K, dtype=torch.int32)
        offsets = new(E + 1, dtype=torch.int64)
        codes, scale, hidden = new(T * K, C // 2), new(T * K, C // 32), new(T * K, 2 * F, dtype=torch.bfloat16)
        codes2, scale2, rows = new(T * K, F // 2), new(T * K, F // 32), new(T * K, C, dtype=torch.bfloat16)
        self.y = new(T, C, dtype=torch.bfloat16)
        router = H.hccl_router_init(experts=E, top_k=K, renormalize=True)

        def bind(stream=None):
            s = dict(stream=stream)
            return [comm.bind_moe_route(router, self.logits, index, weight, **s), comm.bind_moe_plan(index, E, row, offsets, T * K, **s),
                    comm.bind_moe_dispatch_mx(self.x, row, codes, scale, **s), comm.bind_moe_product_mx(codes, scale, *self.w_in, hidden, C, offsets=offsets, **s),
                    comm.bind_moe_quantize_mx(hidden, codes2, scale2, gated=True, limit=offsets[-1:], **s),
                    comm.bind_moe_product_mx(codes2, scale2, *self.w_out, rows, F, offsets=offsets, **s),
                    comm.bind_moe_combine(rows, row, self.y, weight=weight, **s)]

        self.bind, self.index, self.weight = bind, index, weight
        self.out = [index, weight, row, offsets, codes, scale, hidden, codes2, scale2, rows, self.y]

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.out]


def test_a_run_of_them_together(comm):
    """The layer in 4 bits is near the layer of the same weights in 64 bits: what is left is the rounding of rows to 4 bits,
    of which half a step is at most 1/4 of a value (a code below 0.5 apart, which is small beside its block's greatest)."""
    e = Experts(comm)
    for call in e.bind():
        call()
    x, index, weight = host(e.x), host(e.index), host(e.weight)
    want = mx.layer(x, index, weight, host(values(*e.w_in, 256)), host(values(*e.w_out, 96)))[0]
    got = host(e.y)
    assert np.linalg.norm(got - want) < 0.25 * np.linalg.norm(want)


def test_results_are_the_same_in_every_call_and_on_another_stream(comm):
    e = Experts(comm)
    calls = e.bind()
    for call in calls:
        call()
    want = e.results()
    for _ in range(3):
        for t in e.out:
            t.zero_()
        for call in calls:
            call()
        assert all(torch.equal(a, b) for a, b in zip(e.results(), want))
    with SideStream() as side:
        torch.cuda.synchronize()
        for t in e.out:
            t.zero_()
        torch.cuda.synchronize()
        for call in e.bind(side):
            call()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(e.results(), want))


def test_a_captured_run_replays(comm):
    """Captured at its first call; replayed on new inputs with eager work in between."""
    e, eager = Experts(comm), Experts(comm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in e.bind():  # (on the stream that captures)
            call()
    calls = eager.bind()
    for seed in range(4):
        g = torch.Generator(device=DEV).manual_seed(100 + seed)
        e.logits.copy_(torch.randn(e.logits.shape, generator=g, device=DEV))
        e.x.copy_(torch.randn(e.x.shape, generator=g, device=DEV))
        eager.logits.copy_(e.logits)
        eager.x.copy_(e.x)
        graph.replay()
        got = e.results()
        for call in calls:
            call()
        assert all(torch.equal(a, b) for a, b in zip(got, eager.results()))
