"""The whole layer at the ends of the range of scales, rows and hidden values, and tokens that are no numbers and have no expert.

One expert, chosen by every token with weight 1. Sums of n products of a weight and a 16-bit part are off by at most n 2^-23 of
the sum of their sizes, the gate by (1.5 |g| + 8) 2^-24 of itself. The parts of a row's element in fp32 or of a hidden value add up to it but for
less than 2^-133, the least magnitude that a part can have.
"""
import numpy as np
import pytest
import torch

import mx_reference as mx
import paper_2608_00358_amd as H
from test_zz_gpu_moe import DEV, F32, INF, TYPES, host, rounded

pytestmark = pytest.mark.gpu
U8 = torch.uint8
PARTS = {"bf16": 1, "fp16": 2, "fp32": 3}
LEAST = 2.0 ** -133


@pytest.fixture(scope="module")
def comm():
    with H.Comm(1, device=0) as c:
        yield c


def run(comm, x, w_in, w_out, experts=1, logits=None, **kw):
    """w_in and w_out: codes and scales of the held experts, in numpy."""
    T, C = x.shape
    new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
    up = lambda w: [torch.from_numpy(t).to(DEV) for t in w]  # noqa: E731
    held, F = w_in[0].shape[0], w_in[0].shape[1] // 2
    space, out = new(H.hccl_moe_layer_mx_bytes(T, 1, C, F, held), dtype=U8), new(T, C, dtype=x.dtype)
    comm.moe_layer_mx(H.hccl_router_init(experts=experts, top_k=1, renormalize=True), new(T, experts).zero_() if logits is None else logits, x, *up(w_in), *up(w_out),
                      new(T, 1, dtype=torch.int32), new(T, 1), out, workspace=space, **kw)
    torch.cuda.synchronize()
    return out


def random_weights(rng, n, d, scale, greatest=15):
    """One expert's n rows of d random codes, magnitudes up to the code `greatest` & 7, under one scale for each row's blocks."""
    code = (rng.integers(0, (greatest & 7) + 1, (1, n, d)) + 8 * rng.integers(0, 2, (1, n, d))).astype(np.uint8)
    return mx.pack(code), np.broadcast_to(np.asarray(scale, np.uint8).reshape(1, -1, 1), (1, n, mx.blocks(d))).copy()


def check(comm, x, w_in, w_out, dt):
    C, F = x.shape[1], w_in[0].shape[1] // 2
    v, a, b = host(x), mx.values(*w_in, C)[0], mx.values(*w_out, F)[0]
    h, size = v @ a.T, np.abs(v) @ np.abs(a).T
    off = PARTS[dt] * (C + 16) * 2 * F32 * size + (np.abs(v) % LEAST) @ np.abs(a).T
    g, u = h[:, :F], h[:, F:]
    z = mx.silu(g) * u
    dz = 1.1 * off[:, :F] * np.abs(u) + np.abs(mx.silu(g)) * off[:, F:] + 1.1 * off[:, :F] * off[:, F:] + (1.5 * np.abs(g).max() + 8) * F32 * np.abs(z) + LEAST
    bound = dz @ np.abs(b).T + 3 * (F + 32) * 2 * F32 * ((np.abs(z) + dz) @ np.abs(b).T)
    want = z @ b.T
    assert np.abs(want).max() > 1e-3 and (bound < np.abs(want).max() / 10).all()  # (so that it tells something)
    rounded(run(comm, x, w_in, w_out), want, bound)


SIZES = [(1, 64, 32), (3, 512, 256), (7, 100, 45), (18, 256, 96)]


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("T,C,F", SIZES)
@pytest.mark.parametrize("b", [0, 1, 2, 30, 200, 240, 252])
def test_far_scales_of_the_first_products(comm, T, C, F, b, dt):
    """Every scale up to 252, with rows of the opposite size: the least scale's elements are subnormal 16-bit floats."""
    rng = np.random.default_rng(b + C)
    x = rng.choice([-1, 1], (T, C)) * (1 + rng.integers(0, 128, (T, C)) / 128) * 2.0 ** (127 - b - 3)
    x = np.round(x / LEAST) * LEAST if b == 252 else x  # (whole parts)
    x = torch.from_numpy(np.clip(x, -2.0 ** 126, 2.0 ** 126)).to(TYPES[dt]).to(DEV)
    check(comm, x, random_weights(rng, 2 * F, C, b), random_weights(rng, C, F, 122), dt)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("T,C,F", SIZES)
@pytest.mark.parametrize("b", [8, 20, 200, 230, 246])
def test_far_scales_of_the_last_product(comm, T, C, F, b, dt):
    """Hidden values of the opposite size, by ups that are far away and gates that are not."""
    rng = np.random.default_rng(b + C)
    x = torch.from_numpy(rng.normal(size=(T, C))).to(TYPES[dt]).to(DEV)
    scale = np.repeat([124 - int(np.log2(C) / 2), 254 - b - 8], F)
    check(comm, x, random_weights(rng, 2 * F, C, scale), random_weights(rng, C, F, b), dt)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_small_rows(comm, dt):
    """Rows near the least normal number and below it."""
    rng = np.random.default_rng(0)
    for k in (-124, -128, -131):
        x = torch.from_numpy(rng.integers(-8, 9, (5, 96)) * 2.0 ** (k - 2)).to(TYPES[dt]).to(DEV)
        check(comm, x, random_weights(rng, 64, 96, 127 - k - 6 if k > -128 else 248), random_weights(rng, 96, 32, 127), dt)
    x = torch.from_numpy((1 + rng.integers(0, 1 << 23, (5, 96)) * 2.0 ** -23) * 2.0 ** -120).to(TYPES[dt]).to(DEV)  # (in fp32 the last 10 bits are lost)
    check(comm, x, random_weights(rng, 64, 96, 241), random_weights(rng, 96, 32, 127), dt)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
def test_elements_beyond_32_bits_are_infinite(comm, dt):
    """Scales 253 and 254: elements below 2^128 are themselves, others infinite, and what they are multiplied by no number."""
    rng = np.random.default_rng(1)
    x = torch.from_numpy(rng.integers(1, 9, (5, 96)) * rng.choice([-1, 1], (5, 96)) * 2.0 ** -129).to(TYPES[dt]).to(DEV)
    for b, greatest in ((253, 5), (254, 3)):  # codes up to 3, and up to 1.5
        w_in, w_out = random_weights(rng, 64, 96, b, greatest), random_weights(rng, 96, 32, 122)
        check(comm, x, w_in, w_out, dt)
        code = w_in[0][0, 7].copy()
        w_in[0][0, 7, 20] = greatest + 1  # a gate: element 40 is 2^128
        assert not bool(torch.isfinite(run(comm, x, w_in, w_out)[:, np.flatnonzero(mx.values(*w_out, 32)[0, :, 7])]).any())
        w_in[0][0, 7] = code
        w_out = random_weights(rng, 96, 32, 122)
        finite = run(comm, x, w_in, w_out)
        w_out[0][0, 11, 3], w_out[1][0, 11] = greatest + 1, b
        got = run(comm, x, w_in, w_out)
        others = [n for n in range(96) if n != 11]
        assert not bool(torch.isfinite(got[:, 11]).any()) and torch.equal(got[:, others], finite[:, others]) and bool(torch.isfinite(finite).all())


@pytest.mark.parametrize("dt", TYPES)
def test_tokens_that_are_no_numbers_and_have_no_expert_here(comm, dt):
    """Masked, or none of whose experts is held: zeros, whatever their rows hold."""
    rng = np.random.default_rng(2)
    x = torch.from_numpy(rng.normal(size=(6, 70))).to(TYPES[dt]).to(DEV)
    logits = torch.zeros(6, 4, device=DEV)
    logits[[0, 3], 1], logits[[1, 2, 4, 5], 2] = 5.0, 5.0
    x[1, 4], x[2, 69], x[3, 0], x[4, 33] = INF, float("nan"), -INF, float("nan")
    mask = torch.tensor([1, 1, 0, 1, 1, 1], dtype=U8, device=DEV)
    w_in, w_out = random_weights(rng, 80, 70, 122), random_weights(rng, 70, 40, 122)
    both = lambda w: [np.repeat(t, 2, 0) for t in w]  # noqa: E731
    got = run(comm, x, both(w_in), both(w_out), 4, logits, mask=mask, first=0)  # experts 0 and 1: tokens 0 and 3
    assert bool((got[[1, 2, 4, 5]] == 0).all()) and bool(torch.isfinite(got[0]).all()) and not bool(torch.isfinite(got[3]).any())
    got = run(comm, x, both(w_in), both(w_out), 4, logits, mask=mask, first=2)  # experts 2 and 3: tokens 1, 4 and 5; 2 is masked
    assert bool((got[[0, 2, 3]] == 0).all()) and bool(torch.isfinite(got[5]).all()) and not bool(torch.isfinite(got[[1, 4]]).any())
