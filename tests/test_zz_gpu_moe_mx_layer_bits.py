"""How many bits of rows and of hidden values the whole layer keeps, on sums whose results are what is left of two near values.

Every weight row has one or two codes of 1 or -1 under the scale 1, so that a gate is an element of a token and an up one or
the sum of two, exactly; and a result is the difference of two hidden values, which 32 bits hold exactly as well, from
whichever parts they are made. One token's choice of one expert, renormalised, has weight 1. So all that rounds is the gate,
off by (1.5 |g| + 8) 2^-24 of itself, its product, of at most two roundings by 2^-24 of a hidden value each, and the result's type.
"""
import numpy as np
import pytest
import torch

import mx_reference as mx
import paper_2608_00358_amd as H
from test_zz_gpu_moe import DEV, F32, TYPES, host, rounded

pytestmark = pytest.mark.gpu
U8 = torch.uint8


@pytest.fixture(scope="module")
def comm():
    with H.Comm(1, device=0) as c:
        yield c


def packed(w, pad):
    """Weights (rows, n) of 0, 1 and -1 as one expert's codes and scales, rows `pad` bytes longer than they need."""
    code = np.where(w == 0, 0, np.where(w > 0, 2, 10)).astype(np.uint8)
    codes, scale = mx.pack(code), np.full((w.shape[0], mx.blocks(w.shape[1])), 127, np.uint8)
    return [torch.from_numpy(np.pad(t, ((0, 0), (0, pad)), constant_values=77)).to(DEV)[None, :, :t.shape[1]] for t in (codes, scale)]


def run(comm, x, w_in, w_out, pad):
    T, C = x.shape
    F = w_out.shape[1]
    new = lambda *s, dtype=torch.float32: torch.empty(s, dtype=dtype, device=DEV)  # noqa: E731
    space, out = new(H.hccl_moe_layer_mx_bytes(T, 1, C, F, 1), dtype=U8), new(T, C, dtype=x.dtype)
    comm.moe_layer_mx(H.hccl_router_init(experts=1, top_k=1, renormalize=True), new(T, 1).zero_(), x, *packed(w_in, pad), *packed(w_out, pad),
                      new(T, 1, dtype=torch.int32), new(T, 1), out, workspace=space)
    torch.cuda.synchronize()
    return out


# (tokens, columns, inner, bytes behind a weight row): 4, 8 and 16 rows a matrix instruction, whole steps and row ends, aligned and not
SHAPES = [(1, 512, 512, 0), (3, 200, 78, 0), (8, 512, 256, 16), (8, 333, 300, 1), (20, 768, 512, 0), (64, 300, 640, 3)]


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T,C,F,pad", SHAPES)
def test_hidden_values_are_kept_in_32_bits(comm, T, C, F, pad, dt):
    """Two of them that differ by 2^-18 of their size: parts that hold 16 bits would have nothing of that."""
    rng = np.random.default_rng(T + C + F)
    third = C // 3
    x = np.empty((T, C))
    x[:, :third] = rng.uniform(1, 2, (T, third))
    x[:, third:2 * third] = rng.choice([-1.5, -1, 1, 1.5], (T, third)) * 2.0 ** -18
    x[:, 2 * third:] = rng.uniform(0.5, 2, (T, C - 2 * third))
    x = torch.from_numpy(x).to(TYPES[dt]).to(DEV)
    if dt == "fp32":
        x[:, :third] = (x[:, :third] * 32).round() / 32  # (a sum with 2^-18 fits 24 bits)
    w_in, w_out = np.zeros((2 * F, C)), np.zeros((C, F))
    pairs = F // 2
    for p in range(pairs):
        w_in[2 * p:2 * p + 2, 2 * third + rng.integers(C - 2 * third)] = 1  # the gates
        near = rng.integers(third)
        w_in[F + 2 * p:F + 2 * p + 2, near] = 1
        w_in[F + 2 * p + 1, third + rng.integers(third)] = 1
    for n in range(C):
        p = rng.integers(pairs) if n else pairs - 1
        w_out[n, 2 * p], w_out[n, 2 * p + 1] = -1, 1
    v = host(x)
    h = v @ w_in.T
    z = mx.silu(h[:, :F]) * h[:, F:]
    want, size = z @ w_out.T, np.abs(z) @ np.abs(w_out).T
    rounded(run(comm, x, w_in, w_out, pad), want, (1.5 * 2 + 8) * F32 * np.abs(want) + 2 * F32 * size)


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T,C,F,pad", SHAPES)
def test_rows_enter_with_all_their_bits(comm, T, C, F, pad, dt):
    """An up is the difference of two elements that are a few of the type's steps apart, with every bit between."""
    rng = np.random.default_rng(T + C + F)
    half = C // 2
    eps = torch.finfo(TYPES[dt]).eps
    x = np.empty((T, C))
    x[:, :half] = 1 + rng.integers(0, int(1 / eps), (T, half)) * eps
    x[:, half:2 * half] = x[:, :half] + rng.choice([-3, -2, -1, 1, 2, 3], (T, half)) * eps
    x[:, -1] = rng.uniform(0.5, 2, T)
    x = torch.from_numpy(x).to(TYPES[dt]).to(DEV)
    w_in, w_out = np.zeros((2 * F, C)), np.zeros((C, F))
    w_in[:F, -1] = 1
    for f in range(F):
        a = rng.integers(half - 1)
        w_in[F + f, a], w_in[F + f, half + a] = -1, 1
    for n in range(C):
        w_out[n, rng.integers(F) if n else F - 1] = 1
    v = host(x)
    h = v @ w_in.T
    want = (mx.silu(h[:, :F]) * h[:, F:]) @ w_out.T
    rounded(run(comm, x, w_in, w_out, pad), want, (1.5 * 2 + 8 + 2) * F32 * np.abs(want))
