"""Calls of many tokens and short rows: a launch's threads are counted in 32 bits, and each kernel is held to its own.

Results are compared with the same arithmetic in torch where it is one rounded operation for an element, and sums
with their 64-bit values, off by at most n 2^-24 of their terms' sizes for n additions on one path.
"""
import pytest
import torch

import paper_2608_00358_amd as H
from test_zz_gpu_moe import DEV, F32

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def comm():
    with H.Comm(1, device=0) as c:
        yield c


@pytest.mark.parametrize("tokens,cols", [((1 << 22) + 5, 8), ((1 << 22) + 5, 136), ((1 << 22) + 5, 320)])
def test_gradients_of_combine_of_many_tokens(comm, tokens, cols):
    g = torch.Generator(device=DEV).manual_seed(cols)
    grad, z = (torch.randn(tokens, cols, generator=g, device=DEV).to(torch.bfloat16) for _ in range(2))
    weight = torch.rand(tokens, 1, generator=g, device=DEV)
    row = torch.arange(tokens - 1, -1, -1, device=DEV, dtype=torch.int32).view(-1, 1)
    y, gz, gw = torch.empty_like(grad), torch.empty_like(z), torch.full_like(weight, 77)
    comm.moe_combine(z, row, y, weight=weight)
    comm.moe_combine_backward(grad, z, row, weight, gz, gw)
    torch.cuda.synchronize()
    for at in range(0, tokens, 1 << 19):
        part = slice(at, min(at + (1 << 19), tokens))
        r = row[part, 0].long()
        assert torch.equal(y[part], (weight[part] * z[r].float()).to(torch.bfloat16))
        assert torch.equal(gz[r], (weight[part] * grad[part].float()).to(torch.bfloat16))
        terms = grad[part].double() * z[r].double()
        bound = (cols / 64 + 24) * F32 * terms.abs().sum(1) + 1e-37
        assert bool(((gw[part, 0].double() - terms.sum(1)).abs() <= bound).all())


@pytest.mark.parametrize("gated", [False, True])
def test_quantise_of_many_rows(comm, gated):
    rows, cols = (1 << 24) + 3, 4
    g = torch.Generator(device=DEV).manual_seed(5)
    x = torch.randn(rows, 2 * cols if gated else cols, generator=g, device=DEV).to(torch.bfloat16)
    codes, scale = torch.full((rows, cols), 99, device=DEV, dtype=torch.int8), torch.full((rows,), 77.0, device=DEV)
    comm.moe_quantize(x, codes, scale, gated=gated)
    torch.cuda.synchronize()
    v = x.double()
    if gated:
        v = v[:, :cols] * torch.sigmoid(v[:, :cols]) * v[:, cols:]
    m = v.abs().amax(1, keepdim=True)
    # the gate in 32 bits is off by 8 units at most, the scale and the codes' quotient and product by 3 more
    assert bool(((codes.double() - v * 127 / m).abs() <= 0.5 + 127 * 24 * F32).all())
    assert bool(((scale.double() - m[:, 0] / 127).abs() <= 24 * F32 * m[:, 0]).all())


def test_dispatch_in_8_bits_of_many_tokens(comm):
    tokens, cols = (1 << 24) + 3, 3
    g = torch.Generator(device=DEV).manual_seed(6)
    x = torch.randn(tokens, cols, generator=g, device=DEV)
    row = torch.arange(tokens - 1, -1, -1, device=DEV, dtype=torch.int32).view(-1, 1)
    codes, scale = torch.full((tokens, cols), 99, device=DEV, dtype=torch.int8), torch.full((tokens,), 77.0, device=DEV)
    comm.moe_dispatch(x, row, codes, scale=scale)
    torch.cuda.synchronize()
    m = x.double().abs().amax(1, keepdim=True)
    assert bool(((codes.flip(0).double() - x.double() * 127 / m).abs() <= 0.5 + 127 * 8 * F32).all())
    assert bool(((scale.flip(0).double() - m[:, 0] / 127).abs() <= 8 * F32 * m[:, 0]).all())
