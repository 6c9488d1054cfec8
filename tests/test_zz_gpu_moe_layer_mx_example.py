"""The example's decoding layer: 4-bit weights on several ranks, whose results AllReduce adds up.

The layer itself is off by far less than the roundings to 16 bits: each rank's result has one, of 2^-8 of its size, and the
ring's sums over P ranks one at each of P - 1 additions. The parts of a sum are about 1 / sqrt(P) of its size each and do not
line up, so that partial sums are no longer than about the whole; P roundings of at most 2^-8 with a mean square of
1 / sqrt(3) of that: sqrt(P) 2^-8 bounds them for up to 8 ranks, with what one rank's own rounding and the router's product in
32 bits add.
"""
import importlib.util
import os

import pytest

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_layer", _PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("ranks,tokens,experts,top_k,hidden,inner", [(4, 8, 32, 4, 512, 256), (1, 1, 8, 2, 64, 32), (8, 64, 64, 6, 256, 96), (2, 5, 6, 1, 100, 40)])
def test_decoding_layer(example, ranks, tokens, experts, top_k, hidden, inner):
    assert example.decode(ranks, tokens, experts, top_k, hidden, inner) < (ranks + 1) ** 0.5 * 2.0 ** -8
