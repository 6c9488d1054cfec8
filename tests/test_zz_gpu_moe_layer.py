"""The example's layer: all mixture-of-experts operators around the exchange, as a user runs them.

Serving quantises rows and weights twice to 8 bits with a scale of max / 127: an element is off by up to half
a step, max / 254, of a row whose values are about max / 3.5 in size (normal, 512 of them): 0.8 % of a value in
the mean square (step / sqrt(12)), for each of four operands, adding up in squares to 1.6 %; the gate passes
errors on from both factors: 3 % bounds it. Training runs in 32 bits: sums of 64 to 200 terms, 1e-5.

This file comes after those of the resident executor: matrix products of torch make streams that live on,
and with some numbers of live streams the runtime gives the executor's stream the hardware queue of the
default stream, whose work then waits until the executor has been idle for its limit.
"""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("moe_layer", _PATH)
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


@pytest.mark.parametrize("ranks,tokens,experts,top_k", [(8, 48, 32, 4), (1, 1, 8, 2), (4, 33, 64, 6), (2, 300, 4, 1)])
def test_serving_layer(example, ranks, tokens, experts, top_k):
    assert example.serve(ranks=ranks, tokens=tokens, experts=experts, top_k=top_k) < 0.03


@pytest.mark.parametrize("tokens,experts,top_k", [(200, 16, 2), (1, 8, 1), (77, 60, 5)])
def test_training_step(example, tokens, experts, top_k):
    torch.backends.cuda.matmul.allow_tf32 = False
    assert example.train(tokens=tokens, experts=experts, top_k=top_k) < 1e-5
