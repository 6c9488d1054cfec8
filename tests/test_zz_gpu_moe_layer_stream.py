"""The example's serving layer called on a stream that is not the one it was made on.

Its bound calls keep the stream that was current when it was made. The inputs are written, the layer called and the result read
on another one: the layer has to wait for the inputs, do its own torch operations where its bound calls run, and be waited for.
Three passes, each behind work that takes long, against the same passes on the layer's own stream, bit for bit: no
result depends on the stream.
"""
import importlib.util
import os

import pytest
import torch

import paper_2608_00358_amd as H
from gpu_helpers import SideStream

pytestmark = pytest.mark.gpu

_PATH = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples", "moe_layer.py")


def test_serving_layer_called_on_another_stream():
    spec = importlib.util.spec_from_file_location("moe_layer", _PATH)
    example = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(example)
    P, T, E, C, F = 2, 40, 8, 256, 128
    router = H.hccl_router_init(experts=E, top_k=2, renormalize=True)
    weights = example.parameters(0, E, C, F, torch.float32)
    g = torch.Generator(device="cuda:0").manual_seed(3)
    inputs = [torch.randn(T, C, generator=g, device="cuda:0").to(torch.bfloat16) for _ in range(3 * P)]
    slow = torch.randn(4096, 4096, device="cuda:0")

    def passes(layer):
        out = []
        for step in range(3):
            for _ in range(8):
                slow @ slow
            for r in range(P):
                layer.x[r].copy_(inputs[step * P + r])
            out += [t.clone() for t in layer()]
        return out

    with H.Comm(P, device=0) as comm:
        layer = example.ServingLayer(comm, router, *weights, T)
        want = passes(layer)
        torch.cuda.synchronize()
        with SideStream() as side:
            with torch.cuda.stream(side):
                got = passes(layer)
            side.synchronize()
        torch.cuda.synchronize()
        assert comm.async_error() == 0
        for a, b in zip(got, want):
            assert torch.equal(a, b)
