"""Shares among chosen experts whose sigmoid scores are small, on the GPU against 64 bits.

A renormalised weight is a share: however small the chosen experts' scores are, their shares are not, and
neither is the gradient, (g_k - sum_j g_j p_j) p_k (1 - s_k) with the shares p. Tolerances as in
test_zz_gpu_moe.py: 1e-5 for a share (exponentials of differences below 32, sums and quotients in 32 bits), and for
the gradient, whose terms cancel, 4 times that of the terms' size.
"""
import numpy as np
import pytest
import torch

import moe_reference as ref
import paper_2608_00358_amd as H
from test_zz_gpu_moe import DEV, INF, Room, TYPES, check_route, host, rand, rounded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def comm():
    with H.Comm(4, device=0) as c:
        yield c


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("experts", [32, 200, 600])
def test_shares_of_sigmoid_scores_far_below_one(comm, experts, dt):
    rng = np.random.default_rng(experts)
    centers = (0.0, 3.0, -1.0, -20.0, -60.0, -80.0, -86.0, -88.0, -95.0, -103.0, -110.0, -200.0)
    K, T = 4, 2 * len(centers)
    logits = rand(rng, T, experts, dt)
    logits += torch.tensor(centers, device=DEV, dtype=TYPES[dt]).repeat(2)[:, None]
    logits[len(centers) + 6] = -INF
    logits[len(centers) + 6, :2] = -87.0     # two experts that share the weight, and no others
    logits[len(centers) + 7, 1:] -= 100.0    # one that has all but nothing of it beside the others
    cfg = dict(experts=experts, top_k=K, score="sigmoid", renormalize=True, scale=2.5)
    index = check_route(comm, cfg, logits, dt=dt)
    grad = torch.from_numpy(15.0 * rng.normal(size=(T, K)).astype(np.float32)).to(DEV)
    out = Room(T, experts, TYPES[dt])
    comm.moe_route_backward(H.hccl_router_init(**cfg), logits, torch.from_numpy(index.astype(np.int32)).to(DEV), grad, out.view)
    torch.cuda.synchronize()
    out.check()
    l = host(logits)
    want = ref.route_backward(l, index, host(grad), **cfg)
    size = np.zeros((T, experts))
    for t in range(T):
        at = index[t][index[t] >= 0]
        s = ref.scores(l[t], "sigmoid")[at]
        size[t, at] = 2.5 * np.abs(host(grad)[t]).max() * s / s.sum()
    rounded(out.view, want, 4e-5 * size)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
def test_sigmoid_scores_that_are_none(comm, dt):
    """Down to logits of -708 there are scores, and shares, in 64 bits; below them, as under a mask, there is nothing."""
    rng = np.random.default_rng(9)
    low = {"bf16": -1e9, "fp16": -6e4, "fp32": -1e9}[dt]
    logits = rand(rng, 8, 64, dt)
    logits[:2] -= 690.0
    logits[2:4] -= 1000.0
    logits[4:6] = low
    logits[6] = torch.finfo(TYPES[dt]).min
    logits[7, 3:] = low      # three left, which share it all
    cfg = dict(experts=64, top_k=4, score="sigmoid", renormalize=True, scale=1.5)
    index = check_route(comm, cfg, logits, dt=dt)
    grad = torch.from_numpy(rng.normal(size=(8, 4)).astype(np.float32)).to(DEV)
    out = Room(8, 64, TYPES[dt])
    comm.moe_route_backward(H.hccl_router_init(**cfg), logits, torch.from_numpy(index.astype(np.int32)).to(DEV), grad, out.view)
    torch.cuda.synchronize()
    out.check()
    l = host(logits)
    want = ref.route_backward(l, index, host(grad), **cfg)
    size = np.zeros((8, 64))
    for t in (0, 1, 7):
        s = ref.scores(l[t], "sigmoid")[index[t]]
        size[t, index[t]] = 1.5 * np.abs(host(grad)[t]).max() * s / s.sum()
    assert not want[2:7].any()
    rounded(out.view, want, 4e-5 * size)
