"""An operator on a stream of its own while a resident executor runs.

The operator is launched, not handed to the executor, and nothing orders the two. The runtime may give a stream the
executor's hardware queue; its work then waits until the executor has left the device, at the latest at its idle limit. So the
call is made once before (which loads its kernels), and a limit of 3 s bounds the wait. What is checked is that the
operator completes, with the executor still running or ended, and that its results are right.
"""
import pytest
import torch

import paper_2608_00358_amd as H
from gpu_helpers import SideStream

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
IDLE_MS = 3000


def test_an_operator_beside_a_resident_executor():
    g = torch.Generator(device=DEV).manual_seed(1)
    z = torch.randn(64, 256, generator=g, device=DEV)
    row = torch.randperm(64, generator=g, device=DEV).to(torch.int32).view(32, 2)
    want = z[row[:, 0].long()] + z[row[:, 1].long()]
    out = torch.zeros(32, 256, device=DEV)
    send, recv = ([torch.full((4096,), v, device=DEV) for v in (1.0, 2.0)] for _ in range(2))
    with SideStream() as side, H.Comm(2, device=0) as c:
        combine = c.bind_moe_combine(z, row, out, stream=side)
        c.allreduce(send, recv)  # (compiled before the executor takes it)
        combine()
        torch.cuda.synchronize()
        out.zero_()
        torch.cuda.synchronize()
        print("operator beside a resident executor", flush=True)
        with c.resident(blocks=8, idle_ms=IDLE_MS):
            c.allreduce(send, recv)
            c.resident_wait()
            combine()
            side.synchronize()
        torch.cuda.synchronize()
        assert torch.equal(out, want)
        assert all(bool((t == 3.0).all()) for t in recv)
