"""What the Python binding of the mixture-of-experts operators passes on: nothing that its C call could write beyond."""
import inspect

import pytest
import torch

import paper_2608_00358_amd as H


@pytest.fixture()
def comm():
    with H.Comm(4, device=H.NO_DEVICE) as c:
        yield c


def _plan_arrays(T=5, K=2, E=8):
    i32 = torch.int32
    return (torch.zeros(T, K, dtype=i32), E, torch.zeros(T, K, dtype=i32), torch.zeros(E + 1, dtype=torch.int64), T * K)


@pytest.mark.parametrize("n", [0, 1, 3, 5])
def test_rank_counts_hold_a_number_for_every_rank(comm, n):
    counts = torch.zeros(n, dtype=torch.int64)
    for handle in (comm.handle, comm.handle.value):
        with pytest.raises(ValueError):
            H.hccl_moe_plan(handle, *_plan_arrays(), rank_counts=counts)
        H.hccl_moe_plan(handle, *_plan_arrays(), rank_counts=torch.zeros(4, dtype=torch.int64))
        H.hccl_moe_plan(handle, *_plan_arrays())
    for method in (comm.moe_plan, comm.bind_moe_plan):
        with pytest.raises(ValueError):
            method(*_plan_arrays(), rank_counts=counts)


def test_rank_counts_of_a_communicator_that_the_binding_does_not_know(comm, monkeypatch):
    """Nobody can say how many counts such a communicator writes."""
    counts = torch.zeros(4, dtype=torch.int64)
    H.hccl_moe_plan(comm.handle, *_plan_arrays(), rank_counts=counts)
    monkeypatch.setattr(H.hccl, "_comm_ranks", {})
    with pytest.raises(ValueError):
        H.hccl_moe_plan(comm.handle, *_plan_arrays(), rank_counts=counts)
    H.hccl_moe_plan(comm.handle, *_plan_arrays())


def test_a_destroyed_communicator_is_forgotten():
    handle = H.hccl_comm_create(3, H.NO_DEVICE)
    at = handle.value
    assert H.hccl._comm_ranks[at] == 3
    H.hccl_comm_destroy(handle)
    assert at not in H.hccl._comm_ranks


def test_a_workspace_is_packed(comm):
    """Its bytes are those from its address on, which a strided or expanded tensor does not have."""
    T, K, E = 4096, 2, 8
    need = H.hccl_moe_plan_bytes(T, K, E)
    arrays = _plan_arrays(T, K, E)
    comm.moe_plan(*arrays, workspace=torch.zeros(need, dtype=torch.uint8))
    comm.moe_plan(*arrays, workspace=torch.zeros(8, need // 8, dtype=torch.uint8))
    for bad in (torch.zeros(2 * need, dtype=torch.uint8)[::2], torch.zeros(1, dtype=torch.int32).expand(need),
                torch.zeros(need // 8, 16, dtype=torch.uint8)[:, :8]):
        for call in (comm.moe_plan, comm.bind_moe_plan):
            with pytest.raises(ValueError):
                call(*arrays, workspace=bad)


def test_a_bound_call_keeps_its_router(comm):
    """The arrays were checked against the router as it was: a larger one would write beyond them."""
    T, E = 5, 8
    logits, index, weight = torch.zeros(T, E), torch.zeros(T, 2, dtype=torch.int32), torch.zeros(T, 2)
    router = H.hccl_router_init(experts=E, top_k=2)
    calls = [comm.bind_moe_route(router, logits, index, weight),
             comm.bind_moe_route_backward(router, logits, index, weight, torch.zeros_like(logits))]
    router.top_k = E + 1  # (refused where it is read)
    for call in calls:
        call()


@pytest.mark.parametrize("name", ["route", "route_backward", "plan", "dispatch", "combine", "combine_backward", "quantize", "product"])
def test_functions_and_methods_have_one_signature(name):
    """The function takes a communicator's handle first, the methods are those of the communicator."""
    function, method, bind = (list(inspect.signature(f).parameters.values())[1:] for f in (
        getattr(H, f"hccl_moe_{name}"), getattr(H.Comm, f"moe_{name}"), getattr(H.Comm, f"bind_moe_{name}")))
    assert function and all(p.kind is p.POSITIONAL_OR_KEYWORD for p in function)
    assert [(p.name, p.default) for p in function] == [(p.name, p.default) for p in method] == [(p.name, p.default) for p in bind]
