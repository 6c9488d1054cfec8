"""The mixture-of-experts operators without a GPU: argument checks, and the 64-bit reference's gradients."""
import numpy as np
import pytest
import torch

import moe_reference as ref
import paper_2608_00358_amd as H


@pytest.fixture()
def comm():
    with H.Comm(4, device=H.NO_DEVICE) as c:
        yield c


def _i32(*shape):
    return torch.zeros(shape, dtype=torch.int32)


def _router(**kw):
    return H.hccl_router_init(**{"experts": 8, "top_k": 2, **kw})


def test_router_defaults():
    r = H.hccl_router_init(experts=16)
    assert (r.experts, r.top_k, r.score, r.groups, r.top_groups, r.group_top, r.renormalize, r.scale) == (16, 1, 0, 1, 1, 1, 0, 1.0)


@pytest.mark.parametrize("bad", [
    dict(experts=0), dict(experts=1025, top_k=1), dict(top_k=0), dict(top_k=9), dict(experts=64, top_k=33), dict(score=2),
    dict(groups=0), dict(groups=3), dict(experts=66, groups=33), dict(groups=4, top_groups=5), dict(groups=4, top_groups=0),
    dict(group_top=3), dict(groups=4, top_groups=1, top_k=3), dict(scale=float("nan")), dict(scale=float("inf"))])
def test_router_refusals(comm, bad):
    r = _router(**bad)
    logits, index, weight = torch.zeros(3, r.experts), _i32(3, r.top_k), torch.zeros(3, r.top_k)
    with pytest.raises(H.HcclError) as e:
        comm.moe_route(r, logits, index, weight)
    assert e.value.code == 1
    with pytest.raises(H.HcclError) as e:
        comm.moe_route_backward(r, logits, index, weight, torch.zeros_like(logits))
    assert e.value.code == 1


def _refused(code, fn, *a, **kw):
    with pytest.raises(H.HcclError) as e:
        fn(*a, **kw)
    assert e.value.code == code, str(e.value)


def test_good_calls_pass_the_checks_on_a_communicator_without_a_device(comm):
    T, E, K, C = 5, 8, 2, 24
    r = _router()
    logits, index, weight, x = torch.zeros(T, E), _i32(T, K), torch.zeros(T, K), torch.zeros(T, C)
    row, offsets, out = _i32(T, K), torch.zeros(E + 1, dtype=torch.int64), torch.zeros(T * K, C)
    comm.moe_route(r, logits, index, weight, bias=torch.zeros(E), mask=torch.ones(T, dtype=torch.uint8))
    comm.moe_route(r, logits, index, weight, mask=torch.ones(T, dtype=torch.bool))
    comm.moe_route_backward(r, logits, index, weight, torch.zeros_like(logits))
    comm.moe_plan(index, E, row, offsets, T * K, rank_counts=torch.zeros(4, dtype=torch.int64))
    comm.moe_dispatch(x, row, out)
    codes, scale = torch.zeros(T * K, C, dtype=torch.int8), torch.zeros(T * K)
    comm.moe_dispatch(x, row, codes, scale=scale)
    comm.moe_combine(out, row, x, weight=weight)
    comm.moe_combine_backward(x, out, row, weight, torch.zeros_like(out), torch.zeros_like(weight))
    comm.moe_quantize(out, codes, scale)
    comm.moe_quantize(torch.zeros(T * K, 2 * C), codes, scale, gated=True)
    comm.moe_product(codes, scale, torch.zeros(E, 6, C, dtype=torch.int8), torch.zeros(E, 6), torch.zeros(T * K, 6), offsets=offsets)
    assert H.hccl_moe_plan_bytes(T, K, E) == 0
    assert H.hccl_moe_plan_bytes(4096, 2, 64) > 0
    # nothing to do needs no arrays
    empty = torch.zeros(0, C)
    comm.moe_dispatch(empty, _i32(0, K), out)
    comm.moe_combine(out, _i32(0, K), empty)


def test_columns_side_by_side_do_not_overlap(comm):
    both = torch.zeros(6, 20)
    row = _i32(6, 1)
    comm.moe_dispatch(both[:, :10], row, both[:, 10:])
    comm.moe_combine(both[:, 10:], row, both[:, :10])
    _refused(1, comm.moe_dispatch, both[:, :11], row, both[:, 9:])
    _refused(1, comm.moe_combine, both[:, 9:], row, both[:, :11])


def test_refusals(comm):
    T, E, K, C = 5, 8, 2, 24
    r, logits, index, weight = _router(), torch.zeros(T, E), _i32(T, K), torch.zeros(T, K)
    row, x, out = _i32(T, K), torch.zeros(T, C), torch.zeros(T * K, C)
    offsets = torch.zeros(E + 1, dtype=torch.int64)
    lib = H.load()
    h = comm.handle
    # int32 rows, null arrays, wrong strides
    assert lib.hccl_moe_dispatch(h, 4096, C, 3, T, C, 8192, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, None, C, 0, T, C, 8192, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, 4096, C - 1, 0, T, C, 1 << 16, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, 4097, C, 0, T, C, 1 << 16, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, 4096, C, 0, T, C, 1 << 16, 33, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, 4096, C, 0, T, C, 1 << 16, 0, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, 4096, C, 0, 1 << 31, C, 1 << 16, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(h, 4096, 1 << 62, 0, T, C, 1 << 16, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_dispatch(None, 4096, C, 0, T, C, 1 << 16, K, 1 << 20, C, T * K, None, None) == 1
    assert lib.hccl_moe_plan(h, 4096, T, K, 0, 4, 8192, 16384, None, None, 0, None) == 1
    assert lib.hccl_moe_plan(h, 4096, T, K, 1025, 4, 8192, 16384, None, None, 0, None) == 1
    assert lib.hccl_moe_plan(h, 4096, T, K, E, 1 << 31, 8192, 16384, None, None, 0, None) == 1
    assert lib.hccl_moe_plan(h, 4096, T, K, E, 4, 8192, None, None, None, 0, None) == 1
    assert lib.hccl_moe_plan_bytes(T, K, E, None) == 1
    assert lib.hccl_router_init(None) == 1
    # results over inputs
    _refused(1, comm.moe_route, r, logits, index, logits.view(-1)[:T * K].view(T, K))
    _refused(1, comm.moe_route_backward, r, logits, index, weight, logits)
    _refused(1, comm.moe_combine, out, row, out[:T])
    _refused(1, comm.moe_combine_backward, x, out, row, weight, out, torch.zeros_like(weight))
    # ranks that do not divide the experts; a workspace that is needed and missing or small
    _refused(1, comm.moe_plan, index, 6, row, torch.zeros(7, dtype=torch.int64), 10, rank_counts=torch.zeros(4, dtype=torch.int64))
    many = _i32(4096, K)
    _refused(1, comm.moe_plan, many, E, many.clone(), offsets, 8192)
    _refused(1, comm.moe_plan, many, E, many.clone(), offsets, 8192, workspace=torch.zeros(8, dtype=torch.uint8))
    # products: an inner size whose sums could wrap, segments that are no multiple of the experts, experts without segments
    assert lib.hccl_moe_product(h, 1 << 20, 131072, 1 << 24, 4, 131072, 1 << 25, 131072, 1 << 26, 4, 1, None, 0, 1 << 27, 4, 0, None) == 1
    codes, scale, w, ws = torch.zeros(T, C, dtype=torch.int8), torch.zeros(T), torch.zeros(E, 6, C, dtype=torch.int8), torch.zeros(E, 6)
    y = torch.zeros(T, 6)
    _refused(1, comm.moe_product, codes, scale, w, ws, y)
    _refused(1, comm.moe_product, codes, scale, w, ws, y, offsets=torch.zeros(E + 2, dtype=torch.int64))
    _refused(1, comm.moe_product, codes, scale, w[:1], ws[:1], y, offsets=torch.zeros(1, dtype=torch.int64))
    # tensors that do not fit each other
    for call in (lambda: comm.moe_dispatch(x, row, torch.zeros(T * K, C + 1)), lambda: comm.moe_dispatch(x, row, out.to(torch.bfloat16)),
                 lambda: comm.moe_dispatch(x, row.long(), out), lambda: comm.moe_dispatch(x, row, out, scale=torch.zeros(T * K)),
                 lambda: comm.moe_dispatch(x.t().contiguous().t(), row, out), lambda: comm.moe_route(r, logits[:, :7], index, weight),
                 lambda: comm.moe_plan(index, E, row, offsets, 10, rank_counts=torch.zeros(3, dtype=torch.int64)),
                 lambda: comm.moe_product(codes, scale, w.transpose(1, 2).contiguous().transpose(1, 2), ws, y, offsets=offsets),
                 lambda: comm.moe_combine(out, row, x.half())):
        with pytest.raises(ValueError):
            call()


def test_refused_inside_a_group(comm):
    x, row, out = torch.zeros(4, 8), _i32(4, 1), torch.zeros(4, 8)
    H.hccl_group_start(comm.handle)
    _refused(2, comm.moe_dispatch, x, row, out)
    H.hccl_group_end(comm.handle)
    comm.moe_dispatch(x, row, out)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("renormalize", [False, True])
def test_reference_router_gradient_against_differences(score, renormalize):
    rng = np.random.default_rng(3)
    l = rng.normal(size=(4, 12))
    l[1, 5] = -ref.INF
    index, _, _ = ref.route(l, 3, score)
    index[2, 1] = -1
    g = rng.normal(size=(4, 3))
    got = ref.route_backward(l, index, g, score, renormalize, 1.7)
    h = 1e-5
    for t in range(4):
        for e in range(12):
            if l[t, e] == -ref.INF:
                assert got[t, e] == 0
                continue
            up, down = l[t].copy(), l[t].copy()
            up[e] += h
            down[e] -= h
            d = (ref.weights_of(up, index[t], score, renormalize, 1.7) - ref.weights_of(down, index[t], score, renormalize, 1.7)) / (2 * h)
            assert abs((d * g[t]).sum() - got[t, e]) < 1e-8


def test_reference_combine_gradient_against_differences():
    rng = np.random.default_rng(4)
    z, row, w = rng.normal(size=(5, 7)), np.array([[0, 3], [4, -1], [1, 2]]), rng.random((3, 2))
    g = rng.normal(size=(3, 7))
    dz, dw, _ = ref.combine_backward(g, z, row, w, np.zeros((5, 7)))
    f = lambda z_, w_: (ref.combine(z_, row, w_)[0] * g).sum()  # noqa: E731
    h = 1e-6
    for i in range(5):
        for j in range(7):
            e = np.zeros((5, 7))
            e[i, j] = h
            assert abs((f(z + e, w) - f(z - e, w)) / (2 * h) - dz[i, j]) < 1e-7
    for t in range(3):
        for k in range(2):
            e = np.zeros((3, 2))
            e[t, k] = h
            assert abs((f(z, w + e) - f(z, w - e)) / (2 * h) - dw[t, k]) < 1e-7
