"""The mixture-of-experts operators on the GPU against their definitions in 64 bits.

Tolerances follow from the arithmetic. 32-bit results: a softmax score is an exponential (its argument,
a difference below 32 in size, rounded once: 2^-19 relative), a sum of at most 22 roundings and a
quotient; 1e-5 covers them. A sum of n terms in 32 bits is off by at most n 2^-24 of the sum of their
sizes, with n the additions on one path (a lane's own, then the tree over lanes and waves). A result is
rounded to its type once, to nearest: rounding keeps order, so it lies between the roundings of the least
and the greatest value that its 32-bit bound allows, and no tolerance is added for the type.
"""
import numpy as np
import pytest
import torch

import moe_reference as ref
import paper_2608_00358_amd as H
from gpu_helpers import SideStream

pytestmark = pytest.mark.gpu

DEV = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
LOWEST = {"bf16": torch.finfo(torch.bfloat16).min, "fp16": -65504.0, "fp32": torch.finfo(torch.float32).min}
F32 = 2.0 ** -24
INF = float("inf")


@pytest.fixture(scope="module")
def comm():
    with H.Comm(4, device=0) as c:
        yield c


def rand(rng, rows, cols, dt, pad=0, std=1.0, shift=0):
    """Rows of normal values, `pad` elements apart, `shift` elements into their allocation."""
    x = torch.from_numpy(rng.normal(size=(rows, cols + pad)).astype(np.float32) * np.float32(std)).to(TYPES[dt])
    return place(x, shift)[:, :cols]


def place(x, shift=0):
    flat = torch.empty(x.numel() + shift, dtype=x.dtype, device=DEV)
    flat[shift:] = x.reshape(-1).to(DEV)
    return flat[shift:].view(x.shape)


class Room:
    """An output whose surroundings (the padding of its rows, 64 elements on both sides) must stay as they are."""

    def __init__(self, rows, cols, dtype, pad=0, shift=0):
        self.rows, self.cols, self.pad = rows, cols, pad
        n = rows * (cols + pad)
        self.flat = torch.full((n + 128 + shift,), 77, dtype=dtype, device=DEV)
        self.at = 64 + shift
        self.view = self.flat[self.at:self.at + n].view(rows, cols + pad)[:, :cols]

    def check(self):
        f = self.flat.clone()
        f[self.at:self.at + self.rows * (self.cols + self.pad)].view(self.rows, self.cols + self.pad)[:, :self.cols] = 77
        assert bool((f == 77).all()), "wrote outside its rows"


def host(t):
    return t.double().cpu().numpy() if t.is_floating_point() else t.cpu().numpy()


def close(got, want, bound, what=""):
    got = host(got) if torch.is_tensor(got) else got
    bad = ~(np.abs(got - want) <= bound)
    bad &= ~(np.isnan(got) & np.isnan(want)) & ~(got == want)
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {got[bad][0]} for {want[bad][0]}"


def rounded(got, want, bound, what=""):
    """A value within `bound` of `want` (and the rounding to 32 bits that it has anyway), rounded to got's type."""
    want = torch.from_numpy(np.ascontiguousarray(want))
    bound = torch.from_numpy(np.broadcast_to(bound, want.shape).copy()) + F32 * want.abs() + 1e-37
    lo, hi = ((want + s * bound).float().to(got.dtype).double().numpy() for s in (-1, 1))
    v, w = host(got), want.numpy()
    bad = ~((lo <= v) & (v <= hi)) & ~(np.isnan(v) & np.isnan(w))
    assert not bad.any(), f"{what}: {bad.sum()} of {bad.size} off, first at {np.argwhere(bad)[0]}: {v[bad][0]} for {w[bad][0]}"


# ---------------------------------------------------------------------------------------- routing

ROUTERS = [
    dict(experts=8, top_k=2), dict(experts=1, top_k=1), dict(experts=3, top_k=3, renormalize=True),
    dict(experts=60, top_k=4, renormalize=True, scale=2.5), dict(experts=64, top_k=6, score="sigmoid"),
    dict(experts=100, top_k=8, score="sigmoid", bias=True, renormalize=True), dict(experts=128, top_k=8, renormalize=True),
    dict(experts=129, top_k=8, bias=True), dict(experts=192, top_k=6, score="sigmoid", bias=True, groups=8, top_groups=3, group_top=2, renormalize=True),
    dict(experts=256, top_k=32, score="sigmoid", renormalize=True), dict(experts=500, top_k=7), dict(experts=512, top_k=8, groups=32, top_groups=5),
    dict(experts=1000, top_k=17, renormalize=True), dict(experts=1024, top_k=32, score="sigmoid", bias=True, groups=16, top_groups=8),
    dict(experts=64, top_k=4, groups=4, top_groups=2), dict(experts=60, top_k=5, score="sigmoid", groups=20, top_groups=3, group_top=2),
    dict(experts=24, top_k=2, groups=24, top_groups=2), dict(experts=40, top_k=20, score="sigmoid", bias=True),
]


def check_route(comm, cfg, logits, mask=None, dt="fp32", stream=None, bias_host=None):
    cfg = dict(cfg)
    T, E = logits.shape
    K = cfg["top_k"]
    use_bias = cfg.pop("bias", False)
    router = H.hccl_router_init(**cfg)
    bias = None
    if use_bias:
        if bias_host is None:
            bias_host = np.random.default_rng(E).normal(size=E).astype(np.float32) * np.float32(0.1)
        bias = torch.from_numpy(bias_host).to(DEV)
    l = host(logits)
    index, weight, margin = ref.route(l, bias=None if bias is None else bias_host.astype(np.float64), mask=mask, **cfg)
    # scores are held in 32 bits: where less than 2e-6 decides, either order is right
    clear = margin > 2e-6
    assert clear.mean() > 0.8, "the inputs leave too few choices clear"
    gi, gw = Room(T, K, torch.int32), Room(T, K, torch.float32)
    comm.moe_route(router, logits, gi.view, gw.view, bias=bias, mask=None if mask is None else torch.from_numpy(mask).to(DEV), stream=stream)
    torch.cuda.synchronize()
    gi.check(), gw.check()
    assert np.array_equal(host(gi.view)[clear], index[clear])
    close(host(gw.view)[clear], weight[clear], 1e-5 * np.abs(weight[clear]) + 1e-37)
    assert (host(gi.view)[~clear] >= -1).all() and (host(gi.view)[~clear] < E).all()
    return index


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("cfg", ROUTERS, ids=lambda c: "-".join(str(v) for v in c.values()))
def test_route_and_its_gradient(comm, cfg, dt):
    rng = np.random.default_rng(cfg["experts"])
    E, K = cfg["experts"], cfg["top_k"]
    T = 67
    logits = rand(rng, T, E, dt, pad=3, std=1.5, shift=1)
    if E > 8:
        logits[5, : E // 2] = -INF
        logits[6, 1::2] = LOWEST[dt]
        logits[7, 3] = float("nan")
        logits[8, 2:5] = INF if not cfg.get("bias") else 6.0
    logits[9] = -INF          # a row that leaves nothing
    logits[10] = LOWEST[dt] if not cfg.get("bias") and cfg.get("group_top", 1) == 1 else logits[11]
    logits[12] = float("nan")
    mask = (rng.random(T) < 0.9).astype(np.uint8)
    check_route(comm, cfg, logits, mask, dt)
    index = check_route(comm, cfg, logits, None, dt)

    opts = {k: v for k, v in cfg.items() if k != "bias"}
    l = host(logits)
    index[13, 0] = -1
    index[14, K - 1] = E
    grad = torch.from_numpy(rng.normal(size=(T, K)).astype(np.float32)).to(DEV)
    want = ref.route_backward(l, index, host(grad), **opts)
    out = Room(T, E, TYPES[dt], pad=5, shift=1)
    comm.moe_route_backward(H.hccl_router_init(**opts), logits, torch.from_numpy(index.astype(np.int32)).to(DEV), grad, out.view)
    torch.cuda.synchronize()
    out.check()
    # the terms of a token's gradient cancel: their size is that of scale g (/ r) times the scores
    s = np.stack([ref.scores(v, opts.get("score", "softmax")) for v in l])
    some = (index >= 0) & (index < E)
    u = np.where(some, np.take_along_axis(s, np.where(some, index, 0), 1), 0.0)
    r = np.maximum(u.sum(1, keepdims=True), 1e-300) if opts.get("renormalize") else np.ones((T, 1))
    size = abs(opts.get("scale", 1.0)) * np.abs(np.where(some, host(grad), 0)).max(1, keepdims=True) / r * s
    size[u.sum(1) == 0] = 0
    rounded(out.view, want, 4e-5 * size)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
def test_slope_of_a_sigmoid_far_from_zero(comm, dt):
    """s (1 - s), where 1 - s is far below the spacing of numbers near 1."""
    rng = np.random.default_rng(4)
    T, E, K = 40, 64, 4
    logits = rand(rng, T, E, dt, std=10.0)
    index = np.stack([rng.permutation(E)[:K] for _ in range(T)]).astype(np.int32)
    grad = rng.normal(size=(T, K)).astype(np.float32)
    l, want = host(logits), np.zeros((T, E))
    e = np.exp(-np.abs(l))
    np.put_along_axis(want, index, grad.astype(np.float64), 1)
    want *= e / (1.0 + e) ** 2
    out = Room(T, E, TYPES[dt])
    comm.moe_route_backward(H.hccl_router_init(experts=E, top_k=K, score="sigmoid"), logits, torch.from_numpy(index).to(DEV),
                            torch.from_numpy(grad).to(DEV), out.view)
    torch.cuda.synchronize()
    out.check()
    # two exponentials (their arguments: a constant and a product, rounded: 1.5 |l| units; themselves 2), sums (1),
    # reciprocals (2) and two products
    rounded(out.view, want, F32 * (3.0 * np.abs(l) + 12.0) * np.abs(want))


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("experts", [32, 200, 600])
def test_shares_of_chosen_experts_far_below_the_greatest(comm, experts, dt):
    """A bias chooses experts whose softmax scores are too small for 32 bits; among themselves they have shares."""
    rng = np.random.default_rng(experts)
    T, K = 21, 4
    logits = rand(rng, T, experts, dt)
    logits[:, 8:] -= 120.0
    bias = np.linspace(9.0, 5.0, experts).astype(np.float32)
    bias[:8] = 0.0
    cfg = dict(experts=experts, top_k=K, renormalize=True, scale=2.5)
    index = check_route(comm, dict(cfg, bias=True), logits, dt=dt, bias_host=bias)
    assert (index == np.arange(8, 8 + K)).all()
    grad = torch.from_numpy(rng.normal(size=(T, K)).astype(np.float32)).to(DEV)
    out = Room(T, experts, TYPES[dt])
    comm.moe_route_backward(H.hccl_router_init(**cfg), logits, torch.from_numpy(index.astype(np.int32)).to(DEV), grad, out.view)
    torch.cuda.synchronize()
    out.check()
    l = host(logits)
    size = np.zeros((T, experts))
    size[:, 8:8 + K] = 2.5 * np.abs(host(grad)).max(1, keepdims=True)
    want = ref.route_backward(l, index, host(grad), **cfg)
    # sum_k du_k u_k = 0 where weights are renormalised, so experts not chosen have no gradient; in 64 bits that sum
    # is its terms' rounding, which the quotient by r (1e-52) does not make small
    assert np.abs(np.delete(want, range(8, 8 + K), 1)).max() < 1e-14
    want[:, :8], want[:, 8 + K:] = 0.0, 0.0
    rounded(out.view, want, 4e-5 * size)


@pytest.mark.parametrize("tokens", [1, 2, 3, 15, 16, 17, 255, 1025])
@pytest.mark.parametrize("experts", [16, 96, 200, 320, 768])
def test_route_of_any_number_of_tokens(comm, tokens, experts):
    rng = np.random.default_rng(tokens)
    check_route(comm, dict(experts=experts, top_k=5, renormalize=True), rand(rng, tokens, experts, "bf16"))


@pytest.mark.parametrize("dt,low", [("bf16", -1e9), ("fp32", -1e9), ("fp32", -1e30), ("fp16", -6e4)])
@pytest.mark.parametrize("cfg", [dict(experts=128, top_k=8), dict(experts=128, top_k=8, renormalize=True), dict(experts=200, top_k=4, score="sigmoid"),
                                 dict(experts=64, top_k=4, bias=True), dict(experts=64, top_k=4, groups=8, top_groups=2, renormalize=True)],
                         ids=lambda c: "-".join(str(v) for v in c.values()))
def test_route_of_finite_masks(comm, cfg, dt, low):
    """Masks by a great negative number: rows with some experts left, with one, and with none but masked ones."""
    rng = np.random.default_rng(3)
    logits = rand(rng, 30, cfg["experts"], dt)
    logits[:10, ::2] = low
    logits[10:20, 1:] = low
    logits[20:] = low
    if cfg.get("bias"):
        logits[10:] = logits[:1]  # (equal scores of 0 and a bias leave nothing to choose by but the bias)
        logits[10:, 1:] = low
    check_route(comm, cfg, logits, dt=dt)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
def test_route_ties_go_to_the_lowest_expert(comm, dt):
    rng = np.random.default_rng(0)
    for cfg in (dict(experts=64, top_k=8), dict(experts=300, top_k=9, score="sigmoid"), dict(experts=64, top_k=8, groups=8, top_groups=2)):
        x = torch.from_numpy(rng.integers(-2, 3, size=(50, cfg["experts"])).astype(np.float32) / 4)
        x[0] = 0.0
        x[1, ::2], x[1, 1::2] = 0.0, -0.0
        check_route(comm, cfg, x.to(TYPES[dt]).to(DEV), dt=dt)


def test_route_of_a_bias_that_closes_experts(comm):
    rng = np.random.default_rng(1)
    bias = rng.normal(size=32).astype(np.float32)
    bias[3], bias[4], bias[5] = -np.inf, np.nan, 9.0
    logits = rand(rng, 40, 32, "fp32")
    cfg = dict(experts=32, top_k=4, score="sigmoid", bias=True)
    index = check_route(comm, cfg, logits, bias_host=bias)
    assert not np.isin(index, (3, 4)).any() and (index[:, 0] == 5).all()


def test_route_gradient_against_differences(comm):
    """The weights that the kernel gives move as its gradient says (central differences in 32 bits:
    their error is 2e-7 / h + h^2)."""
    rng = np.random.default_rng(2)
    for cfg in (dict(experts=12, top_k=3, renormalize=True), dict(experts=12, top_k=3), dict(experts=12, top_k=3, score="sigmoid", scale=2.0)):
        router = H.hccl_router_init(**cfg)
        l = rng.permutation(12).astype(np.float32)[None] * np.float32(0.3)  # (distances that a step does not bridge)
        g = rng.normal(size=(1, 3)).astype(np.float32)
        h = 2.0 ** -6
        steps = np.concatenate([l] + [l + np.float32(s * h) * np.eye(12, dtype=np.float32)[[e]] for e in range(12) for s in (1, -1)])
        logits = torch.from_numpy(steps).to(DEV)
        index, weight = torch.empty(25, 3, dtype=torch.int32, device=DEV), torch.empty(25, 3, device=DEV)
        comm.moe_route(router, logits, index, weight)
        out = torch.empty(1, 12, device=DEV)
        comm.moe_route_backward(router, logits[:1], index[:1], torch.from_numpy(g).to(DEV), out)
        assert bool((index == index[0]).all())
        w = host(weight)
        got = [((w[1 + 2 * e] - w[2 + 2 * e]) / (2 * h) * g[0]).sum() for e in range(12)]
        close(out[0], np.array(got), 6 * (2e-7 / h + h * h))


# --------------------------------------------------------------------------- plan, dispatch, combine

@pytest.mark.parametrize("tokens,top_k,experts", [
    (0, 2, 8), (1, 1, 1), (1, 8, 64), (37, 4, 64), (64, 1, 3), (1000, 3, 1000), (1024, 4, 1024), (1025, 4, 60), (2048, 8, 128), (40000, 1, 7),
    (20001, 8, 256), (600000, 1, 33)])
def test_plan(comm, tokens, top_k, experts):
    rng = np.random.default_rng(tokens + experts)
    index = np.minimum(rng.integers(0, experts, size=(tokens, top_k)), rng.integers(0, experts, size=(tokens, top_k))).astype(np.int32)
    index[rng.random(index.shape) < 0.05] = -1
    index[rng.random(index.shape) < 0.02] = experts
    index[rng.random(index.shape) < 0.02] = np.iinfo(np.int32).min
    n = tokens * top_k
    for capacity in (n, n // 2, 0):
        flat = index.reshape(-1)
        some = np.nonzero((flat >= 0) & (flat < experts))[0]
        order = some[np.argsort(flat[some], kind="stable")]
        row = np.full(n, -1)
        row[order] = np.arange(order.size)
        row[row >= capacity] = -1
        offsets = np.minimum(np.concatenate([[0], np.cumsum(np.bincount(flat[some], minlength=experts))]), capacity)
        if n < 500:
            slow = ref.plan(np.where((index >= 0) & (index < experts), index, -1), experts, capacity)
            assert np.array_equal(slow[0].reshape(-1), row) and np.array_equal(slow[1], offsets)
        got_row, got_off = Room(tokens, top_k, torch.int32), Room(1, experts + 1, torch.int64)
        ranked = experts % 4 == 0
        counts = torch.full((4,), -7, dtype=torch.int64, device=DEV)
        ws = torch.empty(H.hccl_moe_plan_bytes(tokens, top_k, experts), dtype=torch.uint8, device=DEV)
        comm.moe_plan(torch.from_numpy(index).to(DEV), experts, got_row.view, got_off.view, capacity,
                      rank_counts=counts if ranked else None, workspace=ws if ws.numel() else None)
        torch.cuda.synchronize()
        got_row.check(), got_off.check()
        assert np.array_equal(host(got_row.view).reshape(-1), row)
        assert np.array_equal(host(got_off.view)[0], offsets)
        if ranked:
            assert np.array_equal(host(counts), np.diff(offsets[::experts // 4]))


def routes(rng, tokens, top_k, rows, holes=0.1):
    """Distinct rows for the routes, in no order; some routes have none, some an invalid one."""
    row = rng.permutation(max(rows, tokens * top_k))[: tokens * top_k].astype(np.int32).reshape(tokens, top_k)
    row[rng.random(row.shape) < holes] = -1
    row[rng.random(row.shape) < holes / 4] = np.iinfo(np.int32).min
    if tokens > 2:
        row[1] = -1
    return row


SHAPES = [(1, 1, 1), (70, 3, 128), (33, 6, 129), (21, 7, 250), (1, 4, 4096), (3, 2, 7), (5, 32, 64), (37, 4, 1001), (16, 5, 511), (9, 3, 513), (20, 8, 2048), (6, 6, 5003), (130, 1, 100)]


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("tokens,top_k,cols", SHAPES)
def test_dispatch(comm, tokens, top_k, cols, dt):
    rng = np.random.default_rng(cols)
    for pad, shift, rows in ((0, 0, tokens * top_k), (3, 1, max(1, tokens * top_k - 5)), (16, 8, tokens * top_k + 9)):
        x = rand(rng, tokens, cols, dt, pad, shift=shift)
        x[0, 0] = float("nan")
        row = routes(rng, tokens, top_k, rows)
        out = Room(rows, cols, TYPES[dt], pad, shift)
        comm.moe_dispatch(x, torch.from_numpy(row).to(DEV), out.view)
        torch.cuda.synchronize()
        out.check()
        assert np.array_equal(host(out.view), ref.dispatch(host(x), row, np.full((rows, cols), 77.0)), equal_nan=True)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("tokens,top_k,cols", SHAPES)
def test_combine_and_its_gradients(comm, tokens, top_k, cols, dt):
    rng = np.random.default_rng(cols + 1)
    for pad, shift, rows in ((0, 0, tokens * top_k), (3, 1, max(1, tokens * top_k - 5)), (16, 8, tokens * top_k + 9)):
        z = rand(rng, rows, cols, dt, pad, shift=shift)
        row = routes(rng, tokens, top_k, rows)
        unseen = np.setdiff1d(np.arange(rows), row)
        z[torch.from_numpy(unseen).to(DEV)] = float("nan")  # rows that nobody names
        w = rng.random((tokens, top_k)).astype(np.float32)
        d_row, d_w = torch.from_numpy(row).to(DEV), torch.from_numpy(w).to(DEV)
        zh = np.nan_to_num(host(z))
        for weight in (w, None):
            out = Room(tokens, cols, TYPES[dt], pad, shift)
            comm.moe_combine(z, d_row, out.view, weight=None if weight is None else d_w)
            torch.cuda.synchronize()
            out.check()
            want, size = ref.combine(zh, row, weight)
            rounded(out.view, want, (top_k + 1) * F32 * size, "combine")
        grad = rand(rng, tokens, cols, dt, pad, shift=shift)
        gz, gw = Room(rows, cols, TYPES[dt], pad, shift), Room(tokens, top_k, torch.float32)
        comm.moe_combine_backward(grad, z, d_row, d_w, gz.view, gw.view)
        torch.cuda.synchronize()
        gz.check(), gw.check()
        want_z, want_w, size = ref.combine_backward(host(grad), zh, row, w, np.full((rows, cols), 77.0))
        rounded(gz.view, want_z, 0.0, "grad_z")
        close(gw.view, want_w, (cols / 64 + 24) * F32 * size + 1e-37, "grad_weight")
        # each of them alone
        one, two = torch.full_like(gz.view, 77), torch.full_like(gw.view, 77)
        comm.moe_combine_backward(grad, z, d_row, d_w, grad_z=one)
        comm.moe_combine_backward(grad, z, d_row, d_w, grad_weight=two)
        assert torch.equal(one, gz.view) and torch.equal(two, gw.view)


@pytest.mark.parametrize("dt,tokens,top_k,cols", [("bf16", 9000, 4, 4096), ("fp32", 5000, 3, 5001), ("fp16", 130, 2, 9000), ("bf16", 70000, 8, 300)])
def test_large_calls(comm, dt, tokens, top_k, cols):
    """Calls that move more than the last-level cache, and rows of many vectors, against 64 bits on the GPU."""
    g = torch.Generator(device=DEV).manual_seed(tokens)
    row = torch.randperm(tokens * top_k, generator=g, device=DEV).to(torch.int32).view(tokens, top_k)
    x = torch.randn(tokens, cols, generator=g, device=DEV).to(TYPES[dt])
    rows = torch.empty(tokens * top_k, cols, device=DEV, dtype=TYPES[dt])
    comm.moe_dispatch(x, row, rows)
    for k in range(top_k):
        assert torch.equal(rows[row[:, k].long()], x)
    del rows
    z = torch.randn(tokens * top_k, cols, generator=g, device=DEV).to(TYPES[dt])
    w = torch.rand(tokens, top_k, generator=g, device=DEV)
    y, gz, gw = torch.empty_like(x), torch.empty_like(z), torch.empty_like(w)
    comm.moe_combine(z, row, y, weight=w)
    comm.moe_combine_backward(x, z, row, w, gz, gw)
    torch.cuda.synchronize()
    for at in range(0, tokens, 1000):
        part = slice(at, at + 1000)
        zs = z[row[part].long()].double()
        terms = w[part, :, None].double() * zs
        rounded(y[part], host(terms.sum(1)), (top_k + 1) * F32 * host(terms.abs().sum(1)), "combine")
        products = x[part, None].double() * zs
        close(gw[part], host(products.sum(2)), (cols / 64 + 24) * F32 * host(products.abs().sum(2)), "grad_weight")
        for k in range(top_k):
            rounded(gz[row[part, k].long()], host(w[part, k:k + 1].double() * x[part].double()), 0.0, "grad_z")


def test_gradient_of_dispatch_is_combine_without_weights(comm):
    rng = np.random.default_rng(5)
    T, K, C = 12, 3, 40
    row = routes(rng, T, K, T * K)
    g = rand(rng, T * K, C, "fp32")
    dx = torch.empty(T, C, device=DEV)
    comm.moe_combine(g, torch.from_numpy(row).to(DEV), dx)
    x = rng.normal(size=(T, C))
    f = lambda v: (ref.dispatch(v, row, np.zeros((T * K, C))) * host(g)).sum()  # noqa: E731
    for t, c in ((0, 0), (1, 3), (5, 39), (11, 20)):
        e = np.zeros((T, C))
        e[t, c] = 0.5
        assert abs((f(x + e) - f(x - e)) - float(dx[t, c])) < 1e-5  # (linear: any step is exact)


# --------------------------------------------------------------------------------------- quantize

@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (1, 4096), (3, 7), (17, 515), (5, 2048), (2, 20001), (2050, 33), (2048, 4095), (2100, 4100)])
def test_quantize(comm, rows, cols, dt):
    rng = np.random.default_rng(cols)
    for pad, shift in ((0, 0), (3, 1)):
        x = rand(rng, rows, cols, dt, pad, shift=shift)
        if rows > 2:
            x[0] = 0.0
            x[1, cols - 1] = INF
            x[2, 0] = float("nan")
        if rows > 4:
            x[3] *= 2.0 ** -13
            x[4] = 1e-37 if dt != "fp16" else 0.0
        want, want_scale = ref.quantize(host(x))
        codes, scale = Room(rows, cols, torch.int8, pad, shift), Room(1, rows, torch.float32)
        comm.moe_quantize(x, codes.view, scale.view)
        torch.cuda.synchronize()
        codes.check(), scale.check()
        assert np.array_equal(host(codes.view), want)
        assert np.array_equal(scale.view[0].cpu().numpy(), want_scale, equal_nan=True)
        # to the rows of a dispatch
        if rows < 100:
            row = routes(rng, rows, 2, 2 * rows)
            many, scales = Room(2 * rows, cols, torch.int8, pad, shift), Room(1, 2 * rows, torch.float32)
            comm.moe_dispatch(x, torch.from_numpy(row).to(DEV), many.view, scale=scales.view[0])
            torch.cuda.synchronize()
            many.check(), scales.check()
            assert np.array_equal(host(many.view), ref.dispatch(want.astype(np.float64), row, np.full((2 * rows, cols), 77.0)))
            got = scales.view[0].cpu().numpy()[:, None]
            assert np.array_equal(got, ref.dispatch(want_scale[:, None], row, np.full((2 * rows, 1), 77, np.float32)), equal_nan=True)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,cols", [(1, 1), (7, 2048), (3, 1407), (2049, 72)])
def test_quantize_of_a_gate(comm, rows, cols, dt):
    rng = np.random.default_rng(cols)
    x = rand(rng, rows, 2 * cols, dt, 5, std=2.0)
    v = ref.silu_gate(host(x))
    codes, scale = Room(rows, cols, torch.int8, 3), Room(1, rows, torch.float32)
    comm.moe_quantize(x, codes.view, scale.view, gated=True)
    torch.cuda.synchronize()
    codes.check(), scale.check()
    m = np.abs(v).max(1, keepdims=True)
    # the gate in 32 bits is off by 8 units at most: a code by that, and half of one for the rounding
    close(codes.view, v * 127 / m, 0.5 + 127 * 16 * F32)
    close(scale.view[0], m[:, 0] / 127, 16 * F32 * m[:, 0])


@pytest.mark.parametrize("cols", [13, 61, 131, 509, 1003, 2501, 7003])
@pytest.mark.parametrize("dt", TYPES)
def test_quantize_many_odd_rows(comm, cols, dt):
    """Rows of odd sizes that fill the chip, as themselves and to the rows of a dispatch."""
    g = torch.Generator(device=DEV).manual_seed(cols)
    rows = 5000
    x = torch.randn(rows, cols + 3, generator=g, device=DEV).to(TYPES[dt])[:, 1:cols + 1]
    m = x.float().abs().amax(1, keepdim=True).cpu()
    want = torch.round(x.float().cpu() * (1 / m * 127)).to(torch.int8)
    codes, scale = Room(rows, cols, torch.int8, 2, 1), Room(1, rows, torch.float32)
    comm.moe_quantize(x, codes.view, scale.view)
    row = torch.randperm(2 * rows, generator=g, device=DEV).to(torch.int32).view(rows, 2)
    many, scales = Room(2 * rows, cols, torch.int8, 2, 1), Room(1, 2 * rows, torch.float32)
    comm.moe_dispatch(x, row, many.view, scale=scales.view[0])
    torch.cuda.synchronize()
    for room in (codes, scale, many, scales):
        room.check()
    assert torch.equal(codes.view.cpu(), want) and torch.equal(scale.view[0].cpu(), (m / 127)[:, 0])
    for k in range(2):
        at = row[:, k].long().cpu()
        assert torch.equal(many.view.cpu()[at], want) and torch.equal(scales.view[0].cpu()[at], (m / 127)[:, 0])


def test_quantize_up_to_a_limit_on_the_device(comm):
    rng = np.random.default_rng(0)
    x = rand(rng, 30, 100, "bf16")
    want, want_scale = ref.quantize(host(x))
    for n in (0, 1, 17, 30, 99, -4):
        codes, scale = torch.full((30, 100), 77, dtype=torch.int8, device=DEV), torch.full((30,), 77.0, device=DEV)
        comm.moe_quantize(x, codes, scale, limit=torch.tensor([n], device=DEV))
        k = min(max(n, 0), 30)
        assert np.array_equal(host(codes)[:k], want[:k]) and bool((codes[k:] == 77).all())
        assert np.array_equal(scale.cpu().numpy()[:k], want_scale[:k]) and bool((scale[k:] == 77).all())


# ---------------------------------------------------------------------------------------- product

def check_product(comm, rng, rows, inner, cols, experts, ends, dt, pad=0, shift=0, stream=None):
    def codes(*shape):
        return torch.from_numpy(rng.integers(-128, 128, size=shape).astype(np.int8))

    a, b = place(codes(rows, inner + pad), shift)[:, :inner], place(codes(experts, cols, inner + pad), shift)[:, :, :inner]
    sa = torch.from_numpy((rng.random(rows) + 0.5).astype(np.float32) / 128).to(DEV)
    sb = torch.from_numpy((rng.random((experts, cols)) - 0.5).astype(np.float32) / 128).to(DEV)
    out = Room(rows, cols, TYPES[dt], pad, shift)
    offsets = None if ends is None else torch.tensor(ends, dtype=torch.int64, device=DEV)
    comm.moe_product(a, sa, b, sb, out.view, offsets=offsets, stream=stream)
    torch.cuda.synchronize()
    out.check()
    want = ref.product(a.cpu().numpy(), sa.cpu().numpy(), b.cpu().numpy(), sb.cpu().numpy(), ends, np.full((rows, cols), 77.0))
    rounded(out.view, want, 3 * F32 * np.abs(want))  # (the whole sum to 32 bits, and two products)


@pytest.mark.parametrize("dt", ["bf16", "fp16", "fp32"])
@pytest.mark.parametrize("rows,inner,cols", [
    (1, 1, 1), (1, 4096, 4096), (1, 127, 65), (2, 129, 30), (15, 64, 16), (16, 128, 64), (17, 1000, 100), (33, 2048, 48), (64, 512, 255), (100, 16, 300),
    (128, 256, 128), (129, 1407, 257), (255, 96, 512), (300, 640, 1000), (513, 320, 768), (1000, 2049, 70), (40, 0, 33)])
def test_product_of_one_expert(comm, rows, inner, cols, dt):
    rng = np.random.default_rng(rows + inner)
    check_product(comm, rng, rows, inner, cols, 1, None, dt)
    check_product(comm, rng, rows, inner, cols, 1, [0, rows], dt, pad=16)
    check_product(comm, rng, rows, inner, cols, 1, None, dt, pad=5, shift=1)


@pytest.mark.parametrize("dt", ["bf16", "fp32"])
@pytest.mark.parametrize("rows,inner,cols,experts,sources", [
    (1, 256, 64, 4, 1), (7, 100, 40, 16, 1), (64, 512, 200, 8, 1), (256, 384, 130, 64, 1), (300, 130, 64, 100, 1), (1500, 256, 300, 5, 1),
    (900, 272, 256, 3, 4), (4000, 128, 520, 8, 1), (200, 64, 32, 70, 2)])
def test_product_of_segments(comm, rows, inner, cols, experts, sources, dt):
    """Segments of all lengths, some empty, some rows in none; several sources that use the same experts."""
    rng = np.random.default_rng(rows + experts)
    n = experts * sources
    for skew in (0.0, 3.0):
        p = np.exp(skew * rng.normal(size=n + 1))
        sizes = rng.multinomial(rows, p / p.sum())[:n]
        ends = np.concatenate([[0], np.cumsum(sizes)])
        check_product(comm, rng, rows, inner, cols, experts, ends.tolist(), dt)
    check_product(comm, rng, rows, inner, cols, experts, [0] * (n + 1), dt)
    check_product(comm, rng, rows, inner, cols, experts, [0] * n + [rows], dt, pad=3)
    first = rows // 3
    check_product(comm, rng, rows, inner, cols, experts, [first] + [rows] * n, dt, pad=16)
    # offsets beyond the rows, or that go back, move nothing beyond them
    check_product(comm, rng, rows, inner, cols, experts, [0] + [rows + 1000] * n, dt)


def on_gpu(codes, scale, weights, weight_scale, ends):
    """The product in 64 bits on the GPU, segment by segment (whole sums below 2^53)."""
    out = torch.zeros(codes.shape[0], weights.shape[1], device=DEV, dtype=torch.float64)
    for s, (a, b) in enumerate(zip(ends[:-1], ends[1:])):
        e = s % weights.shape[0]
        if b > a:
            out[a:b] = torch.mm(codes[a:b].double(), weights[e].double().t().contiguous()) * scale[a:b, None].double() * weight_scale[e].double()
    return out


# (rows, columns, experts): sizes for each of the tiles that a product chooses among on 256 CUs
TILES = {"256x256": (6000, 2100, 8), "256x256 dense": (3000, 4100, 1), "128x128": (3000, 1500, 12), "64x128": (1000, 2000, 40), "64x64": (300, 3000, 1),
         "few 16x64": (100, 4096, 30), "few 16x32": (3, 8200, 1), "few 16x16": (9, 300, 1), "few 32x64": (512, 2050, 40), "few 32x32": (48, 4100, 1),
         "few 32x16": (505, 185, 1)}


@pytest.mark.parametrize("inner", [16, 64, 65, 128, 191, 192, 256, 320, 321, 384, 447, 640, 1000])
@pytest.mark.parametrize("tile", TILES)
def test_product_of_every_tile_and_length(comm, tile, inner):
    rows, cols, experts = TILES[tile]
    g = torch.Generator(device=DEV).manual_seed(inner)
    rng = np.random.default_rng(rows + inner)
    sizes = rng.multinomial(rows, rng.dirichlet(np.full(experts, 8.0)))
    ends = np.concatenate([[0], np.cumsum(sizes)]).tolist()
    offsets = torch.tensor(ends, device=DEV) if experts > 1 else None
    dt = ("bf16", "fp16", "fp32")[inner % 3]
    sa, sb = torch.rand(rows, generator=g, device=DEV) / 64, torch.rand(experts, cols, generator=g, device=DEV) / 64
    whole = (inner + 15) // 16 * 16
    for pa, pb in ((whole - inner, whole - inner), (1 + whole - inner, whole - inner), (whole - inner, 1 + whole - inner), (3, 3)):
        a = torch.randint(-128, 128, (rows, inner + pa), generator=g, device=DEV, dtype=torch.int8)[:, :inner]
        w = torch.randint(-128, 128, (experts, cols, inner + pb), generator=g, device=DEV, dtype=torch.int8)[:, :, :inner]
        out = Room(rows, cols, TYPES[dt], pa)
        comm.moe_product(a, sa, w, sb, out.view, offsets=offsets)
        torch.cuda.synchronize()
        out.check()
        want = on_gpu(a, sa, w, sb, ends)
        bound = 4 * F32 * want.abs() + 1e-37
        lo, hi = ((want + s * bound).float().to(TYPES[dt]).double() for s in (-1, 1))
        got = out.view.double()
        bad = ~((lo <= got) & (got <= hi))
        assert not bool(bad.any()), f"{int(bad.sum())} of {bad.numel()} off, first at {bad.nonzero()[0].tolist()}"


def test_product_of_many_segments(comm):
    """More segments than a wave has lanes, in one-row tiles and in large ones, some of them empty."""
    g = torch.Generator(device=DEV).manual_seed(0)
    for rows, cols, experts, sources in ((700, 512, 100, 3), (9000, 1024, 70, 2), (20000, 300, 33, 8)):
        n = experts * sources
        rng = np.random.default_rng(n)
        ends = np.concatenate([[0], np.cumsum(rng.multinomial(rows, rng.dirichlet(np.full(n, 0.7))))]).tolist()
        a = torch.randint(-128, 128, (rows, 96), generator=g, device=DEV, dtype=torch.int8)
        w = torch.randint(-128, 128, (experts, cols, 96), generator=g, device=DEV, dtype=torch.int8)
        sa, sb = torch.rand(rows, generator=g, device=DEV), torch.rand(experts, cols, generator=g, device=DEV)
        out = torch.empty(rows, cols, device=DEV)
        comm.moe_product(a, sa, w, sb, out, offsets=torch.tensor(ends, device=DEV))
        want = on_gpu(a, sa, w, sb, ends)
        assert bool(((out.double() - want).abs() <= 4 * F32 * want.abs()).all())


def test_product_of_rows_that_are_no_numbers(comm):
    """A quantised row with an infinity or NaN gives NaN; a row of zeros gives zeros."""
    rng = np.random.default_rng(0)
    x = rand(rng, 6, 64, "bf16")
    x[1, 5], x[2, 6], x[3] = INF, float("nan"), 0.0
    codes, scale = torch.empty(6, 64, dtype=torch.int8, device=DEV), torch.empty(6, device=DEV)
    comm.moe_quantize(x, codes, scale)
    w = torch.from_numpy(rng.integers(-127, 128, size=(1, 40, 64)).astype(np.int8)).to(DEV)
    out = torch.empty(6, 40, device=DEV)
    comm.moe_product(codes, scale, w, torch.ones(1, 40, device=DEV), out)
    nan = torch.isnan(out).all(1).tolist()
    assert nan == [False, True, True, False, False, False] and bool((out[3] == 0).all()) and bool(torch.isfinite(out[[0, 4, 5]]).all())


def test_product_sums_are_whole(comm):
    """The greatest sums there are: 131 071 products of 2^14."""
    n = 131071
    a = torch.full((3, n), -128, dtype=torch.int8, device=DEV)
    a[1] = 127
    w = torch.full((1, 5, n), -128, dtype=torch.int8, device=DEV)
    out = torch.empty(3, 5, device=DEV)
    comm.moe_product(a, torch.ones(3, device=DEV), w, torch.ones(1, 5, device=DEV), out)
    assert out[0].tolist() == [float(np.float32(n * 16384))] * 5 and out[1].tolist() == [float(np.float32(-n * 127 * 128))] * 5


def test_nothing_to_do(comm):
    """No tokens, rows or columns: nothing is read, and what is left to write is."""
    i32, f32, i8 = (dict(dtype=t, device=DEV) for t in (torch.int32, torch.float32, torch.int8))
    r = H.hccl_router_init(experts=8, top_k=2)
    none = torch.empty(0, 8, **f32)
    comm.moe_route(r, none, torch.empty(0, 2, **i32), torch.empty(0, 2, **f32))
    comm.moe_route_backward(r, none, torch.empty(0, 2, **i32), torch.empty(0, 2, **f32), none)
    comm.moe_dispatch(none, torch.empty(0, 2, **i32), torch.empty(4, 8, **f32))
    comm.moe_dispatch(torch.ones(3, 8, **f32), torch.zeros(3, 2, **i32), none)
    out = torch.full((3, 8), 77.0, device=DEV)
    comm.moe_combine(none, torch.zeros(3, 2, **i32), out)  # rows that there are none of
    assert bool((out == 0).all())
    gw = torch.full((3, 2), 77.0, device=DEV)
    comm.moe_combine_backward(torch.empty(3, 0, **f32), torch.empty(6, 0, **f32), torch.arange(6, **i32).view(3, 2), torch.ones(3, 2, **f32),
                              torch.empty(6, 0, **f32), gw)
    assert bool((gw == 0).all())
    comm.moe_quantize(none, torch.empty(0, 8, **i8), torch.empty(0, **f32))
    scale = torch.full((3,), 77.0, device=DEV)
    comm.moe_quantize(torch.empty(3, 0, **f32), torch.empty(3, 0, **i8), scale)
    assert bool((scale == 0).all())
    comm.moe_product(torch.empty(0, 8, **i8), torch.empty(0, **f32), torch.zeros(2, 4, 8, **i8), torch.ones(2, 4, **f32), torch.empty(0, 4, **f32),
                     offsets=torch.zeros(3, dtype=torch.int64, device=DEV))
    torch.cuda.synchronize()


# ------------------------------------------------------------------- offsets, streams, graphs, order

def test_rows_far_apart(comm):
    """Element offsets beyond 32 bits in every array of rows."""
    step = (1 << 31) + 8
    rng = np.random.default_rng(0)
    big = torch.empty(2 * step + 64, dtype=torch.bfloat16, device=DEV)
    far = big.as_strided((3, 64), (step, 1))
    near = rand(rng, 3, 64, "bf16")
    row = torch.tensor([[2], [0], [1]], dtype=torch.int32, device=DEV)
    comm.moe_dispatch(near, row, far)
    assert torch.equal(far[[2, 0, 1]], near)
    out = torch.empty_like(near)
    comm.moe_combine(far, row, out)
    assert torch.equal(out, near)
    gw = torch.empty(3, 1, device=DEV)
    gz = torch.empty_like(near)
    comm.moe_combine_backward(near, far, row, torch.ones(3, 1, device=DEV), gz, gw)
    assert torch.equal(gz[[2, 0, 1]], near) and torch.allclose(gw[:, 0], (near.float() ** 2).sum(1), rtol=1e-5)
    comm.moe_combine(near, row, far)
    assert torch.equal(far, near[[2, 0, 1]])
    codes, scale = torch.empty(3, 64, dtype=torch.int8, device=DEV), torch.empty(3, device=DEV)
    comm.moe_quantize(far, codes, scale)
    want = ref.quantize(host(far))
    assert np.array_equal(host(codes), want[0])
    index, weight = torch.empty(3, 4, dtype=torch.int32, device=DEV), torch.empty(3, 4, device=DEV)
    comm.moe_route(H.hccl_router_init(experts=64, top_k=4), far, index, weight)
    assert np.array_equal(host(index), ref.route(host(far), 4)[0])
    small = big.view(torch.int8)
    a, o = small.as_strided((3, 64), (step, 1)), big.as_strided((3, 64), (step, 1), 0)
    a.copy_(codes)
    w = torch.from_numpy(rng.integers(-127, 128, size=(1, 64, 64)).astype(np.int8)).to(DEV)
    got, same = torch.empty(3, 64, device=DEV), torch.empty(3, 64, device=DEV)
    comm.moe_product(a, scale, w, torch.ones(1, 64, device=DEV), got)
    comm.moe_product(codes, scale, w, torch.ones(1, 64, device=DEV), same)
    assert torch.equal(got, same)
    far_w = small.as_strided((1, 3, 64), (3 * step, step, 1))
    far_w.copy_(w[:, :3])
    comm.moe_product(codes, scale, far_w, torch.ones(1, 3, device=DEV), got[:, :3])
    assert torch.equal(got[:, :3], same[:, :3])
    comm.moe_product(codes, scale, w, torch.ones(1, 64, device=DEV), o)
    assert torch.equal(o, same.to(torch.bfloat16))


class Layer:
    """One pass through all operators, on preallocated tensors."""

    def __init__(self, comm, T=300, E=16, K=4, C=256, N=128, stream=None):
        g = torch.Generator(device=DEV).manual_seed(1)
        self.x = torch.randn(T, C, generator=g, device=DEV).to(torch.bfloat16)
        self.logits = torch.randn(T, E, generator=g, device=DEV)
        self.w = torch.randint(-127, 128, (E, N, C), generator=g, device=DEV, dtype=torch.int8)
        ws = torch.rand(E, N, generator=g, device=DEV) / 1000
        index, self.weight = torch.empty(T, K, dtype=torch.int32, device=DEV), torch.empty(T, K, device=DEV)
        row, offsets = torch.empty(T, K, dtype=torch.int32, device=DEV), torch.empty(E + 1, dtype=torch.int64, device=DEV)
        codes, scale = torch.empty(T * K, C, dtype=torch.int8, device=DEV), torch.empty(T * K, device=DEV)
        rows, self.y = torch.empty(T * K, N, device=DEV, dtype=torch.bfloat16), torch.empty(T, N, device=DEV, dtype=torch.bfloat16)
        self.gz, self.gw = torch.empty_like(rows), torch.empty_like(self.weight)
        self.gl = torch.empty_like(self.logits)
        dy = torch.randn(T, N, generator=g, device=DEV).to(torch.bfloat16)
        r = H.hccl_router_init(experts=E, top_k=K, renormalize=True)

        def bind(stream=None):
            s = dict(stream=stream)
            return [
                comm.bind_moe_route(r, self.logits, index, self.weight, **s), comm.bind_moe_plan(index, E, row, offsets, T * K, **s),
                comm.bind_moe_dispatch(self.x, row, codes, scale=scale, **s), comm.bind_moe_product(codes, scale, self.w, ws, rows, offsets=offsets, **s),
                comm.bind_moe_combine(rows, row, self.y, weight=self.weight, **s),
                comm.bind_moe_combine_backward(dy, rows, row, self.weight, self.gz, self.gw, **s),
                comm.bind_moe_route_backward(r, self.logits, index, self.gw, self.gl, **s)]

        self.bind, self.calls = bind, bind(stream)
        self.out = [index, self.weight, row, offsets, codes, scale, rows, self.y, self.gz, self.gw, self.gl]

    def __call__(self):
        for call in self.calls:
            call()

    def results(self):
        torch.cuda.synchronize()
        return [t.clone() for t in self.out]


def test_results_are_the_same_in_every_call_and_on_another_stream(comm):
    layer = Layer(comm)
    layer()
    want = layer.results()
    for _ in range(3):
        for t in layer.out:
            t.zero_()
        layer()
        assert all(torch.equal(a, b) for a, b in zip(layer.results(), want))
    with SideStream() as side:
        torch.cuda.synchronize()
        other = Layer(comm, stream=side)
        torch.cuda.synchronize()
        other()
        side.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(other.results(), want))


def test_a_captured_layer_replays(comm):
    """Captured at its first call; replayed on new inputs with eager work in between."""
    layer, eager = Layer(comm), Layer(comm)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        for call in layer.bind():  # (on the stream that captures)
            call()
    for seed in range(4):
        g = torch.Generator(device=DEV).manual_seed(100 + seed)
        layer.logits.copy_(torch.randn(layer.logits.shape, generator=g, device=DEV))
        layer.x.copy_(torch.randn(layer.x.shape, generator=g, device=DEV))
        eager.logits.copy_(layer.logits)
        eager.x.copy_(layer.x)
        graph.replay()
        got = layer.results()
        eager()
        assert all(torch.equal(a, b) for a, b in zip(got, eager.results()))

