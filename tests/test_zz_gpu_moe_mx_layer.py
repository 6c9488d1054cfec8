"""The whole layer for few tokens, with 4-bit weights, against its definition in 64 bits.

Weights and their products with 16-bit parts of a row are exact in 32 bits, so a sum of n of them is off by at most n 2^-23 of
the sum of their sizes (an instruction may cut off what an addition would round); rows of fp16 and fp32 go in two
and three parts. The hidden value's sums' errors pass through the gate with at most their slopes; the gate itself is off by
(1.5 |g| + 8) 2^-24, what is kept of the hidden value by 2^-16 where that is in two parts, the routing weight by 1e-5.
Then one rounding to the result's type, which keeps order.
"""
import numpy as np
import pytest
import torch

import moe_reference as ref
import mx_reference as mx
import paper_2608_00358_amd as H
from gpu_helpers import SideStream
from test_zz_gpu_moe import DEV, F32, INF, TYPES, Room, host, place, rand, rounded
from test_zz_gpu_moe_mx import U8, bytes_of, random_mx, values

pytestmark = pytest.mark.gpu
PARTS, PLANES = {"bf16": 1, "fp16": 2, "fp32": 3}, {"bf16": 2, "fp16": 2, "fp32": 3}


@pytest.fixture(scope="module")
def comm():
    with H.Comm(4, device=0) as c:
        yield c


class Case:
    def __init__(self, rng, T, E, K, C, F, dt, ldt=None, held=None, first=0, pad=0, shift=0, mask=None, **router):
        self.T, self.E, self.K, self.C, self.F, self.dt, self.first, self.held = T, E, K, C, F, dt, first, held or E
        self.logits = rand(rng, T, E, ldt or "fp32", pad, 1.5, shift)
        self.x = rand(rng, T, C, dt, pad, 1.0, shift)
        # scales so that hidden values and results are about 1 in size
        lo = 127 - int(round(np.log2(max(C, 1)) / 2)) - 2
        self.w_in = random_mx(rng, self.held, 2 * F, C, pad=pad, spad=pad // 2, shift=shift, lo=lo - 1, hi=lo + 2)
        lo = 127 - int(round(np.log2(max(F, 1)) / 2)) - 2
        self.w_out = random_mx(rng, self.held, C, F, pad=pad, spad=pad // 2, shift=shift, lo=lo - 1, hi=lo + 2)
        self.mask = mask
        self.router = H.hccl_router_init(experts=E, top_k=K, **router)
        self.options = router
        self.index, self.weight, self.out = Room(T, K, torch.int32), Room(T, K, torch.float32), Room(T, C, TYPES[dt], pad, shift)
        self.need = H.hccl_moe_layer_mx_bytes(T, K, C, F, self.held)
        self.space = Room(1, self.need, U8)

    def args(self):
        space = self.space.flat[self.space.at:self.space.at + self.need] if self.need else None
        return dict(router=self.router, logits=self.logits, x=self.x, w_in=self.w_in[0], w_in_scale=self.w_in[1], w_out=self.w_out[0], w_out_scale=self.w_out[1],
                    index=self.index.view, weight=self.weight.view, out=self.out.view, first=self.first, workspace=space,
                    mask=None if self.mask is None else torch.from_numpy(self.mask).to(DEV))

    def run(self, comm, **kw):
        comm.moe_layer_mx(**self.args(), **kw)
        return self

    def check(self):
        torch.cuda.synchronize()
        for room in (self.index, self.weight, self.out, self.space):
            room.check()
        index, weight, _ = ref.route(host(self.logits), self.K, mask=self.mask, **self.options)
        assert np.array_equal(host(self.index.view), index)
        got = host(self.weight.view)
        assert (np.abs(got - weight) <= 1e-5 * np.abs(weight) + 1e-37).all()
        y, size, spread, greatest = mx.layer(host(self.x), index, weight, host(values(*self.w_in, self.C)), host(values(*self.w_out, self.F)), self.first)
        kept = 0 if self.dt == "fp32" else 2.0 ** -16
        bound = PARTS[self.dt] * (self.C + 16) * 2 * F32 * spread
        bound += (kept + (1.5 * greatest + 8) * F32 + PLANES[self.dt] * (self.F + 32) * 2 * F32 + 1e-5 + 2.0 ** -20) * size
        rounded(self.out.view, y, bound)
        return y


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T,E,K,C,F", [
    (1, 1, 1, 1, 1), (1, 8, 2, 32, 16), (1, 64, 4, 512, 256), (2, 4, 4, 33, 17), (3, 60, 2, 100, 40), (5, 60, 6, 1003, 117), (8, 128, 8, 256, 96), (16, 8, 2, 130, 64),
    (17, 8, 2, 255, 31), (32, 16, 4, 64, 160), (33, 2, 2, 96, 48), (64, 4, 1, 80, 24), (64, 1, 1, 300, 33), (64, 32, 8, 48, 80), (7, 1024, 32, 40, 20),
    (64, 1024, 32, 17, 9), (4, 3, 3, 2050, 513), (2, 5, 1, 7, 1100), (9, 40, 6, 304, 288), (11, 30, 4, 768, 256), (30, 12, 3, 256, 320), (5, 16, 3, 1024, 1280),
    (40, 6, 3, 544, 512), (1, 200, 16, 3000, 270)])
def test_layer(comm, T, E, K, C, F, dt):
    rng = np.random.default_rng(T + E + C)
    Case(rng, T, E, K, C, F, dt, renormalize=True).run(comm).check()
    Case(rng, T, E, K, C, F, dt, ldt=dt if dt == "fp32" else None, pad=3, shift=1, scale=2.5).run(comm).check()


@pytest.mark.parametrize("dt", TYPES)
def test_logits_of_another_type(comm, dt):
    rng = np.random.default_rng(1)
    for ldt in TYPES:
        Case(rng, 6, 24, 3, 64, 48, dt, ldt=ldt, score="sigmoid", renormalize=True).run(comm).check()


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T", [1, 9, 40])
def test_a_ranks_experts(comm, T, dt):
    """The parts of ranks that hold a quarter each add up to the whole; experts of others add nothing."""
    rng = np.random.default_rng(T)
    whole = Case(rng, T, 32, 4, 200, 72, dt, renormalize=True)
    want = whole.run(comm).check()
    total = np.zeros_like(want)
    for first in (0, 8, 16, 24):
        part = Case(rng, T, 32, 4, 200, 72, dt, held=8, first=first, renormalize=True)
        part.logits, part.x = whole.logits, whole.x
        part.w_in, part.w_out = (tuple(t[first:first + 8] for t in w) for w in (whole.w_in, whole.w_out))
        total += part.run(comm).check()
    assert np.abs(total - want).max() <= 1e-12 * np.abs(want).max()


def test_ranks_add_up_their_parts_by_allreduce():
    """The decoding step of a group: every rank has the tokens and a quarter of the experts."""
    rng = np.random.default_rng(3)
    whole = Case(rng, 6, 16, 4, 256, 64, "fp32", renormalize=True)
    with H.Comm(4, device=0) as comm:
        y = whole.run(comm).check()
        parts = []
        for r in range(4):
            part = Case(rng, 6, 16, 4, 256, 64, "fp32", held=4, first=4 * r, renormalize=True)
            part.logits, part.x = whole.logits, whole.x
            part.w_in, part.w_out = (tuple(t[4 * r:4 * r + 4] for t in w) for w in (whole.w_in, whole.w_out))
            part.run(comm)
            parts.append(part.out.view)
        out = [torch.empty(6, 256, device=DEV) for _ in range(4)]
        comm.allreduce([p.reshape(-1) for p in parts], [o.view(-1) for o in out])
        torch.cuda.synchronize()
        assert comm.async_error() == 0
    for o in out:
        assert np.abs(host(o) - y).max() < 1e-4 * np.abs(y).max() + 1e-30


@pytest.mark.parametrize("dt", TYPES)
def test_tokens_without_an_expert(comm, dt):
    """Masked tokens and those whose logits are all -inf have zeros; all of them masked is no special case."""
    rng = np.random.default_rng(4)
    case = Case(rng, 7, 12, 3, 64, 40, dt, mask=np.array([1, 0, 1, 1, 0, 1, 0], np.uint8), renormalize=True)
    case.logits[3] = -INF
    case.logits[5, 2:] = -INF  # (fewer experts than choices)
    y = case.run(comm).check()
    assert (y[[1, 3, 4, 6]] == 0).all() and bool((case.out.view[[1, 3, 4, 6]] == 0).all())
    case = Case(rng, 5, 12, 3, 64, 40, dt, mask=np.zeros(5, np.uint8))
    case.run(comm).check()
    assert bool((case.out.view == 0).all())


def test_many_tokens_of_one_expert(comm):
    """All tokens choose the same two experts: more of them than a matrix instruction has rows."""
    rng = np.random.default_rng(5)
    for T, E in ((16, 40), (17, 40), (31, 200), (64, 8), (64, 200)):
        case = Case(rng, T, E, 2, 96, 56, "bf16", renormalize=True)
        case.logits[:, 3] = 9.0
        case.logits[:, E - 1] = 8.0
        case.run(comm).check()
        assert bool((case.index.view == torch.tensor([3, E - 1], device=DEV)).all())


@pytest.mark.parametrize("dt", TYPES)
def test_a_token_that_is_no_number(comm, dt):
    """Its results are no finite numbers, and no other token's are touched."""
    rng = np.random.default_rng(6)
    case = Case(rng, 9, 6, 2, 100, 48, dt, renormalize=True)
    case.run(comm)
    want = case.out.view.clone()
    case.x[2, 50], case.x[6, 7] = INF, float("nan")
    case.run(comm)
    torch.cuda.synchronize()
    others = [0, 1, 3, 4, 5, 7, 8]
    assert torch.equal(case.out.view[others], want[others])
    assert not bool(torch.isfinite(case.out.view[[2, 6]]).any())


def test_weights_that_are_no_numbers(comm):
    """A scale of 255 in a column of the last product leaves that column alone without a number, for tokens of its expert."""
    rng = np.random.default_rng(7)
    case = Case(rng, 8, 4, 1, 70, 64, "fp32")
    case.w_out[1][2, 33, 1] = 255
    case.run(comm)
    torch.cuda.synchronize()
    want = torch.zeros(8, 70, dtype=torch.bool)
    want[(case.index.view[:, 0] == 2).cpu(), 33] = True
    assert torch.equal(torch.isnan(case.out.view).cpu(), want)


def test_far_rows(comm):
    """Byte offsets beyond 32 bits in every array of rows."""
    rng = np.random.default_rng(8)
    case = Case(rng, 2, 2, 1, 64, 32, "bf16", ldt="bf16")
    want = case.run(comm).out.view.clone()
    step = (1 << 32) + 64
    rows, weights = torch.zeros(2 * step, dtype=U8, device=DEV), torch.zeros(4 * step, dtype=U8, device=DEV)

    def far(t, at):  # two rows
        v = rows.view(t.dtype).as_strided(t.shape, (step // 2, 1), at // 2)
        return v.copy_(t)

    def far_weights(t, at):  # 128 rows
        ld = step // 32
        v = weights.as_strided(t.shape, (t.shape[1] * ld, ld, 1), at)
        return v.copy_(t)

    case.x, case.logits = far(case.x, 0), far(case.logits, 1024)
    case.w_in, case.w_out = (tuple(far_weights(t, at + 64 * n) for n, t in enumerate(w)) for at, w in ((0, case.w_in), (4096, case.w_out)))
    args = case.args()
    args["out"] = far(torch.zeros(2, 64, dtype=torch.bfloat16, device=DEV), 4096)
    comm.moe_layer_mx(**args)
    assert torch.equal(args["out"], want)


def test_results_are_the_same_in_every_call_and_on_another_stream(comm):
    rng = np.random.default_rng(9)
    for T, E, K in ((1, 64, 4), (24, 16, 4)):
        case = Case(rng, T, E, K, 512, 288, "bf16", renormalize=True)
        want = case.run(comm).out.view.clone()
        for _ in range(5):
            case.out.view.zero_(), case.space.flat[case.space.at:case.space.at + case.need].fill_(255)
            assert torch.equal(case.run(comm).out.view, want)
        with SideStream() as side:
            case.out.view.zero_()
            torch.cuda.synchronize()
            case.run(comm, stream=side)
            side.synchronize()
            assert torch.equal(case.out.view, want)


def test_captured_layers_replay(comm):
    """Two graphs, a workspace each, captured at their first call; replayed on new inputs with eager work in between."""
    rng = np.random.default_rng(10)
    cases = [Case(rng, T, 32, 4, 256, 160, "bf16", renormalize=True) for T in (1, 12)]
    graphs = []
    for case in cases:
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        args = case.args()
        with torch.cuda.graph(graph):
            comm.moe_layer_mx(**args)
        graphs.append(graph)
    for _ in range(4):
        for case, graph in zip(cases, graphs):
            case.logits.copy_(rand(rng, case.T, 32, "fp32"))
            case.x.copy_(rand(rng, case.T, 256, "bf16"))
            graph.replay()
        torch.cuda.synchronize()
        for case in cases:
            got = case.out.view.clone()
            case.check()
            case.out.view.zero_()
            assert torch.equal(case.run(comm).out.view, got)


def test_calls_on_two_streams_at_once(comm):
    """Workspaces of their own, no order between them."""
    rng = np.random.default_rng(11)
    cases = [Case(rng, T, 32, 4, 1024, 512, "bf16", renormalize=True) for T in (3, 20)]
    want = [case.run(comm).out.view.clone() for case in cases]
    with SideStream() as side:
        for case in cases:
            case.out.view.zero_()
        torch.cuda.synchronize()
        for _ in range(20):
            cases[0].run(comm)
            cases[1].run(comm, stream=side)
        torch.cuda.synchronize()
    assert all(torch.equal(case.out.view, w) for case, w in zip(cases, want))


@pytest.mark.parametrize("dt", TYPES)
@pytest.mark.parametrize("T,E,K,C,F", [
    (1, 4, 2, 128, 128), (3, 8, 2, 384, 128), (9, 6, 3, 128, 640), (24, 16, 4, 640, 384), (33, 4, 2, 1152, 896), (64, 8, 2, 128, 1408), (5, 90, 8, 2176, 384), (2, 3, 1, 896, 256)])
def test_rows_that_end_with_half_a_step(comm, T, E, K, C, F, dt):
    """Multiples of 128 elements, aligned, with the last expert's rows at the ends of their arrays; and blocks that are no numbers at
    the end of one expert's rows."""
    rng = np.random.default_rng(T + C + F)
    Case(rng, T, E, K, C, F, dt, renormalize=True).run(comm).check()
    Case(rng, T, E, K, C, F, dt, held=max(1, E // 2), first=E - max(1, E // 2)).run(comm).check()
    case = Case(rng, T, E, K, C, F, dt, renormalize=True)
    case.w_in[1][E - 1, :, -1] = 255  # (the last block of one expert's gates and ups)
    case.run(comm)
    torch.cuda.synchronize()
    index, out = host(case.index.view), host(case.out.view.float())
    bad = (index == E - 1).any(1)
    assert np.isnan(out[bad]).all() and np.isfinite(out[~bad]).all()


@pytest.mark.parametrize("ldt", TYPES)
@pytest.mark.parametrize("T,E,K,options", [
    (1, 1, 1, {}), (1, 128, 16, {}), (33, 128, 16, {}), (64, 127, 5, {}), (3, 129, 8, {}), (5, 64, 17, {}), (32, 7, 7, {}), (40, 96, 6, {"groups": 8, "top_groups": 3}),
    (40, 96, 6, {"groups": 8, "top_groups": 8}), (9, 64, 4, {"groups": 4, "top_groups": 2, "group_top": 2})])
def test_routes_are_those_of_the_router_alone(comm, T, E, K, options, ldt):
    """Whichever kernel makes them: equal logits, tokens whose logits are masked in part or all, a bias, padding tokens.

    The weights' sums of up to E terms may be added up in another order: each is off by E 2^-24 of itself at most, and the few
    roundings behind it by 2^-24 each.
    """
    rng = np.random.default_rng(13)
    for score in ("softmax", "sigmoid"):
        for renormalize in (False, True):
            for biased in (False, True):
                case = Case(rng, T, E, K, 64, 32, "bf16", ldt=ldt, score=score, renormalize=renormalize, scale=1.5, **options)
                logits = case.logits
                logits.copy_((logits * 2).round() / 2)  # (many are equal)
                for t, v in ((2, -INF), (4, float("nan")), (6, INF), (8, -1e4)):
                    if t < T:
                        logits[t, :: 1 if t in (2, 8) else 3] = v
                if biased:
                    logits[logits == INF] = 1.0
                bias = torch.from_numpy(rng.integers(-2, 3, E).astype(np.float32) / 4).to(DEV) if biased else None
                case.mask = (rng.random(T) < 0.8).astype(np.uint8)
                mask = torch.from_numpy(case.mask).to(DEV)
                index, weight = torch.empty(T, K, dtype=torch.int32, device=DEV), torch.empty(T, K, device=DEV)
                comm.moe_route(case.router, logits, index, weight, bias=bias, mask=mask)
                case.run(comm, bias=bias)
                torch.cuda.synchronize()
                for room in (case.index, case.weight, case.out, case.space):
                    room.check()
                assert torch.equal(case.index.view, index)
                want, got = weight.double(), case.weight.view.double()
                assert bool(((got - want).abs() <= (2 * E + 16) * 2.0 ** -24 * want.abs() + 1e-37).all())


def test_nothing_to_do(comm):
    rng = np.random.default_rng(12)
    Case(rng, 0, 4, 2, 64, 32, "bf16").run(comm)
    case = Case(rng, 3, 4, 2, 64, 0, "bf16").run(comm)
    torch.cuda.synchronize()
    assert bool((case.out.view == 0).all())
    case = Case(rng, 3, 4, 2, 0, 32, "bf16").run(comm)
    torch.cuda.synchronize()
    assert np.array_equal(host(case.index.view), ref.route(host(case.logits), 2)[0])
