"""Microscaled 4-bit operators of a mixture-of-experts layer, as cases that can be timed and compared.

Rows and weights are held as 4-bit floats (0, 0.5, 1, 1.5, 2, 3, 4, 6 and their negatives, two codes a byte, the
lower half first) with one power of two for every 32 neighbours of a row, kept as its exponent plus 127 in a
byte. A block whose greatest magnitude is m has the least scale 2^s with m < 7 * 2^s, and codes are the nearest
values, ties to the even code. A case names one of three operators with its sizes and types:

  rows      rows -> codes, at once into the experts' order where a row goes to several experts, and read back
  product   rows -> codes -> the product with the 4-bit weights of every row's expert
  layer     logits and rows of a few tokens -> choices, weights and the whole layer's result, with 4-bit
            weights and rows in their own type:  y_t = sum_k w_tk W_out (silu(W_gate x_t) * (W_up x_t))

`prepare` makes what a program holds before the call, `run` makes one pass. Where `own` is false the
operators are computed in their plain form, by elementary tensor operations in 32 bits.
"""
import math

import numpy as np
import torch

own = False

DEVICE = "cuda:0"
TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}
SIZE = {"bf16": 2, "fp16": 2, "fp32": 4}
Ki, Mi = 1024, 1024 * 1024
BLOCK = 32

# Fields that a case leaves out.
DEFAULTS = {
    "rows": {"experts": 0, "top_k": 0, "masked": 0.0, "pad": 0},
    "product": {"gated": False, "top_k": 0, "pad": 0},
    "layer": {"score": "softmax", "renormalize": True, "scale": 1.0, "masked": 0.0, "held": 0, "pad": 0},
}


def listed():
    return [
        # A few tokens of a serving batch, four experts each, with a row length that is no multiple of a block.
        {"name": "rows_serving", "op": "rows", "rows": 37, "experts": 64, "top_k": 4, "cols": 1001, "dtype": "bf16"},
        # A prompt's tokens into the experts' order, and read back by their ranks: what an exchange in 4 bits does
        # at its ends.
        {"name": "rows_prompt", "op": "rows", "rows": 8 * Ki, "experts": 64, "top_k": 4, "cols": 4096, "dtype": "bf16"},
        # Rows of a layer in 32 bits, odd and apart.
        {"name": "rows_odd", "op": "rows", "rows": 3001, "cols": 2051, "dtype": "fp32", "pad": 3},
        # One new token through a dense layer: the weights' bytes are all.
        {"name": "product_one_token", "op": "product", "rows": 1, "experts": 1, "inner": 4096, "cols": 4096, "dtype": "bf16"},
        # A serving batch of 64 tokens, four experts each: a handful of rows for each expert.
        {"name": "product_serving", "op": "product", "rows": 256, "experts": 64, "inner": 2048, "cols": 2048, "dtype": "bf16",
         "top_k": 4},
        # A ragged layer: odd sizes everywhere, the gate of the first product applied on the way in.
        {"name": "product_ragged", "op": "product", "rows": 2999, "experts": 12, "inner": 1407, "cols": 2050, "dtype": "bf16",
         "gated": True},
        # A prompt's rows through 16 experts, the largest call.
        {"name": "product_prompt", "op": "product", "rows": 16 * Ki, "experts": 16, "inner": 4096, "cols": 4096, "dtype": "bf16"},
        # One token of a decoding step through a whole layer.
        {"name": "layer_one_token", "op": "layer", "tokens": 1, "experts": 64, "top_k": 4, "cols": 2048, "inner": 1024, "dtype": "bf16"},
        # A few sequences that decode together, eight of 128 experts each.
        {"name": "layer_few", "op": "layer", "tokens": 8, "experts": 128, "top_k": 8, "cols": 4096, "inner": 1024, "dtype": "bf16"},
        # One rank's experts of a layer whose few tokens every rank has, in 16-bit floats with padding tokens.
        {"name": "layer_rank", "op": "layer", "tokens": 24, "experts": 64, "top_k": 4, "held": 16, "cols": 2048, "inner": 1408,
         "dtype": "fp16", "masked": 0.1},
        # Odd sizes in 32 bits, scores by sigmoids.
        {"name": "layer_odd", "op": "layer", "tokens": 5, "experts": 60, "top_k": 2, "cols": 1003, "inner": 517, "dtype": "fp32",
         "score": "sigmoid", "scale": 2.5, "pad": 1},
        # A decoding batch that reaches most of the experts.
        {"name": "layer_batch", "op": "layer", "tokens": 32, "experts": 64, "top_k": 4, "cols": 4096, "inner": 2048, "dtype": "bf16"},
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm; half of them odd, half multiples of 64."""
    v = int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))
    if rng.random() < 0.5:
        return min(max(lo, v | 1), hi)
    v = max(64, v // 64 * 64)
    return max(lo, v) if v <= hi else hi


def draw(rng):
    op = rng.choice(["rows", "product", "product", "layer", "layer"])
    c = {"op": op, "dtype": rng.choice(["bf16", "bf16", "fp16", "fp32"])}
    if op == "rows":
        if rng.random() < 0.6:
            c["experts"] = rng.choice([8, 16, 60, 64, 128, 256])
            c["top_k"] = rng.choice([1, 2, 4, 6, 8])
            c["masked"] = rng.choice([0.0, 0.0, 0.1])
        c["cols"] = _spread(rng, 32, 8192)
        c["rows"] = _spread(rng, 1, min(32 * Ki, 128 * Mi // c["cols"] // max(1, c.get("top_k", 0))))
        c["pad"] = rng.choice([0, 0, 0, 8, 3])
        return c
    if op == "product":
        c["dtype"] = rng.choice(["bf16", "bf16", "fp16", "fp32"])
        c["experts"] = rng.choice([1, 1, 4, 16, 40, 64, 128])
        c["inner"] = _spread(rng, 32, 8192)
        c["cols"] = _spread(rng, 16, min(8192, 512 * Mi // c["inner"] // c["experts"]))
        c["rows"] = _spread(rng, 1, min(16 * Ki, 16 * Ki * 4096 * 4096 // c["inner"] // c["cols"]))
        if rng.random() < 0.3:
            c["top_k"] = rng.choice([k for k in (1, 2, 4, 8) if k <= c["experts"]])
            c["rows"] = max(c["top_k"], c["rows"] // c["top_k"] * c["top_k"])
        else:
            c["gated"] = rng.random() < 0.3 and c["dtype"] != "fp32"
        c["pad"] = rng.choice([0, 0, 0, 16])
        return c
    c["tokens"] = _spread(rng, 1, 32)
    c["experts"] = rng.choice([8, 16, 60, 64, 96, 128])
    c["top_k"] = rng.choice([1, 2, 4, 6, 8])
    c["held"] = rng.choice([0, 0, c["experts"] // 4])
    c["cols"] = _spread(rng, 64, 4096)
    c["inner"] = _spread(rng, 32, min(4096, 512 * Mi // c["cols"] // c["experts"]))
    c["score"] = rng.choice(["softmax", "softmax", "sigmoid"])
    c["renormalize"] = rng.random() < 0.7
    c["scale"] = rng.choice([1.0, 1.0, 2.5])
    c["masked"] = rng.choice([0.0, 0.0, 0.1])
    c["pad"] = rng.choice([0, 0, 3])
    return c


def _full(case):
    return {**DEFAULTS[case["op"]], **case}


def _generator(seed):
    g = torch.Generator(device=DEVICE)
    g.manual_seed(seed * 1000003 + 29)
    return g


def _normal(g, rows, cols, dtype, pad=0, std=1.0):
    """Rows of normal values, `pad` elements apart."""
    x = torch.randn((rows, cols + pad), generator=g, device=DEVICE, dtype=torch.float32)
    return x.mul_(std).to(TYPES[dtype])[:, :cols]


def _room(rows, cols, dtype, pad=0):
    """A zeroed output of the same layout."""
    return torch.zeros((rows, cols + pad), device=DEVICE, dtype=TYPES[dtype])[:, :cols]


def _blocks(cols):
    return (cols + BLOCK - 1) // BLOCK


# ---- the format, in plain operations -------------------------------------------------------------

def _plain_scales(v):
    """Rows (R, C) in 32 bits to blocks (R, C / 32, 32), zeros behind the last column, and their exponents s."""
    R, C = v.shape
    b = torch.nn.functional.pad(v, (0, _blocks(C) * BLOCK - C)).view(R, _blocks(C), BLOCK)
    part, power = torch.frexp(b.abs().amax(2))  # part in [0.5, 1)
    s = torch.where(part < 0.875, power - 3, power - 2)
    return b, torch.where(part > 0, s, torch.full_like(s, -127)).clamp_(min=-127)


def _plain_round(q):
    """Magnitudes below 7 to the nearest of 0, 0.5, 1, 1.5, 2, 3, 4, 6, ties to the even code (steps of 1/2, 1 and 2
    by powers of two: a tie's even neighbour is the even multiple of the step)."""
    step = torch.where(q < 2, 0.5, torch.where(q < 4, 1.0, 2.0))
    return torch.round(q / step) * step


def _plain_values(v):
    """What rows in 32 bits become when they are held in 4 bits."""
    b, s = _plain_scales(v)
    s = s[..., None]
    # (in two steps of the exponent, each a normal number)
    q = _plain_round(torch.ldexp(torch.ldexp(b.abs(), -(s // 2)), s // 2 - s))
    out = torch.ldexp(torch.ldexp(q, s // 2), s - s // 2) * torch.sign(b)
    return out.view(v.shape[0], -1)[:, :v.shape[1]]


def _pack(v):
    """Rows in 32 bits to packed codes and scale bytes, as a program keeps its weights."""
    b, s = _plain_scales(v)
    q = _plain_round(torch.ldexp(b.abs(), -s[..., None]))
    code = torch.where(q < 2, q * 2, torch.where(q < 4, q + 2, q / 2 + 4)).to(torch.uint8) + 8 * (b < 0).to(torch.uint8)
    code = code.view(v.shape[0], -1)[:, :(v.shape[1] + 1) // 2 * 2]
    return code[:, 0::2] + 16 * code[:, 1::2], (s + 127).to(torch.uint8)


_VALUES = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def _unpack(codes, scale, cols, dtype=torch.float32):
    """Packed codes (..., C / 2) and scale bytes (..., C / 32) to the values that they stand for."""
    table = torch.tensor(_VALUES + tuple(-v for v in _VALUES), device=DEVICE, dtype=dtype)
    pairs = torch.stack([table.repeat(16), table.repeat_interleave(16)], 1)  # a byte's two values
    v = pairs[codes.int()].flatten(-2)
    v = torch.nn.functional.pad(v, (0, _blocks(cols) * BLOCK - v.shape[-1])).view(*v.shape[:-1], -1, BLOCK)
    v = v * torch.exp2(scale.to(dtype) - 127)[..., None]
    return v.flatten(-2)[..., :cols]


def _weights(g, E, N, D):
    """Packed weights of E experts, N rows of D each, about 1 / sqrt(D) in size."""
    codes = torch.empty((E, N, (D + 1) // 2), device=DEVICE, dtype=torch.uint8)
    scale = torch.empty((E, N, _blocks(D)), device=DEVICE, dtype=torch.uint8)
    for e in range(E):
        codes[e], scale[e] = _pack(torch.randn((N, D), generator=g, device=DEVICE).mul_(1.0 / math.sqrt(D)))
    return codes, scale


def _value4(v):
    """The same 4-bit floats in 64 bits, by thresholds: between neighbours, the one nearer; at a tie the even one."""
    R, C = v.shape
    b = torch.zeros((R, _blocks(C) * BLOCK), device=DEVICE, dtype=torch.float64)
    b[:, :C] = v
    b = b.view(R, -1, BLOCK)
    m = b.abs().amax(2, keepdim=True)
    s = torch.floor(torch.log2(torch.where(m > 0, m, torch.ones_like(m)) / 7.0)) + 1.0
    s = torch.where(m >= 7.0 * 2.0 ** s, s + 1, torch.where(m < 7.0 * 2.0 ** (s - 1), s - 1, s)).clamp(min=-127)
    q = b.abs() * 2.0 ** -s
    out = torch.zeros_like(q)
    for border, above, value in ((0.25, True, 0.5), (0.75, False, 1.0), (1.25, True, 1.5), (1.75, False, 2.0),
                                 (2.5, True, 3.0), (3.5, False, 4.0), (5.0, True, 6.0)):
        out = torch.where(q > border if above else q >= border, torch.full_like(out, value), out)
    return (out * 2.0 ** s * torch.sign(b)).view(R, -1)[:, :C]


# ---- rows ----------------------------------------------------------------------------------------

def _routes(T, E, K, g, masked=0.0):
    """The row of every route (T, K) in the experts' order, -1 for padding tokens, and the experts' first rows. Tokens
    have distinct experts, some sought more than others."""
    liking = torch.randn((T, E), generator=g, device=DEVICE) + torch.randn(E, generator=g, device=DEVICE).mul_(0.5)
    expert = liking.topk(K, 1).indices
    kept = T - int(T * masked)
    expert[kept:] = E
    order = expert.flatten().sort(stable=True).indices
    row = torch.empty_like(order)
    row[order] = torch.arange(T * K, device=DEVICE)
    row = torch.where(expert < E, row.view(T, K), torch.full_like(expert, -1)).to(torch.int32)
    counts = torch.bincount(expert.flatten(), minlength=E + 1)[:E]
    return row, torch.cat([counts.new_zeros(1), counts.cumsum(0)])


def _rows_inputs(c, seed):
    g = _generator(seed)
    x = _normal(g, c["rows"], c["cols"], c["dtype"], c["pad"])
    row = _routes(c["rows"], c["experts"], c["top_k"], g, c["masked"])[0] if c["top_k"] else None
    return x, row


def _prepare_rows(c, seed):
    x, row = _rows_inputs(c, seed)
    state = {"case": c, "x": x, "row": row}
    if own:
        import paper_2608_00358_amd as hccl

        R, C = c["rows"] * max(1, c["top_k"]), c["cols"]
        comm = hccl.Comm(1, 0)
        codes = torch.zeros((R, (C + 1) // 2), device=DEVICE, dtype=torch.uint8)
        scale = torch.zeros((R, _blocks(C)), device=DEVICE, dtype=torch.uint8)
        out = _room(R, C, c["dtype"], c["pad"])
        first = comm.bind_moe_dispatch_mx(x, row, codes, scale) if row is not None else comm.bind_moe_quantize_mx(x, codes, scale)
        state.update(comm=comm, calls=[first, comm.bind_moe_dequantize_mx(codes, scale, out)], out=[out], keep=(codes, scale))
    return state


def _into_order(v, row):
    """Rows (T, C) to the rows that `row` (T, K) names; the others are zero."""
    T, K = row.shape
    flat = row.flatten().long()
    out = v.new_zeros((T * K + 1, v.shape[1]))  # (its last row takes what has none)
    out[torch.where(flat >= 0, flat, torch.full_like(flat, T * K))] = v[torch.arange(T * K, device=DEVICE) // K]
    return out[:T * K]


def _run_rows(state):
    out = _plain_values(state["x"].float()).to(state["x"].dtype)
    return [out if state["row"] is None else _into_order(out, state["row"])]


def _exact_rows(c, seed):
    x, row = _rows_inputs(c, seed)
    out = _value4(x.double())
    return [out if row is None else _into_order(out, row)]


# ---- product -------------------------------------------------------------------------------------

def _product_inputs(c, seed):
    g = _generator(seed)
    R, E, D, K = c["rows"], c["experts"], c["inner"], c["top_k"]
    w, ws = _weights(g, E, c["cols"], D)
    if K:  # rows come from tokens, each of which goes to K experts
        row, offsets = _routes(R // K, E, K, g)
        x = _normal(g, R // K, D, c["dtype"], c["pad"])
    else:
        row = None
        p = torch.rand(E, generator=g, device=DEVICE).cpu().double().numpy() + 0.2
        sizes = np.random.default_rng(seed).multinomial(R, p / p.sum())
        offsets = torch.from_numpy(np.concatenate([[0], np.cumsum(sizes)]).astype(np.int64)).to(DEVICE)
        x = _normal(g, R, 2 * D if c["gated"] else D, c["dtype"], c["pad"])
    return x, row, offsets, w, ws


def _prepare_product(c, seed):
    x, row, offsets, w, ws = _product_inputs(c, seed)
    state = {"case": c, "x": x, "row": row, "ends": offsets.tolist(), "w": w, "ws": ws}
    if own:
        import paper_2608_00358_amd as hccl

        R, D = c["rows"], c["inner"]
        comm = hccl.Comm(1, 0)
        codes = torch.empty((R, (D + 31) // 32 * 16), device=DEVICE, dtype=torch.uint8)[:, :(D + 1) // 2]
        scale = torch.empty((R, _blocks(D)), device=DEVICE, dtype=torch.uint8)
        out = _room(R, c["cols"], c["dtype"], c["pad"])
        if row is not None:
            first = comm.bind_moe_dispatch_mx(x, row, codes, scale)
        else:
            first = comm.bind_moe_quantize_mx(x, codes, scale, gated=c["gated"])
        calls = [first, comm.bind_moe_product_mx(codes, scale, w, ws, out, D, offsets=offsets if c["experts"] > 1 else None)]
        state.update(comm=comm, calls=calls, out=[out], keep=(codes, scale, offsets))
    return state


def _run_product(state):
    c, row = state["case"], state["row"]
    D = c["inner"]
    x = state["x"].float()
    if c["gated"]:
        x = x[:, :D] * (1.0 / (1.0 + torch.exp(-x[:, :D]))) * x[:, D:]
    x = _plain_values(x)
    if row is not None:
        x = _into_order(x, row)
    out = torch.empty((c["rows"], c["cols"]), device=DEVICE, dtype=state["x"].dtype)
    for e in range(c["experts"]):
        a, b = state["ends"][e], state["ends"][e + 1]
        if b > a:
            out[a:b] = (x[a:b] @ _unpack(state["w"][e], state["ws"][e], D).t()).to(out.dtype)
    return [out]


def _exact_product(c, seed):
    x, row, offsets, w, ws = _product_inputs(c, seed)
    D = c["inner"]
    x = x.double()
    if c["gated"]:
        x = x[:, :D] * torch.sigmoid(x[:, :D]) * x[:, D:]
    x = _value4(x)
    if row is not None:
        x = _into_order(x, row)
    out = torch.zeros((c["rows"], c["cols"]), device=DEVICE, dtype=torch.float64)
    ends = offsets.tolist()
    for e in range(c["experts"]):
        a, b = ends[e], ends[e + 1]
        if b > a:
            out[a:b] = torch.mm(x[a:b], _unpack(w[e], ws[e], D, torch.float64).t().contiguous())
    return [out]


# ---- layer ---------------------------------------------------------------------------------------

def _layer_inputs(c, seed):
    g = _generator(seed)
    T, E, C, F = c["tokens"], c["experts"], c["cols"], c["inner"]
    held = c["held"] or E
    first = (seed % (E // held)) * held if held < E else 0  # one rank's experts
    logits = _normal(g, T, E, c["dtype"], 0, 1.5)
    x = _normal(g, T, C, c["dtype"], c["pad"])
    w_in, w_out = _weights(g, held, 2 * F, C), _weights(g, held, C, F)
    mask = None
    if c["masked"]:
        mask = (torch.arange(T, device=DEVICE) < T - max(1, int(T * c["masked"]))).to(torch.uint8)
    return logits, mask, x, w_in, w_out, first, held


def _prepare_layer(c, seed):
    logits, mask, x, w_in, w_out, first, held = _layer_inputs(c, seed)
    state = {"case": c, "logits": logits, "mask": mask, "x": x, "w_in": w_in, "w_out": w_out, "first": first, "held": held}
    if own:
        import paper_2608_00358_amd as hccl

        T, K = c["tokens"], c["top_k"]
        comm = hccl.Comm(1, 0)
        router = hccl.hccl_router_init(experts=c["experts"], top_k=K, score=c["score"], renormalize=c["renormalize"], scale=c["scale"])
        index = torch.empty((T, K), device=DEVICE, dtype=torch.int32)
        weight = torch.empty((T, K), device=DEVICE, dtype=torch.float32)
        out = _room(T, c["cols"], c["dtype"], c["pad"])
        space = torch.empty(hccl.hccl_moe_layer_mx_bytes(T, K, c["cols"], c["inner"], held), device=DEVICE, dtype=torch.uint8)
        call = comm.bind_moe_layer_mx(router, logits, x, *w_in, *w_out, index, weight, out, mask=mask, first=first, workspace=space)
        state.update(comm=comm, calls=[call], out=[index, weight, out], keep=space)
    return state


def _run_layer(state):
    c, x = state["case"], state["x"]
    T, C, F = c["tokens"], c["cols"], c["inner"]
    l = state["logits"].float()
    p = torch.exp(l - l.amax(1, keepdim=True))
    p = p / p.sum(1, keepdim=True) if c["score"] == "softmax" else 1.0 / (1.0 + torch.exp(-l))
    index = l.sort(dim=1, descending=True, stable=True).indices[:, :c["top_k"]]
    weight = p.gather(1, index)
    if c["renormalize"]:
        weight = weight / weight.sum(1, keepdim=True)
    weight = weight * c["scale"]
    if state["mask"] is not None:
        on = (state["mask"] != 0)[:, None]
        index, weight = torch.where(on, index, torch.full_like(index, -1)), torch.where(on, weight, torch.zeros_like(weight))
    y = torch.zeros((T, C), device=DEVICE)
    for k in range(c["top_k"]):
        e = index[:, k] - state["first"]
        here = (index[:, k] >= 0) & (e >= 0) & (e < state["held"])
        e = torch.where(here, e, torch.zeros_like(e))
        h = torch.bmm(_unpack(state["w_in"][0][e], state["w_in"][1][e], C), x.float()[:, :, None])[:, :, 0]
        gate, up = h[:, :F], h[:, F:]
        h = gate * (1.0 / (1.0 + torch.exp(-gate))) * up
        z = torch.bmm(_unpack(state["w_out"][0][e], state["w_out"][1][e], F), h[:, :, None])[:, :, 0]
        y += torch.where(here, weight[:, k], torch.zeros_like(weight[:, k]))[:, None] * z
    return [index.to(torch.int32), weight, y.to(x.dtype)]


def _exact_layer(c, seed):
    logits, mask, x, w_in, w_out, first, held = _layer_inputs(c, seed)
    T, C, F, K = c["tokens"], c["cols"], c["inner"], c["top_k"]
    l = logits.double().cpu().numpy()
    s = 1.0 / (1.0 + np.exp(-l)) if c["score"] == "sigmoid" else np.exp(l - l.max(1, keepdims=True))
    if c["score"] == "softmax":
        s /= s.sum(1, keepdims=True)
    index = np.argsort(-l, axis=1, kind="stable")[:, :K].astype(np.int32)
    weight = np.take_along_axis(s, index, 1)
    if c["renormalize"]:
        weight /= weight.sum(1, keepdims=True)
    weight *= c["scale"]
    if mask is not None:
        off = mask.cpu().numpy() == 0
        index[off], weight[off] = -1, 0.0
    y = torch.zeros((T, C), device=DEVICE, dtype=torch.float64)
    rows = x.double()
    for e in range(held):  # expert by expert, the tokens that chose it
        t, k = np.nonzero(index == first + e)
        if not t.size:
            continue
        a = torch.mm(rows[t], _unpack(w_in[0][e], w_in[1][e], C, torch.float64).t().contiguous())
        h = torch.nn.functional.silu(a[:, :F]) * a[:, F:]
        z = torch.mm(h, _unpack(w_out[0][e], w_out[1][e], F, torch.float64).t().contiguous())
        y[t] += torch.from_numpy(weight[t, k]).to(DEVICE)[:, None] * z
    return [torch.from_numpy(index).to(DEVICE), torch.from_numpy(weight).to(DEVICE), y]


# ---- the cases' interface ------------------------------------------------------------------------

def prepare(case, seed):
    c = _full(case)
    return {"rows": _prepare_rows, "product": _prepare_product, "layer": _prepare_layer}[c["op"]](c, seed)


def run(state):
    if own:
        for call in state["calls"]:
            call()
        return state["out"]
    return {"rows": _run_rows, "product": _run_product, "layer": _run_layer}[state["case"]["op"]](state)


def exact(case, seed):
    c = _full(case)
    return {"rows": _exact_rows, "product": _exact_product, "layer": _exact_layer}[c["op"]](c, seed)


def _bytes4(cols):
    """A row of 4-bit floats with its scales."""
    return (cols + 1) // 2 + _blocks(cols)


def work(case):
    c = _full(case)
    size = SIZE[c["dtype"]]
    if c["op"] == "rows":
        T, K, C = c["rows"], c["top_k"], c["cols"]
        kept = T - int(T * c["masked"]) if K else T
        rows = kept * K if K else T  # written in 4 bits, read again, written in the rows' type
        return {"bytes": kept * C * size + T * K * 4 + 2 * rows * _bytes4(C) + T * max(1, K) * C * size, "flops": 0}
    if c["op"] == "product":
        R, E, N, D, K = c["rows"], c["experts"], c["cols"], c["inner"], c["top_k"]
        seen = E * (1.0 - (1.0 - 1.0 / E) ** R)  # experts that have a row: only their weights are read
        read = (R // K if K else R) * D * (2 if c["gated"] else 1) * size + seen * N * _bytes4(D)
        return {"bytes": int(read + R * N * size + (4 * R if K else 0)), "flops": 2 * R * N * D}
    T, E, K, C, F = c["tokens"], c["experts"], c["top_k"], c["cols"], c["inner"]
    kept = T - (max(1, int(T * c["masked"])) if c["masked"] else 0)
    held = c["held"] or E
    seen = held * (1.0 - (1.0 - K / E) ** kept)
    moved = T * (E + 2 * C) * size + T * K * 8 + seen * (2 * F * _bytes4(C) + C * _bytes4(F))
    return {"bytes": int(moved), "flops": int(6 * kept * K * held / E * C * F)}
