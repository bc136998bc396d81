"""Routing and 4-bit experts, as cases to be timed.

Five kinds of call, each in a plain form of elementary torch operations (in 32
bits, rounded once; the choice of experts in 64) and, with `own` set, through
the package's entry points:

* "route"       Router.forward: router logits to expert ids and gates;
* "route-grad"  llep_route_backward: the gates' gradients to the logits';
* "rows"        llep_quantize_rows_mxfp4 and llep_dequantize_rows_mxfp4: rows to
                4-bit floating point (e2m1) with a power of two for every 32
                values, and the values that they stand for;
* "product"     llep_quantize_rows_mxfp4 and llep_mxfp4_matmul: activations to
                such rows, times 4-bit weights;
* "experts"     LLEPLayer.forward_mxfp4: the expert layer with 4-bit weights,
                from token activations to layer outputs.

Sizes are those of the layer configurations in synth.py (hidden and FFN sizes,
experts, top-k, routing skew) with token counts from one to a training batch;
drawn cases also take generic and odd sizes.
"""

from __future__ import annotations

import math

import torch

own = False

# hidden size, FFN size, experts, experts per token
SHAPES = {
    "gpt-oss-20b": (2880, 2880, 32, 4),
    "qwen3-30b-a3b": (2048, 768, 128, 8),
}
INF = math.inf


def _route(T, E, K, dtype, score, renorm=True, bias=False, groups=1, top=1, by="max", masked=0.0,
           scale=1.0):
    """masked: share of the logits, and of whole rows (padding), that are -inf."""
    return {"op": "route", "T": T, "E": E, "K": K, "dtype": dtype, "score": score,
            "renorm": renorm, "bias": bias, "groups": groups, "top": top, "by": by,
            "masked": masked, "scale": scale}


def _route_grad(*args, **kw):
    return {**_route(*args, **kw), "op": "route-grad"}


def _rows(R, D, dtype):
    return {"op": "rows", "R": R, "D": D, "dtype": dtype}


def _product(M, N, K, dtype="bf16"):
    return {"op": "product", "M": M, "N": N, "K": K, "dtype": dtype}


def _experts(T, shape, hot, n_hot, P=8):
    """hot: share of the token-expert pairs on the first n_hot experts, the rest uniform."""
    D, F, E, K = SHAPES[shape] if isinstance(shape, str) else shape
    return {"op": "experts", "T": T, "D": D, "F": F, "E": E, "K": K, "P": P, "hot": hot,
            "n_hot": n_hot}


def listed():
    cases = {
        # one decoded token: scores by sigmoid, a bias for balance, 4 of 8 groups; latency
        "route-token": _route(1, 256, 8, "f32", "sigmoid", bias=True, groups=8, top=4, by="top2",
                              scale=2.5),
        # a training batch, softmax over the chosen experts
        "route-batch": _route(65536, 128, 8, "bf16", "softmax"),
        # the batch that goes with the first one: the groups and the bias for every token
        "route-groups": _route(8192, 256, 8, "f32", "sigmoid", bias=True, groups=8, top=4,
                               by="top2", scale=2.5),
        # the gradient of a training batch, scores over all experts
        "route-grad-batch": _route_grad(32768, 128, 4, "f32", "softmax", renorm=False),
        # of a ragged one of an odd number of experts, padded rows and masked experts among them
        "route-grad-ragged": _route_grad(1777, 37, 2, "bf16", "sigmoid", masked=0.1),
        # an expert layer's gate weights into 4 bits, and back into what a bf16 program reads
        "rows-weights": _rows(92160, 2880, "bf16"),
        # a ragged batch's activations, rows of odd length
        "rows-odd": _rows(333, 1003, "f32"),
        # one decoded token through a projection: latency, and the weights once
        "product-token": _product(1, 7168, 2048),
        # a prompt batch through a projection
        "product-batch": _product(8192, 7168, 2048),
        # decode: a few tokens, most of the experts in use
        "experts-decode": _experts(8, "gpt-oss-20b", 0.5, 4),
        # a ragged prompt over many small experts
        "experts-ragged": _experts(1531, "qwen3-30b-a3b", 0.6, 16),
        # a prompt batch with hot experts
        "experts-prompt": _experts(8192, "gpt-oss-20b", 0.6, 4),
    }
    return [{**c, "name": n} for n, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["route", "route-grad", "rows", "product", "experts"])
    if op in ("route", "route-grad"):
        E = rng.choice([8, 16, 32, 64, 128, 160, 256, 512, _log(rng, 3, 500)])
        K = min(E, rng.choice([1, 2, 4, 6, 8]))
        groups, top, by = 1, 1, "max"
        if E % 8 == 0 and E >= 32 and rng.random() < 0.5:
            groups, top, by = rng.choice([(4, 2), (8, 4), (8, 3)]) + (rng.choice(["max", "top2"]),)
            K = min(K, top * (E // groups))
        make = _route if op == "route" else _route_grad
        most = (65536 * 128 if op == "route" else 32768 * 128) // E
        return make(_log(rng, 1, most), E, K, rng.choice(["bf16", "f32"]),
                    rng.choice(["softmax", "sigmoid"]), rng.random() < 0.6, rng.random() < 0.5,
                    groups, top, by, rng.choice([0.0, 0.0, 0.1, 0.4]), rng.choice([1.0, 2.5]))
    if op == "rows":
        D = rng.choice([64, 768, 1024, 2048, 2880, 4096, 7168, _log(rng, 60, 8000)])
        return _rows(_log(rng, 1, 92160 * 2880 // D), D, rng.choice(["bf16", "bf16", "f32"]))
    if op == "product":
        N, K = (rng.choice([768, 1024, 2048, 2880, 4096, _log(rng, 64, 7000)]) for _ in "NK")
        M = _log(rng, 1, min(16384, 8192 * 7168 * 2048 // (N * K)))
        return _product(M, N, K, rng.choice(["bf16", "bf16", "f32"]))
    E = rng.choice([8, 16, 32, 64, 128])
    K = rng.choice([1, 2, 4, 8])
    D, F = (64 * rng.choice([4, 8, 12, 16, 23, 32, 45]) for _ in "DF")
    most = min(32768 // K, 8192 * 4 * 2880 * 2880 // (K * D * F))
    return _experts(_log(rng, 1, most), (D, F, E, K), rng.choice([0.0, 0.5, 0.9]),
                    rng.choice([1, 4]), rng.choice([1, 4, 8]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _randn(g, *shape, dtype=torch.float32, scale=1.0):
    x = torch.randn(shape, generator=g, device="cuda")
    return (x * scale if scale != 1.0 else x).to(dtype)


def _activations(g, R, D, dtype):
    """Rows whose channels differ in size, as hidden states' do."""
    channel = torch.exp(_randn(g, D, scale=0.5))
    return (torch.randn((R, D), generator=g, device="cuda") * channel).to(dtype)


def _weights4(g, *shape):
    """4-bit weights, rows = output channels: two values a byte (the first in the low half), and
    for every 32 of them the exponent of a power of two, plus 127."""
    *rows, K = shape
    q = torch.randint(0, 256, (*rows, (K + 1) // 2), generator=g, device="cuda", dtype=torch.uint8)
    s = torch.randint(118, 122, (*rows, (K + 31) // 32), generator=g, device="cuda",
                      dtype=torch.uint8)
    return q, s


def _inputs(case, seed):
    """The case's data: the same for either form and for the definition in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], _dtype(case)
    s = {}
    if op in ("route", "route-grad"):
        T, E, K = (case[k] for k in "TEK")
        logits = _randn(g, T, E, scale=1.5)
        if case["masked"]:
            off = torch.rand((T, E), generator=g, device="cuda") < case["masked"]
            off |= torch.rand((T, 1), generator=g, device="cuda") < case["masked"]
            logits = torch.where(off, -INF, logits)
        s["logits"] = logits.to(dt)
        s["bias"] = _randn(g, E, scale=0.1) if case["bias"] else None
        if op == "route-grad":
            s["d_gates"] = _randn(g, T, K, scale=0.1)
            s["ids"], s["gates"] = _plain_route({**s, "case": case}).values()
    elif op == "rows":
        s["x"] = _activations(g, case["R"], case["D"], dt)
    elif op == "product":
        s["x"] = _activations(g, case["M"], case["K"], dt)
        s["w"] = _weights4(g, case["N"], case["K"])
    else:
        T, D, F, E, K = (case[k] for k in "TDFEK")
        s["x"] = _activations(g, T, D, dt)
        hot = torch.rand((T, K), generator=g, device="cuda") < case["hot"]
        some = torch.randint(0, min(case["n_hot"], E), (T, K), generator=g, device="cuda")
        rest = torch.randint(0, E, (T, K), generator=g, device="cuda")
        s["ids"] = torch.where(hot, some, rest).to(torch.int32)
        s["gates"] = torch.softmax(_randn(g, T, K), dim=-1)
        s["w"] = [_weights4(g, E, *nk) for nk in ((F, D), (F, D), (D, F))]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["op"], s["case"] = case["op"], case
    if case["op"] == "experts":
        # rows per expert on the host, which an eager program needs to split its rows
        s["counts"] = torch.bincount(s["ids"].flatten().long(), minlength=case["E"]).tolist()
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    """What a program on the framework keeps: outputs, packed weights, the router, the layer."""
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import LLEPLayer, Mxfp4Experts, Router
    op, cuda = case["op"], dict(device="cuda")
    if op in ("route", "route-grad"):
        T, E, K = (case[k] for k in "TEK")
        how = dict(score=case["score"], groups=case["groups"], top_groups=case["top"],
                   group_score=case["by"], renormalize=case["renorm"], scale=case["scale"])
        if op == "route":
            s["router"] = Router(T, K, E, bias=s["bias"], **how)
        else:
            s["params"] = B.make_route(T, K, E, **how)
            s["d_logits"] = torch.empty_like(s["logits"])
    elif op in ("rows", "product"):
        R, D = s["x"].shape
        s["q"] = torch.empty((R, B.llep_mxfp4_row_bytes(D)), dtype=torch.uint8, **cuda)
        s["scale"] = torch.empty((R, B.llep_mxfp4_scale_bytes(D)), dtype=torch.uint8, **cuda)
        if op == "rows":
            s["values"] = torch.empty_like(s["x"])
        else:
            s["packed"] = B.llep_pack_matrix_mxfp4(*s["w"], K=D)
            s["y"] = torch.empty((R, case["N"]), dtype=_dtype(case), **cuda)
    else:
        T, D, F, E, K, P = (case[k] for k in "TDFEKP")
        s["layer"] = LLEPLayer(T, K, E, P, D, F, math.ceil(1.1 * T * K / P), torch.bfloat16)
        s["experts"] = Mxfp4Experts(*[t for qs in s["w"] for t in qs])


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return {"route": _plain_route, "route-grad": _plain_route_grad, "rows": _plain_rows,
            "product": _plain_product, "experts": _plain_experts}[s["op"]](s)


def _run_own(s):
    from paper_2601_17111_amd import binding as B
    op = s["op"]
    if op == "route":
        ids, gates = s["router"].forward(s["logits"])
        return {"ids": ids, "gates": gates}
    if op == "route-grad":
        B.llep_route_backward(s["params"], s["logits"], s["ids"], s["gates"], s["d_gates"],
                              s["d_logits"])
        return s["d_logits"]
    if op == "rows":
        B.llep_quantize_rows_mxfp4(s["x"], s["q"], s["scale"])
        B.llep_dequantize_rows_mxfp4(s["q"], s["scale"], s["values"])
        return s["values"]
    if op == "product":
        B.llep_quantize_rows_mxfp4(s["x"], s["q"], s["scale"])
        B.llep_mxfp4_matmul(s["q"], s["scale"], s["packed"], s["y"], s["case"]["K"])
        return s["y"]
    return s["layer"].forward_mxfp4(s["ids"], s["gates"], s["x"], s["experts"])


def _scores(logits, kind):
    """Scores in the logits' precision; rows with nothing but -inf: zeros."""
    if kind == "sigmoid":
        return torch.sigmoid(logits)
    most = logits.amax(-1, keepdim=True)
    e = torch.exp(logits - torch.where(most == -INF, 0.0, most))
    total = e.sum(-1, keepdim=True)
    return e / torch.where(total > 0, total, 1.0)


def _best(key, n):
    """The n largest of each row, ties to the lowest index: their indices and values."""
    key, index = torch.sort(key, dim=-1, descending=True, stable=True)
    return index[..., :n], key[..., :n]


def _plain_route(s):
    c, logits, bias = s["case"], s["logits"], s["bias"]
    T, E, K, G = c["T"], c["E"], c["K"], c["groups"]
    # which experts: in 64 bits, as neighbouring keys may be closer than 32 tell apart
    key = logits.double()
    if bias is not None or (G > 1 and c["by"] == "top2"):
        key = _scores(key, c["score"])
        if bias is not None:
            key = key + bias.double()
    key = torch.where(logits == -INF, -INF, key)
    if G > 1:
        of_group = key.view(T, G, E // G)
        if c["by"] == "max":
            group = of_group.amax(-1)
        else:
            two = _best(of_group, 2)[1]
            group = two[..., 0] + torch.where(two[..., 1] == -INF, 0.0, two[..., 1])
        taken = torch.zeros_like(group, dtype=torch.bool).scatter_(1, _best(group, c["top"])[0], True)
        key = torch.where(taken.repeat_interleave(E // G, 1), key, -INF)
    index, key = _best(key, K)
    found = key > -INF
    if c["renorm"] and c["score"] == "softmax":
        gates = _scores(torch.where(found, logits.float().gather(1, index), -INF), "softmax")
    else:
        gates = torch.where(found, _scores(logits.float(), c["score"]).gather(1, index), 0.0)
        if c["renorm"]:
            total = gates.sum(-1, keepdim=True)
            gates = gates / torch.where(total > 0, total, 1.0)
    return {"ids": torch.where(found, index, -1).to(torch.int32), "gates": gates * c["scale"]}


def _plain_route_grad(s):
    c, ids, gates, dg = s["case"], s["ids"].long(), s["gates"], s["d_gates"]
    found = ids >= 0
    at = torch.where(found, ids, 0)
    dg = torch.where(found, dg, 0.0)
    if c["renorm"]:
        dg = dg - (gates * dg).sum(-1, keepdim=True) / c["scale"]
    each = gates * dg
    logits = s["logits"].float()
    if c["score"] == "sigmoid":
        each = each * torch.sigmoid(-logits.gather(1, at))
    out = torch.zeros_like(logits).scatter_add_(1, at, torch.where(found, each, 0.0))
    if c["score"] == "softmax" and not c["renorm"]:
        out = out - _scores(logits, "softmax") * each.sum(-1, keepdim=True)
    return out.to(s["logits"].dtype)


def _plain_quantize(x):
    """x [R, D] in 32 bits: the values on the 4-bit grid, times their blocks' powers of two."""
    R, D = x.shape
    x = torch.nn.functional.pad(x, (0, -D % 32)).view(R, -1, 32)
    # floor(log2(largest)) - 2 (frexp: a fraction in [1/2, 1))
    power = torch.frexp(x.abs().amax(-1, keepdim=True))[1] - 3
    step = torch.exp2(power.clamp(min=-126).float())
    y = (x / step).abs()
    y = torch.where(y < 2, torch.round(y * 2) / 2,
                    torch.where(y < 4, torch.round(y), torch.round(y / 2) * 2)).clamp(max=6)
    return (torch.copysign(y, x) * step).view(R, -1)[:, :D]


def _plain_weights(q, s, K):
    """What 4-bit weights stand for, in 32 bits."""
    table = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6], device=q.device)
    codes = torch.stack((q & 15, q >> 4), -1).view(*q.shape[:-1], -1)[..., :K].int()
    size = table[codes & 7]
    values = torch.where(codes > 7, -size, size)
    steps = torch.exp2(s.float() - 127)
    return values * steps.repeat_interleave(32, -1)[..., :K]


def _plain_rows(s):
    return _plain_quantize(s["x"].float()).to(s["x"].dtype)


def _plain_product(s):
    w = _plain_weights(*s["w"], s["case"]["K"])
    return (_plain_quantize(s["x"].float()) @ w.t()).to(s["x"].dtype)


def _plain_experts(s):
    T, K, D, F = (s["case"][k] for k in "TKDF")
    x = _plain_quantize(s["x"].float())
    order = torch.argsort(s["ids"].flatten(), stable=True)
    used = [e for e, n in enumerate(s["counts"]) if n]
    rows = []
    for e, a in zip(used, x[order // K].split([s["counts"][e] for e in used])):
        wg, wu, wd = (_plain_weights(q[e], z[e], n) for (q, z), n in zip(s["w"], (D, D, F)))
        gate = a @ wg.t()
        rows.append(_plain_quantize(gate * torch.sigmoid(gate) * (a @ wu.t())) @ wd.t())
    rows = torch.cat(rows)
    pairs = torch.empty_like(rows)
    pairs[order] = rows
    return (pairs.view(T, K, D) * s["gates"].unsqueeze(-1)).sum(1).to(s["x"].dtype)


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_choice(s):
    """The experts of every row, one after another."""
    c, l = s["case"], s["logits"].double()
    T, E, G = c["T"], c["E"], c["groups"]
    key = l.clone()
    if s["bias"] is not None or (G > 1 and c["by"] == "top2"):
        if c["score"] == "sigmoid":
            key = 1 / (1 + torch.exp(-l))
        else:
            key = torch.exp(l - torch.logsumexp(l, -1, keepdim=True))
        key = key + (0 if s["bias"] is None else s["bias"].double())
    key[l == -INF] = -INF

    def take(key):
        """The first of the largest, and the keys without it."""
        most = key.amax(-1, keepdim=True)
        place = torch.arange(key.shape[-1], device="cuda")
        first = torch.where(key == most, place, key.shape[-1]).amin(-1, keepdim=True)
        return first, most, key.scatter(-1, first, -INF)

    if G > 1:
        parts = key.view(T, G, E // G)
        _, total, rest = take(parts)
        if c["by"] == "top2":
            second = take(rest)[1]
            total = total + second.masked_fill(second == -INF, 0.0)
        total, out = total.squeeze(-1), torch.full_like(parts, -INF)
        for _ in range(c["top"]):
            first, most, total = take(total)
            at = first.unsqueeze(-1).expand(T, 1, E // G)
            out.scatter_(1, at, parts.gather(1, at))
            # (of used-up groups the first is named again: it stays as it is)
        key = out.view(T, E)
    ids = torch.empty((T, c["K"]), dtype=torch.int32, device="cuda")
    for k in range(c["K"]):
        first, most, key = take(key)
        ids[:, k] = torch.where(most == -INF, -1, first).squeeze(-1)
    return ids


def _exact_gates(s, ids):
    """The gates of these experts, from the definition: e^l over a sum of them, or 1 / (1 + e^-l)."""
    c = s["case"]
    l = s["logits"].double()
    chosen = torch.where(ids >= 0, l.gather(1, ids.clamp(min=0).long()), -INF)
    if c["score"] == "softmax":
        over = torch.logsumexp(chosen if c["renorm"] else l, -1, keepdim=True)
        gates = torch.exp(chosen - over)
        gates = torch.where(ids >= 0, gates, 0.0)
    else:
        gates = 1 / (1 + torch.exp(-chosen))
        if c["renorm"]:
            gates = gates / gates.sum(-1, keepdim=True).clamp(min=1e-300)
    return gates * c["scale"]


def _exact_route_grad(s):
    """Through the Jacobian of the gates of every row."""
    c, ids = s["case"], s["ids"]
    E = c["E"]
    l = s["logits"].double()
    hit = (ids.long().unsqueeze(-1) == torch.arange(E, device="cuda")).double()  # [T, K, E]
    g = _exact_gates(s, ids)
    dg = s["d_gates"].double()
    if c["score"] == "softmax":
        if c["renorm"]:
            over = (hit * (g / c["scale"]).unsqueeze(-1)).sum(1, keepdim=True)
        else:
            top = l.amax(-1, keepdim=True)
            over = torch.softmax(l - torch.where(top == -INF, 0.0, top), -1).nan_to_num(0.0)
            over = over.unsqueeze(1)
        jac = g.unsqueeze(-1) * (hit - over)
    else:
        slope = hit * (1 - 1 / (1 + torch.exp(-l))).unsqueeze(1)
        jac = g.unsqueeze(-1) * slope
        if c["renorm"]:
            jac = jac - (g / c["scale"]).unsqueeze(-1) * jac.sum(1, keepdim=True)
    return (dg.unsqueeze(-1) * jac).sum(1)


def _exact_rows(x):
    """The nearest value of the grid, the even one between two: by comparing with the borders."""
    R, D = x.shape
    out = torch.zeros((R, -(-D // 32) * 32), dtype=torch.float64, device="cuda")
    out[:, :D] = x
    block = out.view(R, -1, 32)
    most = block.abs().amax(-1, keepdim=True)
    power = torch.floor(torch.log2(torch.where(most > 0, most, 1.0)))
    # log2 rounds: put right where it fell on the wrong side of a whole number
    power = power - (torch.exp2(power) > most).double() + (torch.exp2(power + 1) <= most).double()
    step = torch.where(most > 0, torch.exp2(power - 2), 1.0)
    y = (block / step).abs()
    size = torch.zeros_like(y)
    for border, even, value in ((0.25, 0, 0.5), (0.75, 1, 1.0), (1.25, 0, 1.5), (1.75, 1, 2.0),
                                (2.5, 0, 3.0), (3.5, 1, 4.0), (5.0, 0, 6.0)):
        size = torch.where((y >= border) if even else (y > border), value, size)
    return (torch.sign(block) * size * step).view(R, -1)[:, :D]


def _exact_weights(q, s, K):
    grid = [0, 0.5, 1, 1.5, 2, 3, 4, 6]
    table = torch.tensor(grid + [-v for v in grid], dtype=torch.float64, device="cuda")
    w = torch.empty((q.shape[0], 2 * q.shape[1]), dtype=torch.float64, device="cuda")
    w[:, 0::2], w[:, 1::2] = table[q.long() % 16], table[q.long() // 16]
    block = torch.arange(K, device="cuda") // 32
    return w[:, :K] * torch.pow(2.0, s.double() - 127)[:, block]


def _exact_experts(s):
    D, F = s["case"]["D"], s["case"]["F"]
    y = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda")
    x = _exact_rows(s["x"].double())
    for e in range(s["case"]["E"]):
        where = (s["ids"] == e).nonzero()
        if not len(where):
            continue
        wg, wu, wd = (_exact_weights(q[e], z[e], n) for (q, z), n in zip(s["w"], (D, D, F)))
        rows = x[where[:, 0]]
        gate = rows @ wg.t()
        act = _exact_rows(gate / (1 + torch.exp(-gate)) * (rows @ wu.t()))
        y.index_add_(0, where[:, 0], (act @ wd.t()) * s["gates"][where[:, 0], where[:, 1]]
                     .double().unsqueeze(-1))
    return y


def exact(case, seed):
    s = {**_inputs(case, seed), "case": case}
    op = case["op"]
    if op == "route":
        return {"ids": None, "gates": _exact_gates(s, _exact_choice(s))}
    if op == "route-grad":
        return _exact_route_grad(s)
    if op == "rows":
        return _exact_rows(s["x"].double())
    if op == "product":
        return _exact_rows(s["x"].double()) @ _exact_weights(*s["w"], case["K"]).t()
    return _exact_experts(s)


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    op = case["op"]
    size = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if op == "route":
        T, E, K = (case[k] for k in "TEK")
        return {"bytes": size * T * E + 8 * T * K + 4 * E * case["bias"], "flops": 4 * T * E}
    if op == "route-grad":
        T, E, K = (case[k] for k in "TEK")
        # the scores that the formula has: all of them, those of the chosen, none
        read = K if case["score"] == "sigmoid" else 0 if case["renorm"] else E
        return {"bytes": size * T * (E + read) + 12 * T * K, "flops": T * (E + 6 * K)}
    if op == "rows":
        n = case["R"] * case["D"]
        return {"bytes": int(n * (2 * size + 17 / 32)), "flops": 4 * n}
    if op == "product":
        M, N, K = (case[k] for k in "MNK")
        return {"bytes": int(size * M * (K + N) + 17 / 32 * N * K), "flops": 2 * M * N * K}
    T, D, F, E, K = (case[k] for k in "TDFEK")
    R, hot, n_hot = T * K, case["hot"], min(case["n_hot"], E)
    # experts with rows, expected
    rest = (1 - hot) / E
    used = (n_hot * (1 - (1 - rest - hot / n_hot) ** R) + (E - n_hot) * (1 - (1 - rest) ** R))
    return {"bytes": int(used * 3 * D * F * 17 / 32) + 2 * T * D * 2 + 8 * R,
            "flops": 6 * R * D * F}
