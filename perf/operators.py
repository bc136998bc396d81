"""The operators around and inside the expert layer, as cases to be timed.

Four kinds of call, each in a plain form of elementary torch operations (in 32
bits, rounded once) and, with `own` set, through the package's entry points:

* "norm"       llep_block_norm: norm of a block's output, gate, residual scale,
               residual sum, and the norm before the next block;
* "norm-grad"  llep_block_norm_backward: every gradient of it;
* "product"    llep_quantize_rows and llep_int8_matmul: activations to 8 bits
               with a scale per token, times 8-bit weights with a scale per
               channel;
* "experts"    LLEPLayer.forward_int8: the expert layer with 8-bit weights,
               from token activations to layer outputs;
* "clip"       llep_clip_gradients: the norm over all gradients, and the
               clipped gradients.

Sizes are those of the layer configurations in synth.py (hidden and FFN sizes,
experts, top-k, routing skew) with token counts from one to a training batch;
drawn cases also take generic and odd sizes.
"""

from __future__ import annotations

import math

import torch

own = False

EPS = 1e-5
ALPHA = 0.5
MAX_NORM = 1.0

# hidden size, FFN size, experts, experts per token
SHAPES = {
    "gpt-oss-20b": (2880, 2880, 32, 4),
    "qwen3-30b-a3b": (2048, 768, 128, 8),
}


def _norm(T, D, dtype, gate, post=True, pre=True):
    return {"op": "norm", "T": T, "D": D, "dtype": dtype, "gate": gate, "post": post, "pre": pre}


def _norm_grad(T, D, dtype, gate, post=True, pre=True):
    return {**_norm(T, D, dtype, gate, post, pre), "op": "norm-grad"}


def _product(M, N, K, dtype="bf16"):
    return {"op": "product", "M": M, "N": N, "K": K, "dtype": dtype}


def _experts(T, shape, hot, n_hot, P=8):
    """hot: share of the token-expert pairs on the first n_hot experts, the rest uniform."""
    D, F, E, K = SHAPES[shape] if isinstance(shape, str) else shape
    return {"op": "experts", "T": T, "D": D, "F": F, "E": E, "K": K, "P": P, "hot": hot,
            "n_hot": n_hot}


def _clip(kind, D, F, E, n, half):
    """kind "experts": n layers' three expert weight gradients [E, D, F]; "mixed": n tensors of
    sizes from a norm's weights [D] to a projection's [D, F], of odd lengths; every `half`-th in
    bfloat16 (0: none)."""
    return {"op": "clip", "kind": kind, "D": D, "F": F, "E": E, "n": n, "half": half}


def listed():
    cases = {
        # one decoded token between two blocks: latency
        "norm-token": _norm(1, 2880, "bf16", "channel"),
        # a prompt batch between two blocks
        "norm-prompt": _norm(16384, 2880, "bf16", "channel"),
        # a ragged batch in float32, a gate value for every element
        "norm-grad-ragged": _norm_grad(1777, 2048, "f32", "full"),
        # a training batch
        "norm-grad-batch": _norm_grad(8192, 7168, "bf16", "channel"),
        # one decoded token through a projection: latency, and the weights once
        "product-token": _product(1, 7168, 2048),
        # a ragged batch through a projection of odd sizes
        "product-odd": _product(333, 2881, 1003, "f32"),
        # a prompt batch through a projection
        "product-batch": _product(8192, 7168, 2048),
        # decode: a few tokens, most of the experts in use
        "experts-decode": _experts(8, "gpt-oss-20b", 0.5, 4),
        # a ragged prompt over many small experts
        "experts-ragged": _experts(1531, "qwen3-30b-a3b", 0.6, 16),
        # a prompt batch with hot experts
        "experts-prompt": _experts(8192, "gpt-oss-20b", 0.6, 4),
        # the many small and middling tensors of a model's dense part
        "clip-mixed": _clip("mixed", 2048, 768, 1, 61, 3),
        # an expert layer's weight gradients
        "clip-experts": _clip("experts", 2880, 2880, 16, 1, 0),
    }
    return [{**c, "name": n} for n, c in cases.items()]


def _log(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choice(["norm", "norm-grad", "product", "experts", "clip"])
    if op in ("norm", "norm-grad"):
        D = rng.choice([64, 768, 1024, 2048, 2880, 4096, 7168, _log(rng, 60, 8000)])
        T = _log(rng, 1, min(32768, (16384 * 2880 if op == "norm" else 8192 * 7168) // D))
        make = _norm if op == "norm" else _norm_grad
        post, pre = rng.choice([(True, True), (True, True), (False, True), (True, False)])
        return make(T, D, rng.choice(["bf16", "bf16", "f32"]) if T * D < 10 ** 7 else "bf16",
                    rng.choice(["none", "channel", "token", "full"]), post, pre)
    if op == "product":
        N, K = (rng.choice([768, 1024, 2048, 2880, 4096, _log(rng, 64, 7000)]) for _ in "NK")
        M = _log(rng, 1, min(16384, 8192 * 7168 * 2048 // (N * K)))
        return _product(M, N, K, rng.choice(["bf16", "bf16", "f32"]))
    if op == "experts":
        E = rng.choice([8, 16, 32, 64, 128])
        K = rng.choice([1, 2, 4, 8])
        D, F = (64 * rng.choice([4, 8, 12, 16, 23, 32, 45]) for _ in "DF")
        most = min(32768 // K, 8192 * 4 * 2880 * 2880 // (K * D * F))
        return _experts(_log(rng, 1, most), (D, F, E, K), rng.choice([0.0, 0.5, 0.9]),
                        rng.choice([1, 4]), rng.choice([1, 4, 8]))
    if rng.random() < 0.5:
        D, F = (64 * rng.choice([4, 8, 12, 16, 23, 32, 45]) for _ in "DF")
        return _clip("experts", D, F, rng.choice([1, 4, 16]), 1, 0)
    return _clip("mixed", _log(rng, 60, 3000), _log(rng, 60, 3000), 1, _log(rng, 2, 150),
                 rng.choice([0, 2, 3]))


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------

def _dtype(case):
    return torch.bfloat16 if case.get("dtype", "bf16") == "bf16" else torch.float32


def _randn(g, *shape, dtype=torch.float32, scale=1.0, mean=0.0):
    x = torch.randn(shape, generator=g, device="cuda")
    return (x * scale + mean if scale != 1.0 or mean != 0.0 else x).to(dtype)


def _gate_shape(case):
    T, D = case["T"], case["D"]
    return {"channel": (1, D), "token": (T, 1), "full": (T, D)}.get(case["gate"])


def _mixed_shapes(case):
    """Tensor sizes of a model's dense part: norm weights, biases, projections."""
    D, F = case["D"], case["F"]
    cycle = [(D,), (F, D), (D,), (F,), (D // 2 + 1, F), (1,), (D - 1, 33)]
    return [cycle[i % len(cycle)] for i in range(case["n"])]


def _weights8(g, *shape):
    """8-bit weights, rows = output channels, and their scales."""
    q = torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8)
    s = (torch.rand(shape[:-1], generator=g, device="cuda") + 0.5) * (0.035 / 127)
    return q, s


def _inputs(case, seed):
    """The case's data: the same for either form and for the definition in 64 bits."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    op, dt = case["op"], _dtype(case)
    s = {}
    if op in ("norm", "norm-grad"):
        T, D = case["T"], case["D"]
        s["x" if op == "norm" else "r"] = _randn(g, T, D, dtype=dt, scale=1.5)
        s["b"] = _randn(g, T, D, dtype=dt)
        shape = _gate_shape(case)
        s["gate"] = None if shape is None else _randn(g, *shape, dtype=dt, scale=0.3, mean=0.5)
        s["w_post"] = _randn(g, D, dtype=dt, scale=0.1, mean=1.0) if case["post"] else None
        s["w_pre"] = _randn(g, D, dtype=dt, scale=0.1, mean=1.0) if case["pre"] else None
        if op == "norm-grad":
            s["d_r"] = _randn(g, T, D, dtype=dt, scale=0.01)
            s["d_h"] = _randn(g, T, D, dtype=dt, scale=0.01) if case["pre"] else None
    elif op == "product":
        s["x"] = _randn(g, case["M"], case["K"], dtype=dt)
        s["wq"], s["ws"] = _weights8(g, case["N"], case["K"])
    elif op == "experts":
        T, D, F, E, K = (case[k] for k in "TDFEK")
        s["x"] = _randn(g, T, D, dtype=dt)
        hot = torch.rand((T, K), generator=g, device="cuda") < case["hot"]
        some = torch.randint(0, min(case["n_hot"], E), (T, K), generator=g, device="cuda")
        rest = torch.randint(0, E, (T, K), generator=g, device="cuda")
        s["ids"] = torch.where(hot, some, rest).to(torch.int32)
        s["gates"] = torch.softmax(_randn(g, T, K), dim=-1)
        s["w"] = [_weights8(g, E, *nk) for nk in ((F, D), (F, D), (D, F))]
    else:
        if case["kind"] == "experts":
            shapes = [(case["E"], case["D"], case["F"])] * (3 * case["n"])
        else:
            shapes = _mixed_shapes(case)
        half = case["half"]
        s["grads"] = [_randn(g, *shape, dtype=torch.bfloat16 if half and i % half == 0
                             else torch.float32, scale=0.02) for i, shape in enumerate(shapes)]
    return s


def prepare(case, seed):
    s = _inputs(case, seed)
    s["op"], s["case"] = case["op"], case
    if case["op"] == "experts":
        # rows per expert on the host, which an eager program needs to split its rows
        s["counts"] = torch.bincount(s["ids"].flatten().long(), minlength=case["E"]).tolist()
    if case["op"] == "clip":
        s["out"] = [torch.empty_like(t) for t in s["grads"]]
    if own:
        _prepare_own(case, s)
    return s


def _prepare_own(case, s):
    """What a program on the framework keeps: outputs, workspaces, packed weights, the layer."""
    from paper_2601_17111_amd import binding as B
    from paper_2601_17111_amd.layer import Int8Experts, LLEPLayer
    op = case["op"]
    empty = torch.empty_like
    if op == "norm":
        s["r"] = empty(s["x"])
        s["h"] = empty(s["x"]) if case["pre"] else None
    elif op == "norm-grad":
        f32 = dict(dtype=torch.float32, device="cuda")
        s["dx"], s["db"] = empty(s["r"]), empty(s["r"])
        s["d_gate"] = None if s["gate"] is None else torch.empty(s["gate"].shape, **f32)
        for k in ("w_post", "w_pre"):
            s["d" + k] = None if s[k] is None else torch.empty(case["D"], **f32)
        s["ws"] = torch.empty(B.llep_block_norm_backward_workspace_bytes(case["T"], case["D"]),
                              dtype=torch.uint8, device="cuda")
    elif op == "product":
        M, N, K = (case[k] for k in "MNK")
        s["packed"] = B.llep_pack_matrix_int8(s["wq"])
        s["q"] = torch.empty((M, B.llep_int8_row_bytes(K)), dtype=torch.int8, device="cuda")
        s["scale"] = torch.empty(M, dtype=torch.float32, device="cuda")
        s["y"] = torch.empty((M, N), dtype=_dtype(case), device="cuda")
        s["work"] = torch.empty(B.llep_int8_matmul_workspace_bytes(M, N, K), dtype=torch.uint8,
                                device="cuda")
    elif op == "experts":
        T, D, F, E, K, P = (case[k] for k in "TDFEKP")
        s["layer"] = LLEPLayer(T, K, E, P, D, F, math.ceil(1.1 * T * K / P), torch.bfloat16)
        s["experts"] = Int8Experts(*[t for qs in s["w"] for t in qs])
    else:
        s["norm"] = torch.empty(1, dtype=torch.float32, device="cuda")
        s["ws"] = torch.empty(B.llep_clip_gradients_workspace_bytes(), dtype=torch.uint8,
                              device="cuda")


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------

def run(s):
    if own:
        return _run_own(s)
    return {"norm": _plain_norm, "norm-grad": _plain_norm_grad, "product": _plain_product,
            "experts": _plain_experts, "clip": _plain_clip}[s["op"]](s)


def _run_own(s):
    from paper_2601_17111_amd import binding as B
    op = s["op"]
    if op == "norm":
        B.llep_block_norm(s["x"], s["b"], s["gate"], s["w_post"], s["w_pre"], ALPHA, EPS,
                          s["r"], s["h"])
        return {k: s[k] for k in ("r", "h") if s[k] is not None}
    if op == "norm-grad":
        B.llep_block_norm_backward(s["r"], s["b"], s["gate"], s["w_post"], s["w_pre"], ALPHA, EPS,
                                   s["d_r"], s["d_h"], s["dx"], s["db"], s["d_gate"],
                                   s["dw_post"], s["dw_pre"], s["ws"])
        return {k: s[k] for k in ("dx", "db", "d_gate", "dw_post", "dw_pre") if s[k] is not None}
    if op == "product":
        B.llep_quantize_rows(s["x"], s["q"], s["scale"])
        B.llep_int8_matmul(s["q"], s["scale"], s["packed"], s["ws"], s["y"], s["case"]["K"],
                           s["work"])
        return s["y"]
    if op == "experts":
        return s["layer"].forward_int8(s["ids"], s["gates"], s["x"], s["experts"])
    B.llep_clip_gradients(s["grads"], MAX_NORM, s["norm"], s["ws"], out=s["out"])
    return {"norm": s["norm"], "grads": s["out"]}


def _plain_norm(s):
    dt = s["x"].dtype
    r = s["b"].float()
    if s["w_post"] is not None:
        r = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * s["w_post"].float()
    if s["gate"] is not None:
        r = r * s["gate"].float()
    r = s["x"].float() + ALPHA * r
    out = {"r": r.to(dt)}
    if s["w_pre"] is not None:
        h = r * torch.rsqrt((r * r).mean(-1, keepdim=True) + EPS) * s["w_pre"].float()
        out["h"] = h.to(dt)
    return out


def _norm_back(x, e):
    """Gradient of x * rsqrt(mean(x^2) + eps) for the output gradient e, and the normalised x."""
    i = torch.rsqrt((x * x).mean(-1, keepdim=True) + EPS)
    n = x * i
    return i * (e - n * (n * e).mean(-1, keepdim=True)), n


def _plain_norm_grad(s):
    dt = s["r"].dtype
    r, b, total = s["r"].float(), s["b"].float(), s["d_r"].float()
    out = {}
    if s["w_pre"] is not None:
        d_h = s["d_h"].float()
        dx, n = _norm_back(r, d_h * s["w_pre"].float())
        out["dw_pre"] = (d_h * n).sum(0)
        total = total + dx
    gate = None if s["gate"] is None else s["gate"].float()
    m = ALPHA * total if gate is None else ALPHA * total * gate
    db, n = m, b
    if s["w_post"] is not None:
        w = s["w_post"].float()
        db, n = _norm_back(b, m * w)
        out["dw_post"] = (m * n).sum(0)
        n = n * w
    if gate is not None:
        d_gate = ALPHA * total * n
        axes = [a for a in (0, 1) if gate.shape[a] == 1 and d_gate.shape[a] != 1]
        out["d_gate"] = d_gate.sum(axes, keepdim=True) if axes else d_gate
    out["dx"], out["db"] = total.to(dt), db.to(dt)
    return {k: out[k] for k in ("dx", "db", "d_gate", "dw_post", "dw_pre") if k in out}


def _plain_quantize(x):
    """Whole numbers in [-127, 127] (kept in 32 bits) and the scale of each row."""
    most = x.abs().amax(-1, keepdim=True)
    inv = torch.where(most > 0, 127.0 / most, torch.zeros_like(most))
    return torch.round(x * inv), most / 127.0


def _plain_product(s):
    q, scale = _plain_quantize(s["x"].float())
    return ((q @ s["wq"].float().t()) * scale * s["ws"]).to(s["x"].dtype)


def _plain_expert(q, scale, w):
    """One expert on its rows; w: gate, up and down weights with their scales."""
    (wg, sg), (wu, su), (wd, sd) = w
    gate = (q @ wg.float().t()) * scale * sg
    up = (q @ wu.float().t()) * scale * su
    q, scale = _plain_quantize(gate * torch.sigmoid(gate) * up)
    return (q @ wd.float().t()) * scale * sd


def _plain_experts(s):
    T, K, D = s["case"]["T"], s["case"]["K"], s["case"]["D"]
    q, scale = _plain_quantize(s["x"].float())
    order = torch.argsort(s["ids"].flatten(), stable=True)
    token = order // K
    used = [e for e, n in enumerate(s["counts"]) if n]
    sizes = [s["counts"][e] for e in used]
    rows = torch.cat([_plain_expert(a, b, [(w[e], c[e]) for w, c in s["w"]])
                      for e, a, b in zip(used, q[token].split(sizes), scale[token].split(sizes))])
    pairs = torch.empty_like(rows)
    pairs[order] = rows
    return (pairs.view(T, K, D) * s["gates"].unsqueeze(-1)).sum(1).to(s["x"].dtype)


def _plain_clip(s):
    squares = torch.stack([(t.float() * t.float()).sum() for t in s["grads"]])
    norm = torch.sqrt(squares.sum()).reshape(1)
    factor = torch.where(norm > MAX_NORM, MAX_NORM / norm, torch.ones_like(norm))
    return {"norm": norm, "grads": [(t.float() * factor).to(t.dtype) for t in s["grads"]]}


# ---------------------------------------------------------------------------
# the definitions in 64 bits
# ---------------------------------------------------------------------------

def _exact_rms(x):
    return x / (x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS).sqrt()


def _exact_norm(s):
    r = s["b"].double()
    if s["w_post"] is not None:
        r = _exact_rms(r) * s["w_post"].double()
    if s["gate"] is not None:
        r = r * s["gate"].double()
    r = s["x"].double() + ALPHA * r
    if s["w_pre"] is None:
        return {"r": r}
    return {"r": r, "h": _exact_rms(r) * s["w_pre"].double()}


def _exact_norm_grad(s):
    """Through the Jacobian J = (I - x x^T / (D m)) / sqrt(m), m = mean(x^2) + eps, of each norm."""
    def through(x, e):
        m = x.pow(2).sum(-1, keepdim=True) / x.shape[-1] + EPS
        return e / m.sqrt() - x * (x * e).sum(-1, keepdim=True) / (x.shape[-1] * m ** 1.5)
    r, b = s["r"].double(), s["b"].double()
    total, out = s["d_r"].double(), {}
    if s["w_pre"] is not None:
        out["dw_pre"] = (s["d_h"].double() * _exact_rms(r)).sum(0)
        total = total + through(r, s["d_h"].double() * s["w_pre"].double())
    n = b
    if s["w_post"] is not None:
        n = _exact_rms(b) * s["w_post"].double()
    scaled = ALPHA * total
    if s["gate"] is not None:
        d_gate = scaled * n
        if s["gate"].shape[0] != d_gate.shape[0]:
            d_gate = d_gate.sum(0, keepdim=True)
        if s["gate"].shape[1] != d_gate.shape[1]:
            d_gate = d_gate.sum(1, keepdim=True)
        out["d_gate"] = d_gate
        scaled = scaled * s["gate"].double()
    out["db"] = scaled
    if s["w_post"] is not None:
        out["dw_post"] = (scaled * _exact_rms(b)).sum(0)
        out["db"] = through(b, scaled * s["w_post"].double())
    out["dx"] = total
    return {k: out[k] for k in ("dx", "db", "d_gate", "dw_post", "dw_pre") if k in out}


def _exact_rows(x):
    """The 8-bit rows as the real values that they stand for."""
    most = x.abs().max(-1, keepdim=True).values
    step = most / 127
    return torch.where(step > 0, torch.round(x / torch.where(step > 0, step, 1.0)), 0.0) * step


def _exact_experts(s):
    T, K = s["ids"].shape
    y = torch.zeros(s["x"].shape, dtype=torch.float64, device="cuda")
    x = _exact_rows(s["x"].double())
    for e in range(s["w"][0][0].shape[0]):
        where = (s["ids"] == e).nonzero()
        if not len(where):
            continue
        wg, wu, wd = (w[e].double() * c[e].double().unsqueeze(-1) for w, c in s["w"])
        rows = x[where[:, 0]]
        gate = rows @ wg.t()
        act = _exact_rows(gate / (1 + torch.exp(-gate)) * (rows @ wu.t()))
        y.index_add_(0, where[:, 0], (act @ wd.t()) * s["gates"][where[:, 0], where[:, 1]]
                     .double().unsqueeze(-1))
    return y


def exact(case, seed):
    s = _inputs(case, seed)
    op = case["op"]
    if op == "norm":
        return _exact_norm(s)
    if op == "norm-grad":
        return _exact_norm_grad(s)
    if op == "product":
        w = s["wq"].double() * s["ws"].double().unsqueeze(-1)
        return _exact_rows(s["x"].double()) @ w.t()
    if op == "experts":
        return _exact_experts(s)
    norm = math.sqrt(sum(float(t.double().square().sum()) for t in s["grads"]))
    factor = min(1.0, MAX_NORM / norm) if norm > 0 else 1.0
    return {"norm": torch.tensor([norm], dtype=torch.float64),
            "grads": [t.double() * factor for t in s["grads"]]}


# ---------------------------------------------------------------------------
# what a pass cannot do without
# ---------------------------------------------------------------------------

def work(case):
    op = case["op"]
    size = 2 if case.get("dtype", "bf16") == "bf16" else 4
    if op in ("norm", "norm-grad"):
        T, D = case["T"], case["D"]
        gate = {"none": 0, "channel": D, "token": T, "full": T * D}[case["gate"]]
        weights = D * (case["post"] + case["pre"])
        if op == "norm":
            return {"bytes": size * (T * D * (3 + case["pre"]) + gate + weights),
                    "flops": T * D * (3 + 4 * case["post"] + 4 * case["pre"])}
        return {"bytes": size * (T * D * (5 + case["pre"]) + gate + weights)
                + 4 * (gate + weights),
                "flops": T * D * (4 + 9 * case["post"] + 9 * case["pre"])}
    if op == "product":
        M, N, K = (case[k] for k in "MNK")
        return {"bytes": size * M * (K + N) + N * K + 4 * N, "flops": 2 * M * N * K}
    if op == "experts":
        T, D, F, E, K = (case[k] for k in "TDFEK")
        R, hot, n_hot = T * K, case["hot"], min(case["n_hot"], E)
        # experts with rows, expected
        rest = (1 - hot) / E
        used = (n_hot * (1 - (1 - rest - hot / n_hot) ** R) + (E - n_hot) * (1 - (1 - rest) ** R))
        return {"bytes": int(used * 3 * D * F) + 2 * T * D * 2 + 8 * R, "flops": 6 * R * D * F}
    if case["kind"] == "experts":
        total = 3 * case["n"] * case["E"] * case["D"] * case["F"]
        return {"bytes": 8 * total + 4, "flops": 3 * total}
    counts = [math.prod(shape) for shape in _mixed_shapes(case)]
    half = case["half"]
    sizes = [2 if half and i % half == 0 else 4 for i in range(len(counts))]
    return {"bytes": 2 * sum(n * z for n, z in zip(counts, sizes)) + 4, "flops": 3 * sum(counts)}
