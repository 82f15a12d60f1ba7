"""Measured cases of the operators between the proved products of a decoder step.

Four operators, each a call of ``paper_2602_22700_b200.imm``:

  sample          one token per row of logits: temperature, top-k, top-p and min-p filters, and the draw
                  from a given uniform number
  rmsnorm_quant   residual addition, root-mean-square norm, and the int8 operand of the next product with
                  its scales
  moe_dispatch    rows of the tokens sorted by expert (the ragged left operands of the experts' products)
  moe_combine     the experts' output rows back in token order, weighted and added up

``own`` is set by the program that measures: False computes the plain forms with elementary torch
operations, True calls the library.  ``run(state)`` is one pass; everything it needs is in the state.
"""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16, "int8": torch.int8,
          "int32": torch.int32}
SIZES = {"float32": 4, "bfloat16": 2, "float16": 2, "int8": 1, "int32": 4}


def _library():
    from paper_2602_22700_b200 import imm as library
    return library


# ------------------------------------------------------------------ cases


def listed():
    return [
        # one decision of one request: the latency of a decode step, Top-20 as the audited service samples
        {"name": "sample_1x128256", "op": "sample", "rows": 1, "n": 128256, "dtype": "float32", "temperature": 0.8,
         "top_k": 20, "top_p": 0.95, "min_p": 0.0, "mixed": False, "masked": 0.0},
        # a serving batch in which every request brings its own parameters, greedy ones among them
        {"name": "sample_mixed_128x128256", "op": "sample", "rows": 128, "n": 128256, "dtype": "bfloat16", "temperature": 1.0,
         "top_k": 50, "top_p": 0.9, "min_p": 0.05, "mixed": True, "masked": 0.0},
        # replayed decisions of an audited request, nucleus sampling over the whole vocabulary
        {"name": "sample_top_p_1024x128256", "op": "sample", "rows": 1024, "n": 128256, "dtype": "float32", "temperature": 1.0,
         "top_k": 0, "top_p": 0.95, "min_p": 0.0, "mixed": False, "masked": 0.0},
        # the plain distribution: no filter, so every entry's weight counts
        {"name": "sample_plain_512x151936", "op": "sample", "rows": 512, "n": 151936, "dtype": "bfloat16", "temperature": 0.7,
         "top_k": 0, "top_p": 1.0, "min_p": 0.0, "mixed": False, "masked": 0.0},
        # an odd vocabulary (rows at odd addresses), part of it masked by a grammar, one row masked altogether
        {"name": "sample_masked_33x40003", "op": "sample", "rows": 33, "n": 40003, "dtype": "float16", "temperature": 1.2,
         "top_k": 1000, "top_p": 0.98, "min_p": 0.01, "mixed": False, "masked": 0.9},
        # one token of a decode step
        {"name": "norm_1x4096", "op": "norm", "rows": 1, "cols": 4096, "dtype": "bfloat16", "residual": True, "group": 0},
        # the audited decoder block's activations
        {"name": "norm_8192x4096", "op": "norm", "rows": 8192, "cols": 4096, "dtype": "bfloat16", "residual": True, "group": 0},
        # a wide hidden state in 32 bits, one scale per 128 columns, an odd number of rows
        {"name": "norm_group_2047x14336", "op": "norm", "rows": 2047, "cols": 14336, "dtype": "float32", "residual": True, "group": 128},
        # the routed rows of a decode step
        {"name": "dispatch_16x4096", "op": "dispatch", "rows": 16, "cols": 4096, "dtype": "int8", "experts": 8, "top": 2, "dropped": 0.0},
        # the expert batch at its longest token count, some of the tokens padding
        {"name": "dispatch_16384x4096", "op": "dispatch", "rows": 16384, "cols": 4096, "dtype": "int8", "experts": 8, "top": 2, "dropped": 0.02},
        # the accumulators of the experts' down projections back in token order
        {"name": "combine_4096x4096", "op": "combine", "rows": 4096, "cols": 4096, "dtype": "int32", "experts": 8, "top": 2, "dropped": 0.0},
        # many small experts, bf16 rows, an odd width
        {"name": "combine_1021x2051", "op": "combine", "rows": 1021, "cols": 2051, "dtype": "bfloat16", "experts": 64, "top": 6, "dropped": 0.05},
    ]


def _spread(rng, low, high):
    """A whole number in [low, high], spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["sample", "sample", "norm", "dispatch", "combine"])
    if op == "sample":
        n = _spread(rng, 200, 160000)
        rows = _spread(rng, 1, max(1, min(1024, 1024 * 128256 // (2 * n))))
        return {"op": op, "rows": rows, "n": n, "dtype": rng.choice(["float32", "bfloat16", "float16"]),
                "temperature": rng.choice([0.0, 1.0, round(rng.uniform(0.3, 2.0), 3)]),
                "top_k": rng.choice([0, 0, 1, 20, _spread(rng, 2, 2000)]),
                "top_p": rng.choice([1.0, round(rng.uniform(0.05, 0.999), 4)]),
                "min_p": rng.choice([0.0, 0.0, round(rng.uniform(0.001, 0.3), 4)]),
                "mixed": rng.random() < 0.3, "masked": rng.choice([0.0, 0.0, 0.5])}
    if op == "norm":
        group = rng.choice([0, 0, 128])
        cols = 128 * _spread(rng, 1, 128) if group else _spread(rng, 64, 16384)
        rows = _spread(rng, 1, max(1, 8192 * 4096 // cols))
        return {"op": op, "rows": rows, "cols": cols, "dtype": rng.choice(["float32", "bfloat16", "float16"]),
                "residual": rng.random() < 0.7, "group": group}
    experts = rng.choice([2, 8, 60, 128, 256])
    top = rng.randint(1, min(8, experts))
    cols = _spread(rng, 64, 8192)
    rows = _spread(rng, 1, max(1, 16384 * 4096 // (2 * top * cols)))
    return {"op": op, "rows": min(rows, 16384), "cols": cols,
            "dtype": rng.choice(["int8", "bfloat16", "float32"] if op == "dispatch" else ["int32", "bfloat16", "float16", "float32"]),
            "experts": experts, "top": top, "dropped": rng.choice([0.0, 0.1])}


def work(case):
    """Each input read once, each output written once."""
    r = case["rows"]
    if case["op"] == "sample":
        # per entry one subtraction, one scaling, one exponential and one addition
        return {"bytes": r * case["n"] * SIZES[case["dtype"]] + r * 28, "flops": 4 * r * case["n"]}
    c, e = case["cols"], SIZES[case["dtype"]]
    if case["op"] == "norm":
        groups = c // case["group"] if case["group"] else 1
        moved = e * r * c * (3 if case["residual"] else 1) + r * c + 4 * r * groups + 4 * c
        return {"bytes": moved, "flops": 6 * r * c}
    pairs = r * case["top"]
    if case["op"] == "dispatch":
        return {"bytes": e * r * c + e * pairs * c + 12 * pairs + 8 * r, "flops": pairs}
    return {"bytes": e * pairs * c + (2 if case["dtype"] != "float32" else 4) * r * c + 12 * pairs, "flops": 2 * pairs * c}


# ------------------------------------------------------------------ inputs


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * (int(seed) + 1))


def _pick(values, rows, g, dtype):
    table = torch.tensor(values, dtype=dtype, device="cuda")
    return table[torch.randint(len(values), (rows,), generator=g, device="cuda")]


def _prepare_sample(case, g):
    rows, n = case["rows"], case["n"]
    # an approximately normal bulk and a dozen plausible tokens lifted above it, by more in rows where the
    # model is sure of itself (the nucleus then holds a few tokens) than where it is not (tens of thousands)
    x = torch.randn((rows, n), generator=g, device="cuda") * 2.5
    hot = torch.randint(n, (rows, 12), generator=g, device="cuda")
    lift = torch.linspace(17.0, 9.0, 12, device="cuda") * torch.rand((rows, 1), generator=g, device="cuda").sqrt()
    x.scatter_add_(1, hot, lift.expand(rows, 12).contiguous())
    if case["masked"]:
        x.masked_fill_(torch.rand((rows, n), generator=g, device="cuda") < case["masked"], -math.inf)
        if rows > 2:
            x[rows // 2] = -math.inf                      # a padded row
    state = {"logits": x.to(DTYPES[case["dtype"]]), "u": torch.rand(rows, generator=g, device="cuda", dtype=torch.float64),
             "temperature": case["temperature"], "top_k": case["top_k"], "top_p": case["top_p"], "min_p": case["min_p"]}
    if case["mixed"]:
        f32 = torch.float32
        state["temperature"] = _pick([0.0, case["temperature"], 0.6, 0.8, 1.0, 1.3], rows, g, f32)
        state["top_k"] = _pick([0, case["top_k"], 1, 20, 64], rows, g, torch.int32)
        state["top_p"] = _pick([1.0, case["top_p"], 0.95, 0.8], rows, g, f32)
        state["min_p"] = _pick([0.0, case["min_p"], 0.02], rows, g, f32)
    # the buffers a decode loop keeps for the answers
    state["out"] = (torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.float32, device="cuda"),
                    torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, dtype=torch.int32, device="cuda"))
    return state


def _prepare_norm(case, g):
    rows, cols, dt = case["rows"], case["cols"], DTYPES[case["dtype"]]
    x = torch.randn((rows, cols), generator=g, device="cuda")
    # a few channels carry most of the energy, as in a residual stream
    loud = 1.0 + 15.0 * (torch.rand(cols, generator=g, device="cuda") < 0.01).float()
    state = {"x": (x * loud).to(dt), "residual": None, "eps": 1e-5, "group": case["group"],
             "weight": (1.0 + 0.2 * torch.randn(cols, generator=g, device="cuda")).to(dt)}
    if case["residual"]:
        state["residual"] = (3.0 * loud * torch.randn((rows, cols), generator=g, device="cuda")).to(dt)
    groups = cols // case["group"] if case["group"] else 1
    state["out"] = (torch.empty((rows, cols), dtype=torch.int8, device="cuda"),
                    torch.empty((rows, groups), dtype=torch.float32, device="cuda"),
                    torch.empty((rows, cols), dtype=dt, device="cuda") if case["residual"] else None)
    return state


def _routing(case, g):
    """int32 (rows, top): distinct experts per token, popular ones among them; -1 for tokens of padding."""
    rows, experts, top = case["rows"], case["experts"], case["top"]
    score = torch.randn((rows, experts), generator=g, device="cuda") + 0.5 * torch.randn(experts, generator=g, device="cuda")
    ids = score.topk(top, dim=1).indices.to(torch.int32)
    if case["dropped"]:
        ids[torch.rand(rows, generator=g, device="cuda") < case["dropped"]] = -1
    return ids.contiguous()


def _prepare_dispatch(case, g):
    rows, cols, pairs = case["rows"], case["cols"], case["rows"] * case["top"]
    x = torch.randn((rows, cols), generator=g, device="cuda") * 20.0
    x = x.round().clamp(-127, 127).to(torch.int8) if case["dtype"] == "int8" else x.to(DTYPES[case["dtype"]])
    return {"x": x, "ids": _routing(case, g), "experts": case["experts"],
            "scale": torch.rand(rows, generator=g, device="cuda") * 0.1,
            "out": (torch.zeros((pairs, cols), dtype=x.dtype, device="cuda"),      # rows behind the last stay as they are
                    torch.empty(case["experts"] + 1, dtype=torch.int64, device="cuda"),
                    torch.empty((rows, case["top"]), dtype=torch.int32, device="cuda"),
                    torch.zeros(pairs, dtype=torch.float32, device="cuda"),
                    torch.empty(1, dtype=torch.int32, device="cuda"))}


def _prepare_combine(case, g):
    rows, cols, top, pairs = case["rows"], case["cols"], case["top"], case["rows"] * case["top"]
    ids = _routing(case, g).view(-1).to(torch.int64)
    order = torch.argsort(torch.where(ids < 0, torch.full_like(ids, case["experts"]), ids), stable=True)
    position = torch.empty(pairs, dtype=torch.int32, device="cuda")
    position[order] = torch.arange(pairs, dtype=torch.int32, device="cuda")
    position[ids < 0] = -1
    weights = torch.rand((rows, top), generator=g, device="cuda") + 0.05
    state = {"position": position.view(rows, top), "weights": weights / weights.sum(1, keepdim=True), "row_scale": None}
    if case["dtype"] == "int32":
        state["y"] = torch.randint(-200000, 200001, (pairs, cols), generator=g, device="cuda", dtype=torch.int32)
        state["row_scale"] = torch.rand(pairs, generator=g, device="cuda") * 1e-4 + 1e-6
    else:
        state["y"] = torch.randn((pairs, cols), generator=g, device="cuda").to(DTYPES[case["dtype"]])
    to = torch.bfloat16 if case["dtype"] == "int32" else state["y"].dtype
    state["out"] = torch.empty((rows, cols), dtype=to, device="cuda")
    return state


PREPARE = {"sample": _prepare_sample, "norm": _prepare_norm, "dispatch": _prepare_dispatch, "combine": _prepare_combine}


def prepare(case, seed):
    state = PREPARE[case["op"]](case, _generator(seed))
    state["op"] = case["op"]
    return state


# ------------------------------------------------------------------ the plain forms and the library's calls


def _column(value, rows, dtype):
    """A parameter as a column of 64-bit values: per-row ones as they are, a number rounded to the 32 bits it is passed in."""
    t = value if isinstance(value, torch.Tensor) else torch.full((rows,), value, dtype=dtype, device="cuda")
    return t.to(torch.float64 if dtype == torch.float32 else torch.int64).view(rows, 1)


def _sample(s):
    """Entries in the order (logit descending, index ascending); every filter keeps a prefix of it."""
    if own:
        return _library().sample(s["logits"], s["u"], temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"],
                                 min_p=s["min_p"], out=s["out"])
    x = s["logits"].float()
    rows, n = x.shape
    t, k = _column(s["temperature"], rows, torch.float32), _column(s["top_k"], rows, torch.int32)
    p, m = _column(s["top_p"], rows, torch.float32), _column(s["min_p"], rows, torch.float32)
    xs, order = torch.sort(x, dim=1, descending=True, stable=True)
    alive = xs[:, :1] > -math.inf                           # a row with nothing left has no token
    best = torch.where(alive, xs[:, :1], torch.zeros_like(xs[:, :1])).double()
    greedy = t == 0
    w = torch.exp((xs.double() - best) / torch.where(greedy, torch.ones_like(t), t))
    place = torch.arange(n, device=x.device)
    keep = (xs > -math.inf) & ((k <= 0) | (place < k)) & (~greedy | (place < 1))
    w = torch.where(keep, w, torch.zeros_like(w))
    reached = torch.cumsum(w, dim=1)
    before = torch.cat([torch.zeros_like(reached[:, :1]), reached[:, :-1]], dim=1)
    keep &= (p >= 1) | (before < p * reached[:, -1:])       # the shortest prefix that holds p of the mass
    keep &= w >= m
    w = torch.where(keep, w, torch.zeros_like(w))
    spread = torch.empty_like(w).scatter_(1, order, w)      # back in the vocabulary's order
    total = torch.cumsum(spread, dim=1)
    aim = s["u"].view(rows, 1) * total[:, -1:]
    token = (total > aim).to(torch.int8).argmax(dim=1, keepdim=True)
    logprob = torch.log(spread.gather(1, token) / total[:, -1:])
    token = torch.where(alive, token, torch.full_like(token, -1))
    status = torch.where(alive, torch.zeros_like(token), torch.full_like(token, -1))
    return (token.view(rows).to(torch.int32), logprob.view(rows).to(torch.float32), keep.sum(1).to(torch.int32),
            status.view(rows).to(torch.int32))


def _norm(s):
    """h = x + residual, rounded to its type; t = h * weight; q = round(127 t / max|t|); scale = rms norm of the maximum / 127.
    The rounding of q does not depend on the norm (it cancels), so no order of summation can move it."""
    if own:
        return _library().rmsnorm_quant(s["x"], s["weight"], residual=s["residual"], eps=s["eps"], group=s["group"], out=s["out"])
    h = s["x"] if s["residual"] is None else (s["x"].float() + s["residual"].float()).to(s["x"].dtype)
    rows, cols = h.shape
    wide = h.double()
    inverse = 1.0 / torch.sqrt(wide.square().mean(dim=1, keepdim=True) + s["eps"])
    t = (wide * s["weight"].double()).view(rows, -1, s["group"] or cols)
    top = t.abs().amax(dim=2, keepdim=True)
    q = torch.where(top > 0, torch.round(t * 127.0 / top), torch.zeros_like(t))   # 64 bits: values next to a border
    scale = (top.squeeze(2) * inverse / 127.0).float()
    out = (q.view(rows, cols).to(torch.int8), scale)        # whole numbers, and the scales that turn them into values
    return out if s["residual"] is None else out + (h,)


def _dispatch(s):
    if own:
        return _library().moe_dispatch(s["x"], s["ids"], s["experts"], scale=s["scale"], out=s["out"])
    rows, top = s["ids"].shape
    flat = s["ids"].view(-1).to(torch.int64)
    key = torch.where(flat < 0, torch.full_like(flat, s["experts"]), flat)
    order = torch.argsort(key, stable=True)
    counts = (key.view(-1, 1) == torch.arange(s["experts"], device=key.device)).sum(0)
    offsets = torch.cat([torch.zeros_like(counts[:1]), torch.cumsum(counts, 0)])
    place = torch.arange(order.numel(), device=key.device)
    routed = place < offsets[-1]
    token = order // top
    rows_out = torch.where(routed.view(-1, 1), s["x"][token], torch.zeros_like(s["x"][:1]))
    position = torch.empty_like(order).scatter_(0, order, torch.where(routed, place, torch.full_like(place, -1)))
    scale = torch.where(routed, s["scale"][token], torch.zeros_like(s["scale"][:1]))
    return rows_out, offsets, position.view(rows, top).to(torch.int32), scale, torch.zeros(1, dtype=torch.int32, device=key.device)


def _combine(s):
    if own:
        return _library().moe_combine(s["y"], s["position"], weights=s["weights"], row_scale=s["row_scale"], out=s["out"])
    held = s["position"] >= 0
    at = torch.where(held, s["position"], torch.zeros_like(s["position"])).to(torch.int64)
    factor = s["weights"] if s["row_scale"] is None else s["weights"] * s["row_scale"][at]
    factor = torch.where(held, factor, torch.zeros_like(factor))
    return (s["y"][at].float() * factor.unsqueeze(2)).sum(1).to(s["out"].dtype)


RUN = {"sample": _sample, "norm": _norm, "dispatch": _dispatch, "combine": _combine}


def run(state):
    return RUN[state["op"]](state)


# ------------------------------------------------------------------ the definitions in 64 bits


def _at(value, i):
    return value[i].item() if isinstance(value, torch.Tensor) else torch.tensor(value).item()


def _exact_sample(s):
    """Row by row: log of the drawn entry's share of what the filters leave."""
    logits, u = s["logits"].double(), s["u"]
    found = []
    for i in range(logits.shape[0]):
        row = logits[i]
        ranked = torch.argsort(row, descending=True, stable=True)
        ranked = ranked[torch.isfinite(row[ranked])]
        if ranked.numel() == 0:
            found.append(math.nan)
            continue
        t, k, p, m = (_at(s[name], i) for name in ("temperature", "top_k", "top_p", "min_p"))
        if t == 0:
            found.append(0.0)
            continue
        if k > 0:
            ranked = ranked[:k]
        mass = torch.exp((row[ranked] - row[ranked[0]]) / t)
        if p < 1:
            running = mass.cumsum(0)
            held = int((running < p * running[-1]).sum()) + 1
            ranked, mass = ranked[:held], mass[:held]
        left = int((mass >= m).sum())
        ranked, mass = ranked[:left], mass[:left]
        by_index = torch.sort(ranked)
        mass = mass[by_index.indices]
        running = mass.cumsum(0)
        drawn = min(int((running <= u[i] * running[-1]).sum()), left - 1)
        found.append(math.log(float(mass[drawn] / running[-1])))
    return None, torch.tensor(found, dtype=torch.float64), None, None


def _exact_norm(s):
    h = s["x"].double()
    if s["residual"] is not None:
        h = (s["x"].float() + s["residual"].float()).to(s["x"].dtype).double()
    rms = (h.pow(2).sum(1) / h.shape[1] + s["eps"]).sqrt()
    peak = (h * s["weight"].double()).abs().unflatten(1, (-1, s["group"] or h.shape[1])).max(2).values
    scale = peak / (127.0 * rms.unsqueeze(1))
    summed = None if s["residual"] is None else s["x"].double() + s["residual"].double()
    return (None, scale) if summed is None else (None, scale, summed)


def _exact_combine(s):
    out = torch.zeros(s["out"].shape, dtype=torch.float64, device="cuda")
    for j in range(s["position"].shape[1]):
        at = s["position"][:, j].long()
        some = (at >= 0).nonzero().view(-1)
        factor = s["weights"][some, j].double()
        if s["row_scale"] is not None:
            factor = factor * s["row_scale"][at[some]].double()
        out[some] += s["y"][at[some]].double() * factor.view(-1, 1)
    return out


def exact(case, seed):
    s = prepare(case, seed)
    if case["op"] == "sample":
        return _exact_sample(s)
    if case["op"] == "norm":
        return _exact_norm(s)
    return _exact_combine(s) if case["op"] == "combine" else None       # a dispatch moves values, it computes none
