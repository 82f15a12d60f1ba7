"""Measured cases of the operators of a decode step over an 8-bit cache.

Three operators, each a call of ``paper_2602_22700_b200.imm``:

  kv_append       rows of keys and values into a paged int8 cache with one scale per page and head
  kv_attention    causal attention over that cache, for prompts and single tokens, with an optional sliding window
                  and first tokens that stay visible
  verify_draft    drafted tokens against the target's distribution with given uniform numbers, and the token that
                  follows the accepted ones

``own`` is set by the program that measures: False computes the plain forms with elementary torch operations, True
calls the library.  ``run(state)`` is one pass; everything it needs is in the state.
"""
import math
import random

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZES = {"float32": 4, "bfloat16": 2, "float16": 2}


def _library():
    from paper_2602_22700_b200 import imm as library
    return library


# ------------------------------------------------------------------ cases


def listed():
    return [
        # a decode step of a serving batch: one new token per request, histories of all lengths
        {"name": "append_step_64", "op": "append", "batch": 64, "new": 1, "past": 8000, "kv_heads": 8, "dim": 128, "page": 16,
         "dtype": "bfloat16", "spare": 0},
        # prompts of different lengths into empty and half-full pages
        {"name": "append_prompts_5x3000", "op": "append", "batch": 5, "new": 3000, "past": 500, "kv_heads": 8, "dim": 128, "page": 64,
         "dtype": "float16", "spare": 7},
        # one token of one request: the latency of a decode step
        {"name": "attention_1x2000", "op": "attention", "batch": 1, "new": 1, "past": 1999, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "dtype": "bfloat16", "window": 0, "sinks": 0, "spare": 0},
        # one request with a long history: its keys have to be shared out over the whole GPU
        {"name": "attention_1x100001", "op": "attention", "batch": 1, "new": 1, "past": 100000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "dtype": "bfloat16", "window": 0, "sinks": 0, "spare": 0},
        # a serving batch with histories between 500 and 32 thousand tokens
        {"name": "attention_64x32000", "op": "attention", "batch": 64, "new": 1, "past": 32000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 16, "dtype": "bfloat16", "window": 0, "sinks": 0, "spare": 0},
        # a sliding window with first tokens that stay visible, as many key heads as query heads, heads of 80, 32 bits
        {"name": "attention_window_33x9000", "op": "attention", "batch": 33, "new": 1, "past": 9000, "heads": 20, "kv_heads": 20, "dim": 80,
         "page": 32, "dtype": "float32", "window": 2047, "sinks": 4, "spare": 0},
        # four drafted tokens per request checked at once
        {"name": "attention_draft_32x5", "op": "attention", "batch": 32, "new": 5, "past": 6000, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 32, "dtype": "float16", "window": 0, "sinks": 0, "spare": 3},
        # a whole prompt
        {"name": "attention_prompt_4096", "op": "attention", "batch": 1, "new": 4096, "past": 0, "heads": 32, "kv_heads": 8, "dim": 128,
         "page": 64, "dtype": "bfloat16", "window": 0, "sinks": 0, "spare": 0},
        # one request, four drafted tokens, the vocabulary of the audited logits
        {"name": "verify_1x4x128256", "op": "verify", "batch": 1, "drafts": 4, "n": 128256, "dtype": "float32", "temperature": 0.8,
         "mixed": False, "masked": 0.0, "draft": True},
        # a serving batch in which every request has its own temperature, greedy ones among them
        {"name": "verify_mixed_64x4x128256", "op": "verify", "batch": 64, "drafts": 4, "n": 128256, "dtype": "bfloat16", "temperature": 1.0,
         "mixed": True, "masked": 0.0, "draft": True},
        # tokens copied from the prompt: a proposal without a distribution
        {"name": "verify_copied_48x7x151936", "op": "verify", "batch": 48, "drafts": 7, "n": 151936, "dtype": "float32", "temperature": 0.7,
         "mixed": False, "masked": 0.0, "draft": False},
        # an odd vocabulary, part of it masked
        {"name": "verify_masked_33x3x40003", "op": "verify", "batch": 33, "drafts": 3, "n": 40003, "dtype": "float16", "temperature": 1.2,
         "mixed": False, "masked": 0.9, "draft": True},
    ]


def _spread(rng, low, high):
    """A whole number in [low, high], spread over its logarithm."""
    return max(low, min(high, int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))))


def draw(rng):
    op = rng.choice(["append", "attention", "attention", "attention", "verify"])
    if op == "verify":
        n, drafts = _spread(rng, 300, 160000), rng.randint(1, 8)
        return {"op": op, "batch": _spread(rng, 1, max(1, min(256, 64 * 5 * 128256 // ((drafts + 1) * n)))), "drafts": drafts, "n": n,
                "dtype": rng.choice(["float32", "bfloat16", "float16"]), "temperature": rng.choice([0.0, 1.0, round(rng.uniform(0.3, 2.0), 3)]),
                "mixed": rng.random() < 0.3, "masked": rng.choice([0.0, 0.0, 0.5]), "draft": rng.random() < 0.7}
    page, dtype, dim = rng.choice([16, 32, 64, 128]), rng.choice(["bfloat16", "bfloat16", "float16", "float32"]), rng.choice([64, 80, 96, 128])
    kv_heads = rng.choice([1, 2, 4, 8, 16])
    if op == "append":
        batch = _spread(rng, 1, 128)
        return {"op": op, "batch": batch, "new": _spread(rng, 1, max(1, 15000 // batch)), "past": _spread(rng, 1, 4000), "kv_heads": kv_heads,
                "dim": dim, "page": page, "dtype": dtype, "spare": rng.choice([0, 5])}
    group, kind = rng.choice([1, 2, 4, 5, 8]), rng.choice(["token", "token", "draft", "prompt"])
    heads = kv_heads * group
    case = {"op": op, "heads": heads, "kv_heads": kv_heads, "dim": dim, "page": page, "dtype": dtype,
            "window": rng.choice([0, 0, _spread(rng, 30, 5000)]), "sinks": 0, "spare": rng.choice([0, 2])}
    if case["window"]:
        case["sinks"] = rng.choice([0, 4, 70])
    if kind == "prompt":
        # short of the listed prompt's products, in 32 bits by eight times
        pairs = 4096 * 4096 * 32 * 128 // (heads * dim * (8 if dtype == "float32" else 1))
        new = _spread(rng, 30, max(30, min(4096, int(pairs ** 0.5))))
        case.update(batch=max(1, min(8, pairs // (new * new) // 2)), new=new, past=_spread(rng, 1, max(1, new // 2)))
    else:
        new = 1 if kind == "token" else rng.randint(2, 9)
        past = _spread(rng, 10, 32000)
        case.update(batch=_spread(rng, 1, max(1, min(128, 64 * 32000 * 8 // (2 * past * kv_heads * new)))), new=new, past=past)
    return case


def _lengths(case):
    """(new, total) tokens of every sequence, from the case alone: the longest first, the others spread below it."""
    batch, most, past = case["batch"], case["new"], case["past"]
    found = []
    for i in range(batch):
        new = most if most < 10 else max(1, most - (most * 2 * i) // (3 * batch))
        if 1 < most < 10 and i % 3 == 2:
            new = most - 1                                             # a request with one drafted token less
        found.append((new, new + past - (past * i * 63) // (batch * 64)))
    return found


def _visible(case, new, total):
    """Keys that some row of a sequence sees, and pairs of rows and keys."""
    window, sinks = case["window"] or total, case["sinks"]
    first = total - new
    low = max(0, first - window + 1)
    keys = total - low + min(sinks, low)
    pairs = 0
    for at in range(first, total):
        low = max(0, at - window + 1)
        pairs += at + 1 - low + min(sinks, low)
    return keys, pairs


def _agreement(case):
    """About how often a drafted token is taken, as the inputs are made."""
    return 0.82 if case["draft"] else 0.65


def work(case):
    """Each input that the answer needs read once, each output written once."""
    e = SIZES[case["dtype"]]
    if case["op"] == "verify":
        # rows behind the first token that is not taken are not needed
        rate, k = _agreement(case), case["drafts"]
        tested = sum(rate ** i for i in range(k))
        rows = case["batch"] * (tested * (2 if case["draft"] else 1) + rate ** k)
        return {"bytes": int(rows * case["n"] * e) + case["batch"] * (12 * (k + 1) + 16), "flops": int(4 * rows * case["n"])}
    sequences = _lengths(case)
    tokens, width = sum(new for new, _ in sequences), case["kv_heads"] * case["dim"]
    if case["op"] == "append":
        pages = sum((total - 1) // case["page"] - (total - new) // case["page"] + 1 for new, total in sequences)
        return {"bytes": 2 * tokens * width * (e + 1) + pages * (16 * case["kv_heads"] + 4), "flops": 4 * tokens * width}
    keys, pairs = (sum(v) for v in zip(*(_visible(case, new, total) for new, total in sequences)))
    moved = 2 * keys * width + keys // case["page"] * (8 * case["kv_heads"] + 4) + tokens * case["heads"] * (2 * case["dim"] * e + 4)
    return {"bytes": moved, "flops": 4 * pairs * case["heads"] * case["dim"]}


# ------------------------------------------------------------------ inputs


def _generator(seed):
    return torch.Generator(device="cuda").manual_seed(1000003 * (int(seed) + 1))


def _sequences(case, seed, g):
    """Offsets, lengths and page table of the sequences, in an order of the seed; pages lie anywhere in the cache."""
    found, page = _lengths(case), case["page"]
    random.Random(seed).shuffle(found)
    offsets = [0]
    for new, _ in found:
        offsets.append(offsets[-1] + new)
    pages = [-(-total // page) for _, total in found]
    width = max(pages)
    count = sum(pages) + 3
    order = torch.randperm(count, generator=g, device="cuda").to(torch.int32)
    held = torch.tensor(pages, device="cuda").view(-1, 1)
    column = torch.arange(width, device="cuda").view(1, -1)
    first = torch.cumsum(held, 0) - held
    table = torch.where(column < held, order[(first + column).clamp(max=count - 1)], torch.full_like(order[:1], -1))
    return {"offsets": torch.tensor(offsets, dtype=torch.int64, device="cuda"),
            "lengths": torch.tensor([total for _, total in found], dtype=torch.int32, device="cuda"),
            "table": table.contiguous(), "pages": count, "tokens": offsets[-1], "most_new": max(new for new, _ in found)}


def _cache(case, count, g):
    """Entries as a quantised cache holds them: scales that differ between pages and heads by a factor of a few."""
    shape = (count, case["kv_heads"], case["page"], case["dim"])
    cache = [torch.randint(-127, 128, shape, generator=g, device="cuda", dtype=torch.int8) for _ in range(2)]
    scales = [torch.exp(0.7 * torch.randn(shape[:2], generator=g, device="cuda")) * 0.02 for _ in range(2)]
    return cache[0], cache[1], scales[0], scales[1]


def _prepare_append(case, seed, g):
    state = _sequences(case, seed, g)
    state["cache"] = _cache(case, state["pages"], g)
    rows, heads, dim = state["tokens"] + case["spare"], case["kv_heads"], case["dim"]
    # keys and values as parts of one projection's output; some rows are louder than what their page holds
    both = torch.randn((rows, 2 * heads, dim), generator=g, device="cuda") * torch.exp(torch.randn((rows, 2 * heads, 1), generator=g, device="cuda"))
    both = both.to(DTYPES[case["dtype"]])
    state.update(k=both[:, :heads], v=both[:, heads:], out=torch.zeros(case["batch"], dtype=torch.int32, device="cuda"))
    return state


def _prepare_attention(case, seed, g):
    state = _sequences(case, seed, g)
    state["cache"] = _cache(case, state["pages"], g)
    rows = state["tokens"] + case["spare"]
    state["q"] = (1.2 * torch.randn((rows, case["heads"], case["dim"]), generator=g, device="cuda")).to(DTYPES[case["dtype"]])
    state.update(scale=case["dim"] ** -0.5, window=case["window"], sinks=case["sinks"],
                 out=(torch.zeros_like(state["q"]), torch.zeros((rows, case["heads"]), device="cuda")))
    return state


def _prepare_verify(case, seed, g):
    batch, most, n, dt = case["batch"], case["drafts"], case["n"], DTYPES[case["dtype"]]
    held = [most if i % 4 else max(1, most - i % 3) for i in range(batch)]             # drafted tokens of every request
    random.Random(seed).shuffle(held)
    offsets = [0]
    for k in held:
        offsets.append(offsets[-1] + k + 1)
    rows = offsets[-1]
    # a bulk of unlikely tokens and a dozen plausible ones; the draft's logits are the target's with noise
    x = torch.randn((rows, n), generator=g, device="cuda") * 2.0
    hot = torch.randint(n, (rows, 12), generator=g, device="cuda")
    x.scatter_add_(1, hot, torch.linspace(16.0, 9.0, 12, device="cuda").expand(rows, 12).contiguous())
    if case["masked"]:
        x.masked_fill_(torch.rand((rows, n), generator=g, device="cuda") < case["masked"], -math.inf)
    tested = torch.ones(rows, dtype=torch.bool, device="cuda")
    tested[torch.tensor(offsets[1:], device="cuda") - 1] = False                       # the last row of a request has no draft
    tested = tested.nonzero().view(-1)
    y = x[tested] + 0.6 * torch.randn((rows - batch, n), generator=g, device="cuda")
    target, draft = x.to(dt), y.to(dt)
    t = torch.full((batch,), case["temperature"], device="cuda")
    if case["mixed"]:
        t = torch.tensor([0.0, case["temperature"], 0.6, 1.0, 1.3], device="cuda")[torch.randint(5, (batch,), generator=g, device="cuda")]
    owner = torch.repeat_interleave(torch.arange(batch, device="cuda"), torch.tensor(held, device="cuda"))
    warm = torch.where(t > 0, t, torch.full_like(t, 1e-3))[owner].view(-1, 1)
    proposed = torch.multinomial(torch.softmax(draft.float() / warm, 1), 1, generator=g).view(-1)
    tokens = torch.zeros(rows, dtype=torch.int32, device="cuda")
    tokens[tested + 1] = proposed.to(torch.int32)
    return {"target": target, "draft": draft if case["draft"] else None, "tokens": tokens,
            "offsets": torch.tensor(offsets, dtype=torch.int64, device="cuda"), "most": most,
            "u": torch.rand(rows, generator=g, device="cuda", dtype=torch.float64),
            "temperature": t if case["mixed"] else case["temperature"],
            "out": (torch.empty(batch, dtype=torch.int32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda"),
                    torch.empty(batch, dtype=torch.float32, device="cuda"), torch.empty(batch, dtype=torch.int32, device="cuda"))}


PREPARE = {"append": _prepare_append, "attention": _prepare_attention, "verify": _prepare_verify}


def prepare(case, seed):
    state = PREPARE[case["op"]](case, int(seed), _generator(seed))
    state["op"] = case["op"]
    return state


# ------------------------------------------------------------------ the plain forms and the library's calls


def _append(s):
    """A page's scale is the largest magnitude of its entries / 127, so far; where new rows raise it, the entries that the
    page holds already are rounded again.  64 bits: quotients next to a border."""
    if own:
        status = _library().kv_append(s["k"], s["v"], s["cache"], s["table"], s["offsets"], s["lengths"], out=s["out"])
        return s["cache"] + (status,)
    k_cache, v_cache, k_scale, v_scale = s["cache"]
    count, heads, page, dim = k_cache.shape
    rows = torch.arange(s["tokens"], device=k_cache.device)
    owner = torch.searchsorted(s["offsets"], rows, right=True) - 1
    start = s["lengths"].long() - (s["offsets"][1:] - s["offsets"][:-1])
    place = start[owner] + rows - s["offsets"][owner]                   # position of a row in its sequence
    at, slot = s["table"][owner, place // page].long(), place % page
    held = torch.zeros(count, dtype=torch.int64, device=at.device)      # entries that a page holds already
    begun = s["table"].gather(1, (start // page).clamp(max=s["table"].shape[1] - 1).view(-1, 1)).view(-1).long()
    held.scatter_(0, begun.clamp(min=0), start % page)
    touched = torch.zeros(count, dtype=torch.bool, device=at.device)
    touched[at] = True
    for x, cache, scale in ((s["k"], k_cache, k_scale), (s["v"], v_cache, v_scale)):      # keys, values
        wide = x[:s["tokens"]].double()
        top = torch.zeros((count, heads), dtype=torch.float64, device=at.device)
        top.scatter_reduce_(0, at.view(-1, 1).expand(-1, heads), wide.abs().amax(2), "amax")
        old = torch.where(held.view(-1, 1) > 0, scale, torch.zeros_like(scale))
        new = torch.maximum(old, (top / torch.full_like(top, 127.0)).float())
        grown = (touched.view(-1, 1) & (new > old) & (old > 0)).nonzero()
        ratio = (old[grown[:, 0], grown[:, 1]].double(), new[grown[:, 0], grown[:, 1]].double())
        kept = cache[grown[:, 0], grown[:, 1]].double() * ratio[0].view(-1, 1, 1) / ratio[1].view(-1, 1, 1)
        inside = torch.arange(page, device=at.device).view(1, -1, 1) < held[grown[:, 0]].view(-1, 1, 1)
        cache[grown[:, 0], grown[:, 1]] = torch.where(inside, torch.round(kept).to(torch.int8), cache[grown[:, 0], grown[:, 1]])
        per_row = new[at].double().unsqueeze(2)
        q = torch.where(per_row > 0, torch.round(wide / per_row), torch.zeros_like(wide)).clamp(-127, 127)
        cache[at, :, slot] = q.to(torch.int8)
        scale.copy_(torch.where(touched.view(-1, 1), new, scale))
    return s["cache"] + (torch.zeros_like(s["lengths"]),)


def _attention(s):
    """Row i of a sequence stands at position length - new + i and sees the keys up to it: the last `window` of them
    (0: all) and the first `sinks`."""
    if own:
        if "workspace" not in s:
            s["workspace"] = _library().kv_attention_workspace(s["q"], s["cache"], s["table"], s["offsets"])
        return _library().kv_attention(s["q"], s["cache"], s["table"], s["offsets"], s["lengths"], scale=s["scale"], window=s["window"],
                                       sinks=s["sinks"], out=s["out"], workspace=s["workspace"])
    k_cache, v_cache, k_scale, v_scale = s["cache"]
    _, kv_heads, page, dim = k_cache.shape
    batch, width = s["table"].shape
    heads, most, device = s["q"].shape[1], s["most_new"], k_cache.device
    pages = s["table"].clamp(min=0).long()
    k = (k_cache[pages].float() * k_scale[pages].view(batch, width, kv_heads, 1, 1)).transpose(1, 2).reshape(batch, kv_heads, width * page, dim)
    v = (v_cache[pages].float() * v_scale[pages].view(batch, width, kv_heads, 1, 1)).transpose(1, 2).reshape(batch, kv_heads, width * page, dim)
    new = s["offsets"][1:] - s["offsets"][:-1]
    row = torch.arange(most, device=device).view(1, -1)
    real = row < new.view(-1, 1)
    source = torch.where(real, s["offsets"][:-1].view(-1, 1) + row, torch.zeros_like(row))
    q = s["q"][source].float().view(batch, most, kv_heads, heads // kv_heads, dim).permute(0, 2, 3, 1, 4)
    x = (q.reshape(batch, kv_heads, -1, dim) @ k.transpose(2, 3)).mul_(s["scale"]).view(batch, kv_heads, heads // kv_heads, most, width * page)
    place = ((s["lengths"].long() - new).view(-1, 1) + row).unsqueeze(2)
    key = torch.arange(width * page, device=device).view(1, 1, -1)
    seen = (key <= place) & real.unsqueeze(2)
    if s["window"]:
        seen &= (place - key < s["window"]) | (key < s["sinks"])
    x.masked_fill_(~seen.view(batch, 1, 1, most, width * page), -math.inf)
    top = x.amax(4, keepdim=True)
    top = torch.where(top > -math.inf, top, torch.zeros_like(top))
    p = x.sub_(top).exp_()
    total = p.sum(4, keepdim=True)
    y = (p.view(batch, kv_heads, -1, width * page) @ v).view(batch, kv_heads, heads // kv_heads, most, dim) / total
    lse = (torch.log(total) + top).squeeze(4)
    out, out_lse = torch.zeros_like(s["q"]), torch.zeros_like(s["out"][1])
    out[source[real]] = y.permute(0, 3, 1, 2, 4).reshape(batch, most, heads, dim)[real].to(out.dtype)
    out_lse[source[real]] = lse.permute(0, 3, 1, 2).reshape(batch, most, heads)[real]
    return out, out_lse


def _distribution(x, t):
    """softmax(x / t) in 64 bits, by rows; t = 0: all of it on the first of the largest."""
    x, t = x.double(), t.view(-1, 1).double()
    w = torch.exp((x - x.amax(1, keepdim=True)) / torch.where(t > 0, t, torch.ones_like(t)))
    first = torch.zeros_like(w).scatter_(1, x.argmax(1, keepdim=True), 1.0)
    return torch.where(t > 0, w / w.sum(1, keepdim=True), first)


def _verify(s):
    """A drafted token d is taken where u q(d) < p(d); the first that is not is replaced by a token from max(p - q, 0); behind
    the last comes one from p.  64 bits: values next to a border."""
    if own:
        return _library().verify_draft(s["target"], s["draft"], s["tokens"], s["offsets"], s["u"], temperature=s["temperature"], out=s["out"])
    offsets, tokens, most = s["offsets"], s["tokens"].long(), s["most"]
    rows, n = s["target"].shape
    batch, device = offsets.numel() - 1, tokens.device
    request = torch.arange(batch, device=device)
    t = s["temperature"] if isinstance(s["temperature"], torch.Tensor) else torch.full((batch,), s["temperature"], device=device)
    owner = torch.searchsorted(offsets, torch.arange(rows, device=device), right=True) - 1
    p = _distribution(s["target"], t[owner])
    tested = (torch.arange(rows, device=device) + 1 < offsets[owner + 1]).nonzero().view(-1)        # rows with a drafted token
    copied = torch.zeros((tested.numel(), n), dtype=torch.float64, device=device).scatter_(1, tokens[tested + 1].view(-1, 1), 1.0)
    q = copied
    if s["draft"] is not None:
        q = torch.where((t[owner[tested]] > 0).view(-1, 1), _distribution(s["draft"], t[owner[tested]]), copied)
    taken = s["u"][tested] * q.gather(1, tokens[tested + 1].view(-1, 1)).view(-1) < p[tested].gather(1, tokens[tested + 1].view(-1, 1)).view(-1)
    chain = torch.zeros((batch, most), dtype=torch.int64, device=device)
    chain[owner[tested], tested - offsets[owner[tested]]] = taken.to(torch.int64)
    accepted = torch.cumprod(chain, 1).sum(1)
    last = offsets[:-1] + accepted
    refused = (last + 1 < offsets[1:]).view(-1, 1)
    other = q[torch.where(refused.view(-1), last - request, torch.zeros_like(last))]
    left = torch.where(refused, (p[last] - other).clamp(min=0), p[last])
    reached = torch.cumsum(left, 1)
    aim = s["u"][offsets[1:] - 1].view(-1, 1) * reached[:, -1:]
    token = (reached > aim).to(torch.int8).argmax(1, keepdim=True)
    logprob = torch.log(p[last].gather(1, token)).view(-1)
    return accepted.to(torch.int32), token.view(-1).to(torch.int32), logprob.float(), torch.zeros_like(s["out"][3])


RUN = {"append": _append, "attention": _attention, "verify": _verify}


def run(state):
    return RUN[state["op"]](state)


# ------------------------------------------------------------------ the definitions in 64 bits


def _exact_append(s):
    """Scales of the pages, sequence by sequence."""
    scales = [s["cache"][2].double(), s["cache"][3].double()]
    page, table, offsets = s["cache"][0].shape[2], s["table"].tolist(), s["offsets"].tolist()
    for b, total in enumerate(s["lengths"].tolist()):
        new = offsets[b + 1] - offsets[b]
        at = total - new
        while at < total:
            end = min(total, (at // page + 1) * page)
            number = table[b][at // page]
            for x, scale in zip((s["k"], s["v"]), scales):
                part = x[offsets[b] + at - (total - new):offsets[b] + end - (total - new)].double()
                peak = part.abs().flatten(2).amax(2).amax(0) / 127
                scale[number] = torch.maximum(scale[number], peak) if at % page else peak
            at = end
    return None, None, scales[0], scales[1], None


def _exact_attention(s):
    """Sequence by sequence and head by head."""
    k_cache, v_cache, k_scale, v_scale = s["cache"]
    page, dim, heads = k_cache.shape[2], k_cache.shape[3], s["q"].shape[1]
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.zeros(s["q"].shape[:2], dtype=torch.float64, device="cuda")
    offsets, group = s["offsets"].tolist(), heads // k_cache.shape[1]
    for b, total in enumerate(s["lengths"].tolist()):
        a, e = offsets[b], offsets[b + 1]
        number = s["table"][b, :-(-total // page)].long()
        here = torch.arange(total - (e - a), total, device="cuda").view(-1, 1)
        there = torch.arange(total, device="cuda").view(1, -1)
        hidden = there > here
        if s["window"]:
            hidden = hidden | ((there <= here - s["window"]) & (there >= s["sinks"]))
        for h in range(heads):
            kv = h // group
            keys = (k_cache[number, kv].double() * k_scale[number, kv].double().view(-1, 1, 1)).view(-1, dim)[:total]
            values = (v_cache[number, kv].double() * v_scale[number, kv].double().view(-1, 1, 1)).view(-1, dim)[:total]
            logits = s["scale"] * torch.mm(s["q"][a:e, h].double(), keys.t())
            logits[hidden] = -math.inf
            norm = torch.logsumexp(logits, 1)
            out[a:e, h] = torch.mm(torch.exp(logits - norm.view(-1, 1)), values)
            lse[a:e, h] = norm
    return out, lse


def _exact_verify(s):
    """Request by request: log of the target's probability of the token that is returned."""
    offsets, tokens, u = s["offsets"].tolist(), s["tokens"].tolist(), s["u"].tolist()
    found = []
    for b in range(len(offsets) - 1):
        t = s["temperature"][b].item() if isinstance(s["temperature"], torch.Tensor) else torch.tensor(s["temperature"]).item()
        row, end = offsets[b], offsets[b + 1]
        if t == 0:
            found.append(0.0)
            continue
        left = None
        while True:
            p = torch.softmax(s["target"][row].double() / t, 0)
            if row + 1 == end:
                left = p
                break
            d = tokens[row + 1]
            if s["draft"] is None:
                q = torch.zeros_like(p)
                q[d] = 1.0
            else:
                q = torch.softmax(s["draft"][row - b].double() / t, 0)
            if not u[row] * float(q[d]) < float(p[d]):
                left = torch.relu(p - q)
                break
            row += 1
        running = left.cumsum(0)
        drawn = int((running <= u[end - 1] * running[-1]).sum())
        found.append(math.log(float(p[min(drawn, p.numel() - 1)])))
    return None, None, torch.tensor(found, dtype=torch.float64), None


EXACT = {"append": _exact_append, "attention": _exact_attention, "verify": _exact_verify}


def exact(case, seed):
    return EXACT[case["op"]](prepare(case, seed))
