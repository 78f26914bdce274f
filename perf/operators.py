"""The attention cache in 8 bits: the operators that hold, read and shrink it, as cases that can be timed.

A front end that runs its share of the layers token by token holds the keys and values of what it has seen, and so does
the back end that goes on from the features it is sent.  The cache keeps them by pages of 64 tokens of one sequence, in
8 bits with a scale for each page and head; the tokens of a page that is not full yet are kept as bf16.

A case names one pass: `ingest` (a batch of prompts goes into the cache and is read back from it), `step` (new tokens go
into the cache and attend over it: one token, a few drafted ones, or a prompt's chunk), or `evict` (the pages with the least attention leave
the sequences that have too many).  Where `own` is false the pass is made of elementary torch operations.
"""
import math

import torch

own = False

PAGE = 64
TINY = 2.0 ** -119                     # a page whose largest magnitude is below this holds zeros
LARGEST_STEP_TOKENS = 2 * 262016       # cached tokens of the largest step
LARGEST_PAIRS = 8 * 2048 * 2049 // 2 * 32   # query-key pairs of the largest prompt, over its heads
LARGEST_INGEST = 8 * 2048 * 8 * 128    # key elements of the largest batch of prompts
LARGEST_EVICT = 16384 * 8              # weights of the largest eviction

_DTYPE = {"f32": torch.float32, "bf16": torch.bfloat16}


def _step(name, dtype, seqs, past, new, heads, kv_heads, dim, mass):
    c = {"op": "step", "dtype": dtype, "seqs": seqs, "past_lo": past[0], "past_hi": past[1], "new_lo": new[0], "new_hi": new[1],
         "heads": heads, "kv_heads": kv_heads, "dim": dim, "mass": mass}
    return {"name": name, **c} if name else c


def _ingest(name, dtype, seqs, new, kv_heads, dim):
    c = {"op": "ingest", "dtype": dtype, "seqs": seqs, "past_lo": 0, "past_hi": 0, "new_lo": new[0], "new_hi": new[1],
         "heads": kv_heads, "kv_heads": kv_heads, "dim": dim, "mass": False}
    return {"name": name, **c} if name else c


def _evict(name, seqs, tokens, kv_heads, keep, sink, recent):
    c = {"op": "evict", "seqs": seqs, "past_lo": tokens[0], "past_hi": tokens[1], "kv_heads": kv_heads, "keep": keep, "sink": sink, "recent": recent}
    return {"name": name, **c} if name else c


def listed():
    return [
        # one device decodes one token of a short dialogue with a small model: pure latency
        _step("step_one", "bf16", 1, (77, 77), (1, 1), 12, 12, 64, False),
        # the 256 clients of a decoding step at the server, grouped heads, the weights kept for a later eviction
        _step("step_batch", "bf16", 256, (500, 2047), (1, 1), 64, 8, 128, True),
        # two long documents: the work is split over the cache
        _step("step_long", "bf16", 2, (261001, 262015), (1, 1), 32, 8, 128, False),
        # a model in fp32 with a head of its own for every query head
        _step("step_f32", "f32", 32, (100, 700), (1, 1), 12, 12, 64, True),
        # four drafted tokens of each sequence are checked at once; an odd head size
        _step("step_drafts", "bf16", 24, (3000, 5000), (4, 4), 28, 4, 80, False),
        # the prompts of a prefill batch
        _step("prompt_batch", "bf16", 8, (0, 0), (2048, 2048), 32, 8, 128, False),
        # chunks of long prompts behind a prefix that is in the cache, ragged, with their weights
        _step("prompt_chunk", "bf16", 3, (8000, 8200), (400, 700), 32, 8, 128, True),
        # short prompts in fp32, an odd head size and few heads
        _step("prompt_f32", "f32", 4, (0, 200), (100, 333), 10, 2, 80, True),
        # the prompts of a prefill batch go into the cache, whose content is then read for a hand-over
        _ingest("ingest_batch", "bf16", 8, (1500, 2048), 8, 128),
        # token rows of a vision transformer's size
        _ingest("ingest_f32", "f32", 16, (1, 197), 12, 64),
        # one long document gives up half of its pages
        _evict("evict_long", 1, (16384 * 64 - 5, 16384 * 64 - 5), 8, 8192, 4, 64),
        # 256 clients are held to a budget
        _evict("evict_batch", 256, (300, 4100), 8, 32, 1, 4),
    ]


def _log_uniform(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    op = rng.choices(("step", "prompt", "ingest", "evict"), (4, 3, 2, 2))[0]
    dtype = rng.choices(("bf16", "f32"), (3, 1))[0]
    dim = rng.choice((32, 64, 64, 80, 96, 128, 128, 128, 160, 256))
    kv_heads, group = rng.choice((1, 2, 4, 8, 8, 12)), rng.choice((1, 1, 2, 4, 4, 7, 8, 16))
    mass = rng.random() < 0.4
    if op == "evict":
        seqs = _log_uniform(rng, 1, 512)
        pages = _log_uniform(rng, 8, min(16384, max(9, LARGEST_EVICT // (seqs * kv_heads))))
        keep = rng.randint(max(3, pages // 4), pages)
        return _evict("", seqs, (pages * 32, pages * 64 - 1), kv_heads, keep, rng.randint(0, 2), rng.randint(1, max(1, keep // 4)))
    if op == "ingest":
        seqs = _log_uniform(rng, 1, 64)
        most = max(2, min(16384, LARGEST_INGEST // (seqs * kv_heads * dim)))
        new = _log_uniform(rng, 1, most)
        return _ingest("", dtype, seqs, (rng.randint(1, new), new), kv_heads, dim)
    if op == "step":
        seqs, new = _log_uniform(rng, 1, 256), rng.choice((1, 1, 1, 2, 5))
        most = max(64, min(262016, LARGEST_STEP_TOKENS * 8 * 128 // (seqs * new * max(8 * 128, kv_heads * dim * (4 if dtype == "f32" else 1)))))
        past = _log_uniform(rng, 16, most)
        return _step("", dtype, seqs, (rng.randint(past // 2, past), past), (new, new), kv_heads * group, kv_heads, dim, mass)
    seqs, new = _log_uniform(rng, 1, 16), _log_uniform(rng, 6, 4096)
    past = rng.choice((0, 0, _log_uniform(rng, 64, 16384)))
    most = LARGEST_PAIRS * 128 // max(128, dim) // (kv_heads * group) // (4 if dtype == "f32" else 1)
    while seqs * new * (past + new) > most:
        seqs, new, past = max(1, seqs // 2), max(6, new * 3 // 4), past // 2
    return _step("", dtype, seqs, (past // 2, past), (max(1, new // 2), new), kv_heads * group, kv_heads, dim, mass)


def _spread(i, lo, hi):
    return lo + (i * 2654435761 + 12345) % 4294967296 * (hi - lo + 1) // 4294967296


def _lengths(case):
    """Tokens in the cache before the pass and new ones, by sequence.  A sequence that is inside a page starts a new one
    at most by filling it, so that the pass can be made again on the same state (a prefix that is shared is whole pages)."""
    past = [_spread(i, case["past_lo"], case["past_hi"]) for i in range(case["seqs"])]
    if case["op"] == "evict":
        return past, [0] * len(past)
    new = [_spread(3 * i + 1, case["new_lo"], case["new_hi"]) for i in range(case["seqs"])]
    past = [p if p % PAGE == 0 or p % PAGE + n <= PAGE else -(-p // PAGE) * PAGE for p, n in zip(past, new)]
    return past, new


def work(case):
    past, new = _lengths(case)
    G = case["kv_heads"]
    if case["op"] == "evict":
        pages = sum(-(-p // PAGE) for p in past)
        kept = sum(min(-(-p // PAGE), case["keep"] + 1) for p in past)
        return {"bytes": 4 * (pages + kept) * (G + 1) + 4 * (pages - kept), "flops": pages * G}
    D, H, size = case["dim"], case["heads"], 4 if case["dtype"] == "f32" else 2
    total = sum(new)
    if case["op"] == "ingest":
        return {"bytes": 2 * total * G * D * (2 * size + 1), "flops": 4 * total * G * D}
    bytes_ = (2 * G * D + 2 * H * D) * total * size + 4 * H * total
    pairs = 0
    for p, n in zip(past, new):
        full, tail = (p + n) // PAGE, (p + n) % PAGE
        bytes_ += full * G * (2 * PAGE * D + 8) + tail * G * D * 4 + (4 * G * (full + (tail > 0)) if case["mass"] else 0)
        pairs += n * p + n * (n + 1) // 2
    return {"bytes": bytes_, "flops": 4 * D * H * pairs}


# ---- inputs, from the case and the seed alone --------------------------------------------------------------------------


def _inputs(case, seed):
    past, new = _lengths(case)
    gen = torch.Generator(device="cuda")
    gen.manual_seed(int(seed) * 7919 + 17)
    if case["op"] == "evict":
        pages = [p // PAGE for p in past]
        width = max(-(-p // PAGE) for p in past) + 2
        ids = torch.randperm(case["seqs"] * width, generator=gen, device="cuda").to(torch.int32).view(case["seqs"], width)
        # accumulated weights: a few heavy pages and a long tail; in steps of 1/64, so that equal sums are met
        mass = torch.rand(case["seqs"], case["kv_heads"], width, generator=gen, device="cuda").pow(6).mul(4096).round().div(64)
        held = (torch.tensor(past, device="cuda") + PAGE - 1) // PAGE
        mass *= torch.arange(width, device="cuda") < held[:, None, None]
        return {"pages": pages, "width": width, "table": ids, "mass": mass, "lens": torch.tensor(past, dtype=torch.int32, device="cuda")}
    G, D, H, dt = case["kv_heads"], case["dim"], case["heads"], _DTYPE[case["dtype"]]

    def tokens(n, heads, scale):
        x = torch.randn(n, heads, D, generator=gen, device="cuda", dtype=dt)
        # a few channels of every head are far larger than the others, and heads differ in scale
        chan = torch.ones(heads, D, device="cuda", dtype=dt)
        chan[:, :: max(1, D // 3)] = 3.0
        return x * (chan * (0.5 + torch.rand(heads, 1, generator=gen, device="cuda", dtype=dt)) * scale)

    x = {"past": past, "new": new, "old_k": tokens(sum(past), G, 1.0), "old_v": tokens(sum(past), G, 1.0),
         "k": tokens(sum(new), G, 1.0), "v": tokens(sum(new), G, 1.0), "q": tokens(sum(new), H, 0.7)}
    width = max(-(-(p + n) // PAGE) for p, n in zip(past, new))
    x["width"] = width
    # pages are handed out as they come free: in no order
    x["table"] = torch.randperm(case["seqs"] * width, generator=gen, device="cuda").to(torch.int32).view(case["seqs"], width)
    return x


def _starts(counts):
    s = [0]
    for c in counts:
        s.append(s[-1] + c)
    return torch.tensor(s, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    x = _inputs(case, seed)
    seqs = case["seqs"]
    if case["op"] == "evict":
        state = {"case": case, "table": x["table"], "mass": x["mass"], "lens": x["lens"]}
        if own:
            from paper_2511_11608_amd import binding
            state["kv"] = kv = binding.alloc_kv(seqs, case["kv_heads"], 32, seqs * x["width"], x["width"])
            kv.page_table.copy_(x["table"])
            kv.lens.copy_(x["lens"])
            state["out"] = binding.alloc_kv_evict(kv)
        return state
    G, D, H, dt = case["kv_heads"], case["dim"], case["heads"], _DTYPE[case["dtype"]]
    past, new = x["past"], x["new"]
    total = sum(new)
    state = {"case": case, "k": x["k"], "v": x["v"], "q": x["q"], "starts": _starts(new), "max_new": max(new),
             "max_len": max(p + n for p, n in zip(past, new)), "scale": 1.0 / math.sqrt(D)}
    if own:
        from paper_2511_11608_amd import binding
        state["kv"] = kv = binding.alloc_kv(seqs, G, D, seqs * x["width"], x["width"])
        kv.page_table.copy_(x["table"])
        if sum(past):
            kv.lens.copy_(torch.tensor(past, dtype=torch.int32))
            binding.slicer_kv_append(kv, x["old_k"], x["old_v"], _starts(past), max(past))
        kv.lens.copy_(torch.tensor([p + n for p, n in zip(past, new)], dtype=torch.int32))
        if case["op"] == "ingest":
            state["k_out"], state["v_out"] = torch.empty_like(x["k"]), torch.empty_like(x["v"])
        else:
            state["workspace"] = binding.alloc_kv_workspace(kv, H, total, state["max_new"], state["max_len"])
            state["out"] = torch.empty(total, H, D, dtype=dt, device="cuda")
            state["lse"] = torch.empty(total, H, dtype=torch.float32, device="cuda")
            state["mass"] = torch.zeros(seqs, G, x["width"], device="cuda") if case["mass"] else None
        return state
    # the plain cache: codes and scales by page, the tokens of the page that is not full apart; the last page is where
    # what belongs nowhere goes
    n_pages = seqs * x["width"]
    plain = {"codes": torch.zeros(2, n_pages + 1, G, PAGE, D, dtype=torch.int8, device="cuda"),
             "scales": torch.zeros(2, n_pages + 1, G, device="cuda"),
             "tail": torch.zeros(2, seqs, PAGE, G, D, dtype=torch.bfloat16, device="cuda"),
             "table": x["table"].long(), "none": n_pages, "width": x["width"]}
    state["plain"] = plain
    if sum(past):
        zero = torch.zeros(seqs, dtype=torch.long, device="cuda")
        _plain_append(plain, x["old_k"], x["old_v"], _places(past), zero, torch.tensor(past, device="cuda"))
    state["places"], state["past"], state["new"] = _places(new), torch.tensor(past, device="cuda"), torch.tensor(new, device="cuda")
    at = [(b, i) for b, n in enumerate(new) for i in range(n)] if total <= 4096 else None
    if at is None:
        b = torch.repeat_interleave(torch.arange(seqs, device="cuda"), state["new"])
        i = torch.arange(total, device="cuda") - state["starts"][:-1].long()[b]
    else:
        b, i = (torch.tensor(t, device="cuda") for t in zip(*at))
    state["row_seq"], state["row_at"] = b, i
    return state


def _places(counts):
    """[sequences, longest]: where a sequence's tokens are among the packed ones (clamped where it has none)."""
    n = torch.tensor(counts, device="cuda")
    first = torch.cumsum(n, 0) - n
    return (first[:, None] + torch.arange(max(counts), device="cuda")).clamp_(max=max(0, sum(counts) - 1))


# ---- the plain forms ---------------------------------------------------------------------------------------------------


def _plain_append(c, k, v, places, past, new):
    seqs, longest = places.shape
    held = past % PAGE                                          # tokens of the open page
    blocks = -(-(PAGE - 1 + longest) // PAGE)
    j = torch.arange(blocks * PAGE, device="cuda")
    from_new = (j - held[:, None])                              # place among the new tokens of what goes to base + j
    fresh = from_new >= 0
    x = torch.stack([k, v]).to(torch.bfloat16)
    rows = x[:, places.gather(1, from_new.clamp(0, longest - 1))]                      # [2, seqs, blocks * 64, G, D]
    rows = torch.where(fresh[None, :, :, None, None], rows, c["tail"][:, :, (j % PAGE)])
    there = j < (held + new)[:, None]
    rows = torch.where(there[None, :, :, None, None], rows, torch.zeros((), dtype=rows.dtype, device="cuda"))
    # every block as a page: one scale for each head
    blk = rows.view(2, seqs, blocks, PAGE, *rows.shape[3:]).float()
    amax = blk.abs().amax(dim=(3, 5))                                                  # [2, seqs, blocks, G]
    some = amax >= TINY
    # both quotients are the nearest in 32 bits: values of 8 bits lie on borders between two codes
    scale = torch.where(some, (amax.double() / 127).float(), torch.zeros_like(amax))
    inv = torch.where(some, (127 / amax.double()).float(), torch.zeros_like(amax))
    codes = (blk * inv[:, :, :, None, :, None]).round().clamp(-127, 127).to(torch.int8)
    page = torch.arange(blocks, device="cuda")
    full = (page + 1) * PAGE <= (held + new)[:, None]
    at = (past // PAGE)[:, None] + page
    ids = torch.where(full, c["table"].gather(1, at.clamp(max=c["width"] - 1)), c["none"]).view(-1)
    c["codes"][:, ids] = codes.permute(0, 1, 2, 4, 3, 5).reshape(2, seqs * blocks, *c["codes"].shape[2:])
    c["scales"][:, ids] = scale.view(2, seqs * blocks, -1)
    open_at = ((held + new) // PAGE * PAGE)[:, None] + torch.arange(PAGE, device="cuda")
    seq = torch.arange(seqs, device="cuda")[:, None]
    # (a block that was filled leaves the tail as it was: the pass can be made again)
    left = ((held + new) % PAGE > 0)[None, :, None, None, None]
    c["tail"].copy_(torch.where(left, rows[:, seq, open_at.clamp(max=blocks * PAGE - 1)], c["tail"]))


def _plain_held(c):
    """Keys and values by sequence in 32 bits: [2, seqs, G, pages * 64 + 64, D], the open page's tokens last."""
    t = c["table"]
    x = c["codes"][:, t].float() * c["scales"][:, t][..., None, None]                  # [2, seqs, pages, G, 64, D]
    x = x.permute(0, 1, 3, 2, 4, 5).flatten(3, 4)
    return torch.cat([x, c["tail"].permute(0, 1, 3, 2, 4).float()], dim=3)


def _plain_step(s):
    c, case = s["plain"], s["case"]
    _plain_append(c, s["k"], s["v"], s["places"], s["past"], s["new"])
    seqs, G, D, H = case["seqs"], case["kv_heads"], case["dim"], case["heads"]
    R, longest, pages = H // G, s["max_new"], c["width"]
    held_k, held_v = _plain_held(c)
    total_len = s["past"] + s["new"]
    full = total_len // PAGE
    j = torch.arange(pages * PAGE, device="cuda")
    t = torch.arange(PAGE, device="cuda")
    pos = torch.cat([torch.where(j < full[:, None] * PAGE, j, 1 << 40), torch.where(t < (total_len % PAGE)[:, None], full[:, None] * PAGE + t, 1 << 40)], dim=1)
    q = s["q"][s["places"]].float().view(seqs, longest, G, R, D).permute(0, 2, 1, 3, 4).reshape(seqs, G, longest * R, D)
    scores = torch.matmul(q, held_k.transpose(2, 3)).mul_(s["scale"]).view(seqs, G, longest, R, -1)
    last = s["past"][:, None] + torch.arange(longest, device="cuda")                   # the last position that a query sees
    row = torch.arange(longest, device="cuda") < s["new"][:, None]
    seen = (pos[:, None, :] <= last[:, :, None]) & row[:, :, None]
    scores.masked_fill_(~seen[:, None, :, None, :], float("-inf"))
    top = scores.amax(-1, keepdim=True)
    top = torch.where(top == float("-inf"), torch.zeros_like(top), top)
    p = scores.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    p.div_(torch.where(total > 0, total, torch.ones_like(total)))
    out = torch.matmul(p.view(seqs, G, longest * R, -1), held_v).view(seqs, G, longest, R, D)
    b, i = s["row_seq"], s["row_at"]
    out = out[b, :, i].reshape(-1, H, D).to(s["q"].dtype)
    lse = (top + total.log()).squeeze(-1)[b, :, i].reshape(-1, H)
    if not case["mass"]:
        return {"out": out, "lse": lse}
    w = p.sum((2, 3))                                                                  # [seqs, G, tokens]
    mass = torch.zeros(seqs, G, pages + 1, device="cuda")
    mass[:, :, :pages] = w[:, :, : pages * PAGE].view(seqs, G, pages, PAGE).sum(-1)
    mass.scatter_add_(2, full[:, None, None].expand(seqs, G, 1), w[:, :, pages * PAGE:].sum(-1, keepdim=True))
    return {"out": out, "lse": lse, "mass": mass[:, :, :pages]}


def _plain_ingest(s):
    c = s["plain"]
    _plain_append(c, s["k"], s["v"], s["places"], s["past"], s["new"])
    held = _plain_held(c)
    b, i = s["row_seq"], s["row_at"]
    full = s["new"] // PAGE * PAGE
    at = torch.where(i < full[b], i, c["width"] * PAGE + i - full[b])
    k, v = (h[b, :, at].to(s["k"].dtype) for h in held)
    return {"k": k, "v": v}


def _plain_evict(s):
    case, table, mass, lens = s["case"], s["table"], s["mass"], s["lens"]
    seqs, width = table.shape
    keep, sink, recent = case["keep"], case["sink"], case["recent"]
    page = torch.arange(width, device="cuda")
    full = (lens // PAGE)[:, None]
    weight = mass.double().sum(1)
    weight = torch.where((page < sink) | (page >= full - recent), float("inf"), weight)   # always kept
    weight = torch.where(page >= full, float("-inf"), weight)
    order = weight.sort(dim=1, descending=True, stable=True).indices
    stays = torch.zeros_like(weight, dtype=torch.bool).scatter_(1, order[:, :keep], True) if keep < width else torch.ones_like(weight, dtype=torch.bool)
    gone = ~stays & (page < full)
    # the pages that stay in their order, then what stands behind the complete pages; the places left over hold none
    move = gone.to(torch.int64).sort(dim=1, stable=True).indices
    n_gone = gone.sum(1, keepdim=True)
    behind = page >= width - n_gone
    out_table = torch.where(behind, -1, table.gather(1, move))
    out_mass = torch.where(behind[:, None], 0.0, mass.gather(2, move[:, None].expand_as(mass)))
    freed = (~gone).to(torch.int64).sort(dim=1, stable=True).indices
    freed = torch.where(page < n_gone, table.gather(1, freed), -1)
    return {"table": out_table, "lens": lens - PAGE * n_gone[:, 0].to(torch.int32), "mass": out_mass, "freed": freed, "n_freed": n_gone[:, 0].to(torch.int32)}


def run(state):
    case = state["case"]
    if not own:
        return {"step": _plain_step, "ingest": _plain_ingest, "evict": _plain_evict}[case["op"]](state)
    from paper_2511_11608_amd import binding
    kv = state["kv"]
    if case["op"] == "evict":
        o = state["out"]
        binding.slicer_kv_evict(kv, state["mass"], case["keep"], case["sink"], case["recent"], o)
        return {"table": o.page_table, "lens": o.lens, "mass": o.mass, "freed": o.freed, "n_freed": o.n_freed}
    binding.slicer_kv_append(kv, state["k"], state["v"], state["starts"], state["max_new"])
    if case["op"] == "ingest":
        binding.slicer_kv_read(kv, state["starts"], state["max_new"], state["k_out"], state["v_out"])
        return {"k": state["k_out"], "v": state["v_out"]}
    binding.slicer_kv_attend(kv, state["q"], state["starts"], state["max_new"], state["max_len"], state["scale"], state["out"],
                             state["workspace"], lse=state["lse"], mass=state["mass"])
    return {"out": state["out"], "lse": state["lse"], **({"mass": state["mass"]} if case["mass"] else {})}


# ---- the definition in 64 bits -----------------------------------------------------------------------------------------


def _exact_held(x):
    """The values that one sequence's cache stands for, [tokens, G, D] in 64 bits: complete pages by their codes, the others as bf16."""
    x = x.to(torch.bfloat16).double()
    full = x.shape[0] // PAGE * PAGE
    y = x[:full].view(-1, PAGE, *x.shape[1:])
    amax = y.abs().amax(dim=(1, 3), keepdim=True)
    scale = (amax / 127).float().double()
    inv = (127 / amax).float().double()                          # both are held in 32 bits, and so is the scaled value
    codes = (y * inv).float().double().round().clamp(-127, 127)
    y = torch.where(amax >= TINY, codes * scale, torch.zeros_like(y))
    return torch.cat([y.view(full, *x.shape[1:]), x[full:]])


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "evict":
        return _exact_evict(case, x)
    G, H, D = case["kv_heads"], case["heads"], case["dim"]
    past, new = x["past"], x["new"]
    outs, lses, ks, vs = [], [], [], []
    mass = torch.zeros(case["seqs"], G, x["width"], dtype=torch.float64, device="cuda")
    at_old = at_new = 0
    for b in range(case["seqs"]):
        p, n = past[b], new[b]
        k = _exact_held(torch.cat([x["old_k"][at_old: at_old + p], x["k"][at_new: at_new + n]]))
        v = _exact_held(torch.cat([x["old_v"][at_old: at_old + p], x["v"][at_new: at_new + n]]))
        q = x["q"][at_new: at_new + n].double()
        at_old, at_new = at_old + p, at_new + n
        if case["op"] == "ingest":
            ks.append(k)
            vs.append(v)
            continue
        out, lse = torch.empty_like(q), torch.empty(n, H, dtype=torch.float64, device="cuda")
        hidden = torch.arange(p + n, device="cuda") > p + torch.arange(n, device="cuda")[:, None]
        for h in range(H):
            g = h // (H // G)
            s = (q[:, h] @ k[:, g].T.contiguous()) / math.sqrt(D)
            s.masked_fill_(hidden, float("-inf"))
            lse[:, h] = torch.logsumexp(s, 1)
            w = s.sub_(lse[:, h, None]).exp_()
            out[:, h] = w @ v[:, g].contiguous()
            if case["mass"]:
                cols = w.sum(0)
                mass[b, g].index_add_(0, torch.arange(p + n, device="cuda") // PAGE, cols)
        outs.append(out)
        lses.append(lse)
    if case["op"] == "ingest":
        return {"k": torch.cat(ks), "v": torch.cat(vs)}
    return {"out": torch.cat(outs), "lse": torch.cat(lses), **({"mass": mass} if case["mass"] else {})}


def _exact_evict(case, x):
    table, mass, lens = x["table"].tolist(), x["mass"].double(), []
    order = mass.sum(1).tolist()
    width = x["width"]
    new_table, new_mass, freed, counts = [], torch.zeros_like(mass), [], []
    for b, full in enumerate(x["pages"]):
        keep = min(case["keep"], full)
        fixed = [p for p in range(full) if p < case["sink"] or p >= full - case["recent"]] if full > keep else list(range(full))
        free = sorted((p for p in range(full) if case["sink"] <= p < full - case["recent"]), key=lambda p: (-order[b][p], p)) if full > keep else []
        stay = sorted(fixed + free[: keep - len(fixed)])
        rest = stay + list(range(full, width))
        gone = sorted(set(range(full)) - set(stay))
        new_table.append([table[b][p] for p in rest] + [-1] * len(gone))
        new_mass[b, :, : len(rest)] = mass[b][:, torch.tensor(rest, device="cuda")]
        freed.append([table[b][p] for p in gone] + [-1] * (width - len(gone)))
        counts.append(len(gone))
        lens.append(int(x["lens"][b]) - PAGE * len(gone))
    def ints(t):
        return torch.tensor(t, dtype=torch.int32, device="cuda")
    return {"table": ints(new_table), "lens": ints(lens), "mass": new_mass, "freed": ints(freed), "n_freed": ints(counts)}
