"""What a long context keeps, and what a decode step reads of it, as performance cases.

Operators of this library, each beside a plain form in elementary torch operations:

  weights   the attention that new tokens pay to each cached token, summed over heads and new tokens and added to
            what was paid before
  keep      the tokens that stay when a context is cut: its start, its end and the most attended ones between
  bounds    the least and the greatest key of each page, head and element
  scores    for each block (page) and KV head, a bound on the scores that its keys can reach
  select    the blocks that a step attends: the first, the last and those of the largest bounds
  attend    decode attention over the selected blocks

Head counts and lengths are those of ``workloads/synth.py`` and ``perf/cases.py``.

A case is a dict of plain values:
  op        one of the above
  dtype     of the cache: "f32", "bf16" or "fp8" (codes; the queries are bf16)
  batch, hq, hkv, d
  page      tokens per page, 0 for a packed cache (weights)
  lo, hi    context lengths, uniform, drawn from ``mix``; hi bounds the call
  new_lo, new_hi   weights, bounds: new tokens a sequence, uniform (0: all of the context)
  decay     weights: factor of the earlier sums, 0 for none
  budget    keep: tokens that stay; select, attend: blocks
  first, last      keep, select: always kept, of the start and of the end
"""

import math
import random

import torch

own = False

DEVICE = "cuda:0"
K_SCALE, V_SCALE = 2.0 ** -6, 2.0 ** -5  # value = code * scale
FP8_MAX = 448.0


def _case(op, dtype, batch, hq, hkv, d, page, lo, hi, mix=1, new_lo=0, new_hi=0, decay=0.0, budget=0, first=0, last=0):
    return dict(op=op, dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, page=page, lo=lo, hi=hi, mix=mix, new_lo=new_lo,
                new_hi=new_hi, decay=decay, budget=budget, first=first, last=last)


def listed():
    def named(name, *a, **kw):
        return dict(_case(*a, **kw), name=name)

    return [
        # A serving batch's step over FP8 pages: its attention joins the running sums.
        named("weights_fp8_paged64_B8_L1k-7k_M1", "weights", "fp8", 8, 32, 8, 128, 64, 1000, 7000, new_lo=1, new_hi=1,
              decay=0.99),
        # An observation's attention to the cached history, from which the context is about to be cut.
        named("weights_bf16_B1_L24300_M300", "weights", "bf16", 1, 32, 8, 128, 0, 24300, 24300, mix=2, new_lo=300,
              new_hi=300),
        # One agent's history cut to a budget, the prompt and the recent buffer in it.
        named("keep_B1_L24300", "keep", "f32", 1, 32, 8, 128, 0, 24300, 24300, mix=3, budget=6001, first=1000,
              last=2000),
        # The same for a batch of long histories.
        named("keep_B8_L32k-128k", "keep", "f32", 8, 64, 8, 128, 0, 32768, 131072, mix=4, budget=16384, first=777,
              last=7000),
        # A decode step of a full batch: the page of each new token.
        named("bounds_fp8_paged64_B64_M1", "bounds", "fp8", 64, 32, 8, 128, 64, 1000, 7000, mix=5, new_lo=1, new_hi=1),
        # Observations of several agents.
        named("bounds_bf16_paged16_B8_M128-2048", "bounds", "bf16", 8, 32, 8, 128, 16, 8192, 32768, mix=6, new_lo=128,
              new_hi=2048),
        # One user's step over 32K.
        named("scores_bf16_paged64_B1_L32768", "scores", "bf16", 1, 32, 8, 128, 64, 32768, 32768, mix=7),
        # A batch of 128K contexts, FP8.
        named("scores_fp8_paged64_B8_L131072_G8", "scores", "fp8", 8, 64, 8, 128, 64, 131072, 131072, mix=8),
        # One user's step over 32K.
        named("select_paged64_B1_L32768", "select", "bf16", 1, 32, 8, 128, 64, 32768, 32768, mix=9, budget=64, first=1,
              last=2),
        # A full batch with small pages.
        named("select_paged16_B64_L2k-16k", "select", "bf16", 64, 32, 8, 128, 16, 2048, 16384, mix=10, budget=128,
              first=4, last=8),
        # One user's step over 32K: 4096 tokens of it.
        named("attend_bf16_paged64_B1_L32768_K64", "attend", "bf16", 1, 32, 8, 128, 64, 32768, 32768, mix=11, budget=64),
        # A batch of 128K contexts: a sixteenth of each.
        named("attend_bf16_paged64_B8_L131072_G8_K128", "attend", "bf16", 8, 64, 8, 128, 64, 131072, 131072, mix=12,
              budget=128),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_CACHE_BYTES = 1 << 30   # of a drawn case
MAX_WEIGHTS_FLOPS = 6.0e10
MAX_SCORES = 1 << 28        # padded scores of a drawn weights case, as the plain form holds them
MAX_SELECTED = 1 << 26      # padded key elements of a drawn attend case, likewise
MAX_BYTES = 270_000_000     # of a drawn case's work


def draw(rng):
    """One more case: the listed kinds over their ranges (lengths and batches log-uniform, odd sizes included)."""
    op = rng.choice(["weights", "weights", "weights", "keep", "keep", "bounds", "scores", "scores", "select", "attend",
                     "attend"])
    mix = rng.randrange(1 << 30)
    while True:
        hkv = rng.choice([2, 4, 8, 8])
        hq = hkv * rng.choice([1, 2, 4, 4, 8, 16])
        d = rng.choice([128, 128, 64])
        dtype = rng.choice(["bf16", "bf16", "fp8", "fp8", "f32"])
        page = rng.choice([16, 16, 64, 64, 128, 8])
        hi = _log_int(rng, 200, 131072 if op in ("keep", "scores", "select") else 32768)
        lo = max(1, int(hi * rng.uniform(0.1, 1.0)))
        batch = _log_int(rng, 1, 64)
        kw = {}
        if op == "weights":
            page = rng.choice([0, 16, 64, 1])
            m = rng.choice([1, _log_int(rng, 2, min(hi, 512))])
            lo, kw = max(m, lo), dict(new_lo=max(1, int(m * rng.uniform(0.1, 1.0))), new_hi=m,
                                      decay=rng.choice([0.0, 1.0, 0.9]))
        elif op == "bounds":
            m = rng.choice([1, _log_int(rng, 2, hi), 0])
            lo, kw = max(m, lo), dict(new_lo=max(1, int(m * rng.uniform(0.1, 1.0))) if m else 0, new_hi=m)
        elif op == "keep":
            budget = _log_int(rng, 50, 16384)
            first = rng.randint(0, budget // 4)
            page, kw = 0, dict(budget=budget, first=first, last=rng.randint(1, budget // 2))
        elif op in ("select", "attend"):
            budget = _log_int(rng, 2, 256)
            kw = dict(budget=budget, first=rng.randint(0, 1), last=1 if op == "attend" else rng.randint(1, max(1, budget // 2)))
        c = _case(op, dtype, batch, hq, hkv, d, page, lo, hi, mix=mix, **kw)
        lens = _lengths(c)
        caches = {"weights": 1, "bounds": 1, "attend": 2}.get(op, 2.0 / max(page, 1) if op == "scores" else 0)
        if caches * sum(lens) * hkv * d * _elem_bytes(c) > MAX_CACHE_BYTES:
            continue
        if work(c)["bytes"] > MAX_BYTES:
            continue
        if op == "weights" and (work(c)["flops"] > MAX_WEIGHTS_FLOPS or
                                batch * hq * max(_new_tokens(c)) * max(lens) > MAX_SCORES or
                                batch * hkv * max(lens) * d > MAX_SCORES):
            continue
        if op == "keep" and batch * hi > 8 * 131072 or op == "select" and batch * hkv * _pages_of(hi, page) > 1 << 19:
            continue
        if op == "scores" and 2 * batch * hkv * _pages_of(hi, page) * d > MAX_SELECTED:
            continue
        if op == "attend" and batch * hkv * min(budget, _pages_of(hi, page)) * page * d > MAX_SELECTED:
            continue
        return c


# ------------------------------------------------------------------ sizes


def _lengths(case):
    r = random.Random(case["mix"])
    return [r.randint(case["lo"], case["hi"]) for _ in range(case["batch"])]


def _new_tokens(case):
    if case["new_hi"] == 0:
        return _lengths(case)
    r = random.Random(case["mix"] + 1)
    return [min(r.randint(case["new_lo"], case["new_hi"]), n) for n in _lengths(case)]


def _elem_bytes(case):
    return {"f32": 4, "bf16": 2, "fp8": 1}[case["dtype"]]


def _pages_of(n, page):
    return -(-n // page)


def _blocks(case):
    """Selected blocks of each sequence, and the tokens in them (the last block is always among them)."""
    page, got = case["page"], []
    for n in _lengths(case):
        blocks = min(case["budget"], _pages_of(n, page))
        got.append((blocks, (blocks - 1) * page + n - (_pages_of(n, page) - 1) * page))
    return got


def work(case):
    """Each input read once, each output written once."""
    lens, hq, hkv, d, page = _lengths(case), case["hq"], case["hkv"], case["d"], case["page"]
    e, qe, op = _elem_bytes(case), 4 if case["dtype"] == "f32" else 2, case["op"]
    if op == "weights":
        new = _new_tokens(case)
        pairs = sum((n - m) * m + m * (m + 1) // 2 for n, m in zip(lens, new))
        sums = 4 * sum(lens) + (4 * sum(n - m for n, m in zip(lens, new)) if case["decay"] else 0)
        return {"bytes": sum(lens) * hkv * d * e + sum(new) * hq * (d * qe + 4) + sums, "flops": 2 * d * hq * pairs}
    if op == "keep":
        return {"bytes": 4 * sum(lens) + 8 * sum(min(case["budget"], n) for n in lens), "flops": sum(lens)}
    if op == "bounds":
        tokens = blocks = 0
        for n, m in zip(lens, _new_tokens(case)):
            begin = (n - m) // page
            blocks += _pages_of(n, page) - begin
            tokens += n - begin * page
        return {"bytes": (tokens + 2 * blocks) * hkv * d * e, "flops": 2 * tokens * hkv * d}
    blocks = sum(_pages_of(n, page) for n in lens)
    if op == "scores":
        return {"bytes": blocks * hkv * (2 * d * e + 4) + case["batch"] * hq * d * qe, "flops": 4 * d * hq * blocks}
    if op == "select":
        return {"bytes": 4 * hkv * (blocks + 2 * sum(b for b, _ in _blocks(case))), "flops": hkv * blocks}
    tokens = sum(t for _, t in _blocks(case))
    return {"bytes": tokens * 2 * hkv * d * e + case["batch"] * hq * (d * (qe + 4) + 4), "flops": 4 * d * hq * tokens}


# ------------------------------------------------------------------ inputs


def _pair(shape, dtype):
    """K and V caches in one allocation, V's base 256 bytes past K's modulo 512 (the library's advice on placement)."""
    n = math.prod(shape)
    size = torch.empty((), dtype=dtype).element_size()
    gap = (256 - n * size) % 512 // size
    buf = torch.zeros(2 * n + gap, dtype=dtype, device=DEVICE)
    return buf[:n].view(shape), buf[n + gap:2 * n + gap].view(shape)


def _fill(t, g, scale):
    """N(0, 1) values into a cache tensor, in parts (FP8: codes of the values divided by the scale)."""
    rows = t.view(-1, t.shape[-1])
    step = max(1, (1 << 26) // rows.shape[1])
    for i in range(0, rows.shape[0], step):
        part = rows[i:i + step]
        x = torch.randn(part.shape, generator=g, device=t.device)
        if t.dtype == torch.uint8:
            x = (x / scale).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        part.copy_(x)


def _ints(values, dtype):
    return torch.tensor(values, dtype=dtype, device=DEVICE)


def _starts(counts):
    return _ints([sum(counts[:b]) for b in range(len(counts))], torch.int64)


def _dtypes(case):
    """(cache, queries)"""
    return {"f32": (torch.float32, torch.float32), "bf16": (torch.bfloat16, torch.bfloat16),
            "fp8": (torch.uint8, torch.bfloat16)}[case["dtype"]]


def _table(case, g):
    """Pages of every sequence, in a random order of the pool; (block table, pages)."""
    counts = [_pages_of(n, case["page"]) for n in _lengths(case)]
    perm = torch.randperm(sum(counts), generator=g, device=DEVICE).to(torch.int32)
    table = torch.full((len(counts), _pages_of(case["hi"], case["page"])), -1, dtype=torch.int32, device=DEVICE)
    for b, n in enumerate(counts):
        first = sum(counts[:b])
        table[b, :n] = perm[first:first + n]
    return table, sum(counts)


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    lens, hq, hkv, d, page, op = _lengths(case), case["hq"], case["hkv"], case["d"], case["page"], case["op"]
    cache_dtype, q_dtype = _dtypes(case)
    x = dict(case=case, ctx_lens=_ints(lens, torch.int32))
    if op == "keep":
        # Sums of attention weights: a few tokens get most, many nearly the same little, some none that counts.
        w = torch.randn((case["batch"], case["hi"]), generator=g, device=DEVICE).mul_(3).exp_()
        x["weights"] = w.masked_fill_(torch.rand(w.shape, generator=g, device=DEVICE) < 0.05, 0.0)
        shape = (case["batch"], case["budget"])
        x["keep"] = torch.full(shape, -1, dtype=torch.int32, device=DEVICE)
        x["kept"] = torch.zeros(shape, device=DEVICE)
        return x
    if page:
        x["block_table"], total = _table(case, g)
    if op == "select":
        nb = _pages_of(case["hi"], page)
        # Bounds of a head's scores; some blocks are alike.
        s = torch.randn((case["batch"], hkv, nb), generator=g, device=DEVICE).mul_(4)
        x["scores"] = torch.where(torch.rand(s.shape, generator=g, device=DEVICE) < 0.2, s.round(), s)
        x["table"] = torch.full((case["batch"], hkv, case["budget"]), -1, dtype=torch.int32, device=DEVICE)
        x["lens"] = torch.zeros(case["batch"], dtype=torch.int32, device=DEVICE)
        return x
    if op == "scores":
        # Least and greatest of a page's keys, far from 0 by what that many normal values reach.
        x["bounds"] = torch.empty((total, hkv, 2, d), dtype=cache_dtype, device=DEVICE)
        mid, half = (torch.empty((total, hkv, d), device=DEVICE) for _ in range(2))
        _fill(mid, g, 1.0)
        _fill(half, g, 1.0)
        mid.mul_(0.3)
        half.mul_(0.2).add_(math.sqrt(2 * math.log(page + 1))).abs_()
        ends = torch.stack([mid - half, mid + half], dim=2)
        if case["dtype"] == "fp8":
            ends = (ends / K_SCALE).clamp_(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        x["bounds"].copy_(ends)
        x["q"] = torch.randn((case["batch"], hq, d), generator=g, device=DEVICE).to(q_dtype)
        x["scores"] = torch.zeros((case["batch"], hkv, _pages_of(case["hi"], page)), device=DEVICE)
        return x
    pool = (total, page, hkv, d) if page else (sum(lens), hkv, d)
    if op == "attend":
        x["k"], x["v"] = _pair(pool, cache_dtype)
        _fill(x["v"], g, V_SCALE)
    else:
        x["k"] = torch.empty(pool, dtype=cache_dtype, device=DEVICE)
    _fill(x["k"], g, K_SCALE)
    if op == "attend":
        blocks = _blocks(case)
        x["lens"] = _ints([t for _, t in blocks], torch.int32)
        x["table"] = torch.zeros((case["batch"], hkv, max(n for n, _ in blocks)), dtype=torch.int32, device=DEVICE)
        for b, (n, _) in enumerate(blocks):
            # The last block and any others, for each head, in ascending order.
            last = _pages_of(lens[b], page) - 1
            at = torch.rand((hkv, last), generator=g, device=DEVICE).argsort(1)[:, :n - 1].sort(1).values
            at = torch.cat([at, torch.full((hkv, 1), last, device=DEVICE)], dim=1)
            x["table"][b, :, :n] = x["block_table"][b][at]
        x["q"] = torch.randn((case["batch"], hq, d), generator=g, device=DEVICE).to(q_dtype)
        return x
    new = _new_tokens(case)
    x["q_start"], x["q_lens"], x["max_q_len"] = _starts(new), _ints(new, torch.int32), max(new)
    if op == "bounds":
        x["bounds"] = torch.zeros((total, hkv, 2, d), dtype=cache_dtype, device=DEVICE)
        return x
    if not page:
        x["seq_start"] = _starts(lens)
    x["q"] = torch.randn((sum(new), hq, d), generator=g, device=DEVICE).to(q_dtype)
    x["prior"] = torch.rand((case["batch"], case["hi"]), generator=g, device=DEVICE).mul_(6).exp_() if case["decay"] else None
    x["out"] = torch.zeros((case["batch"], case["hi"]), device=DEVICE)
    # What the attention call returned beside its output.
    s, _ = _plain_logits(x)
    top = s.amax(-1, keepdim=True)
    x["lse"] = _packed(x, (s.sub_(top).exp_().sum(-1, keepdim=True).log() + top)[..., 0])
    return x


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:
        from paper_2605_30842_amd.binding import DecodeAttention

        scales = dict(k_scale=K_SCALE, v_scale=V_SCALE) if case["dtype"] == "fp8" else {}
        x["op"] = DecodeAttention(case["hq"], case["hkv"], case["d"], case["dtype"], 1.0 / math.sqrt(case["d"]),
                                  case["batch"], max(case["hi"], case["budget"] * case["page"]), **scales)
    return x


# ------------------------------------------------------------------ one pass


def run(x):
    kind = x["case"]["op"]
    if kind == "weights":
        return dict(weights=_own_weights(x) if own else _plain_weights(x))
    if kind == "keep":
        return dict(zip(("keep", "keep_lens", "kept"), _own_keep(x) if own else _plain_keep(x)))
    if kind == "bounds":
        got = _own_bounds(x) if own else _plain_bounds(x)
        return dict(bounds=got.view(torch.float8_e4m3fn) if x["case"]["dtype"] == "fp8" else got)
    if kind == "scores":
        return dict(scores=_own_scores(x) if own else _plain_scores(x))
    if kind == "select":
        return dict(zip(("table", "lens"), _own_select(x) if own else _plain_select(x)))
    return dict(zip(("out", "lse"), _own_attend(x) if own else _plain_attend(x)))


def _own_weights(x):
    case, more = x["case"], dict(prior=x["prior"], decay=x["case"]["decay"], out=x["out"])
    if case["new_hi"] != 1:  # else one new token a sequence, the step of a decode loop
        more.update(q_start=x["q_start"], q_lens=x["q_lens"], max_q_len=x["max_q_len"])
    if case["page"]:
        return x["op"].attn_weights_paged(x["q"], x["lse"], x["k"], x["block_table"], x["ctx_lens"], case["hi"], **more)
    return x["op"].attn_weights(x["q"], x["lse"], x["k"], x["seq_start"], x["ctx_lens"], case["hi"], **more)


def _own_keep(x):
    case = x["case"]
    keep, _, lens, kept = x["op"].keep_tokens(x["weights"], x["ctx_lens"], case["hi"], case["budget"], first=case["first"],
                                              last=case["last"], keep=x["keep"], kept=x["kept"])
    return keep, lens, kept


def _own_bounds(x):
    case, more = x["case"], {}
    if case["new_hi"] != 1:
        more = dict(q_lens=x["q_lens"], max_q_len=x["max_q_len"])
    return x["op"].block_bounds(x["k"], x["block_table"], x["ctx_lens"], case["hi"], x["bounds"], **more)


def _own_scores(x):
    case = x["case"]
    return x["op"].block_scores(x["q"], x["bounds"], case["page"], x["block_table"], x["ctx_lens"], case["hi"],
                                scores=x["scores"])


def _own_select(x):
    case = x["case"]
    return x["op"].block_select(x["scores"], case["page"], x["block_table"], x["ctx_lens"], case["hi"], case["budget"],
                                first=case["first"], last=case["last"], table=x["table"], lens=x["lens"])


def _own_attend(x):
    case = x["case"]
    lse = torch.empty(x["q"].shape[:2], dtype=torch.float32, device=DEVICE)
    return x["op"].block_forward(x["q"], x["k"], x["v"], x["table"], x["lens"],
                               x["table"].shape[2] * case["page"], lse=lse)


# ------------------------------------------------------------------ the same in elementary operations


def _wide32(case, t, scale):
    if case["dtype"] == "fp8":
        return t.view(torch.float8_e4m3fn).float() * scale
    return t.float()


def _plain_logits(x):
    """Scores of the new tokens, -inf where a token is not seen, [batch, hkv, group, new, keys], and the keys' rows."""
    case, ctx = x["case"], x["ctx_lens"].long()[:, None]
    hkv, group, d = case["hkv"], case["hq"] // case["hkv"], case["d"]
    batch, most, m = case["batch"], max(_lengths(case)), x["max_q_len"]
    key = torch.arange(most, device=DEVICE)[None, :]
    t = torch.minimum(key, ctx - 1)
    if case["page"]:
        seq = torch.arange(batch, device=DEVICE)[:, None]
        rows = x["block_table"][seq, t // case["page"]].long() * case["page"] + t % case["page"]
    else:
        rows = x["seq_start"][:, None] + t
    k = _wide32(case, x["k"].view(-1, hkv, d)[rows], K_SCALE).permute(0, 2, 3, 1).contiguous()  # [batch, hkv, d, most]
    i = torch.arange(m, device=DEVICE)[None, :]
    at = (x["q_start"][:, None] + i).clamp(max=x["q"].shape[0] - 1)
    q = x["q"].float()[at].unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).reshape(batch, hkv, group * m, d)
    s = torch.matmul(q, k).view(batch, hkv, group, m, most).div_(math.sqrt(d))
    seen = (key[:, None] <= (ctx - x["q_lens"].long()[:, None] + i)[..., None]) & (i < x["q_lens"][:, None])[..., None]
    # (A row past a sequence's new tokens sees nothing; its largest score is set to 0 by whoever needs one.)
    return s.masked_fill_(~seen[:, None, None], -math.inf), seen


def _packed(x, t):
    """[batch, hkv, group, new] -> [rows, hq] of the packed new tokens."""
    n = torch.arange(x["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(x["q_start"], n, right=True) - 1
    return t.permute(0, 3, 1, 2)[b, n - x["q_start"][b]].flatten(1, 2).contiguous()


def _plain_weights(x):
    case = x["case"]
    s, _ = _plain_logits(x)
    i = torch.arange(x["max_q_len"], device=DEVICE)[None, :]
    at = (x["q_start"][:, None] + i).clamp(max=x["q"].shape[0] - 1)
    lse = x["lse"][at].unflatten(2, (case["hkv"], -1)).permute(0, 2, 3, 1)
    w = s.sub_(lse[..., None]).exp_().sum((1, 2, 3))  # [batch, keys]
    key = torch.arange(w.shape[1], device=DEVICE)[None, :]
    if case["decay"]:
        old = key < (x["ctx_lens"] - x["q_lens"])[:, None]
        w = w + torch.where(old, x["prior"][:, :w.shape[1]] * case["decay"], 0.0)
    out = x["out"][:, :w.shape[1]]
    out.copy_(torch.where(key < x["ctx_lens"][:, None], w, out))
    return x["out"]


def _largest(scores, lens, count, most, first, last):
    """The places of the `count` entries of each row that are kept, ascending, and which of the `most` columns hold one:
    the first, the last, then the largest, the lower place where two are equal."""
    n = torch.arange(scores.shape[1], device=DEVICE)[None, :]
    live = n < lens[:, None]
    forced = ((n < first) | (n >= lens[:, None] - last)) & live
    ranked = torch.where(forced, math.inf, torch.where(live, scores, -math.inf))
    order = torch.sort(ranked, dim=1, descending=True, stable=True).indices[:, :most]
    held = torch.arange(order.shape[1], device=DEVICE)[None, :] < count[:, None]
    return torch.where(held, order, scores.shape[1]).sort(1).values, held


def _plain_keep(x):
    case = x["case"]
    count = x["ctx_lens"].clamp(max=case["budget"])
    at, held = _largest(x["weights"], x["ctx_lens"], count, case["budget"], case["first"], case["last"])
    keep, kept = x["keep"][:, :at.shape[1]], x["kept"][:, :at.shape[1]]
    keep.copy_(torch.where(held, at, keep))
    kept.copy_(torch.where(held, x["weights"].gather(1, torch.where(held, at, 0)), kept))
    return x["keep"], count, x["kept"]


def _plain_bounds(x):
    case, page, hkv, d = x["case"], x["case"]["page"], x["case"]["hkv"], x["case"]["d"]
    ctx, new = x["ctx_lens"].long(), x["q_lens"].long()
    col = torch.arange(x["block_table"].shape[1], device=DEVICE)[None, :]
    touched = (col >= ((ctx - new) // page)[:, None]) & (col * page < ctx[:, None])
    b, n = touched.nonzero(as_tuple=True)
    pages = x["block_table"][b, n].long()
    live = torch.arange(page, device=DEVICE)[None, :] < (ctx[b] - n * page)[:, None]
    k = x["k"][pages]
    k = (k.view(torch.float8_e4m3fn) if case["dtype"] == "fp8" else k).float()  # a code orders as its value
    live = live[:, :, None, None]
    ends = torch.stack([torch.where(live, k, math.inf).amin(1), torch.where(live, k, -math.inf).amax(1)], dim=2)
    if case["dtype"] == "fp8":
        x["bounds"][pages] = ends.to(torch.float8_e4m3fn).view(torch.uint8)
    else:
        x["bounds"][pages] = ends.to(x["bounds"].dtype)
    return x["bounds"]


def _plain_scores(x):
    case, hkv, d = x["case"], x["case"]["hkv"], x["case"]["d"]
    ends = _wide32(case, x["bounds"][x["block_table"].long().clamp(min=0)], K_SCALE)  # [batch, blocks, hkv, 2, d]
    ends = ends.permute(0, 2, 3, 4, 1).contiguous()  # [batch, hkv, 2, d, blocks]
    q = x["q"].float().view(case["batch"], hkv, -1, d)
    s = torch.matmul(q.clamp(max=0), ends[:, :, 0].contiguous()) + torch.matmul(q.clamp(min=0), ends[:, :, 1].contiguous())
    s = s.amax(2) / math.sqrt(d)
    n = torch.arange(s.shape[2], device=DEVICE)
    live = n * case["page"] < x["ctx_lens"][:, None, None]
    x["scores"].copy_(torch.where(live, s, x["scores"]))
    return x["scores"]


def _plain_select(x):
    case, page, hkv = x["case"], x["case"]["page"], x["case"]["hkv"]
    blocks = (x["ctx_lens"] + page - 1) // page
    count = blocks.clamp(max=case["budget"])
    at, held = _largest(x["scores"].flatten(0, 1), blocks.repeat_interleave(hkv), count.repeat_interleave(hkv),
                        case["budget"], case["first"], case["last"])
    row = torch.arange(at.shape[0], device=DEVICE)[:, None] // hkv
    table = x["table"].view(-1, case["budget"])[:, :at.shape[1]]
    table.copy_(torch.where(held, x["block_table"][row, torch.where(held, at, 0)], table))
    x["lens"].copy_((count - 1) * page + x["ctx_lens"] - (blocks - 1) * page)
    return x["table"], x["lens"]


def _plain_attend(x):
    case, page, hkv, d = x["case"], x["case"]["page"], x["case"]["hkv"], x["case"]["d"]
    batch, most = case["batch"], x["table"].shape[2] * page
    t = torch.arange(most, device=DEVICE)[None, None, :]
    seq, head = (torch.arange(n, device=DEVICE) for n in (batch, hkv))
    t = torch.minimum(t, x["lens"][:, None, None].long() - 1).expand(batch, hkv, most)
    pages = x["table"][seq[:, None, None], head[None, :, None], t // page].long()

    def rows(cache, scale):
        return _wide32(case, cache[pages, t % page, head[None, :, None]], scale)  # [batch, hkv, most, d]

    q = x["q"].float().view(batch, hkv, -1, d)
    s = torch.matmul(q, rows(x["k"], K_SCALE).transpose(2, 3).contiguous()) / math.sqrt(d)
    s = s.masked_fill(torch.arange(most, device=DEVICE) >= x["lens"][:, None, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s = (s - top).exp()
    total = s.sum(-1, keepdim=True)
    out = torch.matmul(s / total, rows(x["v"], V_SCALE))
    return out.flatten(1, 2), (top + total.log())[..., 0].flatten(1, 2)


# ------------------------------------------------------------------ the same in 64 bits


def _wide(case, t, scale):
    if case["dtype"] == "fp8":
        return t.view(torch.float8_e4m3fn).to(torch.float32).to(torch.float64) * scale
    return t.to(torch.float64)


def _exact_rows(case, x, b, n):
    """Cache rows of tokens 0 .. n - 1 of sequence b."""
    if case["page"] == 0:
        begin = int(x["seq_start"][b])
        return torch.arange(begin, begin + n, device=DEVICE)
    pages = x["block_table"][b, :_pages_of(n, case["page"])].to(torch.int64)
    return (pages[:, None] * case["page"] + torch.arange(case["page"], device=DEVICE)).flatten()[:n]


def _exact_weights(case, x):
    out, group, first = x["out"].double().clone(), case["hq"] // case["hkv"], 0
    for b, (n, m) in enumerate(zip(_lengths(case), _new_tokens(case))):
        w = torch.zeros(n, dtype=torch.float64, device=DEVICE)
        if case["decay"]:
            w[:n - m] = x["prior"][b, :n - m].double() * case["decay"]
        rows = _exact_rows(case, x, b, n)
        seen = torch.ones((m, n), dtype=torch.bool, device=DEVICE).tril(n - m)
        for h in range(case["hkv"]):
            k = _wide(case, x["k"].view(-1, case["hkv"], case["d"])[rows, h], K_SCALE).t().contiguous()
            for j in range(h * group, (h + 1) * group):
                s = x["q"][first:first + m, j].double() @ k * case["d"] ** -0.5
                p = torch.exp(s - x["lse"][first:first + m, j, None].double())
                w += (p * seen).sum(0)
        out[b, :n] = w
        first += m
    return dict(weights=out)


def _exact_keep(case, x):
    kept = x["kept"].double().clone()
    for b, n in enumerate(_lengths(case)):
        w, count = x["weights"][b, :n], min(case["budget"], n)
        lo, hi = min(case["first"], n), max(n - case["last"], 0)
        if n > count:
            free = count - lo - (n - hi)
            stay = torch.ones(n, dtype=torch.bool, device=DEVICE)
            stay[lo:hi] = False
            if free > 0:
                least = torch.topk(w[lo:hi], free).values[-1]
                middle = w[lo:hi] > least
                ties = (w[lo:hi] == least).nonzero()[:free - int(middle.sum()), 0]
                middle[ties] = True
                stay[lo:hi] = middle
            w = w[stay]
        kept[b, :count] = w.double()
    return dict(keep=None, keep_lens=None, kept=kept)


def _exact_bounds(case, x):
    page = case["page"]
    out = _wide(case, x["bounds"], 1.0).clone()
    for b, (n, m) in enumerate(zip(_lengths(case), _new_tokens(case))):
        for i in range((n - m) // page, _pages_of(n, page)):
            p = int(x["block_table"][b, i])
            k = _wide(case, x["k"][p, :min(page, n - i * page)], 1.0)
            out[p, :, 0], out[p, :, 1] = k.min(0).values, k.max(0).values
    return dict(bounds=out)


def _exact_scores(case, x):
    out, group = x["scores"].double().clone(), case["hq"] // case["hkv"]
    for b, n in enumerate(_lengths(case)):
        nb = _pages_of(n, case["page"])
        ends = _wide(case, x["bounds"][x["block_table"][b, :nb].long()], K_SCALE)
        for h in range(case["hkv"]):
            best = torch.full((nb,), -math.inf, dtype=torch.float64, device=DEVICE)
            for j in range(h * group, (h + 1) * group):
                q = x["q"][b, j].double()
                reach = torch.maximum(ends[:, h, 0] * q, ends[:, h, 1] * q).sum(1) * case["d"] ** -0.5
                best = torch.maximum(best, reach)
            out[b, h, :nb] = best
    return dict(scores=out)


def _exact_attend(case, x):
    group = case["hq"] // case["hkv"]
    out = torch.zeros((case["batch"], case["hq"], case["d"]), dtype=torch.float64, device=DEVICE)
    lse = torch.zeros((case["batch"], case["hq"]), dtype=torch.float64, device=DEVICE)
    for b, (blocks, tokens) in enumerate(_blocks(case)):
        for h in range(case["hkv"]):
            pages = x["table"][b, h, :blocks].long()
            k = _wide(case, x["k"][pages, :, h].flatten(0, 1)[:tokens], K_SCALE)
            v = _wide(case, x["v"][pages, :, h].flatten(0, 1)[:tokens], V_SCALE)
            for j in range(h * group, (h + 1) * group):
                s = (k * x["q"][b, j].double()).sum(1) * case["d"] ** -0.5
                lse[b, j] = torch.logsumexp(s, 0)
                out[b, j] = (torch.exp(s - lse[b, j])[:, None] * v).sum(0)
    return dict(out=out, lse=lse)


def exact(case, seed):
    x = _inputs(case, seed)
    if case["op"] == "select":
        return None
    return {"weights": _exact_weights, "keep": _exact_keep, "bounds": _exact_bounds, "scores": _exact_scores,
            "attend": _exact_attend}[case["op"]](case, x)
