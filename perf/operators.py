"""What surrounds attention in a program that serves from a KV cache, as performance cases.

Three groups of operators of this library, each beside a plain form in elementary torch operations:

  rope_append  a chunk's queries and keys normalised for each head, rotated to their positions, the keys
               and values stored in the cache in its type
  prefill      attention of a chunk of new tokens over an FP8 cache
  reserve, fork, compact, release
               the pages of a paged cache: pages for new tokens, a second sequence on the same history,
               a context cut to the tokens that stay, pages given back

Head counts and lengths are those of ``workloads/synth.py`` and ``perf/cases.py``: 32 query heads on 8 KV
heads of 128, prompts of a few thousand tokens, observations of 128-2048 new tokens, histories of 8-32K.

A case is a dict of plain values:
  op        "rope", "prefill", "reserve", "fork" or "compact"
  dtype     of the cache: "f32", "bf16" or "fp8" (codes; the queries and new rows are bf16)
  batch, hq, hkv, d
  page      tokens per page, 0 for a packed cache
  lo, hi    context lengths, uniform, drawn from ``mix``; hi bounds the call
  new_lo, new_hi   rope, prefill: new tokens a sequence, uniform (0: all of the context)
  rot       rope: rotated elements of a head
  norm, interleaved   rope: with weights of a norm; pairs of neighbours instead of halves
  gap       rope: positions run ahead of the cache index by so many (a context that was cut)
  layers    fork, compact: layers whose caches share the block table
  forks     fork, compact: children of each sequence
  head_lo, tail   compact: tokens kept of the start and of the end
"""

import math
import random

import torch

own = False

DEVICE = "cuda:0"
K_SCALE, V_SCALE = 2.0 ** -6, 2.0 ** -5  # value = code * scale
EPS = 1e-6
FP8_MAX = 448.0


def _case(op, dtype, batch, hq, hkv, d, page, lo, hi, mix=1, new_lo=0, new_hi=0, rot=0, norm=True,
          interleaved=False, gap=0, layers=1, forks=1, head_lo=0, tail=0):
    return dict(op=op, dtype=dtype, batch=batch, hq=hq, hkv=hkv, d=d, page=page, lo=lo, hi=hi, mix=mix,
                new_lo=new_lo, new_hi=new_hi, rot=rot, norm=norm, interleaved=interleaved, gap=gap, layers=layers,
                forks=forks, head_lo=head_lo, tail=tail)


def listed():
    def named(name, *a, **kw):
        return dict(_case(*a, **kw), name=name)

    return [
        # One user's decode step: the new token's query and key on their way into the cache.
        named("rope_bf16_paged16_B1_M1", "rope", "bf16", 1, 32, 8, 128, 16, 6001, 6001, new_lo=1, new_hi=1, rot=128),
        # The step of a serving batch over an FP8 cache.
        named("rope_fp8_paged64_B64_M1", "rope", "fp8", 64, 32, 8, 128, 64, 1000, 7000, mix=2, new_lo=1, new_hi=1,
              rot=128),
        # Observations of several agents over an FP8 cache; a model that rotates half of each head, in
        # neighbouring pairs, without a norm, at positions after a cut.
        named("rope_fp8_paged16_B8_M128-2048", "rope", "fp8", 8, 64, 8, 128, 16, 8192, 16384, mix=3, new_lo=128,
              new_hi=2048, rot=64, norm=False, interleaved=True, gap=20000),
        # The whole context anew after a summary update, into a packed cache.
        named("rope_bf16_B2_L16384", "rope", "bf16", 2, 32, 8, 128, 0, 16384, 16384, mix=4, rot=128),
        # A few tokens a sequence (drafted ones to verify, short tool answers) over FP8 pages.
        named("prefill_fp8_paged16_B4_L2k-12k_M1-16", "prefill", "fp8", 4, 32, 8, 128, 16, 2000, 12000, mix=5,
              new_lo=1, new_hi=16),
        # One observation of an agent's step over its cached history.
        named("prefill_fp8_paged64_B1_L24300_M300", "prefill", "fp8", 1, 32, 8, 128, 64, 24300, 24300, mix=6,
              new_lo=300, new_hi=300),
        # The whole context prefilled anew.
        named("prefill_fp8_uncached_B1_L8192", "prefill", "fp8", 1, 32, 8, 128, 0, 8192, 8192, mix=7),
        # Pages for the prompts of a small batch, then for its first new token.
        named("reserve_paged64_R8_L1k-7k", "reserve", "bf16", 8, 32, 8, 128, 64, 1000, 7000, mix=8),
        # The same for a full batch with small pages.
        named("reserve_paged16_R64_L2k-16k", "reserve", "fp8", 64, 32, 8, 128, 16, 2048, 16384, mix=9),
        # Four continuations of each of eight histories, over the caches of four layers.
        named("fork_bf16_paged64_B8x4_L8k-32k", "fork", "bf16", 8, 32, 8, 128, 64, 8192, 32768, mix=10, layers=4,
              forks=4),
        # One agent's history, handed on and cut to the prompt and the recent buffer.
        named("compact_bf16_paged16_B1_L24300", "compact", "bf16", 1, 32, 8, 128, 16, 24300, 24300, mix=11,
              head_lo=1000, tail=5001),
        # The same for a batch over an FP8 cache of four layers.
        named("compact_fp8_paged64_B8_L8k-32k", "compact", "fp8", 8, 32, 8, 128, 64, 8192, 32768, mix=12, layers=4,
              head_lo=777, tail=7000),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


MAX_CACHE_BYTES = 1 << 30  # K and V of a drawn case
MAX_ROPE_TOKENS = 32768
MAX_PREFILL_FLOPS = 6.0e11
MAX_SCORES = 1 << 31       # padded scores of a drawn prefill, as the plain form holds them
MAX_MOVED_BYTES = 1 << 28  # rows of a drawn compact


def draw(rng):
    """One more case: the listed kinds over their ranges (lengths and batches log-uniform, odd sizes included)."""
    kind = rng.choice(["step", "step", "chunk", "chunk", "prefill", "prefill", "uncached", "reserve", "fork", "compact"])
    mix = rng.randrange(1 << 30)
    while True:
        hkv = rng.choice([2, 4, 8, 8])
        hq = hkv * rng.choice([1, 2, 4, 4, 8, 16])
        d = rng.choice([128, 128, 64])
        dtype = rng.choice(["bf16", "bf16", "fp8", "fp8", "f32"])
        page = rng.choice([0, 16, 64, 64, 1])
        if kind in ("step", "chunk"):
            hi = _log_int(rng, 200, 16384)
            m = 1 if kind == "step" else _log_int(rng, 2, min(hi, 4096))
            c = _case("rope", dtype, _log_int(rng, 1, 256 if kind == "step" else 16), hq, hkv, d, page,
                      max(m, int(hi * rng.uniform(0.1, 1.0))), hi, mix=mix, new_lo=max(1, int(m * rng.uniform(0.1, 1.0))),
                      new_hi=m, rot=rng.choice([d, d, d // 2]), norm=rng.random() < 0.7,
                      interleaved=rng.random() < 0.3, gap=rng.choice([0, 0, 10000]))
        elif kind in ("prefill", "uncached"):
            hi = _log_int(rng, 200, 24300 if kind == "prefill" else 6000)
            m = _log_int(rng, 1, min(hi, 1024)) if kind == "prefill" else 0
            c = _case("prefill", "fp8", _log_int(rng, 1, 4), hq, hkv, d, page, max(1, m, int(hi * rng.uniform(0.3, 1.0))),
                      hi, mix=mix, new_lo=max(1, int(m * rng.uniform(0.1, 1.0))) if m else 0, new_hi=m)
        elif kind == "reserve":
            hi = _log_int(rng, 200, 16384)
            c = _case("reserve", dtype, _log_int(rng, 1, 64), hq, hkv, d, rng.choice([16, 16, 64, 128]),
                      max(1, int(hi * rng.uniform(0.05, 1.0))), hi, mix=mix)
        else:
            hi = _log_int(rng, 300, 32768)
            tail = _log_int(rng, 1, 7000)
            c = _case(kind, dtype, _log_int(rng, 1, 8), hq, hkv, d, rng.choice([16, 64, 64, 8]),
                      max(1, int(hi * rng.uniform(0.2, 1.0))), hi, mix=mix, layers=rng.randint(1, 4),
                      forks=rng.randint(1, 4) if kind == "fork" else 1,
                      head_lo=rng.randint(0, 1500) if kind == "compact" else 0, tail=tail if kind == "compact" else 0)
        lens = _lengths(c)
        cache = 2 * c["layers"] * sum(lens) * (1 + c["forks"]) * c["hkv"] * c["d"] * _elem_bytes(c)
        w = work(c)
        if cache > MAX_CACHE_BYTES:
            continue
        if c["op"] == "rope" and sum(_new_tokens(c)) > MAX_ROPE_TOKENS:
            continue
        if c["op"] == "prefill" and (w["flops"] > MAX_PREFILL_FLOPS or
                                     c["batch"] * c["hq"] * max(_new_tokens(c)) * max(lens) > MAX_SCORES):
            continue
        if c["op"] == "compact" and w["bytes"] > MAX_MOVED_BYTES:
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


def _kept(case):
    """Positions that stay, for each sequence: the start (part of it may have gone already) and the end."""
    r = random.Random(case["mix"] + 2)
    out = []
    for n in _lengths(case):
        head = min(case["head_lo"], n)
        tail = min(max(1, case["tail"] - r.randint(0, case["tail"] // 4)), n)
        out.append(list(range(head)) + list(range(max(head, n - tail), n)))
    return out


def _elem_bytes(case):
    return {"f32": 4, "bf16": 2, "fp8": 1}[case["dtype"]]


def _pages_of(n, page):
    return -(-n // page)


def work(case):
    """Each input read once, each output written once."""
    lens, hq, hkv, d, page = _lengths(case), case["hq"], case["hkv"], case["d"], case["page"]
    e = _elem_bytes(case)
    qe = 4 if case["dtype"] == "f32" else 2
    row = 2 * hkv * d * e  # K and V of one token
    if case["op"] == "rope":
        new = sum(_new_tokens(case))
        return {"bytes": new * ((2 * hq + 2 * hkv) * d * qe + row + 4 * case["rot"]), "flops": new * (hq + hkv) * d * 8}
    if case["op"] == "prefill":
        new = _new_tokens(case)
        pairs = sum((n - m) * m + m * (m + 1) // 2 for n, m in zip(lens, new))
        return {"bytes": sum(lens) * row + sum(new) * hq * (6 * d + 4), "flops": 4 * d * hq * pairs}
    if case["op"] == "reserve":
        # The old entries and counts go, the new ones come; the counts are looked through once for free pages.
        entries = sum(_pages_of(n, page) for n in lens)
        return {"bytes": 4 * (6 * entries + _pool_pages(case)), "flops": entries}
    entries = case["forks"] * sum(_pages_of(n, page) for n in lens)
    nbytes = 4 * (6 * entries + _pool_pages(case))  # given back and shared anew
    nbytes += case["forks"] * sum(n % page for n in lens) * 2 * row * case["layers"]
    if case["op"] == "compact":
        for kept in _kept(case):
            stay = _unmoved(kept) // page * page
            nbytes += (len(kept) - stay) * (2 * row * case["layers"] + 4)
    return {"bytes": nbytes, "flops": entries}


def _unmoved(kept):
    for t, p in enumerate(kept):
        if t != p:
            return t
    return len(kept)


def _pool_pages(case):
    lens, page = _lengths(case), case["page"]
    held = sum(_pages_of(n, page) for n in lens)
    if case["op"] == "reserve":
        return held + len(lens) + held // 8
    n = held + case["forks"] * len(lens) + held // 8
    return n + (sum(_pages_of(len(k), page) for k in _kept(case)) if case["op"] == "compact" else 0)


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
    rows = t.view(-1, t.shape[-2], t.shape[-1])
    step = max(1, (1 << 26) // (rows.shape[1] * rows.shape[2]))
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


def _inputs(case, seed):
    g = torch.Generator(device=DEVICE).manual_seed(seed)
    lens, hq, hkv, d, page = _lengths(case), case["hq"], case["hkv"], case["d"], case["page"]
    cache_dtype = {"f32": torch.float32, "bf16": torch.bfloat16, "fp8": torch.uint8}[case["dtype"]]
    q_dtype = torch.float32 if case["dtype"] == "f32" else torch.bfloat16
    x = dict(case=case, ctx_lens=_ints(lens, torch.int32))
    if case["op"] in ("rope", "prefill"):
        if page:
            counts = [_pages_of(n, page) for n in lens]
            x["k"], x["v"] = _pair((sum(counts), page, hkv, d), cache_dtype)
            perm = torch.randperm(sum(counts), generator=g, device=DEVICE).to(torch.int32)
            x["block_table"] = torch.full((len(lens), _pages_of(case["hi"], page)), -1, dtype=torch.int32, device=DEVICE)
            for b, n in enumerate(counts):
                first = sum(counts[:b])
                x["block_table"][b, :n] = perm[first:first + n]
        else:
            x["k"], x["v"] = _pair((sum(lens), hkv, d), cache_dtype)
            x["seq_start"] = _starts(lens)
        _fill(x["k"], g, K_SCALE)
        _fill(x["v"], g, V_SCALE)
        new = _new_tokens(case)
        x["q_start"], x["q_lens"], x["max_q_len"] = _starts(new), _ints(new, torch.int32), max(new)
        if case["op"] == "prefill":
            x["q"] = torch.randn((sum(new), hq, d), generator=g, device=DEVICE).to(q_dtype)
            return x
        # The projection's output holds the queries, keys and values of a token side by side.
        qkv = torch.randn((sum(new), hq + 2 * hkv, d), generator=g, device=DEVICE).to(q_dtype)
        x["q"], x["new_k"], x["new_v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        x["q_weight"] = x["k_weight"] = None
        if case["norm"]:
            x["q_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device=DEVICE)).to(q_dtype)
            x["k_weight"] = (1 + 0.2 * torch.randn(d, generator=g, device=DEVICE)).to(q_dtype)
        x["cos_sin"] = _angles(case)
        x["positions"] = None
        if case["gap"]:
            at = [n - m + i + case["gap"] for n, m in zip(lens, new) for i in range(m)]
            x["positions"] = _ints(at, torch.int32)
        return x
    # A pool whose pages are held by the sequences in a random order, the others free.
    total, table_width = _pool_pages(case), _pages_of(case["hi"] + 1, page)
    order = torch.randperm(total, generator=g, device=DEVICE).to(torch.int32).tolist()
    rows = len(lens) * (1 + case["forks"]) if case["op"] != "reserve" else len(lens)
    table, counts, first = [[-1] * table_width for _ in range(rows)], [0] * total, 0
    if case["op"] == "reserve":
        # Some pages are held by others; every eighth or so.
        for p in order[:total - sum(_pages_of(n + 1, page) for n in lens)]:
            counts[p] = 1
        x["ctx_lens"] = _ints([0] * rows, torch.int32)
        x["add"], x["one"] = _ints(lens, torch.int32), _ints([1] * rows, torch.int32)
    else:
        for b, n in enumerate(lens):
            m = _pages_of(n, page)
            table[b][:m] = order[first:first + m]
            for p in table[b][:m]:
                counts[p] = 1
            first += m
        x["ctx_lens"] = _ints(lens + [0] * (rows - len(lens)), torch.int32)
        x["parents"] = _ints([b for b in range(len(lens)) for _ in range(case["forks"])], torch.int32)
    children = list(range(len(lens), rows)) if case["op"] != "reserve" else list(range(rows))
    x["rows"] = _ints(children, torch.int32)
    x["block_table"], x["refcounts"] = _ints(table, torch.int32), _ints(counts, torch.int32)
    x["k"], x["v"] = _pair((case["layers"], total, page, hkv, d), cache_dtype)
    if case["op"] != "reserve":
        _fill(x["k"], g, K_SCALE)
        _fill(x["v"], g, V_SCALE)
    if case["op"] == "compact":
        kept = _kept(case)
        x["keep"] = _ints([p for part in kept for p in part], torch.int32)
        x["keep_start"], x["keep_lens"] = _starts([len(k) for k in kept]), _ints([len(k) for k in kept], torch.int32)
        x["max_keep"] = max(len(k) for k in kept)
    return x


def _angles(case):
    """cos and sin of every position's angles, [positions, rot], in 32 bits from 64-bit angles."""
    half = case["rot"] // 2
    n = case["hi"] + case["gap"]
    freq = 1e6 ** (-torch.arange(half, dtype=torch.float64, device=DEVICE) / half)
    a = torch.arange(n, dtype=torch.float64, device=DEVICE)[:, None] * freq
    return torch.cat([a.cos(), a.sin()], dim=1).to(torch.float32)


def prepare(case, seed):
    x = _inputs(case, seed)
    if own:
        from paper_2605_30842_amd.binding import DecodeAttention, KVPages

        scales = dict(k_scale=K_SCALE, v_scale=V_SCALE) if case["dtype"] == "fp8" else {}
        bound = case["hi"] + (1 if case["op"] == "reserve" else 0)
        x["op"] = DecodeAttention(case["hq"], case["hkv"], case["d"], case["dtype"], 1.0 / math.sqrt(case["d"]),
                                  case["batch"], bound, **scales)
        if case["op"] in ("reserve", "fork", "compact"):
            x["pages"] = KVPages(x["op"], x["k"], x["v"], x["block_table"], x["ctx_lens"], x["refcounts"], bound)
    return x


# ------------------------------------------------------------------ one pass


def _values(x, t):
    """A cache tensor as what it stands for (codes as 8-bit floats)."""
    return t.view(torch.float8_e4m3fn) if x["case"]["dtype"] == "fp8" else t


def run(x):
    kind = x["case"]["op"]
    if kind == "rope":
        q = _own_rope(x) if own else _plain_rope(x)
        return dict(q=q, k=_values(x, x["k"]), v=_values(x, x["v"]))
    if kind == "prefill":
        out, lse = _own_prefill(x) if own else _plain_prefill(x)
        return dict(out=out, lse=lse)
    release, reserve, fork, compact = _own_pages(x) if own else _plain_pages(x)
    release(x["rows"])
    if kind == "reserve":
        short = [reserve(x["add"]), reserve(x["one"])]
    else:
        short = [fork(x["parents"], x["rows"])]
    if kind == "compact":
        short.append(compact(x["rows"], x["keep"], x["keep_start"], x["keep_lens"]))
    got = dict(block_table=x["block_table"], refcounts=x["refcounts"], ctx_lens=x["ctx_lens"], short=short)
    return got if kind == "reserve" else dict(got, k=_values(x, x["k"]), v=_values(x, x["v"]))


def _own_rope(x):
    case, op = x["case"], x["op"]
    more = dict(q_weight=x["q_weight"], k_weight=x["k_weight"], eps=EPS, positions=x["positions"],
                interleaved=case["interleaved"])
    if case["new_hi"] != 1:  # else one new token a sequence, the step of a decode loop
        more.update(q_start=x["q_start"], q_lens=x["q_lens"], max_q_len=x["max_q_len"])
    args = (x["q"], x["new_k"], x["new_v"], x["k"], x["v"])
    if case["page"]:
        return op.rope_append_paged(*args, x["block_table"], x["ctx_lens"], case["hi"], x["cos_sin"], **more)
    return op.rope_append(*args, x["seq_start"], x["ctx_lens"], case["hi"], x["cos_sin"], **more)


def _own_prefill(x):
    case, op = x["case"], x["op"]
    lse = torch.empty(x["q"].shape[:2], dtype=torch.float32, device=DEVICE)
    if case["page"]:
        return op.prefill_paged(x["q"], x["q_start"], x["q_lens"], x["max_q_len"], x["k"], x["v"], x["block_table"],
                                x["ctx_lens"], case["hi"], lse=lse)
    return op.prefill(x["q"], x["q_start"], x["q_lens"], x["max_q_len"], x["k"], x["v"], x["seq_start"], x["ctx_lens"],
                      case["hi"], lse=lse)


def _own_pages(x):
    p = x["pages"]
    return p.release, p.reserve, p.fork, p.compact


# ------------------------------------------------------------------ the same in elementary operations


def _cache_rows(x, b, t):
    """The row of token t of sequence b in a cache seen as [rows, hkv, d]."""
    page = x["case"]["page"]
    if page == 0:
        return x["seq_start"][b] + t
    return x["block_table"][b, t // page].long() * page + t % page


def _turned(y, cos, sin, rot, interleaved):
    if interleaved:
        pairs = y[..., :rot].unflatten(-1, (rot // 2, 2))
        a, b = pairs[..., 0], pairs[..., 1]
        turned = torch.stack([a * cos - b * sin, b * cos + a * sin], dim=-1).flatten(-2)
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
        turned = torch.cat([a * cos - b * sin, b * cos + a * sin], dim=-1)
    return torch.cat([turned, y[..., rot:]], dim=-1)


def _plain_rope(x):
    case, rot = x["case"], x["case"]["rot"]
    n = torch.arange(x["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(x["q_start"], n, right=True) - 1
    t = x["ctx_lens"][b] - x["q_lens"][b] + n - x["q_start"][b]
    angles = x["cos_sin"][(t if x["positions"] is None else x["positions"]).long()][:, None, :]
    cos, sin = angles[..., :rot // 2], angles[..., rot // 2:]

    def normed(y, weight):
        y = y.float()
        return y if weight is None else y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * weight.float()

    def stored(cache, y, scale):
        if case["dtype"] == "fp8":
            y = (y / scale).clamp(-FP8_MAX, FP8_MAX).to(torch.float8_e4m3fn).view(torch.uint8)
        cache.view(-1, case["hkv"], case["d"])[_cache_rows(x, b, t)] = y.to(cache.dtype)

    q = _turned(normed(x["q"], x["q_weight"]), cos, sin, rot, case["interleaved"]).to(x["q"].dtype)
    stored(x["k"], _turned(normed(x["new_k"], x["k_weight"]), cos, sin, rot, case["interleaved"]), K_SCALE)
    stored(x["v"], x["new_v"].float(), V_SCALE)
    return q


def _plain_prefill(x):
    case = x["case"]
    hkv, group, d = case["hkv"], case["hq"] // case["hkv"], case["d"]
    batch, most, m = case["batch"], case["hi"], x["max_q_len"]
    seq = torch.arange(batch, device=DEVICE)[:, None]
    key = torch.arange(most, device=DEVICE)[None, :]
    rows = _cache_rows(x, seq, torch.minimum(key, x["ctx_lens"][:, None].long() - 1))  # [batch, most]

    def heads(cache, scale):
        return (cache.view(torch.float8_e4m3fn).view(-1, hkv, d)[rows].float() * scale).transpose(1, 2)

    k, v = heads(x["k"], K_SCALE), heads(x["v"], V_SCALE)  # [batch, hkv, most, d]
    i = torch.arange(m, device=DEVICE)[None, :]
    at = (x["q_start"][:, None] + i).clamp(max=x["q"].shape[0] - 1)
    q = x["q"].float()[at].unflatten(2, (hkv, group)).permute(0, 2, 3, 1, 4).reshape(batch, hkv, group * m, d)
    s = torch.matmul(q, k.transpose(2, 3).contiguous()).view(batch, hkv, group, m, most) / math.sqrt(d)
    last = x["ctx_lens"][:, None] - x["q_lens"][:, None] + i  # [batch, m]
    s = s.masked_fill((key[:, None, :] > last[..., None])[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    s = (s - top).exp()
    total = s.sum(-1, keepdim=True)
    out = torch.matmul((s / total).view(batch, hkv, group * m, most), v.contiguous()).view(batch, hkv, group, m, d)
    lse = (top + total.log())[..., 0]
    # Back to the packed rows.
    n = torch.arange(x["q"].shape[0], device=DEVICE)
    b = torch.searchsorted(x["q_start"], n, right=True) - 1
    i = n - x["q_start"][b]
    return out.permute(0, 3, 1, 2, 4)[b, i].flatten(1, 2), lse.permute(0, 3, 1, 2)[b, i].flatten(1, 2)


def _plain_pages(x):
    case, page = x["case"], x["case"]["page"]
    table, counts, ctx = x["block_table"], x["refcounts"], x["ctx_lens"]
    total, width = counts.shape[0], table.shape[1]
    col = torch.arange(width, device=DEVICE)[None, :]
    zero = torch.zeros((), dtype=torch.int32, device=DEVICE)

    def pages_of(n):
        return (n + page - 1) // page

    def add(pages, mask, step):
        counts.index_add_(0, torch.where(mask, pages, zero).flatten(), (mask * step).flatten().int())

    def take(mask):
        """Free pages for the entries of the mask, in their order, lowest page first; all of them or none."""
        free = counts == 0
        rank = torch.where(free, free.cumsum(0) - 1, total)
        listing = torch.zeros(total + 1, dtype=torch.int32, device=DEVICE)
        listing.scatter_(0, rank, torch.arange(total, dtype=torch.int32, device=DEVICE))
        want = mask.flatten().cumsum(0) - 1
        short = (mask.sum() - free.sum()).clamp(min=0).to(torch.int32)
        mask = mask & (short == 0)
        pages = listing[want.clamp(0, total)].view(mask.shape)
        add(pages, mask, 1)
        return pages, mask, short

    def release(rows):
        rows = rows.long()
        held = col < pages_of(ctx[rows])[:, None]
        add(table[rows], held, -1)
        table[rows] = torch.where(held, -1, table[rows])
        ctx[rows] = 0

    def reserve(more):
        mask = (col >= pages_of(ctx)[:, None]) & (col < pages_of(ctx + more)[:, None])
        pages, mask, short = take(mask)
        table.copy_(torch.where(mask, pages, table))
        ctx.copy_(torch.where(short == 0, ctx + more, ctx))
        return short

    def move(src, dst, mask):
        """Rows src to rows dst of every layer where the mask holds."""
        dst = torch.where(mask, dst, src).flatten()
        for_all = (case["layers"], total * page, case["hkv"], case["d"])
        x["k"].view(for_all)[:, dst] = x["k"].view(for_all)[:, src.flatten()]
        x["v"].view(for_all)[:, dst] = x["v"].view(for_all)[:, src.flatten()]

    def fork(parents, children):
        parents, children = parents.long(), children.long()
        n = ctx[parents].long()
        whole, rest = n // page, n % page
        pages, got, short = take((col == whole[:, None]) & (rest > 0)[:, None])
        shared = (col < whole[:, None]) & (short == 0)
        add(table[parents], shared, 1)
        table[children] = torch.where(got, pages, torch.where(shared, table[parents], table[children]))
        ctx[children] = torch.where(short == 0, n, ctx[children]).to(torch.int32)
        last = whole.clamp(max=width - 1)
        src = table[parents, last].long().clamp(min=0)[:, None] * page + torch.arange(page, device=DEVICE)
        dst = table[children, last].long().clamp(min=0)[:, None] * page + torch.arange(page, device=DEVICE)
        move(src, dst, (torch.arange(page, device=DEVICE) < rest[:, None]) & (short == 0))
        return short

    def compact(rows, keep, start, length):
        rows, length = rows.long(), length.long()[:, None]
        t = torch.arange(x["max_keep"], device=DEVICE)[None, :]
        live = t < length
        p = torch.where(live, keep[torch.where(live, start[:, None] + t, 0)].long(), 0)
        stay = ((p == t) & live).int().cumprod(1).sum(1, keepdim=True) // page
        old, n = table[rows], ctx[rows].long()[:, None]
        pages, got, short = take((col >= stay) & (col < pages_of(length)))
        ok = short == 0
        gone = (col >= stay) & (col < pages_of(n)) & ok
        add(old, gone, -1)
        new = torch.where(got, pages, torch.where(gone, -1, old))
        table[rows] = new
        ctx[rows] = torch.where(ok, length, n)[:, 0].to(torch.int32)
        src = old.gather(1, p // page).long() * page + p % page
        dst = new.gather(1, torch.where(live, t, 0) // page).long() * page + t % page
        move(src, dst, live & (t >= stay * page) & ok)
        return short

    return release, reserve, fork, compact


# ------------------------------------------------------------------ the same in 64 bits


def _wide(case, t, scale):
    if case["dtype"] == "fp8":
        return t.view(torch.float8_e4m3fn).to(torch.float32).to(torch.float64) * scale
    return t.to(torch.float64)


def _exact_rows(x, b, n):
    page, t = x["case"]["page"], torch.arange(n, device=DEVICE)
    if page == 0:
        return int(x["seq_start"][b]) + t
    return x["block_table"][b, :_pages_of(n, page)].long()[t // page] * page + t % page


def _exact_rope(case, x):
    half, d = case["rot"] // 2, case["d"]
    scales = (K_SCALE, V_SCALE) if case["dtype"] == "fp8" else (1.0, 1.0)
    k = _wide(case, x["k"], 1.0)
    v = _wide(case, x["v"], 1.0)

    def made(y, weight, at):
        y = y.to(torch.float64)
        if weight is not None:
            y = y / torch.sqrt(torch.sum(y * y, -1, keepdim=True) / d + EPS) * weight.to(torch.float64)
        z = y.clone()
        turn = torch.complex(at[:, :half].to(torch.float64), at[:, half:].to(torch.float64))[:, None, :]
        if case["interleaved"]:
            first, second = slice(0, 2 * half, 2), slice(1, 2 * half, 2)
        else:
            first, second = slice(0, half), slice(half, 2 * half)
        turned = torch.complex(y[..., first].contiguous(), y[..., second].contiguous()) * turn
        z[..., first], z[..., second] = turned.real, turned.imag
        return z

    q, first = [], 0
    for b, (n, m) in enumerate(zip(_lengths(case), _new_tokens(case))):
        part = slice(first, first + m)
        first += m
        at = x["cos_sin"][torch.arange(n - m, n, device=DEVICE) + case["gap"]]
        rows = _exact_rows(x, b, n)[n - m:]
        q.append(made(x["q"][part], x["q_weight"], at))
        new_k, new_v = made(x["new_k"][part], x["k_weight"], at) / scales[0], x["new_v"][part].double() / scales[1]
        if case["dtype"] == "fp8":
            new_k, new_v = new_k.clamp(-FP8_MAX, FP8_MAX), new_v.clamp(-FP8_MAX, FP8_MAX)
        k.view(-1, case["hkv"], d)[rows] = new_k
        v.view(-1, case["hkv"], d)[rows] = new_v
    return dict(q=torch.cat(q), k=k, v=v)


def _exact_prefill(case, x):
    group, d = case["hq"] // case["hkv"], case["d"]
    out = torch.zeros(x["q"].shape, dtype=torch.float64, device=DEVICE)
    lse = torch.zeros(x["q"].shape[:2], dtype=torch.float64, device=DEVICE)
    first = 0
    for b, (n, m) in enumerate(zip(_lengths(case), _new_tokens(case))):
        rows = _exact_rows(x, b, n)
        for h in range(case["hq"]):
            k = _wide(case, x["k"].view(-1, case["hkv"], d)[rows, h // group], K_SCALE)
            v = _wide(case, x["v"].view(-1, case["hkv"], d)[rows, h // group], V_SCALE)
            for i in range(0, m, 1024):
                j = min(i + 1024, m)
                part = slice(first + i, first + j)
                s = (x["q"][part, h].to(torch.float64) @ k.t()) / math.sqrt(d)
                seen = torch.arange(n, device=DEVICE)[None, :] <= n - m + torch.arange(i, j, device=DEVICE)[:, None]
                s = torch.where(seen, s, -math.inf)
                lse[part, h] = torch.logsumexp(s, 1)
                out[part, h] = torch.exp(s - lse[part, h][:, None]) @ v
        first += m
    return dict(out=out, lse=lse)


def _exact_pages(case, x):
    """The pages by hand, one at a time."""
    page, lens = case["page"], _lengths(case)
    table, counts, ctx = x["block_table"].tolist(), x["refcounts"].tolist(), x["ctx_lens"].tolist()
    rows = x["rows"].tolist()
    k, v = _wide(case, x["k"], 1.0), _wide(case, x["v"], 1.0)
    lowest = 0

    def fresh():
        nonlocal lowest
        while counts[lowest] != 0:
            lowest += 1
        counts[lowest] = 1
        return lowest

    def copy(src, dst):
        if src:
            for cache in (k, v):
                flat = cache.view(case["layers"], -1, case["hkv"], case["d"])
                flat[:, _ints(dst, torch.int64)] = flat[:, _ints(src, torch.int64)]

    short = [0]
    if case["op"] == "reserve":
        short = [0, 0]
        for n, grown in ((0, lens), (lens, [m + 1 for m in lens])):
            for r in rows:
                have = _pages_of(n[r], page) if n else 0
                for i in range(have, _pages_of(grown[r], page)):
                    table[r][i] = fresh()
                ctx[r] = grown[r]
    else:
        for parent, child in zip(x["parents"].tolist(), rows):
            n = ctx[parent]
            for i in range(n // page):
                table[child][i] = table[parent][i]
                counts[table[child][i]] += 1
            if n % page:
                i = n // page
                table[child][i] = fresh()
                copy([table[parent][i] * page + o for o in range(n % page)],
                     [table[child][i] * page + o for o in range(n % page)])
            ctx[child] = n
    if case["op"] == "compact":
        short = [0, 0]
        lowest = 0
        gone = []
        for r, kept in zip(rows, _kept(case)):
            stay, old, n = _unmoved(kept) // page, list(table[r]), ctx[r]
            for i in range(stay, len(table[r])):
                if i < _pages_of(n, page):
                    gone.append(old[i])
                    table[r][i] = -1
                if i < _pages_of(len(kept), page):
                    table[r][i] = fresh()
            moved = range(stay * page, len(kept))
            copy([old[kept[t] // page] * page + kept[t] % page for t in moved],
                 [table[r][t // page] * page + t % page for t in moved])
            ctx[r] = len(kept)
        for p in gone:
            counts[p] -= 1
    got = dict(block_table=_ints(table, torch.int32), refcounts=_ints(counts, torch.int32),
               ctx_lens=_ints(ctx, torch.int32), short=short)
    return got if case["op"] == "reserve" else dict(got, k=k, v=v)


def exact(case, seed):
    x = _inputs(case, seed)
    return {"rope": _exact_rope, "prefill": _exact_prefill}.get(case["op"], _exact_pages)(case, x)
