"""The operators of an 8-bit cache over which their speed is measured.

A server that decodes in blocks keeps its cache in 8 bits (e4m3 with a power of two for each page
and head) and its page tables on the GPU: before a block each sequence takes the pages that it
needs, and after the round gives back those that rejected tokens leave empty ("reserve"); the
block's keys and values are rotated and quantised into the pages ("append8"); its queries attend
over them ("attend8").  ``run`` computes one pass in plain torch operations in 32 bits, or, with
``own``, through the binding.

A case's fields:
  op        "reserve" (retrace_kv_reserve), "append8" (retrace_kv_append_fp8),
            "attend8" (retrace_attend_fp8);
  B n ctx   sequences, most new tokens of one, most cached tokens of one;
  ragged    lengths differ by sequence (fixed by the case, not by the seed);
  page      slots of a page;
 append8 and attend8:
  Hq Hkv D  query heads, key/value heads, head size;
  dtype     of q, k, v and the output: "bf16" or "f32";
  rot, interleaved       append8: rotated dimensions, and which of them pair up;
  window, sinks, causal  attend8: the mask.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _reserve(name, B, n, ctx, page, ragged=False):
    return {"name": name, "op": "reserve", "B": B, "n": n, "ctx": ctx, "page": page, "ragged": ragged}


def _append(name, B, n, ctx, Hq, Hkv, D, page, rot=0, interleaved=False, ragged=False, dtype="bf16"):
    return {"name": name, "op": "append8", "B": B, "n": n, "ctx": ctx, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "rot": rot or D, "interleaved": interleaved, "ragged": ragged, "dtype": dtype}


def _attend(name, B, n, ctx, Hq, Hkv, D, page, window=0, sinks=0, causal=True, ragged=False, dtype="bf16"):
    return {"name": name, "op": "attend8", "B": B, "n": n, "ctx": ctx, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "window": window, "sinks": sinks, "causal": causal, "ragged": ragged, "dtype": dtype}


def listed():
    return [
        # A few users' next tokens: all latency.
        _reserve("pages-token", 8, 1, 2048, 16, ragged=True),
        # The verify block (16 drafts and the anchor) of the serving batch.
        _reserve("pages-block", 256, 17, 1024, 16, ragged=True),
        # A queue of prompts of many lengths, which is cancelled again.
        _reserve("pages-prompts", 2048, 2000, 0, 64, ragged=True),
        # One user's next token.
        _append("append-token", 1, 1, 2048, 32, 8, 128, 16),
        # The verify block of the serving batch.
        _append("append-block", 256, 17, 1024, 32, 8, 128, 16, ragged=True),
        # Prompts of many lengths at once, half the dimensions rotated in adjacent pairs, fp32.
        _append("append-prompts-f32", 8, 1501, 0, 20, 4, 96, 64, rot=48, interleaved=True, ragged=True, dtype="f32"),
        # One user's next token over a long conversation.
        _attend("token-16k", 1, 1, 16384, 32, 8, 128, 16),
        # The verify block of a medium batch, contexts of many lengths.
        _attend("block-16k", 64, 17, 16384, 32, 8, 128, 16, ragged=True),
        # The serving batch's next token in a layer with a sliding window and sinks.
        _attend("window-tokens", 256, 1, 8000, 64, 8, 64, 32, window=1024, sinks=4, ragged=True),
        # Two long documents: a drafter's block, whose positions see each other both ways.
        _attend("block-128k", 2, 16, 131072, 16, 2, 128, 64, causal=False),
        # A second chunk of prompts, over the first one in the cache.
        _attend("prompts-2k", 4, 2048, 2048, 32, 8, 128, 16, ragged=True),
        # fp32 queries: the toy model's blocks.
        _attend("block-f32", 16, 9, 1000, 8, 4, 64, 16, ragged=True, dtype="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    while True:
        case = _draw(rng)
        if _fits(case):
            return case


def _fits(case):
    """No more work than the largest listed case, and lengths that the plain form's tables have room for."""
    w, most = work(case), MOST[case["op"]]
    if w["bytes"] > most["bytes"] or w["flops"] > most["flops"]:
        return False
    end = case["ctx"] + case["n"]
    if case["op"] == "reserve":
        return case["B"] * end // case["page"] <= 1 << 22
    # a window's cache lies in memory as a whole
    return case["B"] * end * case["Hkv"] * case["D"] <= 2 << 30 and case["op"] == "append8" or \
        case["B"] * end * max(case["Hkv"] * case["D"], case["n"] * case["Hq"]) <= 2 << 30


def _draw(rng):
    op = rng.choice(["reserve", "append8", "attend8", "attend8"])
    form = rng.choice(["token", "block", "prompt"])
    case = {"op": op, "n": {"token": 1, "block": rng.randint(2, 33), "prompt": _spread(rng, 100, 4096)}[form],
            "page": rng.choice([8, 16, 16, 32, 48, 64, 128, 256]), "ragged": rng.random() < 0.7}
    if op == "reserve":
        return dict(case, B=_spread(rng, 1, 4096), ctx=rng.choice([0, _spread(rng, 1, 20000)]))
    Hkv = rng.choice([1, 2, 3, 4, 8, 10])
    case.update(Hkv=Hkv, Hq=Hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), D=rng.choice([64, 64, 80, 96, 128, 128, 128]),
                dtype=rng.choice(["bf16", "bf16", "bf16", "f32"]), B=_spread(rng, 1, 256) if form != "prompt" else rng.randint(1, 8))
    if op == "append8":
        return dict(case, ctx=_spread(rng, 1, 2000), rot=rng.choice([case["D"], case["D"] // 2]), interleaved=rng.random() < 0.4)
    case["ctx"] = _spread(rng, 1, 100000) if form != "prompt" else rng.choice([0, _spread(rng, 1, 4000)])
    window = rng.choice([0, 0, _spread(rng, 16, 8192)])
    return dict(case, window=window, sinks=rng.choice([0, 1, 4, 130]) if window else 0, causal=form != "block" or rng.random() < 0.7)


def _lengths(case):
    """New and cached tokens of each sequence: a user's program knows them, so does work()."""
    B, n, ctx = case["B"], case["n"], case["ctx"]
    if not case["ragged"]:
        return [n] * B, [ctx] * B
    rng = random.Random("%d %d %d" % (B, n, ctx))
    # A block has one size for every sequence; prompts have their own.
    new = [n if n <= 33 else n if b == 0 else rng.randint(max(1, n // 8), n) for b in range(B)]
    return new, [ctx if b == 0 else rng.randint(ctx // 8, ctx) for b in range(B)]


def _committed(case):
    """Tokens that stay after the round: some of a block's, none of a cancelled prompt's."""
    new, cached = _lengths(case)
    return [c + b * 7 % (n + 1) if n <= 33 else c for b, (n, c) in enumerate(zip(new, cached))]


def _visible(case, n, c):
    """Keys that any row of a sequence sees, and keys seen by its rows in all."""
    w, s, end = case["window"], case["sinks"], c + n
    if not w:
        return end, sum(c + i + 1 for i in range(n)) if case["causal"] else n * end
    first = max(0, c - w + 1)
    total = 0
    for i in range(n):
        hi, lo = (c + i if case["causal"] else end - 1), max(0, c + i - w + 1)
        total += hi - lo + 1 + min(s, lo)
    return end - first + min(s, first), total


def work(case):
    new, cached = _lengths(case)
    T, page = sum(new), case["page"]
    if case["op"] == "reserve":
        kept = _committed(case)
        moved = sum(-(-(c + n) // page) - -(-k // page) for n, c, k in zip(new, cached, kept))
        # lengths and pages held, read and written by both calls; pages from the stack into the table and back
        return {"bytes": 2 * 16 * case["B"] + 4 * case["B"] + 16 * moved + 8 * T, "flops": 0}
    size = 2 if case["dtype"] == "bf16" else 4
    D, Hq, Hkv = case["D"], case["Hq"], case["Hkv"]
    if case["op"] == "append8":
        pages = sum((c + n - 1) // page - c // page + 1 for n, c in zip(new, cached))
        return {"bytes": T * ((2 * Hq + 2 * Hkv) * size + 2 * Hkv) * D + T * case["rot"] * 4 + 4 * pages * Hkv + 8 * case["B"],
                "flops": 3 * T * (Hq + Hkv) * case["rot"] + 4 * T * Hkv * D}
    keys, seen = (sum(x) for x in zip(*(_visible(case, n, c) for n, c in zip(new, cached))))
    return {"bytes": 2 * T * Hq * D * size + keys * Hkv * (2 * D + 2 / page) + 8 * case["B"], "flops": 4 * seen * Hq * D}


# No drawn case has more work than the largest listed one of its operator.
MOST = {op: {k: max(work(c)[k] for c in listed() if c["op"] == op) for k in ("bytes", "flops")} for op in ("reserve", "append8", "attend8")}


def _rope(positions, rot, device):
    """cos and sin per position and pair, [positions, rot / 2, 2], base 10000."""
    a = torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot
    t = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * (10000.0 ** -a)
    return torch.stack([t.cos(), t.sin()], -1).float().contiguous()


def _tables(ends, page, width, total, order, device):
    """A page table [B, width] from the first entries of `order` (-1 past a sequence's end), and the pages of each row."""
    need = torch.tensor([-(-e // page) for e in ends], dtype=torch.int64, device=device)
    first = need.cumsum(0) - need
    col = torch.arange(width, device=device)
    return torch.where(col < need[:, None], order[(first[:, None] + col).clamp(max=total - 1)], -1).to(torch.int32).contiguous(), need


def _int32(values, device):
    return torch.tensor(values, dtype=torch.int32, device=device)


def prepare(case, seed):
    dev = "cuda"
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    new, cached = _lengths(case)
    B, page, T = case["B"], case["page"], sum(new)
    start = _int32([0] + torch.tensor(new).cumsum(0).tolist(), dev)
    ends = [n + c for n, c in zip(new, cached)]
    width = -(-max(ends) // page)
    s = {"case": case, "cache_len": _int32(cached, dev)}
    if case["op"] == "reserve":
        # a cache a little larger than what the sequences need
        total = sum(-(-e // page) for e in ends) + 64
        order = torch.randperm(total, generator=gen, device=dev)
        s["table"], need = _tables(cached, page, width, total, order, dev)
        held = int(need.sum())
        s["held"] = need.to(torch.int32)
        s["free"] = torch.cat([order[held:], order[:held]]).to(torch.int32)
        s["counts"] = _int32([total - held, 0], dev)
        s["new_len"], s["kept_len"], s["none"] = _int32(new, dev), _int32(_committed(case), dev), _int32([0] * B, dev)
        s["q_start"] = torch.empty(B + 1, dtype=torch.int32, device=dev)
        s["slots"] = torch.empty(T, dtype=torch.int64, device=dev)
        if own:
            from paper_2608_29748_gb300 import binding as rt

            s["pool"] = rt.PagePool(s["table"], page, s["free"], s["counts"], s["held"])
        return s
    dt, Hq, Hkv, D = DTYPES[case["dtype"]], case["Hq"], case["Hkv"], case["D"]
    total = sum(-(-e // page) for e in ends)
    order = torch.randperm(total, generator=gen, device=dev)
    s["table"], _ = _tables(ends, page, width, total, order, dev)
    # keys and values with a spread near one; pages and heads differ by powers of two
    for name in "kv":
        s[name + "_cache"] = torch.empty((total, page, Hkv, D), dtype=torch.bfloat16, device=dev).normal_(0.0, 90.0, generator=gen).clamp_(-448.0, 448.0).to(
            torch.float8_e4m3fn)
        s[name + "_exp"] = torch.randint(-8, -5, (total, Hkv), generator=gen, device=dev).to(torch.int8)
    # Blocks of one size need no list of where each sequence's tokens start.
    s["q_start"] = None if len(set(new)) == 1 else start
    s["T"], s["most"] = T, max(new)
    if case["op"] == "append8":
        # One projection's output: q, k and v of a token side by side.
        qkv = torch.empty((T, Hq + 2 * Hkv, D), dtype=dt, device=dev).normal_(generator=gen)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["rope"] = _rope(case["ctx"] + case["n"], case["rot"], dev)
    else:
        # Scores with a spread of 2 or so, so that some keys matter more than others.
        s["q"] = torch.empty((T, Hq, D), dtype=dt, device=dev).normal_(0.0, 2.0, generator=gen)
    s["out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
    if own:
        from paper_2608_29748_gb300 import binding as rt

        s["cache"] = rt.KvCacheFp8(s["k_cache"], s["v_cache"], s["table"], s["k_exp"], s["v_exp"])
        if case["op"] == "attend8":
            s["ws"] = rt.AttendWorkspace(Hq, Hkv, D, torch.float8_e4m3fn)
    return s


def _plain_reserve_once(s, cache_len, new_len, q_start, slots):
    page, table, free, counts = s["case"]["page"], s["table"], s["free"], s["counts"]
    B, width = table.shape
    c, n, held = cache_len.long(), new_len.long().clamp(min=0), s["held"].long()
    need = ((c + n).clamp(0, width * page) + page - 1) // page
    count = counts[0].long()
    take, give = (need - held).clamp(min=0), (held - need).clamp(min=0)
    take_before, give_before = take.cumsum(0) - take, give.cumsum(0) - give
    got = torch.minimum((count - take_before).clamp(min=0), take)
    left, back = count - got.sum(), give.sum()
    col = torch.arange(width, device=table.device)
    k, g = col - held[:, None], col - need[:, None]
    taken = free[(count - 1 - take_before[:, None] - k).clamp(0, free.numel() - 1)]
    giving = (g >= 0) & (g < give[:, None])
    to = torch.where(giving, left + back - 1 - give_before[:, None] - g, free.numel())
    longer = torch.cat([free, free[:1]])
    longer[to.view(-1)] = table.view(-1)
    free.copy_(longer[:-1])
    fresh = torch.where((k >= 0) & (k < got[:, None]), taken, -1)
    table.copy_(torch.where(giving | ((k >= 0) & (k < take[:, None])), fresh, table))
    s["held"].copy_(torch.where(give > 0, need, held + got))
    counts.copy_(torch.stack([left + back, take.sum() - got.sum()]))
    if slots is None:
        return
    T = slots.numel()
    upto = n.cumsum(0)
    q_start.copy_(torch.cat([upto[:1] * 0, upto]).clamp(max=T))
    t = torch.arange(T, device=table.device)
    b = torch.searchsorted(upto, t, right=True).clamp(max=B - 1)
    p = c[b] + t - (upto - n)[b]
    where = table.long()[b, (p // page).clamp(0, width - 1)]
    there = (t < upto[-1]) & (p >= 0) & (p < width * page) & (where >= 0)
    slots.copy_(torch.where(there, where * page + p % page, -1))


def _plain_reserve(s):
    _plain_reserve_once(s, s["cache_len"], s["new_len"], s["q_start"], s["slots"])
    _plain_reserve_once(s, s["kept_len"], s["none"], None, None)


def _tokens(s):
    """Sequence and place in it of every new token."""
    T, B, dev = s["T"], s["case"]["B"], s["cache_len"].device
    t = torch.arange(T, device=dev)
    if s["q_start"] is None:
        n = T // B
        return t // n, t % n
    start = s["q_start"].long()
    b = torch.searchsorted(start, t, right=True) - 1
    return b, t - start[b]


def _rotated(x, cs, rot, interleaved):
    """x [T, H, D] in fp32 with its first `rot` dimensions rotated by cs [T, rot/2, 2]."""
    c, s = cs[:, None, :, 0], cs[:, None, :, 1]
    r = x[..., :rot]
    if interleaved:
        a, b = r[..., 0::2], r[..., 1::2]
        turned = torch.stack([a * c - b * s, b * c + a * s], -1).flatten(-2)
    else:
        a, b = r[..., :rot // 2], r[..., rot // 2:]
        turned = torch.cat([a * c - b * s, b * c + a * s], -1)
    return torch.cat([turned, x[..., rot:]], -1)


def _two(e):
    """2 ** e in fp32."""
    return ((e.to(torch.int32) + 127) << 23).view(torch.float32)


def _e4m3(x):
    return x.clamp(-448.0, 448.0).to(torch.float8_e4m3fn)


def _quantise(s, x, cache, exps, page, slot):
    """x [T, H, D] in fp32 into the slots of `cache`, with the pages' powers of two."""
    P, size = cache.shape[:2]
    most = torch.zeros(exps.shape, device=x.device).index_reduce_(0, page, torch.where(x.isnan(), 0.0, x.abs()).amax(-1).clamp(max=3e38), "amax")
    first = torch.full((P,), size, device=x.device).index_reduce_(0, page, slot, "amin")
    m, e = torch.frexp(most)
    fit = torch.where(most > 0, e - 9 + (m > 0.875), -40).clamp(-40, 40)
    old = exps.int().clamp(-40, 40)
    first = first[:, None]
    now = torch.where(first == size, exps.int(), torch.where(first > 0, torch.maximum(fit, old), fit))
    # A sequence's first page may hold tokens already.
    at = s["table"].long()[torch.arange(s["case"]["B"], device=x.device), s["cache_len"].long() // size]
    held = cache[at].float()
    moved = _e4m3(held * _two((old - now)[at].clamp(min=-126))[:, None, :, None])
    keep = (torch.arange(size, device=x.device) < first[at])[:, :, None, None] & ((now > old) & (first < size))[at][:, None, :, None]
    bits = cache.view(torch.uint8)
    bits[at] = torch.where(keep, moved.view(torch.uint8), bits[at])
    exps.copy_(now.to(torch.int8))
    bits[page, slot] = _e4m3(x * _two(-now)[page][:, :, None]).view(torch.uint8)


def _plain_append(s):
    case = s["case"]
    b, i = _tokens(s)
    pos = s["cache_len"].long()[b] + i
    page, slot = s["table"].long()[b, pos // case["page"]], pos % case["page"]
    cs = s["rope"][pos]
    s["out"].copy_(_rotated(s["q"].float(), cs, case["rot"], case["interleaved"]))
    _quantise(s, _rotated(s["k"].float(), cs, case["rot"], case["interleaved"]), s["k_cache"], s["k_exp"], page, slot)
    _quantise(s, s["v"].float(), s["v_cache"], s["v_exp"], page, slot)


def _plain_attend(s):
    case = s["case"]
    B, n, Hq, Hkv, D = case["B"], s["most"], case["Hq"], case["Hkv"], case["D"]
    G, dev = Hq // Hkv, s["q"].device
    b, i = _tokens(s)
    q = torch.zeros((B, n, Hq, D), device=dev)
    q[b, i] = s["q"].float()
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    table = s["table"].long().clamp(min=0)
    value = lambda x, e: (x.view(torch.uint8)[table].view(torch.float8_e4m3fn).float() * _two(e[table])[:, :, None, :, None]).reshape(  # noqa: E731
        B, -1, Hkv, D).transpose(1, 2)
    k, v = value(s["k_cache"], s["k_exp"]), value(s["v_cache"], s["v_exp"])
    j = torch.arange(k.shape[2], device=dev)
    c = s["cache_len"].long()[:, None]
    new = torch.zeros(B, dtype=torch.int64, device=dev).index_add_(0, b, torch.ones_like(b))[:, None]
    p = c + torch.arange(n, device=dev)
    hi = p if case["causal"] else (c + new - 1).expand(B, n)
    seen = j <= hi[:, :, None]
    if case["window"]:
        seen &= (j > p[:, :, None] - case["window"]) | (j < case["sinks"])
    seen = seen[:, None, :, None, :].expand(B, 1, n, G, j.numel()).reshape(B, 1, n * G, j.numel())
    x = torch.matmul(q * (1.0 / math.sqrt(D)), k.transpose(2, 3))
    x = x.masked_fill_(~seen, -math.inf)
    x = x.sub_(x.amax(-1, keepdim=True).clamp(min=-3e38)).exp_()
    total = x.sum(-1, keepdim=True)
    written = (j < c + new)[:, None, :, None]
    o = torch.matmul(x, torch.where(written, v, 0.0))
    o = torch.where(total > 0, o / total, 0.0)
    o = o.view(B, Hkv, n, G, D).permute(0, 2, 1, 3, 4).reshape(B, n, Hq, D)
    s["out"].copy_(o[b, i])


def run(s):
    case = s["case"]
    if not own:
        {"reserve": _plain_reserve, "append8": _plain_append, "attend8": _plain_attend}[case["op"]](s)
    else:
        from paper_2608_29748_gb300 import binding as rt

        if case["op"] == "reserve":
            # before the block, and after its round: rejected tokens' pages go back
            rt.retrace_kv_reserve(s["cache_len"], s["new_len"], s["pool"], q_start=s["q_start"], slots=s["slots"])
            rt.retrace_kv_reserve(s["kept_len"], s["none"], s["pool"])
        elif case["op"] == "append8":
            rt.retrace_kv_append_fp8(s["q"], s["k"], s["v"], s["cache"], s["cache_len"], s["rope"], s["out"], q_start=s["q_start"],
                                     interleaved=case["interleaved"])
        else:
            rt.retrace_attend_fp8(s["q"], s["cache"], s["cache_len"], s["out"], s["ws"], q_start=s["q_start"], window=case["window"],
                                  sinks=case["sinks"], causal=case["causal"])
    names = {"reserve": ("table", "held", "free", "counts", "q_start", "slots"), "append8": ("out", "k_cache", "v_cache", "k_exp", "v_exp"),
             "attend8": ("out",)}[case["op"]]
    return {x: s[x] for x in names}


def _exact_reserve(s):
    case = s["case"]
    page = case["page"]
    new, cached = _lengths(case)
    table, held = s["table"].cpu().tolist(), s["held"].cpu().tolist()
    free, count = s["free"].cpu().tolist(), int(s["counts"][0])
    slots = []
    for b, (n, c) in enumerate(zip(new, cached)):
        while held[b] * page < c + n:
            count -= 1
            table[b][held[b]] = free[count]
            held[b] += 1
        slots += [table[b][p // page] * page + p % page for p in range(c, c + n)]
    back = []
    for b, k in enumerate(_committed(case)):
        keep = -(-k // page)
        back += table[b][keep:held[b]]
        table[b][keep:held[b]] = [-1] * (held[b] - keep)
        held[b] = keep
    for x in reversed(back):
        free[count] = x
        count += 1
    i32 = lambda v: torch.tensor(v, dtype=torch.int32)  # noqa: E731
    return {"table": i32(table), "held": i32(held), "free": i32(free), "counts": i32([count, 0]),
            "q_start": i32([0] + torch.tensor(new).cumsum(0).tolist()), "slots": torch.tensor(slots, dtype=torch.int64)}


def _exact_e4m3(x):
    """The e4m3 value nearest to each x, the even one of two: steps of 2 ** -9 up to 2 ** -6, an eighth of the power of two below x from there."""
    _, e = torch.frexp(x)
    step = torch.exp2((e.clamp(min=-5) - 4).double())
    return (torch.round(x / step) * step).clamp(-448.0, 448.0)


def _exact_append(s):
    case = s["case"]
    rot, size = case["rot"], case["page"]
    new, cached = _lengths(case)
    caches = {x: s[x + "_cache"].double() for x in "kv"}
    exps = {x: s[x + "_exp"].clone() for x in "kv"}
    q = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    pairs = torch.arange(rot // 2, device=q.device)
    first, second = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + rot // 2)
    t = 0
    for b, (n, c) in enumerate(zip(new, cached)):
        # The table's values are inputs: the rotation multiplies complex numbers by them.
        turn = torch.view_as_complex(s["rope"][c:c + n].double())[:, None, :]
        rows = {}
        for name in "qkv":
            x = s[name][t:t + n].double()
            if name != "v":
                z = torch.complex(x[..., first], x[..., second]) * turn
                x[..., first], x[..., second] = z.real, z.imag
            rows[name] = x
        q[t:t + n] = rows["q"]
        p = c
        while p < c + n:
            end = min(c + n, (p // size + 1) * size)
            page, a, z = int(s["table"][b, p // size]), p % size, p % size + end - p
            for name in "kv":
                x = rows[name][p - c:end - c]
                e = torch.ceil(torch.log2(x.abs().amax((0, 2)) / 448.0)).clamp(-40.0, 40.0)
                old = exps[name][page].double()
                if a > 0:
                    e = torch.maximum(e, old)
                    caches[name][page, :a] = _exact_e4m3(caches[name][page, :a] * torch.exp2(old - e)[:, None])
                caches[name][page, a:z] = _exact_e4m3(x * torch.exp2(-e)[:, None])
                exps[name][page] = e.to(torch.int8)
            p = end
        t += n
    return {"out": q, "k_cache": caches["k"], "v_cache": caches["v"], "k_exp": exps["k"], "v_exp": exps["v"]}


def _exact_attend(s):
    case = s["case"]
    Hkv, D, page, w = case["Hkv"], case["D"], case["page"], case["window"]
    G = case["Hq"] // Hkv
    new, cached = _lengths(case)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    t = 0
    for b, (n, c) in enumerate(zip(new, cached)):
        j = torch.arange(c + n, device=out.device)
        at, slot = s["table"][b].long()[torch.div(j, page, rounding_mode="floor")], j.remainder(page)
        k, v = (s[x + "_cache"].view(torch.uint8)[at, slot].view(torch.float8_e4m3fn).double() * torch.exp2(s[x + "_exp"][at].double())[:, :, None] for x in "kv")
        for h in range(Hkv):
            # Rows in pieces, so that the scores of a long prompt fit.
            for i0 in range(0, n, 1024):
                i = torch.arange(i0, min(n, i0 + 1024), device=out.device)
                last = (c + i if case["causal"] else torch.full_like(i, c + n - 1))[:, None]
                hidden = j > last
                if w:
                    hidden |= (j <= c + i[:, None] - w) & (j >= case["sinks"])
                x = torch.einsum("ngd,jd->ngj", s["q"][t + i, h * G:(h + 1) * G].double(), k[:, h]) / math.sqrt(D)
                x.masked_fill_(hidden[:, None, :], -math.inf)
                out[t + i, h * G:(h + 1) * G] = torch.einsum("ngj,jd->ngd", torch.softmax(x, -1), v[:, h])
        t += n
    return {"out": out}


def exact(case, seed):
    s = prepare(case, seed)
    return {"reserve": _exact_reserve, "append8": _exact_append, "attend8": _exact_attend}[case["op"]](s)
