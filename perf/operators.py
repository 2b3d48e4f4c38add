"""The operators around a round over which their speed is measured.

What a decoding loop runs next to a round: the keys and values of a token, a
draft block or a prompt go into a paged cache with the position rotation
("append"), their queries attend over that cache, with a sliding window and
sinks or without ("attend"), and logits become tokens ("sample").  Each case is
one call.  ``run`` computes it in plain torch operations in 32 bits, or, with
``own``, through the binding.

A case's fields:
  op        "append" (retrace_kv_append), "attend" (retrace_attend), "sample"
            (retrace_sample);
  dtype     "bf16" or "f32";
 append and attend:
  B n ctx   sequences, most new tokens of one, most cached tokens of one;
  ragged    lengths differ by sequence (fixed by the case, not by the seed);
  Hq Hkv D  query heads, key/value heads, head size;
  page      slots of a page;
  rot, interleaved       append: rotated dimensions, and which of them pair up;
  window, sinks, causal  attend: the mask;
 sample:
  B R V     sequences, rows of each (draft positions), vocabulary;
  top_k top_p min_p temperature   of every sequence, or with `mixed` the most
            of each where sequences differ (greedy ones among them);
  std       of the logits' bulk, above which 32 tokens a row stand out.
"""

import math
import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _append(name, B, n, ctx, Hq, Hkv, D, page, rot=0, interleaved=False, ragged=False, dtype="bf16"):
    return {"name": name, "op": "append", "B": B, "n": n, "ctx": ctx, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "rot": rot or D, "interleaved": interleaved, "ragged": ragged, "dtype": dtype}


def _attend(name, B, n, ctx, Hq, Hkv, D, page, window=0, sinks=0, causal=True, ragged=False, dtype="bf16"):
    return {"name": name, "op": "attend", "B": B, "n": n, "ctx": ctx, "Hq": Hq, "Hkv": Hkv, "D": D, "page": page,
            "window": window, "sinks": sinks, "causal": causal, "ragged": ragged, "dtype": dtype}


def _sample(name, B, R, V, top_k=0, top_p=1.0, min_p=0.0, temperature=1.0, mixed=False, std=2.0, dtype="bf16"):
    return {"name": name, "op": "sample", "B": B, "R": R, "V": V, "top_k": top_k, "top_p": top_p, "min_p": min_p,
            "temperature": temperature, "mixed": mixed, "std": std, "dtype": dtype}


def listed():
    return [
        # One user's next token: all latency.
        _append("append-token", 1, 1, 2048, 32, 8, 128, 16),
        # The verify block (16 drafts and the anchor) of the serving batch.
        _append("append-block", 256, 17, 1024, 32, 8, 128, 16, ragged=True),
        # Prompts of many lengths at once, half the dimensions rotated in adjacent pairs, fp32.
        _append("append-prompts-f32", 8, 1501, 0, 20, 4, 96, 64, rot=48, interleaved=True, ragged=True, dtype="f32"),
        # One user's next token over a short conversation.
        _attend("token-2k", 1, 1, 2048, 32, 8, 128, 16),
        # The verify block of a medium batch, contexts of many lengths.
        _attend("block-8k", 64, 17, 8192, 32, 8, 128, 16, ragged=True),
        # The serving batch's next token in a layer with a sliding window and sinks.
        _attend("window-tokens", 256, 1, 8000, 64, 8, 64, 32, window=1024, sinks=4, ragged=True),
        # Two long documents: a drafter's block, whose positions see each other both ways.
        _attend("block-128k", 2, 16, 131072, 16, 2, 128, 64, causal=False),
        # Prompts, the first layer's whole attention.
        _attend("prompts-4k", 4, 4096, 0, 32, 8, 128, 16, ragged=True),
        # fp32 throughout: the toy model's blocks.
        _attend("block-f32", 16, 9, 1000, 8, 4, 64, 16, ragged=True, dtype="f32"),
        # The drafter's block of one user, the evaluation's filter.
        _sample("draft-1", 1, 16, 151936, top_k=20, top_p=0.95),
        # The drafter's blocks of the serving batch: each user has settings of their own.
        _sample("draft-256", 256, 16, 151936, top_k=200, top_p=0.95, min_p=0.02, temperature=1.2, mixed=True),
        # A smaller vocabulary of odd size in fp32, nearly no filter.
        _sample("open-f32", 48, 11, 32003, top_p=0.98, dtype="f32"),
    ]


def _spread(rng, lo, hi):
    """A whole number between lo and hi, even over its logarithm."""
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    while True:
        case = _draw(rng)
        w, most = work(case), MOST[case["op"]]
        if w["bytes"] <= most["bytes"] and w["flops"] <= most["flops"]:
            return case


def _draw(rng):
    op = rng.choice(["append", "attend", "attend", "sample"])
    dtype = rng.choice(["bf16", "bf16", "bf16", "f32"])
    if op == "sample":
        return {"op": op, "B": _spread(rng, 1, 256), "R": rng.randint(1, 17), "V": _spread(rng, 1000, 200000),
                "top_k": rng.choice([0, 1, _spread(rng, 2, 1000)]), "top_p": rng.choice([1.0, rng.uniform(0.5, 0.99)]),
                "min_p": rng.choice([0.0, rng.uniform(0.005, 0.2)]), "temperature": rng.uniform(0.5, 1.5),
                "mixed": rng.random() < 0.5, "std": rng.uniform(0.7, 3.0), "dtype": dtype}
    Hkv = rng.choice([1, 2, 3, 4, 8, 10])
    case = {"op": op, "Hq": Hkv * rng.choice([1, 2, 3, 4, 5, 7, 8]), "Hkv": Hkv, "D": rng.choice([64, 64, 80, 96, 128, 128, 128]),
            "page": rng.choice([8, 16, 16, 32, 48, 64, 128, 256]), "ragged": rng.random() < 0.7, "dtype": dtype}
    form = rng.choice(["token", "block", "prompt"])
    case["n"] = {"token": 1, "block": rng.randint(2, 33), "prompt": _spread(rng, 100, 4096)}[form]
    case["B"] = _spread(rng, 1, 256) if form != "prompt" else rng.randint(1, 8)
    if op == "append":
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
    size = 2 if case["dtype"] == "bf16" else 4
    if case["op"] == "sample":
        rows = case["B"] * case["R"]
        # One maximum, one exponential and one sum per logit.
        return {"bytes": rows * (case["V"] * size + 12) + 16 * case["B"], "flops": 4 * rows * case["V"]}
    new, cached = _lengths(case)
    T, D, Hq, Hkv = sum(new), case["D"], case["Hq"], case["Hkv"]
    if case["op"] == "append":
        return {"bytes": T * (Hq + 2 * Hkv) * D * size * 2 + T * case["rot"] * 4 + 8 * case["B"], "flops": 3 * T * (Hq + Hkv) * case["rot"]}
    keys, seen = (sum(x) for x in zip(*(_visible(case, n, c) for n, c in zip(new, cached))))
    return {"bytes": 2 * T * Hq * D * size + keys * Hkv * D * 2 * size + 8 * case["B"], "flops": 4 * seen * Hq * D}


# No drawn case has more work than the largest listed one of its operator.
MOST = {op: {k: max(work(c)[k] for c in listed() if c["op"] == op) for k in ("bytes", "flops")} for op in ("append", "attend", "sample")}


def _rope(positions, rot, device):
    """cos and sin per position and pair, [positions, rot / 2, 2], base 10000."""
    a = torch.arange(0, rot, 2, dtype=torch.float64, device=device) / rot
    t = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * (10000.0 ** -a)
    return torch.stack([t.cos(), t.sin()], -1).float().contiguous()


def _paged(case, gen):
    """Caches, page table (pages in random order, -1 past a sequence's end) and lengths, on the GPU."""
    dev, dt = "cuda", DTYPES[case["dtype"]]
    new, cached = _lengths(case)
    page, B = case["page"], case["B"]
    need = torch.tensor([-(-(n + c) // page) for n, c in zip(new, cached)], dtype=torch.int64)
    total, width = int(need.sum()), int(need.max())
    order = torch.randperm(total, generator=gen, device=dev)
    first = (need.cumsum(0) - need).to(dev)
    col = torch.arange(width, device=dev)
    table = torch.where(col < need.to(dev)[:, None], order[(first[:, None] + col).clamp(max=total - 1)], -1).to(torch.int32).contiguous()
    shape = (total, page, case["Hkv"], case["D"])
    k, v = (torch.empty(shape, dtype=dt, device=dev).normal_(generator=gen) for _ in range(2))
    start = torch.tensor([0] + new, dtype=torch.int64).cumsum(0).to(torch.int32).to(dev)
    return {"k_cache": k, "v_cache": v, "table": table, "cache_len": torch.tensor(cached, dtype=torch.int32, device=dev),
            # Blocks of one size need no list of where each sequence's tokens start.
            "q_start": None if len(set(new)) == 1 else start, "T": sum(new), "most": max(new)}


def prepare(case, seed):
    dev, dt = "cuda", DTYPES[case["dtype"]]
    gen = torch.Generator(device=dev)
    gen.manual_seed(int(seed))
    if case["op"] == "sample":
        B, R, V = case["B"], case["R"], case["V"]
        logits = torch.empty((B, R, V), dtype=torch.float32, device=dev).normal_(0.0, case["std"], generator=gen)
        at = torch.randint(0, V, (B, R, 32), generator=gen, device=dev)
        logits.scatter_add_(2, at, 2.0 + 8.0 * torch.rand((B, R, 32), generator=gen, device=dev))
        s = {"logits": logits.to(dt), "uniforms": torch.rand((B, R), generator=gen, device=dev)}
        part = torch.rand((4, B), generator=gen, device=dev) if case["mixed"] else torch.ones((4, B), device=dev)
        greedy = torch.arange(B, device=dev) % 8 == 5
        T = case["temperature"] * (0.5 + 0.5 * part[0])
        s["temperature"] = torch.where(greedy, 0.0, T) if case["mixed"] else T
        s["top_k"] = torch.ceil(part[1] * case["top_k"]).to(torch.int32)
        s["top_p"] = 1.0 - (1.0 - case["top_p"]) * part[2]
        s["min_p"] = case["min_p"] * part[3]
        s["tokens"] = torch.empty((B, R), dtype=torch.int32, device=dev)
        s["probs"] = torch.empty((B, R), dtype=torch.float32, device=dev)
        return {"case": case, **s}
    s = {"case": case, **_paged(case, gen)}
    T, Hq, Hkv, D = s["T"], case["Hq"], case["Hkv"], case["D"]
    if case["op"] == "append":
        # One projection's output: q, k and v of a token side by side.
        qkv = torch.empty((T, Hq + 2 * Hkv, D), dtype=dt, device=dev).normal_(generator=gen)
        s["q"], s["k"], s["v"] = qkv[:, :Hq], qkv[:, Hq:Hq + Hkv], qkv[:, Hq + Hkv:]
        s["rope"] = _rope(case["ctx"] + case["n"], case["rot"], dev)
    else:
        # Scores with a spread of 2, so that some keys matter more than others.
        s["q"] = torch.empty((T, Hq, D), dtype=dt, device=dev).normal_(0.0, 2.0, generator=gen)
    s["out"] = torch.empty((T, Hq, D), dtype=dt, device=dev)
    if own:
        from paper_2608_29748_gb300 import binding as rt

        s["cache"] = rt.KvCache(s["k_cache"], s["v_cache"], s["table"])
        if case["op"] == "attend":
            s["ws"] = rt.AttendWorkspace(Hq, Hkv, D, dt)
    return s


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


def _plain_append(s):
    case = s["case"]
    b, i = _tokens(s)
    pos = s["cache_len"].long()[b] + i
    page, slot = s["table"].long()[b, pos // case["page"]], pos % case["page"]
    cs = s["rope"][pos]
    s["out"].copy_(_rotated(s["q"].float(), cs, case["rot"], case["interleaved"]))
    s["k_cache"][page, slot] = _rotated(s["k"].float(), cs, case["rot"], case["interleaved"]).to(s["k"].dtype)
    s["v_cache"][page, slot] = s["v"]
    return {"q": s["out"], "k": s["k_cache"], "v": s["v_cache"]}


def _plain_attend(s):
    case = s["case"]
    B, n, Hq, Hkv, D = case["B"], s["most"], case["Hq"], case["Hkv"], case["D"]
    G, dev = Hq // Hkv, s["q"].device
    b, i = _tokens(s)
    q = torch.zeros((B, n, Hq, D), device=dev)
    q[b, i] = s["q"].float()
    q = q.view(B, n, Hkv, G, D).permute(0, 2, 1, 3, 4).reshape(B, Hkv, n * G, D)
    table = s["table"].long()
    k, v = (x[table.clamp(min=0)].reshape(B, -1, Hkv, D).float().transpose(1, 2) for x in (s["k_cache"], s["v_cache"]))
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
    return s["out"]


def _plain_sample(s):
    B, R, V = s["logits"].shape
    each = lambda x: x[:, None].expand(B, R).reshape(-1, 1)  # noqa: E731
    x = s["logits"].float().reshape(B * R, V) + 0.0
    x = torch.where(x.isnan(), -math.inf, x)
    T, k, p, least = each(s["temperature"]), each(s["top_k"]).long(), each(s["top_p"]), each(s["min_p"])
    greedy = T <= 0
    inv, k = torch.where(greedy, 1.0, 1.0 / T), torch.where(greedy, 1, torch.where((k <= 0) | (k > V), V, k))
    top = x.amax(-1, keepdim=True)
    e = (torch.where(x == top, 0.0, x - top) * inv).exp()
    w = (e * 2147483648.0).round().long()
    order = x.sort(dim=-1, descending=True, stable=True)[1]
    ranked = w.gather(-1, order)
    upto = ranked.cumsum(-1)
    before = upto - ranked
    mass = upto.gather(-1, k - 1)
    rank = torch.arange(V, device=x.device)
    keep = (rank < k) & ((before.double() < p.double() * mass.double()) | (p >= 1) | (rank == 0)) & (e.gather(-1, order) >= least)
    del ranked, upto, before
    w = w * torch.zeros_like(keep).scatter_(-1, order, keep)
    upto = w.cumsum(-1)
    total = upto[:, -1:]
    u = s["uniforms"].reshape(-1, 1)
    at = torch.minimum((u.double() * total.double()).floor().long(), total - 1)
    token = (upto <= at).sum(-1, keepdim=True)
    none = top == -math.inf
    prob = (e.gather(-1, token.clamp(max=V - 1)).double() * 2147483648.0 / total.double()).float()
    s["tokens"].copy_(torch.where(none, -1, token).view(B, R))
    s["probs"].copy_(torch.where(none, 0.0, prob).view(B, R))
    return {"tokens": s["tokens"], "probs": s["probs"]}


def run(s):
    case = s["case"]
    if not own:
        return {"append": _plain_append, "attend": _plain_attend, "sample": _plain_sample}[case["op"]](s)
    from paper_2608_29748_gb300 import binding as rt

    if case["op"] == "append":
        rt.retrace_kv_append(s["q"], s["k"], s["v"], s["cache"], s["cache_len"], s["rope"], s["out"], q_start=s["q_start"],
                             interleaved=case["interleaved"])
        return {"q": s["out"], "k": s["k_cache"], "v": s["v_cache"]}
    if case["op"] == "attend":
        rt.retrace_attend(s["q"], s["cache"], s["cache_len"], s["out"], s["ws"], q_start=s["q_start"], window=case["window"],
                          sinks=case["sinks"], causal=case["causal"])
        return s["out"]
    rt.retrace_sample(s["logits"], s["uniforms"], s["tokens"], s["probs"], temperature=s["temperature"], top_k=s["top_k"],
                      top_p=s["top_p"], min_p=s["min_p"])
    return {"tokens": s["tokens"], "probs": s["probs"]}


def _exact_append(s):
    case = s["case"]
    rot, page = case["rot"], case["page"]
    new, cached = _lengths(case)
    k, v = s["k_cache"].double(), s["v_cache"].double()
    q = torch.empty(s["q"].shape, dtype=torch.float64, device=k.device)
    pairs = torch.arange(rot // 2, device=k.device)
    first, second = (2 * pairs, 2 * pairs + 1) if case["interleaved"] else (pairs, pairs + rot // 2)
    t = 0
    for b, (n, c) in enumerate(zip(new, cached)):
        pos = torch.arange(c, c + n, device=k.device)
        # The table's values are inputs: the rotation multiplies complex numbers by them.
        turn = torch.view_as_complex(s["rope"][pos].double())[:, None, :]
        where = s["table"][b].long()[torch.div(pos, page, rounding_mode="floor")], pos.remainder(page)
        for src, put in ((s["q"], None), (s["k"], k)):
            x = src[t:t + n].double()
            z = torch.complex(x[..., first], x[..., second]) * turn
            x[..., first], x[..., second] = z.real, z.imag
            if put is None:
                q[t:t + n] = x
            else:
                put[where] = x
        v[where] = s["v"][t:t + n].double()
        t += n
    return {"q": q, "k": k, "v": v}


def _exact_attend(s):
    case = s["case"]
    Hkv, D, page, w = case["Hkv"], case["D"], case["page"], case["window"]
    G = case["Hq"] // Hkv
    new, cached = _lengths(case)
    out = torch.empty(s["q"].shape, dtype=torch.float64, device=s["q"].device)
    t = 0
    for b, (n, c) in enumerate(zip(new, cached)):
        j = torch.arange(c + n, device=out.device)
        where = s["table"][b].long()[torch.div(j, page, rounding_mode="floor")], j.remainder(page)
        k, v = s["k_cache"][where].double(), s["v_cache"][where].double()
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
    return out


def _exact_sample(s):
    B, R, V = s["logits"].shape
    probs = torch.zeros((B, R), dtype=torch.float64, device=s["logits"].device)
    for b in range(B):
        x = s["logits"][b].double()
        T, k = float(s["temperature"][b]), int(s["top_k"][b])
        if T <= 0:
            probs[b] = 1.0
            continue
        full = torch.softmax(x / T, -1)
        best, order = torch.sort(full, dim=-1, descending=True, stable=True)
        keep = torch.ones_like(best, dtype=torch.bool)
        if 0 < k < V:
            keep[:, k:] = False
        chosen = best * keep
        chosen /= chosen.sum(-1, keepdim=True)
        if float(s["top_p"][b]) < 1:
            keep[:, 1:] &= (chosen.cumsum(-1) - chosen)[:, 1:] < float(s["top_p"][b])
        keep &= best >= float(s["min_p"][b]) * best[:, :1]
        full.mul_(torch.zeros_like(keep).scatter_(-1, order, keep))
        full /= full.sum(-1, keepdim=True)
        u = s["uniforms"][b].double()[:, None]
        token = torch.searchsorted(full.cumsum(-1), u, right=True).clamp(max=V - 1)
        probs[b] = full.gather(-1, token)[:, 0]
    return {"tokens": None, "probs": probs}


def exact(case, seed):
    return {"append": _exact_append, "attend": _exact_attend, "sample": _exact_sample}[case["op"]](prepare(case, seed))
