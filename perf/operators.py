"""The operators of a serving step over a paged key/value cache, as cases that can be timed and compared.

A profile table says what a step of a served model takes at a load; these are the parts of such a step that depend on the lengths of the
requests in it.  The kinds:

  plan     dyn_kv_step: block tables and slot maps from request lengths, pages handed out and taken back
  append   dyn_rope_append: rotary positions, new keys and values into the cache's pages
  attend   dyn_paged_attention: attention of each request's new tokens over its pages
  step     the three one after the other, as a serving step makes them

Where `own` is false, `run` computes them in elementary torch operations in 32 bits (angles in 64); where it is true, it calls this library.
`exact` computes the same in 64 bits, request by request.  Lengths follow from the case alone (which request has which length, from the seed).
"""
import math

import numpy as np
import torch

own = False

_TYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "e4m3": torch.float8_e4m3fn}
_E4M3_MAX = 448.0


# ---- the cases ----------------------------------------------------------------------------------------------

def _case(kind, name=None, **kw):
    # n_req requests; `chunked` of them bring a chunk of up to `chunk` new tokens, the others one token; up to `context` tokens are in the
    # cache already (`spread`: how much the shortest is below the longest); `released` of them are through and give their pages back;
    # `room`: free pages as a share of what the step asks for
    c = {"kind": kind, "n_req": 64, "chunked": 0, "chunk": 1, "context": 4096, "spread": 0.9, "released": 0, "room": 1.5, "page": 16,
         "q_heads": 64, "kv_heads": 8, "dim": 128, "type": "bf16", "cache": "bf16", "window": 0, "sinks": 0,
         "rotary": 128, "interleaved": False, "stretch": 1.0}
    c.update(kw)
    if name is not None:
        c["name"] = name
    return c


def listed():
    return [
        # an instance that generates for 64 requests: one token each.  Latency
        _case("plan", "plan-decode"),
        # a thousand requests, some of them with chunks of their prompts, some through, and too few pages for the last ones
        _case("plan", "plan-mixed", n_req=999, chunked=100, chunk=509, context=16384, released=41, room=0.9),
        # a queue of three thousand prompts admitted at once: 1.6 million tokens
        _case("plan", "plan-prompts", n_req=3000, chunked=3000, chunk=1021, context=0, page=32),
        # 64 new tokens of grouped heads (64 over 8): latency
        _case("append", "append-decode"),
        # a long chunk, neighbouring pairs rotated in three quarters of the head, positions stretched, an 8-bit cache
        _case("append", "append-chunk-8bit", n_req=9, chunked=9, chunk=911, context=8192, q_heads=32, type="fp16", cache="e4m3", rotary=96, interleaved=True, stretch=4.0, page=64),
        # one request of a short conversation: the smallest call, latency
        _case("attend", "attend-decode-one", n_req=1, context=1531),
        # an instance that generates for 64 requests of mixed lengths
        _case("attend", "attend-decode", context=8192),
        # three documents of up to 131072 tokens in 8 bits
        _case("attend", "attend-decode-long-8bit", n_req=3, context=131072, spread=0.5, cache="e4m3", page=64),
        # chunks of two prompts over what is there of them, a key head for each query head, heads of 80
        _case("attend", "attend-chunk", n_req=2, chunked=2, chunk=1000, context=12000, spread=0.3, q_heads=24, kv_heads=24, dim=80, rotary=80, type="fp16", cache="fp16", page=32),
        # a prompt of 8192 tokens from its start
        _case("attend", "attend-prompt", n_req=1, chunked=1, chunk=8192, context=0, q_heads=32),
        # chunks of four long documents under a sliding window with four first tokens that stay visible
        _case("attend", "attend-window", n_req=4, chunked=4, chunk=512, context=32768, spread=0.4, window=4096, sinks=4),
        # a whole step: three chunks of prompts beside 45 requests that generate
        _case("step", "step-mixed", n_req=48, chunked=3, chunk=256, context=4000, q_heads=32),
    ]


def _lengths(c):
    """(tokens in the cache, new tokens) of the requests, in an order that the seed changes: evenly spread quantiles, short ones more often."""
    B = c["n_req"]
    u = (np.arange(B) + 1.0) / B
    ctx = np.rint(c["context"] * (1.0 - c["spread"] * (1.0 - u * u)) if B > 1 else c["context"] * np.ones(1)).astype(np.int64)
    ctx = ctx[(np.arange(B) * 7919) % B] if B > 1 and B % 7919 else ctx       # which lengths come with chunks
    new = np.ones(B, dtype=np.int64)
    n = c["chunked"]
    if n:
        new[:n] = np.rint(c["chunk"] * (0.05 + 0.95 * (np.arange(n) + 1.0) / n)).clip(1)
    if c["released"]:
        new[-c["released"]:] = -1
    return ctx, new


def _pages(c):
    """(columns of the block table, pages in use, pages that the step asks for, pages of the cache)."""
    ctx, new = _lengths(c)
    P, n = c["page"], np.maximum(new, 0)
    used = -(-ctx // P)
    asked = int((-(-(ctx + n) // P) - used).sum())
    cols = int((-(-(ctx + n) // P)).max()) + 1
    free = int(math.ceil(asked * c["room"])) + 1
    return cols, int(used.sum()), asked, int(used.sum()) + free


def _pairs(c):
    """Visible (query token, key) pairs, and keys that some query token of their request sees."""
    ctx, new = _lengths(c)
    pairs = keys = 0
    for a, n in zip(ctx.tolist(), np.maximum(new, 0).tolist()):
        if not n:
            continue
        p = np.arange(a, a + n, dtype=np.int64)
        seen = p + 1
        if c["window"]:
            low = np.maximum(p - c["window"] + 1, 0)
            seen = p - low + 1 + np.minimum(low, c["sinks"])
            keys += int(a + n - low[0] + min(low[0], c["sinks"]))
        else:
            keys += a + n
        pairs += int(seen.sum())
    return pairs, keys


def _cost(c):
    """(elements of the padded score table, multiplications over it): what the plain form pays."""
    ctx, new = _lengths(c)
    table = c["n_req"] * c["q_heads"] * int(new.max()) * int((ctx + new).max())
    return table, table * c["dim"]


def draw(rng):
    log = lambda lo, hi: int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))  # noqa: E731
    # shares of the draws as the serving loop makes the calls: attention most of all
    kind = rng.choice(["plan", "append", "attend", "attend", "attend", "step"])
    t = rng.choice(["bf16", "fp16"])
    kv = rng.choice([1, 2, 4, 8, 8])
    dim = rng.choice([64, 80, 96, 128, 128])
    c = _case(kind, page=rng.choice([16, 16, 32, 64, 128]), type=t, cache=rng.choice([t, t, "e4m3"]), kv_heads=kv, q_heads=kv * rng.choice([1, 3, 4, 6, 8]),
              dim=dim, rotary=rng.choice([dim, dim, dim // 2]), interleaved=rng.random() < 0.5, stretch=rng.choice([1.0, 1.0, 4.0, 8.0]), spread=round(rng.uniform(0.2, 0.95), 2))
    if kind == "plan":
        B = log(1, 3000)
        c.update(n_req=B, chunked=rng.randint(0, B), chunk=log(1, 1021), context=log(1, 16384), released=rng.randint(0, B // 8), room=round(rng.uniform(0.8, 1.5), 2))
        c["chunked"] = min(c["chunked"], B - c["released"])
        return c
    if kind == "append":
        B = log(1, 256)
        c.update(n_req=B, chunked=rng.randint(0, B), context=log(16, 8192))
        c["chunk"] = log(1, max(2, 4900 // max(1, c["chunked"])))
        return c
    if rng.random() < 0.3:
        c.update(window=log(64, 8192), sinks=rng.choice([0, 1, 4, 16]))
    if kind == "attend" and rng.random() < 0.5:                     # one token each
        c.update(n_req=log(1, 128), context=log(16, 131072))
        while c["n_req"] * c["context"] > 300_000:
            c["n_req"], c["context"] = max(1, c["n_req"] * 2 // 3), c["context"] * 3 // 4
        return c
    c.update(n_req=log(1, 48), chunk=log(2, 4096), context=log(1, 32768))
    c["chunked"] = rng.randint(1, c["n_req"])
    while _cost(c)[0] > 1.5e9 or c["n_req"] * (c["context"] + c["chunk"]) > 300_000:
        c["n_req"], c["chunk"], c["context"] = max(1, c["n_req"] * 2 // 3), max(2, c["chunk"] * 3 // 4), max(1, c["context"] * 3 // 4)
        c["chunked"] = min(c["chunked"], c["n_req"])
    return c


# ---- inputs -------------------------------------------------------------------------------------------------

def _frequencies(c):
    """Angle per position of each rotated pair.  Stretched positions: slow pairs are slowed by the factor, fast ones are left, a ramp in between."""
    w = 10000.0 ** (-np.arange(c["rotary"] // 2, dtype=np.float64) * 2.0 / c["rotary"])
    if c["stretch"] != 1.0:
        turns = 8192.0 * w / (2.0 * math.pi)
        part = np.clip((turns - 1.0) / (32.0 - 1.0), 0.0, 1.0)
        w = w / c["stretch"] * (1.0 - part) + w * part
    return w


def prepare(case, seed):
    c, dev = case, torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(int(seed) * 1000003 + 17)
    host = np.random.RandomState((int(seed) * 7 + 5) % (1 << 31))
    ctx, new = _lengths(c)
    order = host.permutation(c["n_req"])
    ctx, new = ctx[order], new[order]
    n = np.maximum(new, 0)
    P = c["page"]
    cols, used, asked, N = _pages(c)
    have, last = -(-ctx // P), -(-(ctx + n) // P)
    pool = torch.randperm(N, generator=g, device=dev).to(torch.int32)
    col = torch.arange(cols, device=dev)[None]
    d = lambda a, t=torch.int32: torch.from_numpy(np.ascontiguousarray(a)).to(device=dev, dtype=t)  # noqa: E731
    s = {"case": c, "n_token": int(n.sum()), "max_new": int(n.max()), "max_kv": int((ctx + n).max()), "ctx_len": d(ctx), "new_len": d(new)}
    # pages in use: the first of a shuffled pool; the ring of free ones starts anywhere
    start = d(np.cumsum(have) - have)[:, None]
    s["block_table"] = torch.where(col < d(have)[:, None], pool[(start + col).clamp(max=N - 1).long()], torch.full((), -1, dtype=torch.int32, device=dev))
    first = int(host.randint(0, N))
    ring = torch.zeros(N, dtype=torch.int32, device=dev)
    ring[(first + torch.arange(N - used, device=dev)) % N] = pool[used:]
    s["free_pages"], s["free_state"] = ring, torch.tensor([first, N - used], dtype=torch.int32, device=dev)
    if c["kind"] == "plan":
        return s
    # grouped heads; queries that pick some keys over others
    T, H, G, D = s["n_token"], c["q_heads"], c["kv_heads"], c["dim"]
    t = _TYPES[c["type"]]
    r = lambda *shape: torch.randn(*shape, generator=g, device=dev, dtype=torch.float32)  # noqa: E731
    quant = c["cache"] == "e4m3"
    s["k_scale"] = (0.01 + 0.01 * torch.rand(G, generator=g, device=dev)) if quant else None
    s["v_scale"] = (0.01 + 0.01 * torch.rand(G, generator=g, device=dev)) if quant else None
    for x in ("k", "v"):
        a = torch.empty(N, G, P, D, dtype=_TYPES[c["cache"]], device=dev)
        for i in range(0, N, 4096):
            f = r(min(4096, N - i), G, P, D)
            a[i:i + 4096] = (f / s[x + "_scale"][:, None, None] if quant else f).to(a.dtype)
        s[x + "_cache"] = a
    s["inv_freq"], s["rope_scale"] = _frequencies(c), 1.0 if c["stretch"] == 1.0 else 0.1 * math.log(c["stretch"]) + 1.0
    s["scale"] = 1.0 / math.sqrt(D)
    s["workspace"] = torch.zeros(96 << 20, dtype=torch.uint8, device=dev)     # what such a program keeps for its steps, zero when it is made
    if c["kind"] in ("append", "step"):
        qkv = r(T, H + 2 * G, D).to(t)                                        # one product's output: queries, keys and values side by side
        qkv[:, :H] *= 2.0
        s["q"], s["k"], s["v"] = qkv[:, :H], qkv[:, H:H + G], qkv[:, H + G:]
    else:
        s["q"] = (2.0 * r(T, H, D)).to(t)
    if c["kind"] != "step":                                                   # a step makes these itself
        for x, v in zip(("cu_new", "kv_len", "next_len", "pos", "slot", "block_table", "free_pages", "free_state"), _plain_step(s)):
            if x in ("cu_new", "kv_len", "pos", "slot", "block_table"):
                s[x] = v
    return s


# ---- the plain forms ----------------------------------------------------------------------------------------

def _plain_step(s):
    P, T = s["case"]["page"], s["n_token"]
    c, n = s["ctx_len"].long(), s["new_len"].long()
    table, ring = s["block_table"], s["free_pages"]
    N, (B, cols) = ring.numel(), table.shape
    first, count = s["free_state"].long()
    gone, n = n < 0, n.clamp(min=0)
    have = (c + P - 1) // P
    need = (c + n + P - 1) // P - have
    before = need.cumsum(0) - need
    fits = (need == 0) | (before + need <= count)
    taken = (need * fits).sum()
    back = have * gone
    back_at = back.cumsum(0) - back
    cu = torch.cat([torch.zeros(1, dtype=torch.int64, device=c.device), n.cumsum(0)])
    col = torch.arange(cols, device=c.device)[None]
    fresh = (col >= have[:, None]) & (col < (have + need)[:, None]) & fits[:, None]
    table = torch.where(fresh, ring[(first + before[:, None] + col - have[:, None]) % N], table)
    to = torch.where(gone[:, None] & (col < have[:, None]), (first + count + back_at[:, None] + col) % N, N)
    ring = torch.cat([ring, ring[:1]]).scatter(0, to.reshape(-1), table.reshape(-1))[:N]
    of = torch.repeat_interleave(torch.arange(B, device=c.device), n, output_size=T)
    pos = c[of] + torch.arange(T, device=c.device) - cu[of]
    slot = table[of, pos // P].long() * P + pos % P
    pos, slot = torch.where(fits[of], pos, -1), torch.where(fits[of], slot, -1)
    kv = torch.where(fits & ~gone, c + n, 0)
    nxt = torch.where(gone, 0, torch.where(fits, c + n, c))
    state = torch.stack([(first + taken) % N, count - taken + back.sum()])
    i = torch.int32
    return cu.to(i), kv.to(i), nxt.to(i), pos.to(i), slot.to(i), table, ring, state.to(i)


def _rotate(c, x, cos, sin):
    r = c["rotary"]
    x = x.float()
    if c["interleaved"]:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
    else:
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
    return torch.cat([y, x[..., r:]], -1)


def _plain_append(s, pos, slot):
    c = s["case"]
    angle = pos.double()[:, None, None] * torch.from_numpy(s["inv_freq"]).to(pos.device)
    cos, sin = (angle.cos() * s["rope_scale"]).float(), (angle.sin() * s["rope_scale"]).float()
    q, k, v = _rotate(c, s["q"], cos, sin), _rotate(c, s["k"], cos, sin), s["v"].float()
    if s["k_scale"] is not None:
        k, v = ((x / f[:, None]).clamp(-_E4M3_MAX, _E4M3_MAX) for x, f in ((k, s["k_scale"]), (v, s["v_scale"])))
    there = (slot >= 0).nonzero()[:, 0]
    page, at = slot[there].long() // c["page"], slot[there].long() % c["page"]
    # 8 bits are written as bytes: torch has no indexed store for them
    for cache, x in ((s["k_cache"], k), (s["v_cache"], v)):
        x = x[there].to(cache.dtype)
        if x.element_size() == 1:
            cache.view(torch.uint8)[page, :, at] = x.view(torch.uint8)
        else:
            cache[page, :, at] = x
    return q.to(s["q"].dtype)


def _plain_attend(s, q, table, cu, kv):
    c = s["case"]
    B, P, H, G, D = c["n_req"], c["page"], c["q_heads"], c["kv_heads"], c["dim"]
    n, cols, dev = s["max_new"], -(-s["max_kv"] // c["page"]), q.device
    cu, kv = cu.long(), kv.long()
    page = table[:, :cols].clamp(min=0).long()
    j = torch.arange(cols * P, device=dev)
    look = lambda x, f: x.view(torch.uint8)[page].view(x.dtype).float() * (1.0 if f is None else f[:, None, None]) if x.element_size() == 1 else x[page].float()  # noqa: E731
    k = look(s["k_cache"], s["k_scale"]).transpose(1, 2).reshape(B, G, cols * P, D)
    v = look(s["v_cache"], s["v_scale"]).transpose(1, 2).reshape(B, G, cols * P, D)
    v = torch.where((j < kv[:, None])[:, None, :, None], v, 0.0)
    i = torch.arange(n, device=dev)
    count = cu[1:] - cu[:-1]
    rows = (cu[:-1, None] + i).clamp(max=max(0, q.shape[0] - 1))
    x = q[rows].float().view(B, n, G, H // G, D).permute(0, 2, 3, 1, 4).reshape(B, G, H // G * n, D)
    score = (torch.matmul(x, k.transpose(2, 3).contiguous()) * s["scale"]).view(B, G, H // G, n, cols * P)
    p = (kv - count)[:, None] + i
    seen = j <= p[..., None]
    if c["window"]:
        seen &= (j > p[..., None] - c["window"]) | (j < c["sinks"])
    score = torch.where(seen[:, None, None], score, -math.inf)
    some = seen.any(-1)[:, None, None, :, None]
    score = score.sub_(torch.where(some, score.amax(-1, keepdim=True), 0.0)).exp_()
    total = score.sum(-1, keepdim=True)
    o = torch.matmul(score.view(B, G, H // G * n, cols * P), v).view(B, G, H // G, n, D)
    o = torch.where(some, o / total, 0.0).permute(0, 3, 1, 2, 4).reshape(B, n, H, D)
    of = torch.repeat_interleave(torch.arange(B, device=dev), count, output_size=q.shape[0])
    return o[of, torch.arange(q.shape[0], device=dev) - cu[of]].to(q.dtype)


_STEP = ("cu_new", "kv_len", "next_len", "pos", "slot", "block_table", "free_pages", "free_state")


def _plain(s):
    kind = s["case"]["kind"]
    if kind == "plan":
        return dict(zip(_STEP, _plain_step(s)))
    if kind == "append":
        return {"q": _plain_append(s, s["pos"], s["slot"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if kind == "attend":
        return {"out": _plain_attend(s, s["q"], s["block_table"], s["cu_new"], s["kv_len"])}
    p = dict(zip(_STEP, _plain_step(s)))
    q = _plain_append(s, p["pos"], p["slot"])
    return {"out": _plain_attend(s, q, p["block_table"], p["cu_new"], p["kv_len"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"], **p}


# ---- the library's --------------------------------------------------------------------------------------------

def _own(s):
    import paper_2408_00741_amd as dyn
    c = s["case"]

    def plan():
        return dyn.dyn_kv_step(s["ctx_len"], s["new_len"], s["n_token"], s["block_table"], s["free_pages"], s["free_state"], c["page"])

    def append(pos, slot):
        return dyn.dyn_rope_append(s["q"], s["k"], s["v"], pos, slot, s["k_cache"], s["v_cache"], s["inv_freq"], interleaved=c["interleaved"],
                                   rope_scale=s["rope_scale"], k_scale=s["k_scale"], v_scale=s["v_scale"])

    def attend(q, table, cu, kv):
        return dyn.dyn_paged_attention(q, s["k_cache"], s["v_cache"], table, cu, kv, s["max_new"], s["max_kv"], scale=s["scale"], window=c["window"],
                                       n_sink=c["sinks"], k_scale=s["k_scale"], v_scale=s["v_scale"], workspace=s["workspace"])

    if c["kind"] == "plan":
        return plan()
    if c["kind"] == "append":
        return {"q": append(s["pos"], s["slot"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"]}
    if c["kind"] == "attend":
        return {"out": attend(s["q"], s["block_table"], s["cu_new"], s["kv_len"])}
    p = plan()
    q = append(p["pos"], p["slot"])
    return {"out": attend(q, p["block_table"], p["cu_new"], p["kv_len"]), "k_cache": s["k_cache"], "v_cache": s["v_cache"], **p}


def run(state):
    return _own(state) if own else _plain(state)


# ---- what a pass cannot do without ------------------------------------------------------------------------------

def work(case):
    c = case
    ctx, new = _lengths(c)
    T, B, P = int(np.maximum(new, 0).sum()), c["n_req"], c["page"]
    H, G, D = c["q_heads"], c["kv_heads"], c["dim"]
    e, ce = 2, 1 if c["cache"] == "e4m3" else 2
    nbytes = flops = 0
    if c["kind"] in ("plan", "step"):
        back = int((-(-ctx // P))[new < 0].sum())
        fresh = min(_pages(c)[2], int(math.ceil(_pages(c)[2] * c["room"])) + 1)
        nbytes += 8 * B + 12 * B + 8 * T + 8 * fresh + 8 * back
        flops += 4 * T
    if c["kind"] in ("append", "step"):
        nbytes += T * D * (2 * H * e + 2 * G * (e + ce)) + 8 * T
        flops += T * (H + G) * c["rotary"] * 3
    if c["kind"] in ("attend", "step"):
        pairs, keys = _pairs(c)
        nbytes += 2 * keys * G * D * ce + 2 * T * H * D * e + 4 * (keys // P)
        flops += 4 * pairs * H * D
    return {"bytes": nbytes, "flops": flops}


# ---- the definition in 64 bits ------------------------------------------------------------------------------------

def _exact_step(s):
    P = s["case"]["page"]
    table, ring = s["block_table"].cpu().numpy().copy(), s["free_pages"].cpu().numpy().copy()
    first, count = (int(x) for x in s["free_state"].cpu())
    N, at, taken, end = ring.size, 0, 0, 0
    cu, kv, nxt, pos, slot = [0], [], [], [], []
    for b, (c, n) in enumerate(zip(s["ctx_len"].cpu().tolist(), s["new_len"].cpu().tolist())):
        have = -(-c // P)
        if n < 0:
            for i in range(have):
                ring[(first + count + end + i) % N] = table[b, i]
            end += have
            kv.append(0), nxt.append(0), cu.append(cu[-1])
            continue
        need = -(-(c + n) // P) - have
        ok = need == 0 or at + need <= count
        for i in range(need if ok else 0):
            table[b, have + i] = ring[(first + at + i) % N]
        p = np.arange(c, c + n)
        pos.append(p if ok else np.full(n, -1))
        slot.append(table[b, p // P].astype(np.int64) * P + p % P if ok else np.full(n, -1))
        kv.append(c + n if ok else 0), nxt.append(c + n if ok else c), cu.append(cu[-1] + n)
        at, taken = at + need, taken + (need if ok else 0)
    i = lambda a: torch.from_numpy(np.asarray(a).astype(np.int32)).cuda()  # noqa: E731
    none = np.zeros(0)
    return i(cu), i(kv), i(nxt), i(np.concatenate(pos or [none])), i(np.concatenate(slot or [none])), i(table), i(ring), i([(first + taken) % N, count - taken + end])


def _exact_append(s, pos, slot):
    c = s["case"]
    r, D = c["rotary"], c["dim"]
    w = torch.from_numpy(s["inv_freq"]).cuda()
    turn = torch.polar(torch.full((), s["rope_scale"], dtype=torch.float64, device="cuda"), pos.double()[:, None] * w)[:, None]
    lo = torch.arange(r // 2, device="cuda") * (2 if c["interleaved"] else 1)
    hi = lo + (1 if c["interleaved"] else r // 2)

    def rotated(x):
        y = x.double().clone()
        z = torch.complex(y[..., lo], y[..., hi]) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    q, k, v = rotated(s["q"]), rotated(s["k"]), s["v"].double()
    caches = []
    ok = slot >= 0
    for name, x in (("k", k), ("v", v)):
        f = s[name + "_scale"]
        if f is not None:
            x = (x / f.double()[:, None]).clamp(-_E4M3_MAX, _E4M3_MAX)
        cache = s[name + "_cache"].double()
        flat = cache.transpose(1, 2).reshape(-1, c["kv_heads"], D)             # [slot][head][dim]
        flat[slot[ok].long()] = x[ok]
        caches.append(flat.view(-1, c["page"], c["kv_heads"], D).transpose(1, 2))
    return q, caches[0], caches[1]


def _exact_attend(s, q, k_cache, v_cache, table, cu, kv):
    c = s["case"]
    P, H, G = c["page"], c["q_heads"], c["kv_heads"]
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    cu, kv = cu.cpu().tolist(), kv.cpu().tolist()
    for b in range(c["n_req"]):
        n, L = cu[b + 1] - cu[b], kv[b]
        if not n or not L:
            continue
        pages = table[b, :-(-L // P)].long()
        p = torch.arange(L - n, L, device=q.device)[:, None]
        j = torch.arange(L, device=q.device)
        hidden = (j > p) | ((j <= p - c["window"]) & (j >= c["sinks"])) if c["window"] else j > p
        for g in range(G):
            k, v = (x[:, g].reshape(-1, c["dim"])[(pages[:, None] * P + torch.arange(P, device=q.device)).view(-1)[:L]] for x in (k_cache, v_cache))
            k, v = (x.double() * (1.0 if f is None else f[g].double()) for x, f in ((k, s["k_scale"]), (v, s["v_scale"])))
            for h in range(g * (H // G), (g + 1) * (H // G)):
                a = (q[cu[b]:cu[b + 1], h].double() @ k.T * s["scale"]).masked_fill_(hidden, -math.inf)
                out[cu[b]:cu[b + 1], h] = torch.softmax(a, 1) @ v
    return out


def exact(case, seed):
    s = prepare(case, seed)
    kind = case["kind"]
    if kind == "plan":
        return dict(zip(_STEP, _exact_step(s)))
    if kind == "append":
        return dict(zip(("q", "k_cache", "v_cache"), _exact_append(s, s["pos"], s["slot"])))
    if kind == "attend":
        k, v = (x.float() if x.element_size() == 1 else x for x in (s["k_cache"], s["v_cache"]))
        return {"out": _exact_attend(s, s["q"], k, v, s["block_table"], s["cu_new"], s["kv_len"])}
    p = dict(zip(_STEP, _exact_step(s)))
    q, k, v = _exact_append(s, p["pos"], p["slot"])
    # what attention reads is what a step holds: rounded to the types of the queries and of the cache
    held = [x.to(s["k_cache"].dtype).float() for x in (k, v)]
    o = _exact_attend(s, q.to(s["q"].dtype), held[0], held[1], p["block_table"], p["cu_new"], p["kv_len"])
    return {"out": o, "k_cache": k, "v_cache": v, **p}
