"""The operators around streamed video attention, as cases to time and compare.

A video that is generated in pieces keeps the K and V of what it has already shown in a paged cache held in 8 bits, and
every new piece (a few latent frames, or a single token) goes through four calls on one stream: the plan that gives the
piece's tokens their pages, the rotary positions of its Q and K, the store of K and V into the pages, and attention
over the cache. One case is one call of one of them. The rotary positions serve whole clips and their backward pass too.

The plain forms below are elementary torch operations in 32 bits (angles in 64), rounded once at the end.
"""

import math

import torch

own = False

D = 128
E_MIN = -100  # smallest exponent of a page's scale
GRID_480P = (21, 30, 52)
GRID_720P = (21, 45, 80)
FRAME_480P = 30 * 52
DTYPES = {"bf16": torch.bfloat16, "fp16": torch.float16, "fp32": torch.float32}


# ---- cases ------------------------------------------------------------------


def _rope(name, batch, heads, kv_heads, T, H, W, dims, dtype="bf16", tokens=0, layout="bhnd", pairing="pairs", order="raster",
          inverse=False, theta=10000.0, t0=0):
    """tokens: 0 is the whole grid, else that many tokens of it by their ids (negative ones among them)."""
    return dict(name=name, op="rope", batch=batch, heads=heads, kv_heads=kv_heads, T=T, H=H, W=W, dt=dims[0], dy=dims[1],
                dx=dims[2], dtype=dtype, tokens=tokens, layout=layout, pairing=pairing, order=order, inverse=inverse,
                theta=theta, t0=t0)


def _plan(name, streams, new, held, page, retire=0):
    """streams that each bring up to `new` tokens to up to `held` cached ones; `retire` of them end and give back."""
    return dict(name=name, op="plan", streams=streams, new=new, held=held, page=page, retire=retire)


def _store(name, streams, new, held, page, heads, layout="bnhd"):
    return dict(name=name, op="store", streams=streams, new=new, held=held, page=page, heads=heads, layout=layout)


def _attn(name, streams, new, held, page, heads, kv_heads, frame=0, window=0, ragged=True, layout="bnhd"):
    """new: query tokens a stream; held: cached tokens a stream, the new ones among them; ragged: both spread out below that."""
    return dict(name=name, op="attn", streams=streams, new=new, held=held, page=page, heads=heads, kv_heads=kv_heads,
                frame=frame, window=window, ragged=ragged, layout=layout)


def listed():
    return [
        # One token of each of 16 streams, far into their videos: latency.
        _rope("rope_tokens", 1, 40, 40, 4096, 30, 52, (32, 48, 48), tokens=16, layout="bnhd"),
        # The backward pass of one GPU's five heads of a 480p clip in 32 bits, in the layout of the projections.
        _rope("rope_480p_backward", 1, 5, 5, *GRID_480P, (44, 42, 42), dtype="fp32", layout="bnhd", inverse=True),
        # Q and K of the whole 720p clip, forty heads, as the attention layer takes them.
        _rope("rope_720p", 1, 40, 40, *GRID_720P, (32, 48, 48)),
        # Pages for one more token of each of 64 streams.
        _plan("plan_tokens", 64, 1, 16000, 64),
        # A chunk of three latent 480p frames for each of up to 16 streams, some of which have ended.
        _plan("plan_chunks", 16, 3 * FRAME_480P, 30000, 64, retire=3),
        # Those 64 tokens into their pages, forty heads.
        _store("store_tokens", 64, 1, 1000, 64, 40),
        # A chunk of three latent 480p frames into the cache.
        _store("store_chunk", 1, 3 * FRAME_480P, 2000, 64, 40),
        # The smallest attention: one token of one stream, one GPU's five heads, a short cache.
        _attn("attn_token", 1, 1, 1001, 64, 5, 5),
        # One token of each of 64 streams, lengths of every size, shared key heads.
        _attn("attn_tokens", 64, 1, 16000, 64, 32, 8),
        # One token against a long clip's cache (111,600 tokens), forty heads.
        _attn("attn_token_long", 1, 1, 111600, 64, 40, 40, ragged=False),
        # Chunks of unequal length, causal by token and windowed, small pages.
        _attn("attn_chunks", 6, 700, 6000, 16, 12, 4, frame=1, window=4000),
        # The largest: a chunk of three 480p frames over the whole clip's cache, causal by frame.
        _attn("attn_chunk_480p", 1, 3 * FRAME_480P, 21 * FRAME_480P, 64, 40, 40, frame=FRAME_480P, ragged=False),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    """A case of the listed ones' ranges."""
    op = rng.choice(("rope", "plan", "store", "attn", "attn"))
    page = rng.choice((16, 32, 64, 64, 128))
    layout = rng.choice(("bhnd", "bnhd"))
    while True:
        if op == "rope":
            grid = (_log_int(rng, 1, 31), _log_int(rng, 8, 45), _log_int(rng, 8, 80))
            heads = _log_int(rng, 1, 40)
            c = _rope(None, rng.choice((1, 1, 2)), heads, rng.choice((heads, 0, max(1, heads // 4))), *grid,
                      rng.choice(((32, 48, 48), (44, 42, 42), (16, 24, 24))), dtype=rng.choice(("bf16", "bf16", "fp16", "fp32")),
                      tokens=rng.choice((0, 0, _log_int(rng, 1, 5000))), layout=layout,
                      pairing=rng.choice(("pairs", "halves")), order=rng.choice(("raster", "ids")),
                      inverse=rng.choice((False, True)), theta=rng.choice((10000.0, 256.0, 1000000.0)), t0=rng.choice((0, 7, 100000)))
            fits = c["batch"] * heads * (c["tokens"] or grid[0] * grid[1] * grid[2]) <= 40 * 75600
        elif op == "plan":
            new = rng.choice((1, _log_int(rng, 1, 4680)))
            c = _plan(None, _log_int(rng, 1, 256), new, _log_int(rng, 1, 30000), page, retire=rng.choice((0, 0, 1, 3)))
            fits = c["streams"] * new <= 16 * 4680 * 2 and c["retire"] < c["streams"]
        elif op == "store":
            new = rng.choice((1, _log_int(rng, 1, 4680)))
            c = _store(None, _log_int(rng, 1, 64), new, _log_int(rng, 1, 2000), page, _log_int(rng, 1, 40), layout=layout)
            fits = c["streams"] * new <= 4680 * 2 and c["streams"] * (c["held"] + new) * c["heads"] <= 64 * 1000 * 40
        else:
            group = rng.choice((1, 1, 4, 8))
            kv_heads = _log_int(rng, 1, 40 // group)
            new = rng.choice((1, 1, _log_int(rng, 1, 4680)))
            held = _log_int(rng, max(new, 2), 111600)
            c = _attn(None, _log_int(rng, 1, 64), new, held, page, group * kv_heads, kv_heads, frame=rng.choice((0, 1, 1, 256, FRAME_480P)),
                      window=rng.choice((0, 0, 300, 4000)), ragged=rng.choice((True, True, False)), layout=layout)
            scores = c["streams"] * c["heads"] * new * held
            fits = scores <= 40 * 4680 * 32760 and c["streams"] * held * kv_heads <= 111600 * 40
        if fits:
            c.pop("name")
            return c


# ---- inputs -----------------------------------------------------------------


def _gen(seed, salt=0):
    return torch.Generator(device="cuda").manual_seed(1000003 * seed + salt)


def _rows(gen, batch, heads, tokens, layout, dtype, spread=True):
    """Unit normal activations [batch, heads, tokens, D], channels of unequal size, in the layout's order in memory."""
    shape = (batch, heads, tokens, D) if layout == "bhnd" else (batch, tokens, heads, D)
    x = torch.randn(shape, generator=gen, device="cuda")
    if spread:
        x *= torch.exp(0.5 * torch.randn(D, generator=gen, device="cuda"))
    x = x.to(dtype)
    return x if layout == "bhnd" else x.transpose(1, 2)


def _lengths(case):
    """(cached tokens before, new tokens) of every stream, spread over the case's range, long streams among short ones."""
    n = case["streams"]
    if not case.get("ragged", True):
        return [case["held"]] * n, [case["new"]] * n
    spread = [((11 * k + 5) % n + 0.5) / n if math.gcd(11, n) == 1 else (k + 0.5) / n for k in range(n)]
    return ([int(case["held"] * a ** 1.5) for a in spread],
            [max(1, int(case["new"] * (0.3 + 0.7 * ((7 * k + 3) % n + 0.5) / n))) for k in range(n)])


def _pool(gen, lens, page, heads):
    """A pool somewhat larger than needed, pages in no order: (pages, block table)."""
    need = [-(-n // page) for n in lens]
    pages = sum(need) + 3
    order = torch.randperm(pages, generator=gen, device="cuda").to(torch.int32)
    width = max(need) + 2
    at = torch.tensor([0] + need, device="cuda").cumsum(0)
    col = torch.arange(width, device="cuda")
    idx = at[:-1, None] + col
    table = torch.where(col < torch.tensor(need, device="cuda")[:, None], order[idx.clamp(max=pages - 1)], -1)
    return pages, table.to(torch.int32).contiguous()


def _codes(gen, pages, heads, page):
    """Codes of normal values, as a store leaves them, and exponents near those of unit activations."""
    x = torch.randn(pages, heads, page, D, generator=gen, device="cuda", dtype=torch.bfloat16)
    codes = (x * 80).clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
    exps = torch.randint(-7, -4, (pages, heads), generator=gen, device="cuda", dtype=torch.int32)
    return codes, exps


def prepare(case, seed):
    gen = _gen(seed)
    i32 = dict(dtype=torch.int32, device="cuda")
    if case["op"] == "rope":
        n = case["tokens"] or case["T"] * case["H"] * case["W"]
        s = {"q": _rows(gen, case["batch"], case["heads"], n, case["layout"], DTYPES[case["dtype"]]), "k": None, "ids": None}
        if case["kv_heads"]:
            s["k"] = _rows(gen, case["batch"], case["kv_heads"], n, case["layout"], DTYPES[case["dtype"]])
        if case["tokens"]:
            s["ids"] = torch.randint(-1, case["T"] * case["H"] * case["W"], (case["batch"], n), generator=gen, **i32)
        elif case["order"] == "ids":
            s["ids"] = torch.randperm(n, generator=gen, device="cuda").to(torch.int32)
    elif case["op"] == "plan":
        held, new = _lengths(case)
        new[1:1 + case["retire"]] = [-1] * case["retire"]
        pages, table = _pool(gen, held, case["page"], 1)
        need = [max(0, -(-(h + max(0, n)) // case["page"])) for h, n in zip(held, new)]
        width = max(need) + 2
        grown = torch.full((len(held), width), -1, **i32)
        grown[:, :table.shape[1]] = table[:, :width]
        more = sum(need) + 5
        used = -(-torch.tensor(held) // case["page"])
        ring = torch.randperm(more, generator=gen, device="cuda").to(torch.int32) + pages  # pages that nobody holds
        ring = torch.cat([ring, torch.full((int(used.sum()) + 3,), -1, **i32)])
        s = {"held": torch.tensor(held, **i32), "new": torch.tensor(new, **i32), "table": grown, "ring": ring,
             "state": torch.tensor([0, more, 0], **i32), "tokens": sum(max(0, n) for n in new) + 7}
    elif case["op"] == "store":
        held, new = _lengths(case)
        pages, table = _pool(gen, [h + n for h, n in zip(held, new)], case["page"], case["heads"])
        n = sum(new)
        row = torch.repeat_interleave(torch.arange(len(new)), torch.tensor(new)).cuda()
        start = torch.tensor([0] + new).cumsum(0).cuda()
        pos = torch.arange(n, device="cuda") - start[row] + torch.tensor(held, device="cuda")[row]
        slots = table[row, pos // case["page"]] * case["page"] + pos % case["page"]
        s = {"k": _rows(gen, 1, case["heads"], n, case["layout"], torch.bfloat16), "v": _rows(gen, 1, case["heads"], n, case["layout"], torch.bfloat16),
             "slots": slots.to(torch.int32)}
        s["k8"], s["k_exp"] = _codes(gen, pages, case["heads"], case["page"])
        s["v8"], s["v_exp"] = _codes(gen, pages, case["heads"], case["page"])
    else:
        held, new = _lengths(case)
        new = [min(case["new"], n) for n in new]
        held = [max(h, n) for h, n in zip(held, new)]
        pages, table = _pool(gen, held, case["page"], case["kv_heads"])
        s = {"q": _rows(gen, 1, case["heads"], sum(new), case["layout"], torch.bfloat16, spread=False), "table": table,
             "kv_len": torch.tensor(held, **i32), "q_start": torch.tensor([0] + new, **i32).cumsum(0).to(torch.int32), "max_q": max(new)}
        s["k8"], s["k_exp"] = _codes(gen, pages, case["kv_heads"], case["page"])
        s["v8"], s["v_exp"] = _codes(gen, pages, case["kv_heads"], case["page"])
    s["case"] = dict(case)
    return s


# ---- one pass ---------------------------------------------------------------


def run(s):
    c = s["case"]
    if own:
        return _run_own(s, c)
    return {"rope": _plain_rope, "plan": _plain_plan, "store": _plain_store, "attn": _plain_attn}[c["op"]](s, c)


def _run_own(s, c):
    import paper_2607_16190_amd as fva

    if c["op"] == "rope":
        return fva.fva_rope(s["q"], s["k"], (c["H"], c["W"]), (c["dt"], c["dy"], c["dx"]), ids=s["ids"], origin=(c["t0"], 0, 0),
                            theta=c["theta"], pairing=fva.FVA_ROPE_PAIRS if c["pairing"] == "pairs" else fva.FVA_ROPE_HALVES,
                            inverse=c["inverse"])
    if c["op"] == "plan":
        kv_len, q_start, slots, ids, state = fva.fva_cache_plan(s["held"], s["new"], s["state"], s["ring"], s["table"], c["page"], s["tokens"])
        return kv_len, q_start, slots, ids, state, s["table"], s["ring"]
    if c["op"] == "store":
        fva.fva_cache_store(s["k"], s["v"], s["slots"], s["k8"], s["v8"], s["k_exp"], s["v_exp"])
        return s["k8"].view(torch.float8_e4m3fn), s["v8"].view(torch.float8_e4m3fn), s["k_exp"], s["v_exp"]
    return fva.fva_attn_cache(s["q"], s["k8"], s["v8"], s["k_exp"], s["v_exp"], s["table"], s["kv_len"], s["q_start"], s["max_q"],
                              frame=c["frame"], window=c["window"])


def _angles(c, ids, n):
    """Angles in 64 bits of n tokens and every rotated pair; (t, y, x) of a token from its id, none for a negative id."""
    p = torch.arange(n, device="cuda") if ids is None else ids.long()
    t, y, x = c["t0"] + p // (c["H"] * c["W"]), p // c["W"] % c["H"], p % c["W"]
    freq = [torch.tensor(float(c["theta"]), dtype=torch.float64, device="cuda") ** (-2.0 * torch.arange(d // 2, device="cuda", dtype=torch.float64) / d)
            for d in (c["dt"], c["dy"], c["dx"])]
    a = torch.cat([pos[..., None].double() * f for pos, f in zip((t, y, x), freq)], -1)
    a = torch.where(p[..., None] < 0, 0.0, a)
    return -a if c["inverse"] else a


def _rotate(x, cos, sin, pairing):
    r = 2 * cos.shape[-1]
    f = x.float()
    a, b = (f[..., 0:r:2], f[..., 1:r:2]) if pairing == "pairs" else (f[..., : r // 2], f[..., r // 2: r])
    u, v = a * cos - b * sin, a * sin + b * cos
    rot = torch.stack((u, v), -1).flatten(-2) if pairing == "pairs" else torch.cat((u, v), -1)
    return torch.cat((rot, f[..., r:]), -1).to(x.dtype)


def _plain_rope(s, c):
    a = _angles(c, s["ids"], s["q"].shape[2])
    cos, sin = a.cos().float(), a.sin().float()
    if a.dim() == 3:
        cos, sin = cos[:, None], sin[:, None]
    q = _rotate(s["q"], cos, sin, c["pairing"])
    return q if s["k"] is None else (q, _rotate(s["k"], cos, sin, c["pairing"]))


def _plain_plan(s, c):
    held, new, table, ring, state, page = s["held"].long(), s["new"].long(), s["table"], s["ring"], s["state"].long(), c["page"]
    cap = ring.shape[0]
    add = new.clamp(min=0)
    old_pages = -(-held // page)
    need = torch.where(new < 0, 0, -(-(held + add) // page) - old_pages)
    wide = old_pages + need <= table.shape[1]
    need = torch.where(wide, need, 0)
    upto = need.cumsum(0)
    fits = wide & ((need == 0) | (upto <= state[1]))
    kv_len = torch.where(new < 0, 0, torch.where(fits, held + add, held))
    first = upto - need
    q_start = torch.cat([add.new_zeros(1), add.cumsum(0)])
    # new pages from the front of the ring
    col = torch.arange(table.shape[1], device="cuda")
    which = col - old_pages[:, None]
    take = (which >= 0) & (which < need[:, None]) & fits[:, None]
    popped = ring[(state[0] + (first[:, None] + which).clamp(0, cap - 1)) % cap]
    table.copy_(torch.where(take, popped, table))
    # the pages of streams that have ended to its back
    back = torch.where(new < 0, old_pages, 0)
    behind = back.cumsum(0) - back
    gives = col < back[:, None]
    at = (state[0] + state[1] + behind[:, None] + col) % cap
    spare = torch.cat([ring, ring[:1]])
    spare.scatter_(0, torch.where(gives, at, cap).flatten(), table.flatten())
    ring.copy_(spare[:cap])
    taken = torch.where(fits, need, 0).sum()
    state_out = torch.stack([(state[0] + taken) % cap, state[1] - taken + back.sum(), (~fits).sum()])
    r = torch.arange(s["tokens"], device="cuda")
    b = (torch.searchsorted(q_start, r, right=True) - 1).clamp(max=len(held) - 1)
    pos = held[b] + r - q_start[b]
    real = (r < q_start[-1]) & fits[b]
    page_of = table[b, (pos // page).clamp(0, table.shape[1] - 1)]
    slots = torch.where(real, page_of * page + pos % page, -1)
    ids = torch.where(real, pos, -1)
    return (*(v.to(torch.int32) for v in (kv_len, q_start, slots, ids, state_out)), table, ring)


def _exponent(amax):
    """Smallest e >= E_MIN with amax <= 448 * 2^e."""
    m, x = torch.frexp(amax)
    return torch.where(amax > 0, x - 9 + (m > 0.875).int(), E_MIN).clamp(min=E_MIN)


def _plain_store(s, c):
    page = c["page"]
    slots = s["slots"].long()
    at, off = slots // page, slots % page
    pages, heads = s["k_exp"].shape
    col = torch.arange(page, device="cuda")
    first = torch.full((pages,), page, device="cuda").index_reduce_(0, at, off, "amin")
    touched = first < page
    k = _plain_store_one(s["k"], s["k8"], s["k_exp"], at, off, first, touched, col)
    v = _plain_store_one(s["v"], s["v8"], s["v_exp"], at, off, first, touched, col)
    return k, v, s["k_exp"], s["v_exp"]


def _plain_store_one(x, x8, x_exp, at, off, first, touched, col):
    f = x[0].transpose(0, 1).float()  # [tokens, heads, D]
    amax = torch.zeros(x_exp.shape, device="cuda").index_reduce_(0, at, f.abs().amax(-1), "amax")
    kept = torch.where((first > 0)[:, None], x_exp, E_MIN)
    e = torch.where(touched[:, None], torch.maximum(_exponent(amax), kept), x_exp)
    codes = x8.view(torch.float8_e4m3fn)
    old = codes.float() * torch.exp2((x_exp - e).float())[..., None, None]
    keep = (touched[:, None] & (col < first[:, None]))[:, None, :, None]
    x8.copy_(torch.where(keep, old.to(torch.float8_e4m3fn).view(torch.uint8), x8))
    x8[at, :, off] = (f * torch.exp2(-e.float())[at][..., None]).to(torch.float8_e4m3fn).view(torch.uint8)
    x_exp.copy_(e)
    return codes


def _visible(c, kv_len, q_len, rows, keys):
    """Which of `keys` positions the query rows [streams, rows] see."""
    p = (kv_len - q_len)[:, None] + rows
    end = torch.div(p, c["frame"], rounding_mode="floor") * c["frame"] + c["frame"] if c["frame"] else kv_len[:, None].expand_as(p)
    lo = (end - c["window"]).clamp(min=0) if c["window"] else torch.zeros_like(end)
    hi = torch.minimum(end, kv_len[:, None])
    return (keys >= lo[..., None]) & (keys < hi[..., None]) & (rows < q_len[:, None])[..., None]


def _plain_attn(s, c):
    q, table, page = s["q"][0].transpose(0, 1), s["table"].long().clamp(min=0), c["page"]  # [tokens, heads, D]
    kv_len, start = s["kv_len"].long(), s["q_start"].long()
    q_len = start[1:] - start[:-1]
    S, G, KH = len(kv_len), c["heads"] // c["kv_heads"], c["kv_heads"]
    rows = torch.arange(s["max_q"], device="cuda")
    at = (start[:-1, None] + rows).clamp(max=q.shape[0] - 1)

    def cached(x8, x_exp):  # [streams, kv heads, keys, D]
        x = x8.view(torch.float8_e4m3fn)[table].float() * torch.exp2(x_exp[table].float())[..., None, None]
        return x.transpose(1, 2).reshape(S, KH, -1, D)

    qs = q[at].float().reshape(S, s["max_q"], KH, G, D).permute(0, 2, 3, 1, 4).reshape(S, KH, G * s["max_q"], D)
    k = cached(s["k8"], s["k_exp"])
    p = torch.matmul(qs, k.transpose(2, 3)).mul_(1.0 / math.sqrt(D))
    del k
    seen = _visible(c, kv_len, q_len, rows.expand(S, -1), torch.arange(p.shape[-1], device="cuda"))
    p = p.view(S, KH, G, s["max_q"], -1).masked_fill_(~seen[:, None, None], -math.inf)
    p.sub_(p.amax(-1, keepdim=True).clamp_(min=-1e30)).exp_()
    total = p.sum(-1, keepdim=True)
    v = cached(s["v8"], s["v_exp"])
    o = torch.matmul(p.view(S, KH, G * s["max_q"], -1), v).view(S, KH, G, s["max_q"], D)
    o = torch.where(total > 0, o / total, 0.0).to(q.dtype)
    o = o.permute(0, 3, 1, 2, 4).reshape(S, s["max_q"], c["heads"], D)
    return o[rows < q_len[:, None]].transpose(0, 1)[None]


# ---- work and exact values --------------------------------------------------


def work(case):
    if case["op"] == "rope":
        n = case["tokens"] or case["T"] * case["H"] * case["W"]
        rows = case["batch"] * (case["heads"] + case["kv_heads"]) * n
        size = 4 if case["dtype"] == "fp32" else 2
        ids = 4 * n if case["tokens"] or case["order"] == "ids" else 0
        return {"bytes": 2 * rows * D * size + ids, "flops": 3 * rows * (case["dt"] + case["dy"] + case["dx"])}
    held, new = _lengths(case)
    page = case["page"]
    if case["op"] == "plan":
        grown = sum(-(-(h + n) // page) - -(-h // page) for h, n in zip(held, new))
        return {"bytes": 16 * len(held) + 8 * grown + 8 * sum(new), "flops": 4 * sum(new)}
    if case["op"] == "store":
        n = sum(new)
        return {"bytes": n * case["heads"] * (2 * D * 2 + 2 * D) + 4 * n, "flops": 4 * n * case["heads"] * D}
    pairs = keys = 0
    for h, n in zip(held, new):
        n = min(n, case["new"])
        h = max(h, n)
        lo_all = h
        f, w = case["frame"], case["window"]
        for i in range(n):
            p = h - n + i
            end = (p // f + 1) * f if f else h
            lo, hi = max(0, end - w) if w else 0, min(end, h)
            pairs += max(0, hi - lo)
            lo_all = min(lo_all, lo)
        keys += h - lo_all
    rows = sum(min(n, case["new"]) for n in new)
    return {"bytes": 2 * D * keys * case["kv_heads"] + 2 * rows * case["heads"] * D * 2, "flops": 4.0 * D * pairs * case["heads"]}


def _e4m3(codes):
    """The values of E4M3 codes in 64 bits, from the format's definition."""
    c = codes.long()
    sign, ex, m = 1.0 - 2.0 * (c >> 7), (c >> 3) & 15, (c & 7).double()
    return sign * torch.where(ex == 0, m * 2.0 ** -9, (8 + m) * torch.exp2((ex - 10).double()))


def exact(case, seed):
    if case["op"] == "plan":
        return None  # whole numbers only
    s = prepare(case, seed)
    if case["op"] == "rope":
        return _exact_rope(case, s)
    if case["op"] == "store":
        k, v = _exact_store(case, s["k"], s["k8"], s["k_exp"], s["slots"]), _exact_store(case, s["v"], s["v8"], s["v_exp"], s["slots"])
        return k, v, None, None
    if sum(s["kv_len"].tolist()) * s["max_q"] * case["heads"] > 4e10:
        return None
    return _exact_attn(case, s)


def _exact_rope(case, s):
    n = s["q"].shape[2]
    ids = torch.arange(n, device="cuda").expand(case["batch"], -1) if s["ids"] is None else s["ids"].long().expand(case["batch"], -1)
    W, H = case["W"], case["H"]
    axes = (torch.div(ids, H * W, rounding_mode="floor") + case["t0"], torch.div(ids, W, rounding_mode="floor") % H, ids % W)
    phase = [pos.double()[..., None] * torch.exp(-math.log(case["theta"]) * torch.arange(0, d, 2, device="cuda", dtype=torch.float64) / d)
             for pos, d in zip(axes, (case["dt"], case["dy"], case["dx"]))]
    phase = torch.cat(phase, -1) * (ids >= 0)[..., None]
    turn = torch.polar(torch.ones_like(phase), -phase if case["inverse"] else phase)[:, None]
    r = 2 * turn.shape[-1]

    def one(x):
        y = torch.empty(x.shape, dtype=torch.float64, device="cuda")
        for h in range(x.shape[1]):
            f = x[:, h: h + 1].double()
            pairs = f[..., :r].unflatten(-1, (-1, 2)) if case["pairing"] == "pairs" else f[..., :r].unflatten(-1, (2, -1)).transpose(-1, -2)
            z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
            y[:, h: h + 1] = torch.cat(((z if case["pairing"] == "pairs" else z.transpose(-1, -2)).flatten(-2), f[..., r:]), -1)
        return y

    return one(s["q"]) if s["k"] is None else (one(s["q"]), one(s["k"]))


def _exact_store(case, x, x8, x_exp, slots):
    """x * 2^-e where a token was written, the old value times its change of scale before the first of them in its page."""
    page = case["page"]
    y = _e4m3(x8)
    rows = x[0].transpose(0, 1).double()
    where = slots.tolist()
    by_page = {}
    for r, t in enumerate(where):
        by_page.setdefault(t // page, []).append((r, t % page))
    for p, got in by_page.items():
        f = rows[[r for r, _ in got]]
        amax = f.abs().amax(-1).amax(0)
        e = torch.ceil(torch.log2(amax.clamp(min=1e-300) / 448)).clamp(min=E_MIN)  # exact at powers of two times 448
        first = min(o for _, o in got)
        if first:
            e = torch.maximum(e, x_exp[p].double())
        y[p, :, :first] *= torch.exp2(x_exp[p].double() - e)[:, None, None]
        y[p][:, [o for _, o in got]] = (f * torch.exp2(-e)[None, :, None]).transpose(0, 1)
    return y


def _exact_attn(case, s):
    out = torch.zeros(s["q"].shape, dtype=torch.float64, device="cuda")
    group = case["heads"] // case["kv_heads"]
    start = s["q_start"].tolist()
    for b, n in enumerate(s["kv_len"].tolist()):
        m = start[b + 1] - start[b]
        if not n or not m:
            continue
        pages = s["table"][b, : -(-n // case["page"])].long()
        i = torch.arange(n - m, n, device="cuda")[:, None]
        j = torch.arange(n, device="cuda")[None]
        end = (i // case["frame"] + 1) * case["frame"] if case["frame"] else torch.full_like(i, n)
        hide = (j >= end) | (j < end - case["window"]) if case["window"] else (j >= end).expand(m, n)
        for h in range(case["kv_heads"]):
            k, v = ((_e4m3(s[a + "8"][pages, h]) * torch.exp2(s[a + "_exp"][pages, h].double())[:, None, None]).flatten(0, 1)[:n] for a in "kv")
            for g in range(h * group, (h + 1) * group):
                w = s["q"][0, g, start[b]: start[b + 1]].double() @ k.T / D ** 0.5
                w = torch.nan_to_num(torch.softmax(w.masked_fill(hide, -math.inf), -1))
                out[0, g, start[b]: start[b + 1]] = w @ v
    return out
