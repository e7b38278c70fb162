"""Serving on a cache held in 4 bits: the operators between a layer's projections and its attention, as a user's program
calls them, and the same operators in elementary torch operations.

Four kinds of pass:

  rope      the rotation of queries or keys by their positions, or of their gradients back (``inverse``).
  plan      the pages, positions and row numbers of the tokens that a step brings, from the requests' lengths.
  store     cache4_append() of new tokens' keys and values (rotated on the way), and the rows read back.
  attend    cache4_attend(): new tokens over the pages of their requests, or over a weighted coreset of them.

A row of the cache holds one token's key and value of one head.  Each stretch of 16 numbers has a scale s of 8 bits (5
exponent bits, 3 mantissa bits: the upper bits of a 16-bit float), the nearest to the largest magnitude over 6, and the
numbers are the nearest of 0, 1/2, 1, 3/2, 2, 3, 4 and 6 times s, signed.
"""
import math

import numpy as np
import torch

own = False

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
ITEM = {"f32": 4, "bf16": 2}
GROUP = 16                                      # numbers that share a scale
LARGEST = 61440.0                               # six times the largest scale
LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)


def listed():
    return [
        # The rotation of one new token's queries in a batch of 8 sequences: latency.
        dict(name="rope_token", kind="rope", batch=8, heads=32, n=1, d=128, rotary=128, layout="halves", scaling="plain", dtype="bf16",
             first=32768, inverse=False, packed=True),
        # A long prompt's queries, out of a projection that keeps queries, keys and values of a token together.
        dict(name="rope_prompt", kind="rope", batch=1, heads=32, n=32768, d=128, rotary=128, layout="pairs", scaling="plain", dtype="bf16",
             first=0, inverse=False, packed=True),
        # Gradients turned back in a fine-tuning step at lengthened contexts: half of the head is rotated.
        dict(name="rope_back_f32", kind="rope", batch=3, heads=12, n=4097, d=64, rotary=32, layout="halves", scaling="ramp", dtype="f32",
             first=100000, inverse=True, packed=False),
        # A decode step of 256 requests, one token each.
        dict(name="plan_decode", kind="plan", batch=256, page=64, longest=16384, new=1, ragged=False, short=False),
        # Prompts of all lengths that arrive together, more than the free pages hold.
        dict(name="plan_prompts", kind="plan", batch=61, page=16, longest=32768, new=8191, ragged=True, short=True),
        # A decode step of 16 requests into the cache.
        dict(name="store_token", kind="store", batch=16, q_heads=32, kv_heads=8, d=128, rotary=128, layout="halves", scaling="plain",
             dtype="bf16", page=64, longest=8192, new=1, ragged=False),
        # Prompts of a batch into the cache.
        dict(name="store_prompts", kind="store", batch=5, q_heads=32, kv_heads=8, d=128, rotary=128, layout="pairs", scaling="smooth",
             dtype="bf16", page=32, longest=0, new=8192, ragged=True),
        # The same of a small fp32 layer, part of its head rotated.
        dict(name="store_prompts_f32", kind="store", batch=4, q_heads=12, kv_heads=12, d=64, rotary=48, layout="halves", scaling="linear",
             dtype="f32", page=16, longest=0, new=1024, ragged=True),
        # One new token of a long-context chat over the coreset of its prompt: latency.
        dict(name="attend_coreset_1", kind="attend", batch=1, q_heads=32, kv_heads=8, d=128, dtype="bf16", page=64, longest=131072,
             new=1, ragged=False, core=2048),
        # A decode step of 48 requests of all lengths: the cache is read once, from memory.
        dict(name="attend_decode_48", kind="attend", batch=48, q_heads=32, kv_heads=8, d=128, dtype="bf16", page=64, longest=32768,
             new=1, ragged=True, core=0),
        # Up to 7 drafted tokens of each request looked at together, in an fp32 layer.
        dict(name="attend_drafts_f32", kind="attend", batch=6, q_heads=12, kv_heads=12, d=64, dtype="f32", page=16, longest=8191,
             new=7, ragged=True, core=0),
        # A prompt's queries over the coreset that its own rows were reduced to.
        dict(name="attend_coreset_8192", kind="attend", batch=1, q_heads=32, kv_heads=8, d=128, dtype="bf16", page=128, longest=32768,
             new=8192, ragged=False, core=1024),
    ]


def draw(rng):
    """One more case of the same ranges; none costs more than the largest listed one of its kind."""
    log = lambda a, b: int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))  # noqa: E731
    kind = rng.choice(["rope", "rope", "plan", "plan", "store", "store", "attend", "attend", "attend", "attend"])
    d = rng.choice([64, 128, 128])
    kv_heads = rng.choice([1, 2, 4, 8])
    rep = rng.choice([1, 2, 3, 4, 8])
    rotary = rng.choice([d, d, d // 2, 2 * rng.randint(4, d // 2)])
    dtype = rng.choice(["f32", "bf16", "bf16"])
    turn = dict(layout=rng.choice(["halves", "pairs"]), scaling=rng.choice(["plain", "linear", "base", "ramp", "smooth"]))
    page = rng.choice([16, 32, 64, 128, 256])
    if kind == "rope":
        heads, batch = kv_heads * min(rep, 4), rng.randint(1, 9)
        return dict(kind="rope", batch=batch, heads=heads, n=log(1, 1048576 / (heads * batch) / ITEM[dtype]), d=d, rotary=rotary, **turn, dtype=dtype,
                    first=log(1, 1000000), inverse=rng.random() < 0.3, packed=rng.random() < 0.5)
    if kind == "plan":
        batch = log(1, 300)
        return dict(kind="plan", batch=batch, page=page, longest=log(16, 32768), new=log(1, 400000 / batch), ragged=rng.random() < 0.7, short=rng.random() < 0.5)
    if kind == "store":
        batch = rng.randint(1, 20)
        longest = rng.choice([0, log(16, 8192)])
        new = log(1, 320000 / (batch * kv_heads * max(rep, 2)))
        return dict(kind="store", batch=batch, q_heads=kv_heads * rep, kv_heads=kv_heads, d=d, rotary=rotary, **turn, dtype=dtype, page=page,
                    longest=longest, new=new, ragged=rng.random() < 0.7)
    if rng.random() < 0.4:
        core = log(20, 4096)
        batch = rng.randint(1, 4)
        n = rng.randint(core, 32768)
        new = rng.choice([1, 1, log(1, 8192 * 32 * 1024 / (core * batch * kv_heads * rep))])
        return dict(kind="attend", batch=batch, q_heads=kv_heads * rep, kv_heads=kv_heads, d=d, dtype=dtype if new < 512 else "bf16", page=page, longest=n,
                    new=new, ragged=False, core=core)
    batch = rng.randint(1, 32)
    return dict(kind="attend", batch=batch, q_heads=kv_heads * rep, kv_heads=kv_heads, d=d, dtype=dtype, page=page,
                longest=log(32, min(32768, 4000000 / (batch * kv_heads))), new=rng.choice([1, 1, rng.randint(2, 9)]), ragged=rng.random() < 0.8, core=0)


# ------------------------------------------------------------------------------------------------
# rotation
# ------------------------------------------------------------------------------------------------
SCALING = {"plain": {}, "linear": dict(factor=4.0), "base": dict(factor=8.0), "ramp": dict(factor=16.0, original=4096),
           "smooth": dict(factor=8.0, original=8192, low=1.0, high=4.0)}


def _frequencies(rotary, scaling):
    """(radians per position of each pair, factor on the rotated numbers) as numpy float64."""
    base, o = 10000.0, SCALING[scaling]
    i = np.arange(rotary // 2, dtype=np.float64)
    if scaling == "base":
        base *= o["factor"] ** (rotary / (rotary - 2.0))
    f = base ** (-2.0 * i / rotary)
    if scaling == "linear":
        return f / o["factor"], 1.0
    turns = o.get("original", 0) * f / (2 * math.pi)           # of a pair over the original length
    if scaling == "ramp":
        # pairs of more than 32 turns keep their frequency, those of less than one are slowed, a ramp over the pair's number between
        where = lambda t: rotary * math.log(o["original"] / (t * 2 * math.pi)) / (2 * math.log(base))  # noqa: E731
        lo, hi = max(0.0, math.floor(where(32.0))), min(rotary - 1.0, math.ceil(where(1.0)))
        keep = 1.0 - np.clip((i - lo) / max(hi - lo, 0.001), 0.0, 1.0)
        return f * keep + f / o["factor"] * (1.0 - keep), 0.1 * math.log(o["factor"]) + 1.0
    if scaling == "smooth":
        keep = np.clip((turns - o["low"]) / (o["high"] - o["low"]), 0.0, 1.0)
        return f * keep + f / o["factor"] * (1.0 - keep), 1.0
    return f, 1.0


def _turn(x, positions, freq, factor, layout, inverse):
    """float32 x [..., n, d] rotated by float64 angles positions [..., n] * freq, whose cosines and sines are rounded to 32 bits."""
    ang = positions.double()[..., None] * freq
    c, s = (ang.cos() * factor).float(), (ang.sin() * (-factor if inverse else factor)).float()
    r = 2 * freq.numel()
    y = x.clone()
    if layout == "halves":
        a, b = x[..., :r // 2], x[..., r // 2:r]
        y[..., :r // 2], y[..., r // 2:r] = a * c - b * s, b * c + a * s
    else:
        a, b = x[..., 0:r:2], x[..., 1:r:2]
        y[..., 0:r:2], y[..., 1:r:2] = a * c - b * s, b * c + a * s
    return y


# ------------------------------------------------------------------------------------------------
# rows of the cache
# ------------------------------------------------------------------------------------------------
def _row_bytes(d):
    return d + d // 8 + (8 if d == 64 else 0)


def _scale_bits(a):
    """The scale of each group from its largest magnitude: nearest to a / 6, 5 exponent and 3 mantissa bits."""
    q = a.clamp(max=LARGEST) / 6.0
    u = q.view(torch.int32)
    normal = ((u + 0x7ffff + ((u >> 20) & 1)) >> 20) - (112 << 3)
    small = (q * 131072.0).round().to(torch.int32)
    return torch.where(q < 2.0 ** -14, small, normal)


def _quantise(x):
    """float32 x [..., d] -> (codes int [..., d] of 4 bits, scale bits int [..., d / 16])."""
    g = x.unflatten(-1, (-1, GROUP))
    bits = _scale_bits(g.abs().amax(-1))
    s = (bits << 7).to(torch.int16).view(torch.float16).float()[..., None]
    y = torch.where(s > 0, g / s, torch.zeros_like(g)).abs()
    code = ((y > 0.25).int() + (y >= 0.75).int() + (y > 1.25).int() + (y >= 1.75).int() + (y > 2.5).int() + (y >= 3.5).int() + (y > 5.0).int())
    code = code + 8 * (g.signbit()).int()
    return code.flatten(-2), bits


def _value(code, bits):
    levels = torch.tensor(LEVELS + tuple(-v for v in LEVELS), device=code.device)
    s = (bits.int() << 7).to(torch.int16).view(torch.float16).float()
    return (levels[code.long()].unflatten(-1, (-1, GROUP)) * s[..., None]).flatten(-2)


def _pack(k, v):
    """Rows [..., row bytes] of float32 k and v [..., d]: codes of the key (two a byte, the even one low), of the value, scales of both."""
    d = k.shape[-1]
    kc, ks = _quantise(k)
    vc, vs = _quantise(v)
    two = lambda c: (c[..., 0::2] | (c[..., 1::2] << 4)).to(torch.uint8)  # noqa: E731
    parts = [two(kc), two(vc), ks.to(torch.uint8), vs.to(torch.uint8)]
    row = torch.cat(parts, -1)
    return torch.nn.functional.pad(row, (0, _row_bytes(d) - row.shape[-1]))


def _unpack(rows, d):
    """float32 (k, v) [..., d] of rows [..., row bytes]."""
    four = lambda b: torch.stack([b & 15, b >> 4], -1).flatten(-2)  # noqa: E731
    h, g = d // 2, d // GROUP
    return (_value(four(rows[..., :h]), rows[..., 2 * h:2 * h + g]),
            _value(four(rows[..., h:2 * h]), rows[..., 2 * h + g:2 * h + 2 * g]))


# ------------------------------------------------------------------------------------------------
# inputs
# ------------------------------------------------------------------------------------------------
def _randn(g, *shape):
    return torch.randn(shape, generator=g, device="cuda")


def _sizes(count, longest, ragged):
    """Lengths of `count` requests as numpy int32: all the longest, or spread over the logarithm."""
    if not ragged or longest < 2:
        return np.full(count, longest, np.int32)
    n = np.exp((np.arange(count) + 0.5) / count * math.log(longest)).round().astype(np.int32)
    n[-1] = longest
    return n


def _lengths(g, count, longest, ragged):
    """The same on the GPU, dealt to the requests in an order of the seed's."""
    n = torch.tensor(_sizes(count, longest, ragged), device="cuda")
    return n[torch.randperm(count, generator=g, device="cuda")].contiguous()


def prepare(case, seed):
    c = case
    g = torch.Generator(device="cuda").manual_seed(seed)
    s = {"case": c, "seed": seed}
    if c["kind"] in ("rope", "store"):
        freq, factor = _frequencies(c["rotary"], c["scaling"])
        s["freq"], s["factor"] = torch.tensor(freq, device="cuda"), factor
        if own:
            import paper_2606_10944_b200 as elm
            s["rope"] = elm.Rope(c["rotary"], layout=c["layout"], scaling=c["scaling"], **SCALING[c["scaling"]])
    if c["kind"] == "rope":
        B, H, n, d = c["batch"], c["heads"], c["n"], c["d"]
        # a token's heads together, with room for its keys and values beside them where `packed`
        wide = H + 2 * max(1, H // 4) if c["packed"] else H
        x = _randn(g, B, n, wide, d).to(DTYPES[c["dtype"]])
        s["x"] = x[:, :, :H].transpose(1, 2)
        start = torch.randint(0, c["first"] + 1, (B, 1), generator=g, device="cuda")
        s["positions"] = (start + torch.arange(n, device="cuda")).to(torch.int32)
        return s
    B, page = c["batch"], c["page"]
    s["n_new"] = _lengths(g, B, c["new"], c["ragged"])
    longest = max(c["longest"], 1) if c["kind"] == "attend" else c["longest"]
    had = _lengths(g, B, longest, c["ragged"])
    if c["kind"] == "plan":
        cap = longest + c["new"]
        max_pages = -(-cap // page)
        s["length"] = had
        held = (had + page - 1) // page
        need = (had + s["n_new"] + page - 1) // page - held
        total_held, total_need = int(held.sum()), int(need.sum())
        free = total_need * 3 // 4 if c["short"] else total_need + 7
        order = torch.randperm(total_held + free, generator=g, device="cuda").to(torch.int32)
        table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
        table[torch.arange(max_pages, device="cuda") < held[:, None]] = order[:total_held]
        s["table"], s["free"] = table, order[total_held:].contiguous()
        s["free_count"] = torch.full((1,), free, dtype=torch.int32, device="cuda")
        s["tokens"] = int(s["n_new"].sum()) + (5 if c["ragged"] else 0)      # a step padded to a round size
        return s
    # requests whose tables are filled already, pages in no order
    length = had if c["kind"] == "attend" else had + s["n_new"]
    max_pages = -(-int(length.max()) // page) + 1
    held = (length + page - 1) // page
    pages = int(held.sum()) + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, max_pages), -1, dtype=torch.int32, device="cuda")
    table[torch.arange(max_pages, device="cuda") < held[:, None]] = order[:int(held.sum())]
    s["table"], s["length"] = table, length
    H, d, rb = c["kv_heads"], c["d"], _row_bytes(c["d"])
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[1:] = s["n_new"].cumsum(0)
    s["cu"], T = cu, int(cu[-1])
    if c["kind"] == "store":
        s["rows"] = torch.zeros(pages, H, page, rb, dtype=torch.uint8, device="cuda")
        wide = _randn(g, T, c["q_heads"] + 2 * H, d)
        wide[:, c["q_heads"]:c["q_heads"] + H] *= torch.exp(0.7 * _randn(g, 1, H, d))      # channels of keys differ in size
        wide = wide.to(DTYPES[c["dtype"]])
        s["Q"], s["K"], s["V"] = wide[:, :c["q_heads"]], wide[:, c["q_heads"]:c["q_heads"] + H], wide[:, c["q_heads"] + H:]
        b = torch.repeat_interleave(torch.arange(B, device="cuda"), s["n_new"].long())
        pos = had[b].long() + torch.arange(T, device="cuda") - cu[b].long()
        s["positions"] = pos.to(torch.int32)
        s["slots"] = table[b, pos // page] * page + (pos % page).to(torch.int32)
        s["n_read"] = int(s["n_new"].max())
        if c["longest"]:                                        # the rows that were added, by their numbers in the request
            j = torch.minimum(torch.arange(s["n_read"], device="cuda"), s["n_new"][:, None] - 1)
            s["idx"] = (had[:, None] + j).to(torch.int32)[:, None].expand(B, H, -1).contiguous()
        return s
    # rows of every page; the channels of keys differ in size, as they do behind a projection
    rows = torch.empty(pages * H * page, rb, dtype=torch.uint8, device="cuda")
    channel = torch.exp(0.5 * _randn(g, d))
    for part in rows.split(1 << 20):
        part.copy_(_pack(_randn(g, part.shape[0], d) * channel, _randn(g, part.shape[0], d)))
    s["rows"] = rows.view(pages, H, page, rb)
    q_std = 1.0 / float(channel.square().mean().sqrt())
    if c["core"]:
        s["Q"] = (_randn(g, B, c["q_heads"], c["new"], d) * q_std).to(DTYPES[c["dtype"]])
        n, nc = c["longest"], c["core"]
        edge = (torch.arange(nc + 1, device="cuda") * n) // nc
        u = torch.rand(B, H, nc, generator=g, device="cuda")
        s["idx"] = torch.minimum(edge[:-1] + (u * (edge[1:] - edge[:-1])).long(), edge[1:] - 1).to(torch.int32)
        level = (torch.arange(nc, device="cuda") * 6) // nc
        s["w"] = (2.0 ** level.float() / n).expand(B, H, nc).contiguous()
    else:
        # every request has its new tokens in the cache already
        s["length"] = torch.maximum(length, s["n_new"]).minimum(held * page)
        s["Q"] = (_randn(g, T, c["q_heads"], d) * q_std).to(DTYPES[c["dtype"]])
    return s


# ------------------------------------------------------------------------------------------------
# one pass
# ------------------------------------------------------------------------------------------------
def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(state):
    import paper_2606_10944_b200 as elm
    s, c = state, state["case"]
    if c["kind"] == "rope":
        return elm.rope(s["x"], s["positions"], s["rope"], inverse=c["inverse"])
    if c["kind"] == "plan":
        plan = elm.page_plan(s["table"], s["length"], s["n_new"], s["free"], s["free_count"], c["page"], s["tokens"])
        return plan.start, plan.length, plan.free_count, plan.cu, plan.positions, plan.slots, s["table"]
    if c["kind"] == "store":
        q = elm.cache4_append(s["rows"], s["K"], s["V"], s["slots"], rope=s["rope"], positions=s["positions"], Q=s["Q"])
        if c["longest"]:
            k, v = elm.cache4_read(s["rows"], s["table"], s["n_read"], idx=s["idx"], dtype=DTYPES[c["dtype"]])
        else:
            k, v = elm.cache4_read(s["rows"], s["table"], s["n_read"], length=s["length"], dtype=DTYPES[c["dtype"]])
        return q, k, v
    if c["core"]:
        return elm.cache4_attend(s["Q"], s["rows"], s["table"], idx=s["idx"], w=s["w"])
    return elm.cache4_attend(s["Q"], s["rows"], s["table"], length=s["length"], cu=s["cu"], max_q=c["new"])


def _run_plain(state):
    s, c = state, state["case"]
    if c["kind"] == "rope":
        return _turn(s["x"].float(), s["positions"][:, None], s["freq"], s["factor"], c["layout"], c["inverse"]).to(s["x"].dtype)
    if c["kind"] == "plan":
        return _plan_plain(s, c)
    if c["kind"] == "store":
        t = s["positions"][:, None]
        q = _turn(s["Q"].float(), t, s["freq"], s["factor"], c["layout"], False).to(s["Q"].dtype)
        k = _value(*_quantise(_turn(s["K"].float(), t, s["freq"], s["factor"], c["layout"], False)))
        v = _value(*_quantise(s["V"].float()))
        # by request: row j of request b is its j-th new token; a request with fewer has zeros, or its last one again
        at = s["cu"][:-1, None] + torch.arange(s["n_read"], device="cuda")
        there = at < s["cu"][1:, None]
        at = torch.minimum(at, s["cu"][1:, None] - 1).clamp(min=0).long()
        show = (lambda x: x[at].transpose(1, 2)) if c["longest"] else (lambda x: (x[at] * there[..., None, None]).transpose(1, 2))
        return q, show(k).to(s["K"].dtype).contiguous(), show(v).to(s["V"].dtype).contiguous()
    return _attend_plain(s, c)


def _plan_plain(s, c):
    page, table, n, had, T = c["page"], s["table"], s["n_new"], s["length"], s["tokens"]
    B, max_pages = table.shape
    cu = torch.zeros(B + 1, dtype=torch.int32, device="cuda")
    cu[1:] = n.cumsum(0)
    held, want = (had + page - 1) // page, (had + n + page - 1) // page
    fits = (had + n <= max_pages * page) & (cu[1:] <= T)
    need = torch.where(fits, want - held, torch.zeros_like(want))
    upto = need.cumsum(0).to(torch.int32)
    ok = fits & ((need == 0) | (upto <= s["free_count"]))
    j = torch.arange(max_pages, device="cuda", dtype=torch.int32)
    new = ok[:, None] & (j >= held[:, None]) & (j < want[:, None])
    nth = s["free_count"] - 1 - ((upto - need - held)[:, None] + j)
    table = torch.where(new, s["free"][nth.clamp(0, max(0, s["free"].numel() - 1)).long()] if s["free"].numel() else table, table)
    t = torch.arange(T, device="cuda", dtype=torch.int32)
    b = torch.searchsorted(cu[1:].contiguous(), t, right=True).clamp(max=B - 1)
    valid = (t < cu[-1]) & ok[b]
    pos = torch.where(valid, had[b] + t - cu[b], torch.full_like(t, -1))
    at = pos.clamp(min=0)
    slot = torch.where(valid, table[b, (at // page).long()] * page + at % page, torch.full_like(t, -1))
    minus = torch.full_like(had, -1)
    left = s["free_count"] - torch.where(ok, need, torch.zeros_like(need)).sum().to(torch.int32)
    return torch.where(ok, had, minus), torch.where(ok, had + n, had), left, cu, pos, slot, table


def _attend_plain(s, c):
    page, H, d, B = c["page"], c["kv_heads"], c["d"], c["batch"]
    rep = c["q_heads"] // H
    if c["core"]:
        at = s["idx"].long()                                    # [B, H, n]
        seen = None
        bias = s["w"].log()[:, :, None, None]
        q = s["Q"].float().view(B, H, rep, c["new"], d)
    else:
        n = int(s["table"].shape[1]) * page
        at = torch.arange(n, device="cuda").expand(B, H, n)
        # query j of request b (of n_b) sees the rows up to its own
        j = torch.arange(c["new"], device="cuda")
        cu = s["cu"].long()
        count = (cu[1:] - cu[:-1])[:, None]
        upto = s["length"][:, None] - count + j + 1              # rows that are seen
        seen = (torch.arange(n, device="cuda") < upto[..., None])[:, None, None]
        bias = 0.0
        take = torch.minimum(cu[:-1, None] + j, cu[1:, None] - 1)
        q = s["Q"].float()[take].view(B, c["new"], H, rep, d).permute(0, 2, 3, 1, 4)
    pages = s["table"].long()[torch.arange(B, device="cuda")[:, None, None], at // page].clamp(min=0)
    k, v = _unpack(s["rows"][pages, torch.arange(H, device="cuda")[:, None], at % page], d)
    logits = (q.flatten(2, 3) @ k.transpose(-1, -2)).view(B, H, rep, -1, k.shape[2]) / math.sqrt(d) + bias
    if seen is not None:
        logits = logits.masked_fill(~seen, -math.inf)
    p = torch.exp(logits - logits.amax(-1, keepdim=True))
    o = ((p / p.sum(-1, keepdim=True)).flatten(2, 3) @ v).view(B, H, rep, -1, d)
    if c["core"]:
        return o.reshape(B, H * rep, c["new"], d).to(s["Q"].dtype)
    valid = j < count                                            # back to the tokens one after the other
    return o.permute(0, 3, 1, 2, 4).flatten(2, 3)[valid].to(s["Q"].dtype)


# ------------------------------------------------------------------------------------------------
# the definition, in 64 bits
# ------------------------------------------------------------------------------------------------
def _exact_rotate(x, pos, freq, factor, layout, sign):
    x = x.double()
    z = torch.polar(torch.full_like(pos, factor, dtype=torch.float64)[..., None].expand(*pos.shape, freq.numel()).contiguous(),
                    sign * (pos.double()[..., None] * freq))
    r = 2 * freq.numel()
    turned = x[..., :r]
    if layout == "halves":
        turned = torch.view_as_real(torch.complex(turned[..., :r // 2].contiguous(), turned[..., r // 2:].contiguous()) * z).transpose(-1, -2).flatten(-2)
    else:
        turned = torch.view_as_real(torch.view_as_complex(turned.unflatten(-1, (-1, 2)).contiguous()) * z).flatten(-2)
    return torch.cat([turned, x[..., r:]], -1)


def _exact_grid(x):
    """The nearest numbers that the cache can hold, from float64 x [..., d]."""
    g = x.unflatten(-1, (-1, GROUP))
    q = g.abs().amax(-1, keepdim=True).clamp(max=LARGEST) / 6.0
    step = torch.exp2(torch.floor(torch.log2(q.clamp(min=2.0 ** -14))) - 3)
    s = torch.round(q / step) * step
    y = torch.where(s > 0, g / s.clamp(min=2.0 ** -17), torch.zeros_like(g)).abs().clamp(max=6.0)
    # numbers up to 2 in halves, up to 4 in ones, above in twos; torch.round takes ties to even
    half = torch.where(y < 2, torch.round(2 * y) / 2, torch.where(y < 4, torch.round(y), 2 * torch.round(y / 2)))
    return (torch.copysign(half, g) * s).flatten(-2)


def exact(case, seed):
    c = case
    if c["kind"] == "plan":
        return None
    s = prepare(case, seed)
    if c["kind"] == "rope":
        return _exact_rotate(s["x"], s["positions"][:, None].expand(s["x"].shape[:3]), s["freq"], s["factor"], c["layout"], -1.0 if c["inverse"] else 1.0)
    if c["kind"] == "store":
        spin = lambda x: _exact_rotate(x, s["positions"][:, None].expand(x.shape[:2]), s["freq"], s["factor"], c["layout"], 1.0)  # noqa: E731
        k, v = _exact_grid(spin(s["K"])), _exact_grid(s["V"].double())
        out = []
        for x in (k, v):
            y = torch.zeros(c["batch"], c["kv_heads"], s["n_read"], c["d"], dtype=torch.float64, device="cuda")
            for b in range(c["batch"]):
                i, j = int(s["cu"][b]), int(s["cu"][b + 1])
                y[b, :, :j - i] = x[i:j].transpose(0, 1)
                if c["longest"] and j > i:
                    y[b, :, j - i:] = x[j - 1][:, None]
            out.append(y)
        return spin(s["Q"]), out[0], out[1]
    d, page = c["d"], c["page"]
    rep = c["q_heads"] // c["kv_heads"]
    number = torch.tensor([sign * v for sign in (1, -1) for v in LEVELS], dtype=torch.float64, device="cuda")

    def numbers(raw, first, scales):
        byte = raw[:, first:first + d // 2].long()
        out = torch.empty(raw.shape[0], d, dtype=torch.float64, device="cuda")
        out[:, 0::2], out[:, 1::2] = number[byte % 16], number[byte // 16]
        e = raw[:, scales:scales + d // GROUP].double()
        power, part = torch.floor(e / 8), e % 8
        scale = torch.where(power > 0, (1 + part / 8) * torch.exp2(power - 15), part * 2.0 ** -17)
        return out * scale.repeat_interleave(GROUP, 1)

    out = torch.zeros(s["Q"].shape, dtype=torch.float64, device="cuda")
    for b in range(c["batch"]):
        for h in range(c["kv_heads"]):
            if c["core"]:
                at, lw = s["idx"][b, h].long(), s["w"][b, h].double().log()
                q = s["Q"][b, h * rep:(h + 1) * rep].double()
                n_b = limit = None
            else:
                n = int(s["length"][b])
                at, lw = torch.arange(n, device="cuda"), 0.0
                q = s["Q"][int(s["cu"][b]):int(s["cu"][b + 1]), h * rep:(h + 1) * rep].double().transpose(0, 1)
                n_b = q.shape[1]
                limit = n - n_b + 1 + torch.arange(n_b, device="cuda")
            raw = s["rows"][s["table"][b].long()[at // page], h, at % page]
            a = q @ numbers(raw, 0, d).T / d ** 0.5 + lw
            if limit is not None:
                a = torch.where(at < limit[:, None], a, -torch.inf)
            o = torch.softmax(a, -1) @ numbers(raw, d // 2, d + d // GROUP)
            if c["core"]:
                out[b, h * rep:(h + 1) * rep] = o
            else:
                out[int(s["cu"][b]):int(s["cu"][b + 1]), h * rep:(h + 1) * rep] = o.transpose(0, 1)
    return out


# ------------------------------------------------------------------------------------------------
# what a pass cannot do without
# ------------------------------------------------------------------------------------------------
def work(case):
    c = case
    if c["kind"] == "rope":
        numbers = c["batch"] * c["heads"] * c["n"]
        return {"bytes": numbers * c["d"] * 2.0 * ITEM[c["dtype"]] + 4.0 * c["batch"] * c["n"], "flops": 3.0 * numbers * c["rotary"]}
    new = float(_sizes(c["batch"], c["new"], c["ragged"]).sum())
    if c["kind"] == "plan":
        # lengths, counts and starts of the requests; a position and a row number per token; a table entry and a free page per new page
        return {"bytes": 24.0 * c["batch"] + 8.0 * new + 8.0 * new / c["page"], "flops": 4.0 * new}
    d, rb = c["d"], _row_bytes(c["d"])
    if c["kind"] == "store":
        item = ITEM[c["dtype"]]
        read_back = new * c["kv_heads"] * 2 * d * item
        stored = new * c["kv_heads"] * (2 * d * item + 2.0 * rb)
        return {"bytes": 2.0 * new * c["q_heads"] * d * item + stored + read_back + 8.0 * new, "flops": new * 3.0 * (c["q_heads"] + c["kv_heads"]) * c["rotary"]}
    qo = 2.0 * ITEM[c["dtype"]] * d * c["q_heads"]
    if c["core"]:
        return {"bytes": qo * c["batch"] * c["new"] + c["batch"] * c["kv_heads"] * c["core"] * (rb + 8.0), "flops": 4.0 * d * c["batch"] * c["q_heads"] * c["new"] * c["core"]}
    seen = float(_sizes(c["batch"], c["longest"], c["ragged"]).sum())
    return {"bytes": qo * new + seen * (c["kv_heads"] * rb + 4.0 / c["page"]), "flops": 4.0 * d * c["q_heads"] * seen * new / c["batch"]}
