"""Operators of a paged serving iteration, each in a plain form and as the library's own call.

Four operators:

``append_rope``    the new tokens' K is rotated by its position and appended to the paged cache with V,
                   and q is rotated for the attention that follows
``append_4bit``    the new tokens' K/V are quantised to 4 bits and appended to a 4-bit paged cache, and
                   read back as the values the cache now stands for
``window``         grouped-query attention of every new token over its last ``window`` keys and the
                   first ``sinks`` keys of its context
``attend_4bit``    grouped-query attention of every new token over its whole context in a 4-bit cache

A case is an iteration: ``chunks`` prefill chunks of ``chunk_len`` new tokens each (on prefixes of
``prefix_lo`` .. ``prefix_hi`` tokens), then ``decodes`` sequences with one new token (contexts of
``ctx_lo`` .. ``ctx_hi``, log-uniform).  ``lens`` seeds the lengths, so that they belong to the case.

Layouts: pool planes ``[pages][kv heads][16][d]``; a tile ``(page, kv head)`` of a 4-bit plane is 16
token rows of d / 2 bytes, then 16 x d / 32 bf16 steps.  A group of 32 consecutive elements shares a
step s; code c (0..15) stands for (c - 8) s.  The d / 8 words (32 bits, lowest nibble first) of a row
are stored in the order t * (d / 32) + g for the elements 32 g + 8 t .. + 7.
"""
import math
import random

import torch

own = False

PAGE = 16
GROUP = 32
DEVICE = "cuda:0"
SHAPE_S1 = dict(hq=8, hkv=2, d=64)
SHAPE_8B = dict(hq=32, hkv=8, d=128)
SHAPE_70B = dict(hq=64, hkv=8, d=128)
SHAPES = (SHAPE_S1, SHAPE_8B, SHAPE_70B, dict(hq=8, hkv=8, d=64), dict(hq=8, hkv=4, d=64), dict(hq=6, hkv=2, d=128),
          dict(hq=5, hkv=1, d=128))


def _case(op, shape, chunks=0, chunk_len=1, prefix_lo=0, prefix_hi=0, decodes=0, ctx_lo=1, ctx_hi=1, lens=1, **more):
    return dict(op=op, **shape, chunks=chunks, chunk_len=chunk_len, prefix_lo=prefix_lo, prefix_hi=prefix_hi,
                decodes=decodes, ctx_lo=ctx_lo, ctx_hi=ctx_hi, lens=lens, **more)


def listed():
    neox = dict(rotary=128, interleaved=False, base=500000.0)
    return [
        # four users far into long documents, small model: one layer's append is all latency
        dict(name="rope_decode_4_far", **_case("append_rope", SHAPE_S1, decodes=4, ctx_lo=65536, ctx_hi=131072, lens=11,
                                               rotary=64, interleaved=False, base=1000000.0)),
        # a decode-heavy iteration; a partly rotated head, pairs next to one another
        dict(name="rope_decode_128_partial", **_case("append_rope", SHAPE_70B, decodes=128, ctx_lo=256, ctx_hi=2048, lens=12,
                                                     rotary=64, interleaved=True, base=10000.0)),
        # a prefill iteration at the token budget a scheduler fills
        dict(name="rope_prefill_8x1024", **_case("append_rope", SHAPE_8B, chunks=8, chunk_len=1024, prefix_lo=0, prefix_hi=4096,
                                                 lens=13, **neox)),
        # the same two kinds of iteration on a 4-bit cache
        dict(name="quant_decode_64", **_case("append_4bit", SHAPE_8B, decodes=64, ctx_lo=128, ctx_hi=8192, lens=21)),
        dict(name="quant_prefill_8x1000", **_case("append_4bit", SHAPE_8B, chunks=8, chunk_len=1000, prefix_lo=0, prefix_hi=4096,
                                                  lens=22)),
        # one user, a short window with four sinks
        dict(name="window_decode_1", **_case("window", SHAPE_8B, decodes=1, ctx_lo=20001, ctx_hi=20001, lens=31, window=512, sinks=4)),
        # a decode-heavy ragged batch, many contexts shorter than the window
        dict(name="window_decode_64", **_case("window", SHAPE_8B, decodes=64, ctx_lo=128, ctx_hi=8192, lens=32, window=1024, sinks=4)),
        # a mixed iteration of a layer with a window
        dict(name="window_mixed_8x512_120", **_case("window", SHAPE_8B, chunks=8, chunk_len=512, prefix_lo=0, prefix_hi=4096,
                                                    decodes=120, ctx_lo=256, ctx_hi=4096, lens=33, window=1024, sinks=4)),
        # one user of a small model
        dict(name="kv4_decode_1", **_case("attend_4bit", SHAPE_S1, decodes=1, ctx_lo=513, ctx_hi=513, lens=41)),
        # a decode-heavy ragged batch over a 4-bit cache
        dict(name="kv4_decode_64", **_case("attend_4bit", SHAPE_8B, decodes=64, ctx_lo=128, ctx_hi=8192, lens=42)),
        # long documents: what a 4-bit cache is for
        dict(name="kv4_decode_16_long", **_case("attend_4bit", SHAPE_70B, decodes=16, ctx_lo=32768, ctx_hi=65536, lens=43)),
        # prefill chunks beside decode rows
        dict(name="kv4_mixed_8x512_120", **_case("attend_4bit", SHAPE_8B, chunks=8, chunk_len=512, prefix_lo=0, prefix_hi=4096,
                                                 decodes=120, ctx_lo=256, ctx_hi=4096, lens=44)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(lo * math.exp(rng.random() * math.log((hi + 1) / lo)))))


def draw(rng):
    op = rng.choice(["append_rope", "append_4bit", "window", "attend_4bit"])
    shape = rng.choice(SHAPES)
    chunks = chunk_len = prefix_hi = decodes = 0
    kind = rng.choice(["decode", "decode", "prefill", "mixed"])
    if kind != "decode":
        chunks, prefix_hi = rng.randint(1, 8), _log_int(rng, 1, 4096)
        rows = 8192 if op.startswith("append") else 4096 * 32 // max(32, shape["hq"])
        chunk_len = _log_int(rng, 2, rows // chunks if op.startswith("append") else min(700, rows // chunks))
    if kind != "prefill":
        decodes = _log_int(rng, 1, 100)
    ctx_hi = _log_int(rng, 1, 8192 if decodes <= 64 else 4096)
    more = {}
    if op == "append_rope":
        rotary = 16 * rng.randint(1, shape["d"] // 16)
        more = dict(rotary=rotary, interleaved=rng.random() < 0.5, base=rng.choice([10000.0, 500000.0, 1000000.0]))
    elif op == "window":
        more = dict(window=_log_int(rng, 1, 4096), sinks=rng.choice([0, 0, 1, 4, 16, 33]))
    return _case(op, shape, chunks=chunks, chunk_len=chunk_len, prefix_hi=prefix_hi, decodes=decodes,
                 ctx_lo=_log_int(rng, 1, ctx_hi), ctx_hi=ctx_hi, lens=rng.randint(1, 1 << 30), **more)


def _lengths(case):
    """(new tokens, context length with them) of every sequence: prefill chunks first, then decode rows."""
    rng = random.Random(case["lens"])
    q = [case["chunk_len"]] * case["chunks"] + [1] * case["decodes"]
    ctx = [rng.randint(case["prefix_lo"], case["prefix_hi"]) + case["chunk_len"] for _ in range(case["chunks"])]
    ctx += [_log_int(rng, case["ctx_lo"], case["ctx_hi"]) for _ in range(case["decodes"])]
    return q, ctx


def work(case):
    q_lens, ctx_lens = _lengths(case)
    hq, hkv, d, n = case["hq"], case["hkv"], case["d"], sum(q_lens)
    plane_row = hkv * d * 2                                   # one token's K (or V) in bf16
    plane_row4 = hkv * (d // 2 + d // GROUP * 2)              # the same in 4 bits
    if case["op"] == "append_rope":
        return {"bytes": n * (2 * hq * d * 2 + 4 * plane_row), "flops": 0}
    if case["op"] == "append_4bit":                           # read, written in 4 bits, and read back from there
        return {"bytes": n * 2 * (plane_row + 2 * plane_row4 + plane_row), "flops": 0}
    keys = pairs = 0
    window, sinks = case.get("window", 1 << 30), case.get("sinks", 0)
    for ql, cl in zip(q_lens, ctx_lens):
        first = max(0, cl - ql - window + 1)                  # first key of the first row's window
        keys += cl - first + min(sinks, first)
        for p in range(cl - ql, cl):
            lo = max(0, p - window + 1)
            pairs += p + 1 - lo + min(sinks, lo)
    row = plane_row if case["op"] == "window" else plane_row4
    return {"bytes": keys * 2 * row + n * hq * (2 * d * 2 + 4), "flops": 4 * d * hq * pairs}


# ------------------------------------------------------------------- state --

class _Handles:
    """The library's pool, plan and workspace of a state: what a serving loop holds while it runs an iteration's layers."""

    def __init__(self, case, s):
        import paper_2604_07144_b200 as ap
        self.ap = ap
        four = case["op"] in ("append_4bit", "attend_4bit")
        create = ap.kv_pool_create_4bit if four else ap.kv_pool_create
        self.pool = create(s["pages"], case["hkv"], case["d"], s["k_pool"], s["v_pool"])
        table = s["table"].cpu().numpy()
        if case["op"] == "window":
            self.plan = ap.plan_create_windowed(self.pool, s["q_lens"], s["ctx_lens"], table, case["hq"], case["window"], case["sinks"])
        else:
            self.plan = ap.plan_create(self.pool, s["q_lens"], s["ctx_lens"], table, case["hq"])
        self.workspace = torch.empty(max(256, ap.plan_workspace_bytes(self.plan)), dtype=torch.uint8, device=DEVICE)

    def __del__(self):
        if getattr(self, "plan", None) is not None:
            self.ap.plan_destroy(self.plan)
        if getattr(self, "pool", None) is not None:
            self.ap.kv_pool_destroy(self.pool)


def _quantise(x):
    """(codes, steps) of [..., d] values: codes int32 [..., d], steps float32 [..., d / 32].

    A group's step is max |x| / 7 rounded up to 5 significant bits, so every (c - 8) s is a bf16 number."""
    g = x.float().unflatten(-1, (-1, GROUP))
    top = g.abs().amax(-1)
    bits = (top / torch.full_like(top, 7.0)).view(torch.int32)       # a true division: top / 7.0 would multiply by 1/7
    step = ((bits + 0x7FFFF) & ~0x7FFFF).view(torch.float32)
    safe = torch.where(step > 0, step, torch.ones_like(step))
    codes = torch.round(g / safe[..., None]).to(torch.int32) + 8
    return codes.flatten(-2), step


def _pack(codes):
    """int32 codes [..., d] -> the d / 2 bytes of a stored row."""
    d = codes.shape[-1]
    w = codes.unflatten(-1, (d // GROUP, 4, 8)).transpose(-3, -2).reshape(*codes.shape[:-1], d // 2, 2)
    return (w[..., 0] | (w[..., 1] << 4)).to(torch.uint8)


def _unpack(rows, d):
    """The d / 2 bytes of stored rows -> int32 codes [..., d]."""
    b = rows.to(torch.int32)
    c = torch.stack((b & 15, b >> 4), -1).flatten(-2)
    return c.unflatten(-1, (4, d // GROUP, 8)).transpose(-3, -2).reshape(*rows.shape[:-1], d)


def _code_view(plane, d):
    """[pages, kv heads, 16, d / 2] view of a 4-bit plane's codes."""
    return plane[:, :, :PAGE * d // 2].unflatten(-1, (PAGE, d // 2))


def _step_view(plane, d):
    """[pages, kv heads, 16, d / 32] view of its steps, in bf16."""
    return plane[:, :, PAGE * d // 2:].view(torch.bfloat16).unflatten(-1, (PAGE, d // GROUP))


def prepare(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    q_lens, ctx_lens = _lengths(case)
    n = sum(q_lens)
    need = [-(-c // PAGE) for c in ctx_lens]
    pages = max(1, math.ceil(1.25 * sum(need)))
    order = torch.randperm(pages, generator=gen, device=DEVICE, dtype=torch.int32)
    starts = torch.tensor([sum(need[:i]) for i in range(len(need))], device=DEVICE)
    col = torch.arange(max(need), device=DEVICE)
    used = col[None, :] < torch.tensor(need, device=DEVICE)[:, None]
    table = torch.where(used, order[(starts[:, None] + col[None, :]).clamp_max(pages - 1)], -1)

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=torch.bfloat16)

    s = dict(case=case, q_lens=q_lens, ctx_lens=ctx_lens, pages=pages, table=table, n=n)
    s["ctx"] = torch.tensor(ctx_lens, device=DEVICE)
    seq = torch.repeat_interleave(torch.arange(len(q_lens), device=DEVICE), torch.tensor(q_lens, device=DEVICE))
    first = torch.tensor([sum(q_lens[:i]) for i in range(len(q_lens))], device=DEVICE)
    s["pos"] = s["ctx"][seq] - torch.tensor(q_lens, device=DEVICE)[seq] + torch.arange(n, device=DEVICE) - first[seq]
    s["page"], s["slot"] = table[seq, s["pos"] // PAGE].long(), s["pos"] % PAGE     # where each new token goes
    # q, k and v as one projection leaves them: slices of its rows
    qkv = normal(n, hq + 2 * hkv, d)
    s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
    if case["op"] in ("append_4bit", "attend_4bit"):
        s["k"], s["v"] = s["k"].contiguous(), s["v"].contiguous()
        for plane in ("k_pool", "v_pool"):
            s[plane] = torch.empty(pages, hkv, PAGE * (d // 2 + d // GROUP * 2), dtype=torch.uint8, device=DEVICE)
            codes, steps = _quantise(normal(pages, hkv, PAGE, d))
            _code_view(s[plane], d).copy_(_pack(codes))
            _step_view(s[plane], d).copy_(steps)
        s["k_read"] = torch.empty(n, hkv, d, dtype=torch.bfloat16, device=DEVICE)
        s["v_read"] = torch.empty_like(s["k_read"])
    else:
        s["k_pool"], s["v_pool"] = normal(pages, hkv, PAGE, d), normal(pages, hkv, PAGE, d)
    if case["op"] == "append_rope":
        s["q_rot"] = torch.empty(n, hq, d, dtype=torch.bfloat16, device=DEVICE)
    else:
        s["q"] = s["q"].contiguous()
        s["out"] = torch.empty(n, hq, d, dtype=torch.bfloat16, device=DEVICE)
        s["lse"] = torch.empty(n, hq, dtype=torch.float32, device=DEVICE)
    if own:
        s["lib"] = _Handles(case, s)
    return s


# --------------------------------------------------------------------- run --

def run(s):
    return {"append_rope": _run_append_rope, "append_4bit": _run_append_4bit, "window": _run_attention,
            "attend_4bit": _run_attention}[s["case"]["op"]](s)


def _run_append_rope(s):
    c = s["case"]
    if own:
        lib = s["lib"]
        lib.ap.kv_append_rope(lib.pool, lib.plan, s["k"], s["v"], q=s["q"], q_rot=s["q_rot"], rotary_dim=c["rotary"],
                              interleaved=c["interleaved"], base=c["base"])
        return {"q": s["q_rot"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}
    half = c["rotary"] // 2
    freq = c["base"] ** (-torch.arange(half, device=DEVICE, dtype=torch.float64) / half)
    angle = s["pos"].double()[:, None] * freq                 # far positions: an angle needs 64 bits
    cos, sin = angle.cos().float()[:, None, :], angle.sin().float()[:, None, :]

    def rotate(x):
        x = x.float()
        r = x[..., :c["rotary"]]
        if c["interleaved"]:
            a, b = r[..., 0::2], r[..., 1::2]
            r = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = r[..., :half], r[..., half:]
            r = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        return torch.cat((r, x[..., c["rotary"]:]), -1).bfloat16()

    s["k_pool"][s["page"], :, s["slot"]] = rotate(s["k"])
    s["v_pool"][s["page"], :, s["slot"]] = s["v"]
    s["q_rot"].copy_(rotate(s["q"]))
    return {"q": s["q_rot"], "k_pool": s["k_pool"], "v_pool": s["v_pool"]}


def _run_append_4bit(s):
    if own:
        lib = s["lib"]
        lib.ap.kv_append(lib.pool, lib.plan, s["k"], s["v"])
        lib.ap.kv_read_new(lib.pool, lib.plan, s["k_read"], s["v_read"])
        return {"k": s["k_read"], "v": s["v_read"]}
    d = s["case"]["d"]

    def append(plane, x, back):
        codes, steps = _quantise(x)
        _code_view(plane, d)[s["page"], :, s["slot"]] = _pack(codes)
        _step_view(plane, d)[s["page"], :, s["slot"]] = steps.bfloat16()
        back.copy_(_values(plane, d, s["page"], s["slot"]))

    append(s["k_pool"], s["k"], s["k_read"])
    append(s["v_pool"], s["v"], s["v_read"])
    return {"k": s["k_read"], "v": s["v_read"]}


def _values(plane, d, page, slot):
    """The rows [..., kv heads, d] that a 4-bit plane stands for at (page, slot), in float32."""
    codes = _unpack(_code_view(plane, d)[page, :, slot], d)
    steps = _step_view(plane, d)[page, :, slot].float()
    return ((codes - 8).unflatten(-1, (-1, GROUP)) * steps[..., None]).flatten(-2)


def _run_attention(s):
    c = s["case"]
    if own:
        lib = s["lib"]
        lib.ap.attention_iteration(lib.pool, lib.plan, s["q"], s["out"], s["lse"], lib.workspace)
        return {"out": s["out"], "lse": s["lse"]}
    split = c["chunks"] * c["chunk_len"]
    if c["chunks"]:
        _attend(s, slice(0, c["chunks"]), slice(0, split), c["chunk_len"])
    if c["decodes"]:
        _attend(s, slice(c["chunks"], None), slice(split, None), 1)
    return {"out": s["out"], "lse": s["lse"]}


def _attend(s, seqs, rows, t):
    """Attention of `t` new tokens of each of the sequences `seqs` (rows `rows` of q): gather, mask, softmax."""
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    ctx, table, pos = s["ctx"][seqs], s["table"][seqs], s["pos"][rows].view(-1, t)
    longest = max(s["ctx_lens"][seqs])
    window, sinks = min(c.get("window", longest), longest), min(c.get("sinks", 0), longest)
    # candidate keys of a sequence: the sinks, then everything from the first row's window on
    recent = ctx[:, None] - t - window + 1 + torch.arange(min(window + t - 1, longest + window), device=DEVICE)
    sink = torch.arange(sinks, device=DEVICE).expand(len(ctx), sinks)
    key = torch.cat((sink, torch.where(recent >= sinks, recent, -1)), 1)
    key = torch.where(key < ctx[:, None], key, -1)
    at = key.clamp_min(0)
    page, slot = torch.gather(table, 1, at // PAGE).clamp_min(0).long(), at % PAGE
    if c["op"] == "window":
        k, v = s["k_pool"][page, :, slot].float(), s["v_pool"][page, :, slot].float()
    else:
        k, v = _values(s["k_pool"], d, page, slot), _values(s["v_pool"], d, page, slot)
    seen = (key[:, None] >= 0) & (key[:, None] <= pos[..., None])
    seen &= (key[:, None] > pos[..., None] - window) | (key[:, None] < sinks)          # [B, t, L]
    q = s["q"][rows].float().view(-1, t, hkv, hq // hkv, d).permute(0, 2, 3, 1, 4)     # [B, kv head, group, t, d]
    x = torch.matmul(q.flatten(2, 3), k.permute(0, 2, 3, 1)).unflatten(2, (hq // hkv, t)) / math.sqrt(d)
    x = torch.where(seen[:, None, None], x, float("-inf"))
    top = x.amax(-1, keepdim=True)
    p = torch.exp(x - top)
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v.transpose(1, 2)).unflatten(2, (hq // hkv, t)) / total
    s["out"][rows] = o.permute(0, 3, 1, 2, 4).reshape(-1, hq, d).bfloat16()
    s["lse"][rows] = (top + total.log()).squeeze(-1).permute(0, 3, 1, 2).reshape(-1, hq)


# ------------------------------------------------------------------- exact --

def exact(case, seed):
    s = prepare(case, seed)
    return {"append_rope": _exact_rope, "append_4bit": _exact_append_4bit, "window": _exact_attention,
            "attend_4bit": _exact_attention}[case["op"]](s)


def _exact_rope(s):
    """The pair (a, b) of pair number i at position p as the complex number a + ib, turned by p base^(-2 i / rotary)."""
    c = s["case"]
    r = c["rotary"]
    theta = torch.tensor([c["base"] ** (-2.0 * i / r) for i in range(r // 2)], dtype=torch.float64, device=DEVICE)
    turn = torch.polar(torch.ones(s["n"], 1, r // 2, dtype=torch.float64, device=DEVICE), (s["pos"].double()[:, None] * theta)[:, None])
    at = torch.arange(r, device=DEVICE)
    first, second = (at[0::2], at[1::2]) if c["interleaved"] else (at[:r // 2], at[r // 2:])

    def rotate(x):
        y = x.double().clone()
        z = torch.complex(y[..., first], y[..., second]) * turn
        y[..., first], y[..., second] = z.real, z.imag
        return y

    k_pool, v_pool = s["k_pool"].double(), s["v_pool"].double()
    k_pool[s["page"], :, s["slot"]] = rotate(s["k"])
    v_pool[s["page"], :, s["slot"]] = s["v"].double()
    return {"q": rotate(s["q"]), "k_pool": k_pool, "v_pool": v_pool}


def _exact_append_4bit(s):
    """Each value goes to the nearest multiple (ties to the even one) of its group's step, found with frexp in 64 bits."""
    def value(x):
        x = x.double().unflatten(-1, (-1, GROUP))
        top = x.abs().amax(-1, keepdim=True)
        m, e = torch.frexp(top / torch.full_like(top, 7.0))
        step = torch.ldexp(torch.ceil(m * 32.0), e - 5)
        return torch.where(step > 0, torch.round(x / step.clamp_min(1e-300)) * step, torch.zeros_like(x)).flatten(-2)

    return {"k": value(s["k"]), "v": value(s["v"])}


def _exact_attention(s):
    c = s["case"]
    hq, hkv, d = c["hq"], c["hkv"], c["d"]
    out, lse, row = [], [], 0
    for b, (ql, cl) in enumerate(zip(s["q_lens"], s["ctx_lens"])):
        pages = s["table"][b, :-(-cl // PAGE)].long()
        k, v = (_exact_tokens(c, s[plane], pages)[:, :cl] for plane in ("k_pool", "v_pool"))      # [kv head, cl, d]
        q = s["q"][row:row + ql].double().permute(1, 0, 2).reshape(hkv, hq // hkv, ql, d)
        x = torch.einsum("hgtd,hjd->hgtj", q, k) * d ** -0.5
        j, p = torch.arange(cl, device=DEVICE)[None], torch.arange(cl - ql, cl, device=DEVICE)[:, None]
        hidden = j > p
        if c["op"] == "window":
            hidden |= (j <= p - c["window"]) & (j >= c["sinks"])
        x.masked_fill_(hidden, -math.inf)
        lse.append(torch.logsumexp(x, -1).reshape(hq, ql).T)
        out.append(torch.einsum("hgtj,hjd->thgd", torch.softmax(x, -1), v).reshape(ql, hq, d))
        row += ql
    return {"out": torch.cat(out), "lse": torch.cat(lse)}


def _exact_tokens(c, plane, pages):
    """[kv head, 16 * pages, d] in 64 bits: the cached rows of the listed pages."""
    d, tiles = c["d"], plane[pages]
    if c["op"] == "window":
        return tiles.double().permute(1, 0, 2, 3).flatten(1, 2)
    groups = d // GROUP
    rows = tiles[..., :PAGE * d // 2].reshape(*tiles.shape[:2], PAGE, d // 2).long()
    steps = tiles[..., PAGE * d // 2:].contiguous().view(torch.bfloat16).reshape(*tiles.shape[:2], PAGE, groups).double()
    element = torch.arange(d, device=DEVICE)
    word = (element % GROUP) // 8 * groups + element // GROUP          # the stored word that holds the element
    code = rows[..., word * 4 + element % 8 // 2] >> (4 * (element % 2)) & 15
    return ((code - 8).double() * steps[..., element // GROUP]).permute(1, 0, 2, 3).flatten(1, 2)
