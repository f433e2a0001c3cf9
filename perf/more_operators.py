"""Operators of a hybrid model's layers over an iteration's packed rows, each in a plain form and as the library's own call.

Three operators:

``conv``     short causal convolution over each sequence's rows, with the last inputs of every sequence kept in a state slot
``scan``     selective state space scan over each sequence's rows, with every sequence's state kept in a slot
``prompt``   causal grouped-query attention of whole prompts, read from q, k, v as one projection leaves them

A ``conv`` or ``scan`` case is an iteration: ``chunks`` prefill chunks of ``chunk_lo`` .. ``chunk_hi`` new tokens (the first
``fresh`` of them begin their sequence), then ``decodes`` sequences with one new token.  A ``prompt`` case is ``batch`` prompts
of ``len_lo`` .. ``len_hi`` tokens.  Lengths are log-uniform; ``lens`` seeds them, so that they belong to the case.
"""
import math
import random

import torch

own = False

DEVICE = "cuda:0"
SHAPE_S1 = dict(hq=8, hkv=2, d=64)
SHAPE_8B = dict(hq=32, hkv=8, d=128)
SHAPE_70B = dict(hq=64, hkv=8, d=128)
SHAPES = (SHAPE_S1, SHAPE_8B, SHAPE_70B, dict(hq=8, hkv=8, d=64), dict(hq=8, hkv=4, d=64), dict(hq=6, hkv=2, d=128),
          dict(hq=5, hkv=1, d=128))
MOST_SCAN = 8192 * 8192 * 16                 # tokens x channels x states of the largest case
MOST_PAIRS = 32 * 8192 * 8192                # (head, row, key) triples of the largest padded batch of prompts


def _conv(channels, width, chunks=0, chunk_lo=1, chunk_hi=1, fresh=0, decodes=0, lens=1, bias=True, silu=True):
    return dict(op="conv", channels=channels, width=width, chunks=chunks, chunk_lo=chunk_lo, chunk_hi=chunk_hi, fresh=fresh,
                decodes=decodes, lens=lens, bias=bias, silu=silu)


def _scan(channels, states, chunks=0, chunk_lo=1, chunk_hi=1, fresh=0, decodes=0, lens=1, gate=True):
    return dict(op="scan", channels=channels, states=states, chunks=chunks, chunk_lo=chunk_lo, chunk_hi=chunk_hi, fresh=fresh,
                decodes=decodes, lens=lens, gate=gate)


def _prompt(shape, batch, len_lo, len_hi, lens=1):
    return dict(op="prompt", **shape, batch=batch, len_lo=len_lo, len_hi=len_hi, lens=lens)


def listed():
    return [
        # a decode-heavy iteration of a large layer
        dict(name="conv_decode_64", **_conv(8192, 4, decodes=64, lens=11)),
        # a prefill iteration at the token budget a scheduler fills
        dict(name="conv_prefill_8x1024", **_conv(8192, 4, chunks=8, chunk_lo=1024, chunk_hi=1024, fresh=4, lens=12)),
        # ragged chunks beside single tokens, a small layer of an odd width, no bias, nothing after it
        dict(name="conv_mixed_ragged", **_conv(1544, 3, chunks=12, chunk_lo=2, chunk_hi=700, fresh=6, decodes=37, lens=13,
                                               bias=False, silu=False)),
        # one user of a small model: a layer is all latency
        dict(name="scan_decode_1", **_scan(1536, 16, decodes=1, lens=21)),
        # a decode-heavy iteration of a large layer: the states are what is read
        dict(name="scan_decode_128", **_scan(8192, 16, decodes=128, lens=22)),
        # one long prompt
        dict(name="scan_prompt_1x8192", **_scan(4096, 16, chunks=1, chunk_lo=8192, chunk_hi=8192, fresh=1, lens=23)),
        # a prefill iteration at the token budget
        dict(name="scan_prefill_8x1024", **_scan(8192, 16, chunks=8, chunk_lo=1024, chunk_hi=1024, fresh=4, lens=24)),
        # ragged chunks beside single tokens, larger states, no gate
        dict(name="scan_mixed_ragged", **_scan(2056, 64, chunks=9, chunk_lo=2, chunk_hi=600, fresh=5, decodes=61, lens=25,
                                               gate=False)),
        # many short prompts (queries to embed, classify or rank)
        dict(name="prompt_64_short", **_prompt(SHAPE_8B, 64, 1, 64, lens=31)),
        # a ragged batch of ordinary prompts
        dict(name="prompt_16_ragged", **_prompt(SHAPE_8B, 16, 100, 2000, lens=32)),
        # documents on a layer with many heads
        dict(name="prompt_3_documents", **_prompt(SHAPE_70B, 3, 1500, 3000, lens=33)),
        # one long document
        dict(name="prompt_1x8192", **_prompt(SHAPE_8B, 1, 8192, 8192, lens=34)),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(lo * math.exp(rng.random() * math.log((hi + 1) / lo)))))


def draw(rng):
    op = rng.choice(["conv", "scan", "prompt"])
    seed = rng.randint(1, 1 << 30)
    if op == "prompt":
        shape = rng.choice(SHAPES)
        batch = _log_int(rng, 1, 64)
        most = min(8192, 16384 // batch, math.isqrt(MOST_PAIRS // (batch * max(32, shape["hq"]))))
        len_hi = _log_int(rng, 1, most)
        return _prompt(shape, batch, _log_int(rng, 1, len_hi), len_hi, lens=seed)
    channels = 8 * _log_int(rng, 8, 1024)
    states = rng.choice([16, 16, 16, 8, 32, 64]) if op == "scan" else 16
    rows = min(16384, MOST_SCAN // (channels * states))
    kind = rng.choice(["decode", "prefill", "prefill", "mixed"])
    more = {}
    if kind != "decode":
        chunks = _log_int(rng, 1, 16)
        chunk_hi = _log_int(rng, 2, max(2, min(8192, rows // chunks // 2)))
        more = dict(chunks=chunks, chunk_lo=_log_int(rng, 2, chunk_hi), chunk_hi=chunk_hi, fresh=rng.randint(0, chunks))
    if kind != "prefill":
        more["decodes"] = _log_int(rng, 1, max(1, min(256, rows // 2)))
    if op == "conv":
        return _conv(channels, rng.choice([2, 3, 4, 4]), lens=seed, bias=rng.random() < 0.7, silu=rng.random() < 0.7, **more)
    return _scan(channels, states, lens=seed, gate=rng.random() < 0.7, **more)


def _lengths(case):
    """(new tokens, context length with them) of every sequence."""
    rng = random.Random(case["lens"])
    if case["op"] == "prompt":
        q = [_log_int(rng, case["len_lo"], case["len_hi"]) for _ in range(case["batch"])]
        return q, q
    q = [_log_int(rng, case["chunk_lo"], case["chunk_hi"]) for _ in range(case["chunks"])]
    ctx = [n if i < case["fresh"] else n + rng.randint(1, 4096) for i, n in enumerate(q)]
    return q + [1] * case["decodes"], ctx + [rng.randint(2, 8192) for _ in range(case["decodes"])]


def work(case):
    q_lens, ctx_lens = _lengths(case)
    n, seqs = sum(q_lens), len(q_lens)
    kept = sum(c > q for q, c in zip(q_lens, ctx_lens))                     # sequences whose state is read
    if case["op"] == "prompt":
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        pairs = sum(q * (q + 1) // 2 for q in q_lens)
        return {"bytes": n * (2 * hq * d * 2 + 2 * hkv * d * 2 + 4 * hq), "flops": 4 * d * hq * pairs}
    c = case["channels"]
    if case["op"] == "conv":
        w = case["width"]
        return {"bytes": 4 * n * c + 2 * (w - 1) * c * (kept + seqs) + 2 * w * c, "flops": 2 * w * n * c}
    s = case["states"]
    row = 2 * c * (4 if case["gate"] else 3) + 4 * s                        # x, dt, out (and z), B and C
    return {"bytes": n * row + 4 * c * s * (kept + seqs) + 4 * c * (s + 2), "flops": 6 * n * c * s}


# ------------------------------------------------------------------- state --

class _Handles:
    """The library's pool and plan of a state: what a serving loop holds while it runs an iteration's layers."""

    def __init__(self, case, s):
        import paper_2604_07144_b200 as ap
        self.ap = ap
        self.pool = self.plan = None
        if case["op"] == "prompt":
            self.close = ap.prompt_plan_destroy, ap.kv_pool_destroy
            self.pool = ap.kv_pool_create(1, case["hkv"], case["d"])
            self.plan = ap.prompt_plan_create(self.pool, s["q_lens"], case["hq"])
            return
        self.close = ap.state_plan_destroy, ap.state_pool_destroy
        states, width = case.get("states", 16), case.get("width", 4)
        self.pool = ap.state_pool_create(s["slots"], case["channels"], states, width, s.get("conv"), s.get("state"))
        self.plan = ap.state_plan_create(self.pool, s["q_lens"], s["ctx_lens"], s["slot"].cpu().numpy())
        self.workspace = torch.empty(max(256, ap.state_plan_workspace_bytes(self.plan)), dtype=torch.uint8, device=DEVICE)

    def __del__(self):
        if getattr(self, "plan", None) is not None:
            self.close[0](self.plan)
        if getattr(self, "pool", None) is not None:
            self.close[1](self.pool)


def prepare(case, seed):
    gen = torch.Generator(DEVICE).manual_seed(seed)
    q_lens, ctx_lens = _lengths(case)
    n, seqs = sum(q_lens), len(q_lens)
    s = dict(case=case, q_lens=q_lens, ctx_lens=ctx_lens, n=n)
    lens = torch.tensor(q_lens, device=DEVICE)
    s["len"] = lens
    s["first"] = torch.cumsum(lens, 0) - lens                               # row of each sequence's first new token
    s["seq"] = torch.repeat_interleave(torch.arange(seqs, device=DEVICE), lens)
    s["pos"] = torch.arange(n, device=DEVICE) - s["first"][s["seq"]]        # row within its sequence's new tokens

    def normal(*shape, dtype=torch.bfloat16):
        return torch.randn(*shape, generator=gen, device=DEVICE, dtype=dtype)

    if case["op"] == "prompt":
        hq, hkv, d = case["hq"], case["hkv"], case["d"]
        qkv = normal(n, hq + 2 * hkv, d)                                    # q, k and v as one projection leaves them
        s["q"], s["k"], s["v"] = qkv[:, :hq], qkv[:, hq:hq + hkv], qkv[:, hq + hkv:]
        s["out"] = torch.empty(n, hq, d, dtype=torch.bfloat16, device=DEVICE)
        s["lse"] = torch.empty(n, hq, dtype=torch.float32, device=DEVICE)
    else:
        c = case["channels"]
        s["slots"] = math.ceil(1.25 * seqs)
        s["slot"] = torch.randperm(s["slots"], generator=gen, device=DEVICE)[:seqs].int()
        s["kept"] = torch.tensor(ctx_lens, device=DEVICE) > lens            # sequences that go on from their slot
        xz = normal(n, 2 * c)                                               # input and gate as one projection leaves them
        s["x"], s["z"] = xz[:, :c], xz[:, c:]
        s["out"] = torch.empty(n, c, dtype=torch.bfloat16, device=DEVICE)
    if case["op"] == "conv":
        s["conv"] = normal(s["slots"], case["width"] - 1, c)
        s["weight"] = (normal(c, case["width"], dtype=torch.float32) / math.sqrt(case["width"])).bfloat16()
        s["bias"] = normal(c) if case["bias"] else None
    elif case["op"] == "scan":
        states, rank = case["states"], 8 * max(1, c // 128)
        s["dt"] = (0.7 * normal(n, c, dtype=torch.float32)).bfloat16()
        proj = normal(n, rank + 2 * states)                                 # B and C lie behind the step's low-rank part
        s["b"], s["c"] = proj[:, rank:rank + states], proj[:, rank + states:]
        # steps of 0.001 to 0.1 before the input moves them, decays of 1 to `states`: how such layers begin, and stay near
        step = torch.exp(torch.rand(c, generator=gen, device=DEVICE) * math.log(100.0) + math.log(0.001))
        s["dt_bias"] = torch.log(torch.expm1(step))
        s["a"] = -torch.arange(1, states + 1, device=DEVICE, dtype=torch.float32) * torch.exp(0.2 * normal(c, states, dtype=torch.float32))
        s["skip"] = 1.0 + 0.2 * normal(c, dtype=torch.float32)
        s["state"] = 0.3 * normal(s["slots"], c, states, dtype=torch.float32)
    if own:
        s["lib"] = _Handles(case, s)
    return s


# --------------------------------------------------------------------- run --

def run(s):
    return {"conv": _run_conv, "scan": _run_scan, "prompt": _run_prompt}[s["case"]["op"]](s)


def _run_conv(s):
    case = s["case"]
    if own:
        lib = s["lib"]
        lib.ap.conv_iteration(lib.pool, lib.plan, s["x"], s["weight"], s["out"], bias=s["bias"], silu=case["silu"])
        return {"out": s["out"], "conv": s["conv"]}
    w = case["width"]
    # what each tap of each row sees: a row of x, or (before the sequence's first new token) a row of its slot
    slot = s["slot"].long()
    old = torch.where(s["kept"][:, None, None], s["conv"][slot], 0).flatten(0, 1)          # [sequences * (w - 1), channels]
    rows = torch.cat((old, s["x"]))
    back = torch.arange(1 - w, 1, device=DEVICE)

    def at(seq, pos):                                          # row of `rows` at a position of a sequence, -1: the slot's last
        return torch.where(pos >= 0, len(old) + s["first"][seq] + pos, (seq + 1) * (w - 1) + pos)

    taps = rows[at(s["seq"][:, None], s["pos"][:, None] + back)]                            # [n, w, channels]
    y = (taps.float() * s["weight"].float().T).sum(1)
    if s["bias"] is not None:
        y = y + s["bias"].float()
    if case["silu"]:
        y = y / (1 + torch.exp(-y))
    s["out"].copy_(y)
    seq = torch.arange(len(slot), device=DEVICE)[:, None]
    s["conv"][slot] = rows[at(seq, s["len"][:, None] + back[:-1])]
    return {"out": s["out"], "conv": s["conv"]}


def _run_scan(s):
    case = s["case"]
    if own:
        lib = s["lib"]
        lib.ap.scan_iteration(lib.pool, lib.plan, s["x"], s["dt"], s["a"], s["b"], s["c"], s["out"],
                              z=s["z"] if case["gate"] else None, d_skip=s["skip"], dt_bias=s["dt_bias"], softplus=True,
                              workspace=lib.workspace)
        return {"out": s["out"], "state": s["state"]}
    x = s["x"].float()
    dt = s["dt"].float() + s["dt_bias"]
    dt = dt.clamp_min(0) + torch.log1p(torch.exp(-dt.abs()))
    decay = torch.exp(dt[:, :, None] * s["a"])                                              # [n, channels, states]
    h = (dt * x)[:, :, None] * s["b"].float()[:, None]
    slot, first = s["slot"].long(), s["first"]
    h[first] += decay[first] * torch.where(s["kept"][:, None, None], s["state"][slot], 0)
    decay[first] = 0                                           # nothing comes over from the sequence before
    k = 1
    while k < max(s["q_lens"]):                                # h[t] takes in its last 1, 2, 4, ... tokens
        h[k:] += decay[k:] * h[:-k]
        decay[k:] = decay[k:] * decay[:-k]
        k *= 2
    y = (h * s["c"].float()[:, None]).sum(-1) + s["skip"] * x
    if case["gate"]:
        z = s["z"].float()
        y = y * (z / (1 + torch.exp(-z)))
    s["out"].copy_(y)
    s["state"][slot] = h[first + s["len"] - 1]
    return {"out": s["out"], "state": s["state"]}


def _run_prompt(s):
    case = s["case"]
    if own:
        lib = s["lib"]
        lib.ap.prompt_attention(lib.pool, lib.plan, s["q"], s["k"], s["v"], s["out"], s["lse"])
        return {"out": s["out"], "lse": s["lse"]}
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    longest, seqs = max(s["q_lens"]), len(s["q_lens"])

    def padded(x):                                             # [prompts, kv heads, heads of a group, longest, d]
        y = torch.zeros(seqs, longest, *x.shape[1:], device=DEVICE)
        y[s["seq"], s["pos"]] = x.float()
        return y.unflatten(2, (hkv, -1)).permute(0, 2, 3, 1, 4)

    q, k, v = padded(s["q"]), padded(s["k"]), padded(s["v"])
    x = torch.matmul(q.flatten(2, 3), k[:, :, 0].transpose(-1, -2)).unflatten(2, (hq // hkv, longest))
    x /= math.sqrt(d)
    at = torch.arange(longest, device=DEVICE)
    x.masked_fill_(at[None, :] > at[:, None], float("-inf"))   # (a padded row sees keys of zeros)
    top = x.amax(-1, keepdim=True)
    p = x.sub_(top).exp_()
    total = p.sum(-1, keepdim=True)
    o = torch.matmul(p.flatten(2, 3), v[:, :, 0]).unflatten(2, (hq // hkv, longest)) / total
    rows = lambda y: y.permute(0, 3, 1, 2, 4)[s["seq"], s["pos"]].flatten(1, 2)              # noqa: E731
    s["out"].copy_(rows(o))
    s["lse"].copy_(rows(top + total.log())[..., 0])
    return {"out": s["out"], "lse": s["lse"]}


# ------------------------------------------------------------------- exact --

def exact(case, seed):
    s = prepare(case, seed)
    return {"conv": _exact_conv, "scan": _exact_scan, "prompt": _exact_prompt}[case["op"]](s)


def _exact_conv(s):
    """Sequence by sequence: a convolution of the old inputs followed by the new ones."""
    case, w = s["case"], s["case"]["width"]
    out, conv, row = [], s["conv"].double(), 0
    kernel = s["weight"].double()
    for ql, cl, slot in zip(s["q_lens"], s["ctx_lens"], s["slot"].tolist()):
        old = conv[slot] if cl > ql else torch.zeros_like(conv[slot])
        u = torch.cat((old, s["x"][row:row + ql].double()))
        y = sum(u[j:j + ql] * kernel[:, j] for j in range(w))
        out.append(y if s["bias"] is None else y + s["bias"].double())
        conv[slot] = u[ql:]
        row += ql
    out = torch.cat(out)
    return {"out": out * torch.sigmoid(out) if case["silu"] else out, "conv": conv}


def _exact_scan(s):
    """Token by token, all sequences at once."""
    case = s["case"]
    slot, lens, first, kept = s["slot"].tolist(), s["q_lens"], s["first"].tolist(), s["kept"].tolist()
    order = sorted(range(len(lens)), key=lambda i: -lens[i])
    state = s["state"].double()
    h = torch.stack([state[slot[i]] * kept[i] for i in order])
    a, out = s["a"].double(), torch.empty(s["n"], case["channels"], dtype=torch.float64, device=DEVICE)
    begin = torch.tensor([first[i] for i in order], device=DEVICE)
    live = len(order)
    for t in range(lens[order[0]]):
        while lens[order[live - 1]] <= t:
            live -= 1
        rows = begin[:live] + t
        x = s["x"][rows].double()
        dt = torch.nn.functional.softplus(s["dt"][rows].double() + s["dt_bias"].double(), threshold=200)
        h[:live] = h[:live] * torch.exp(dt[..., None] * a) + (dt * x)[..., None] * s["b"][rows].double()[:, None]
        out[rows] = torch.einsum("bcn,bn->bc", h[:live], s["c"][rows].double()) + x * s["skip"].double()
    for k, i in enumerate(order):
        state[slot[i]] = h[k]
    if case["gate"]:
        z = s["z"].double()
        out = out * z * torch.sigmoid(z)
    return {"out": out, "state": state}


def _exact_prompt(s):
    case = s["case"]
    hq, hkv, d = case["hq"], case["hkv"], case["d"]
    out, lse, row = [], [], 0
    for n in s["q_lens"]:
        q, k, v = (s[name][row:row + n].double().transpose(0, 1) for name in ("q", "k", "v"))
        o, l = [], []
        for g in range(hkv):
            x = torch.einsum("htd,jd->htj", q[g * hq // hkv:(g + 1) * hq // hkv], k[g]) * d ** -0.5
            x.masked_fill_(torch.ones(n, n, dtype=torch.bool, device=DEVICE).triu(1), -math.inf)
            l.append(torch.logsumexp(x, -1))
            o.append(torch.softmax(x, -1) @ v[g])
        out.append(torch.cat(o).transpose(0, 1))
        lse.append(torch.cat(l).T)
        row += n
    return {"out": torch.cat(out), "lse": torch.cat(lse)}
