"""The serving operators whose speed counts: a review step over a paged cache, operator by operator.

Four kinds of call:
  attend  csd_paged_attention: a chunk of new tokens of each sequence over the paged cache that holds their keys
  store   csd_paged_append and csd_paged_read of the same rows: what the cache holds of them (bf16, or 8 bits with a scale a row)
  read    csd_paged_read of whole sequences
  verify  csd_spec_verify: drafted tokens against the target's probabilities, with given random numbers

Pools are [page][kv head][slot][dimension]; a sequence's pages lie anywhere.  Slots that no sequence has written hold NaN.
An 8-bit row is e4m3 numbers times 2^e, e the smallest whole number (at least -100) with max|x| <= 448 * 2^e, stored as e + 127.
"""
import math

import numpy as np
import torch

own = False

GOLDEN = (0.6180339887498949, 0.7548776662466927)
LEAST = -100                    # least exponent of an 8-bit row's scale
SCRATCH = 48 << 20


def listed():
    return [
        # the draft model's decode of one sequence: latency
        {"name": "attend_draft_m1", "kind": "attend", "seqs": 1, "rows_lo": 1, "rows_hi": 1, "kv_lo": 203, "kv_hi": 203, "heads": 12, "kv_heads": 12,
         "dim": 64, "page": 16, "pool": "bf16", "rows": "bf16", "tree": False},
        # three sequences' blocks as the library's own model hands them over, in 32 bits
        {"name": "attend_review_f32", "kind": "attend", "seqs": 3, "rows_lo": 3, "rows_hi": 5, "kv_lo": 77, "kv_hi": 301, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 64, "pool": "bf16", "rows": "f32", "tree": False},
        # trees of candidates of eight sequences, 8-bit cache
        {"name": "attend_tree_8x12", "kind": "attend", "seqs": 8, "rows_lo": 12, "rows_hi": 12, "kv_lo": 77, "kv_hi": 2048, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 32, "pool": "e4m3", "rows": "bf16", "tree": True},
        # one token of each of 64 sequences, grouped heads: streams the cache
        {"name": "attend_decode_64", "kind": "attend", "seqs": 64, "rows_lo": 1, "rows_hi": 1, "kv_lo": 500, "kv_hi": 8000, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 16, "pool": "bf16", "rows": "bf16", "tree": False},
        # a prompt on an empty cache
        {"name": "attend_prompt_1000", "kind": "attend", "seqs": 1, "rows_lo": 1000, "rows_hi": 1000, "kv_lo": 0, "kv_hi": 0, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 64, "pool": "bf16", "rows": "bf16", "tree": False},
        # a chunk of a long prompt, grouped heads, behind a long 8-bit cache: the products count
        {"name": "attend_chunk_8bit", "kind": "attend", "seqs": 2, "rows_lo": 400, "rows_hi": 700, "kv_lo": 9000, "kv_hi": 15000, "heads": 32, "kv_heads": 8,
         "dim": 128, "page": 64, "pool": "e4m3", "rows": "bf16", "tree": False},
        # the new rows of a review of eight sequences, quantised as they are written: latency
        {"name": "store_review_8x5", "kind": "store", "seqs": 8, "rows_lo": 3, "rows_hi": 5, "kv_lo": 77, "kv_hi": 2048, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 16, "pool": "e4m3", "rows": "f32"},
        # prompts of several sequences
        {"name": "store_prompts", "kind": "store", "seqs": 6, "rows_lo": 500, "rows_hi": 2500, "kv_lo": 0, "kv_hi": 128, "heads": 32, "kv_heads": 32,
         "dim": 128, "page": 64, "pool": "e4m3", "rows": "bf16"},
        # whole sequences read back, as for a hand-over to another program
        {"name": "read_context", "kind": "read", "seqs": 16, "rows_lo": 300, "rows_hi": 4000, "kv_lo": 0, "kv_hi": 0, "heads": 8, "kv_heads": 8,
         "dim": 128, "page": 32, "pool": "e4m3", "rows": "bf16"},
        # one sequence's drafts: latency
        {"name": "verify_1x4_v32000", "kind": "verify", "seqs": 1, "k": 4, "vocab": 32000, "sigma": 0.5, "cut": 0.0, "law": "f32"},
        # a large batch over a large vocabulary, ragged drafts, laws cut to their likely entries
        {"name": "verify_256x8_v128256", "kind": "verify", "seqs": 256, "k": 8, "vocab": 128256, "sigma": 0.5, "cut": 0.001, "law": "f32"},
        # statistical drafts (point masses) in a middling batch, laws in 16 bits
        {"name": "verify_point_16x5", "kind": "verify", "seqs": 16, "k": 5, "vocab": 32128, "sigma": 0.0, "cut": 0.0, "law": "bf16"},
    ]


def _between(rng, lo, hi):
    """A whole number from lo to hi, spread over its logarithm."""
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["attend", "attend", "attend", "attend", "store", "read", "verify", "verify"])
    if kind == "verify":
        c = {"kind": kind, "seqs": _between(rng, 1, 200), "k": rng.randint(1, 12), "vocab": _between(rng, 500, 128256), "sigma": rng.choice([0.0, 0.1, 0.5, 2.0]),
             "cut": rng.choice([0.0, 0.001, 0.02]), "law": rng.choice(["f32", "f32", "bf16"])}
        c["seqs"] = max(1, min(c["seqs"], (256 * 9 * 128256) // ((c["k"] + 1) * c["vocab"])))
        return c
    kv_heads = rng.choice([1, 2, 5, 8, 12, 32])
    c = {"kind": kind, "seqs": _between(rng, 1, 64), "heads": kv_heads, "kv_heads": kv_heads, "dim": rng.choice([64, 128, 128]),
         "page": rng.choice([16, 32, 64, 128]), "pool": rng.choice(["bf16", "e4m3"]), "rows": rng.choice(["bf16", "bf16", "f32"])}
    if kind != "attend":
        most = max(2, 48_000_000 // (c["seqs"] * kv_heads * c["dim"]))
        hi = _between(rng, 1, min(4000, most))
        c |= {"rows_lo": _between(rng, 1, hi), "rows_hi": hi, "kv_lo": 0, "kv_hi": rng.randint(0, 300) if kind == "store" else 0}
        return c
    c["heads"] = kv_heads * rng.choice([1, 1, 2, 4, 7]) if kv_heads <= 12 else kv_heads
    # tokens a sequence: one, a review, or a chunk; the keys behind them as far as the largest listed case's work allows
    size = rng.choice(["decode", "review", "review", "chunk"])
    hi = {"decode": 1, "review": rng.randint(2, 17), "chunk": _between(rng, 18, 1000 if c["rows"] == "bf16" else 60)}[size]
    if size == "chunk":
        c["seqs"] = min(c["seqs"], 6)
    c |= {"rows_lo": _between(rng, 1, hi), "rows_hi": hi, "tree": size == "review" and rng.random() < 0.4}
    most = min(500_000_000 // (c["seqs"] * kv_heads * c["dim"]), 500_000_000 // (c["seqs"] * c["heads"] * hi), 20000)
    far = _between(rng, 1, max(2, most - hi))
    c |= {"kv_lo": rng.choice([0, _between(rng, 1, far)]), "kv_hi": far}
    return c


def _lens(case):
    """Rows and cached positions of each sequence, spread over their ranges; the first has the most of both."""
    def spread(lo, hi, by):
        return [hi - int((hi - lo) * ((s * by) % 1.0) + 0.5) for s in range(case["seqs"])]
    return spread(case["rows_lo"], case["rows_hi"], GOLDEN[0]), spread(case["kv_lo"], case["kv_hi"], GOLDEN[1])


def _dtype(name):
    return {"f32": torch.float32, "bf16": torch.bfloat16, "e4m3": torch.float8_e4m3fn}[name]


def _drafts(case):
    """Drafts of each sequence: from none to k."""
    k = case["k"]
    return [k - int((k + 1) * ((s * GOLDEN[0]) % 1.0) * 0.5) for s in range(case["seqs"])]


def _power(e):
    """2^e in 32 bits for whole e from -126 to 127, put together from its bits (pow may be off by an ulp)."""
    return ((e.int() + 127) << 23).view(torch.float32)


def _quantise(x):
    """Rows [..., dimension] in 32 bits as e4m3 numbers and exponents."""
    a = x.abs().amax(-1)
    m, e = torch.frexp(a)                                   # a = m * 2^e, m in [0.5, 1): 448 * 2^n = 0.875 * 2^(n + 9)
    e = torch.where(a > 0, e - 9 + (m > 0.875).to(e.dtype), LEAST).clamp_min(LEAST)
    return (x * _power(-e)[..., None]).to(torch.float8_e4m3fn), (e + 127).to(torch.uint8)


def _values(rows, exponents):
    """What stored rows [..., dimension] stand for, in 32 bits."""
    x = rows.float()
    return x if exponents is None else x * _power(exponents.int() - 127)[..., None]


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed))
    normal = lambda *shape: torch.randn(*shape, generator=g, device="cuda")  # noqa: E731
    if case["kind"] == "verify":
        return _prepare_verify(case, g)
    rows, kv = _lens(case)
    P, H, D, S = case["page"], case["kv_heads"], case["dim"], case["seqs"]
    need = [(r + n + P - 1) // P for r, n in zip(rows, kv)]
    n_pages = sum(need) + 3
    order = torch.randperm(n_pages, generator=g, device="cuda").int()
    table = torch.zeros(S, max(need), dtype=torch.int32)
    at = np.concatenate([[0], np.cumsum(need)])
    order = order.cpu()
    for s in range(S):
        table[s, :need[s]] = order[at[s]:at[s + 1]]
    s = {"kind": case["kind"], "page": P, "rows": sum(rows), "most": max(rows), "keys": max(r + n for r, n in zip(rows, kv)),
         "table": table.cuda(), "row_start": torch.tensor(np.concatenate([[0], np.cumsum(rows)]), dtype=torch.int32, device="cuda"),
         "kv_len": torch.tensor(kv, dtype=torch.int32, device="cuda"), "type": _dtype(case["rows"]), "scratch": torch.zeros(SCRATCH, dtype=torch.uint8, device="cuda")}
    # slots that hold a position (of those a store writes, none yet); the others are NaN
    held = torch.zeros(n_pages * P, dtype=torch.bool, device="cuda")
    position = torch.arange(max(need) * P, device="cuda")
    filled = s["kv_len"] if case["kind"] == "store" else s["kv_len"] + torch.tensor(rows, device="cuda")
    slot = s["table"].long()[:, position // P] * P + position % P
    held[slot[position[None] < filled[:, None]]] = True
    held = held.view(n_pages, 1, P, 1)
    for name in ("k", "v"):
        x = normal(n_pages, H, P, D).masked_fill_(~held, math.nan)
        if case["pool"] == "e4m3":
            s[name], s[name + "_exp"] = _quantise(x.nan_to_num_(0.0).mul_(torch.exp(0.5 * normal(n_pages, H, P, 1))))
            s[name].view(torch.uint8).masked_fill_(~held, 0x7F)             # NaN
            s[name + "_exp"].masked_fill_(~held[..., 0], 255)
        else:
            s[name], s[name + "_exp"] = x.bfloat16(), None
    if case["kind"] == "store":
        for name in ("k_new", "v_new"):
            s[name] = (normal(sum(rows), H, D) * torch.exp(0.5 * normal(sum(rows), H, 1))).to(s["type"])
    if case["kind"] == "attend":
        s["q"] = (normal(sum(rows), case["heads"], D) * 1.5).to(s["type"])
        s["scale"] = 1.0 / math.sqrt(D)
        s["tree"] = _trees(rows, g) if case["tree"] else None
    if own:
        from paper_2312_11462_b200 import binding as b
        s["pool"] = b.KvPool(s["k"], s["v"], s["k_exp"], s["v_exp"])
        s["batch"] = b.PagedBatch(s["table"], s["row_start"], s["kv_len"], s["rows"], s["most"])
    return s


def _trees(rows, g):
    """A row's ancestors in its sequence's block and itself, as bits: each row's parent is an earlier row."""
    up = torch.rand(sum(rows), generator=g, device="cuda").cpu().tolist()
    masks, at = [], 0
    for n in rows:
        mine = []
        for r in range(n):
            mine.append((mine[int(up[at + r] * r)] if r else 0) | 1 << r)
        masks += mine
        at += n
    return torch.tensor(masks, dtype=torch.int64, device="cuda")


def _prepare_verify(case, g):
    S, k, V = case["seqs"], case["k"], case["vocab"]

    def law(x):
        x = x.softmax(-1)
        if case["cut"]:
            x = torch.where(x < case["cut"] * x.amax(-1, keepdim=True), 0.0, x)
            x = x / x.sum(-1, keepdim=True)
        return x.to(_dtype(case["law"]))

    logits = 3.0 * torch.randn(S, k + 1, V, generator=g, device="cuda")
    p = law(logits)
    if case["sigma"]:
        q = law(logits[:, :k] + case["sigma"] * torch.randn(S, k, V, generator=g, device="cuda"))
        tokens = torch.multinomial(q.view(S * k, V).float(), 1, generator=g).view(S, k).int()
    else:                        # statistical drafts: often the likeliest token, else any
        q = None
        tokens = torch.where(torch.rand(S, k, generator=g, device="cuda") < 0.8, logits[:, :k].argmax(-1), torch.randint(V, (S, k), generator=g, device="cuda")).int()
    return {"kind": "verify", "p": p, "q": q, "tokens": tokens, "n": torch.tensor(_drafts(case), dtype=torch.int32, device="cuda"),
            "u": torch.rand(S, k + 1, generator=g, device="cuda")}


def run(state):
    s = state
    if own:
        from paper_2312_11462_b200 import binding as b
        if s["kind"] == "verify":
            return b.csd_spec_verify(s["p"], s["q"], s["tokens"], s["u"], s["n"])
        if s["kind"] == "attend":
            return b.csd_paged_attention(s["q"], s["pool"], s["batch"], s["scale"], tree_mask=s["tree"], workspace=s["scratch"])
        if s["kind"] == "store":
            b.csd_paged_append(s["pool"], s["batch"], s["k_new"], s["v_new"])
        return b.csd_paged_read(s["pool"], s["batch"], s["type"])
    if s["kind"] == "verify":
        return _verify(s["p"], s["q"], s["tokens"], s["u"], s["n"])
    if s["kind"] == "attend":
        return _attend(s)
    page, slot = _places(s)
    if s["kind"] == "store":
        for name in ("k", "v"):
            x = s[name + "_new"].float()
            if s[name + "_exp"] is None:
                s[name][page, :, slot] = x.bfloat16()
            else:
                x, e = _quantise(x)
                s[name].view(torch.uint8)[page, :, slot] = x.view(torch.uint8)
                s[name + "_exp"][page, :, slot] = e
    return tuple(_values(_take(s[n], page, slot), None if s[n + "_exp"] is None else s[n + "_exp"][page, :, slot]).to(s["type"]) for n in ("k", "v"))


def _take(pool, page, slot):
    """Rows [..., kv head, dimension] of the pool."""
    if pool.dtype == torch.float8_e4m3fn:
        return pool.view(torch.uint8)[page, :, slot].view(torch.float8_e4m3fn)
    return pool[page, :, slot]


def _sequence(s):
    """Of each new row, its sequence and its place in the sequence's chunk."""
    r = torch.arange(s["rows"], device="cuda")
    seq = torch.searchsorted(s["row_start"][1:].long(), r, right=True)
    return seq, r - s["row_start"][seq]


def _places(s):
    """Page and slot of each new row."""
    seq, i = _sequence(s)
    at = s["kv_len"][seq] + i
    return s["table"][seq, at // s["page"]].long(), at % s["page"]


def _attend(s):
    H, D = s["k"].shape[1], s["k"].shape[3]
    S, N, R, G = len(s["kv_len"]), s["keys"], s["most"], s["q"].shape[1] // H
    rows = s["row_start"][1:] - s["row_start"][:-1]
    at = torch.arange(N, device="cuda")
    page, slot = s["table"].long()[:, at // s["page"]], (at % s["page"]).expand(S, N)
    there = at < (s["kv_len"] + rows)[:, None]                                              # [S, N]

    def keys(name):
        x = _values(_take(s[name], page, slot), None if s[name + "_exp"] is None else s[name + "_exp"][page, :, slot])
        return torch.where(there[..., None, None], x, 0.0).transpose(1, 2)                  # [S, H, N, D]

    i = torch.arange(R, device="cuda")
    mine = (s["row_start"][:-1, None] + i).clamp_max(s["rows"] - 1).long()                  # [S, R]
    q = s["q"].float()[mine].view(S, R, H, G, D).permute(0, 2, 3, 1, 4).reshape(S, H, G * R, D)
    if s["tree"] is None:
        sees = at <= (s["kv_len"][:, None] + i)[..., None]
    else:
        new = at - s["kv_len"][:, None, None]                                               # [S, 1, N]
        sees = (new < 0) | ((s["tree"][mine][..., None] >> new.clamp(0, 63)) & 1).bool() & (new < 64)
    sees = (sees & there[:, None])[:, None, None].expand(S, 1, G, R, N).reshape(S, 1, G * R, N)
    x = (q @ keys("k").transpose(2, 3)).mul_(s["scale"]).masked_fill_(~sees, -math.inf)
    top = x.amax(-1, keepdim=True)
    x = x.sub_(torch.where(top == -math.inf, 0.0, top)).exp_()
    total = x.sum(-1, keepdim=True)
    out = (x @ keys("v")) / torch.where(total > 0, total, 1.0)
    out = out.view(S, H, G, R, D).permute(0, 3, 1, 2, 4).reshape(S, R, H * G, D)
    seq, i = _sequence(s)
    return out[seq, i].to(s["type"])


def _verify(p, q, tokens, u, n):
    S, k1, V = p.shape
    k, each = k1 - 1, torch.arange(S, device="cuda")
    x = tokens.long()
    px = p[:, :k].gather(2, x[..., None])[..., 0].double()
    qx = q.gather(2, x[..., None])[..., 0].double() if q is not None else torch.ones_like(px)
    passed = (u[:, :k].double() * qx < px) & (torch.arange(k, device="cuda") < n[:, None])
    a = passed.long().cumprod(1).sum(1)                                                     # accepted
    law, refused, last = p[each, a].double(), (a < n)[:, None], a.clamp_max(k - 1)
    if q is not None:
        left = (law - q[each, last].double()).clamp_min(0.0)
    else:
        left = law.scatter(1, x[each, last][:, None], 0.0)
    mass = torch.where(refused & (left.sum(1, keepdim=True) > 0), left, law)
    cum = mass.cumsum(1)
    token = (cum > u[:, k:].double() * cum[:, -1:]).int().argmax(1)
    i = torch.arange(k1, device="cuda")
    out = torch.where(i < a[:, None], torch.nn.functional.pad(x, (0, 1)), -1)
    return a.int(), torch.where(i == a[:, None], token[:, None], out).int()


def work(case):
    if case["kind"] == "verify":
        size = 2 if case["law"] == "bf16" else 4
        # the numbers of the tests, and one law for the token (two where the sequence's drafts are refused: not counted)
        laws = sum(case["vocab"] + n * (1 if case["sigma"] == 0 else 2) for n in _drafts(case))
        return {"bytes": size * laws + case["seqs"] * (case["k"] + 1) * 12, "flops": 3 * case["seqs"] * case["vocab"]}
    rows, kv = _lens(case)
    D, H, size = case["dim"], case["kv_heads"], 2 if case["rows"] == "bf16" else 4
    row = 2 * H * (2 * D if case["pool"] == "bf16" else D + 1)                              # bytes of a position in the pool
    if case["kind"] == "attend":
        return {"bytes": sum(r + n for r, n in zip(rows, kv)) * row + 2 * sum(rows) * case["heads"] * D * size,
                "flops": 4 * D * case["heads"] * sum(r * n + (r * (r + 1) // 2) for r, n in zip(rows, kv))}
    new = 2 * sum(rows) * H * D
    return {"bytes": (2 if case["kind"] == "store" else 1) * (sum(rows) * row + new * size), "flops": new}


def exact(case, seed):
    """From the definitions, in 64 bits, a sequence at a time."""
    s = prepare(case, seed)
    if case["kind"] == "verify":
        return _exact_verify(s)
    rows, kv = _lens(case)
    table, P, D = s["table"].cpu().tolist(), case["page"], case["dim"]
    scales = torch.tensor([2.0 ** (i - 127) for i in range(256)], dtype=torch.float64, device="cuda")       # (a power by pow() may be off by an ulp)
    at = np.concatenate([[0], np.cumsum(rows)])

    def stored(name, seq, a, b):
        """Positions a to b - 1 of a sequence: [position, kv head, dimension] in 64 bits."""
        got = []
        for page in range(a // P, (b - 1) // P + 1):
            x = s[name][table[seq][page]].double()
            if s[name + "_exp"] is not None:
                x = x * scales[s[name + "_exp"][table[seq][page]].long()][..., None]
            got.append(x[:, max(a - page * P, 0):min(b - page * P, P)])
        return torch.cat(got, 1).transpose(0, 1)

    def kept(x):
        """What the pool keeps of new rows."""
        if case["pool"] == "bf16":
            return x.bfloat16().double()
        x = x.double()
        top = x.abs().amax(-1, keepdim=True)
        unit = scales[torch.searchsorted(448.0 * scales, top).clamp_min(LEAST + 127)]     # the first that reaches the largest
        y = (x / unit).view(-1, D)
        binade = torch.frexp(y)[1].clamp_min(-5) - 1                        # of values below 2^-6 that of the subnormals
        step = scales[(binade - 3 + 127).long()]
        return (torch.round(y / step) * step).view_as(x) * unit

    if case["kind"] == "store":
        return kept(s["k_new"]), kept(s["v_new"])
    if case["kind"] == "read":
        return tuple(torch.cat([stored(name, i, 0, r) for i, r in enumerate(rows)]) for name in ("k", "v"))
    out, group = torch.zeros(s["rows"], case["heads"], case["dim"], dtype=torch.float64, device="cuda"), case["heads"] // case["kv_heads"]
    for i, (r, n) in enumerate(zip(rows, kv)):
        k, v = stored("k", i, 0, n + r), stored("v", i, 0, n + r)
        hidden = torch.ones(r, n + r, dtype=torch.bool, device="cuda").triu(n + 1)
        if s["tree"] is not None:
            bits = s["tree"][at[i]:at[i] + r].cpu().tolist()
            hidden[:, n:] = torch.tensor([[not (m >> j) & 1 for j in range(r)] for m in bits], device="cuda")
        for h in range(case["heads"]):
            q = s["q"][at[i]:at[i] + r, h].double()
            x = torch.softmax((q @ k[:, h // group].T * s["scale"]).masked_fill(hidden, -math.inf), -1)
            out[at[i]:at[i] + r, h] = x @ v[:, h // group]
    return out


def _exact_verify(s):
    S, k1, V = s["p"].shape
    u, tokens, n = s["u"].cpu().double().numpy(), s["tokens"].cpu().numpy(), s["n"].cpu().numpy()
    law = lambda t, i, j: t[i, j].cpu().double().numpy()  # noqa: E731
    accepted, out = np.zeros(S, np.int32), np.full((S, k1), -1, np.int32)
    for i in range(S):
        left = None
        for j in range(n[i]):
            p, x = law(s["p"], i, j), tokens[i, j]
            q = law(s["q"], i, j) if s["q"] is not None else np.eye(1, V, x)[0]
            if not u[i, j] * q[x] < p[x]:
                left = np.maximum(p - q, 0.0) if s["q"] is not None else np.where(np.arange(V) == x, 0.0, p)
                left = left if left.sum() > 0 else p
                break
            out[i, j], accepted[i] = x, j + 1
        left = law(s["p"], i, n[i]) if left is None else left
        out[i, accepted[i]] = np.searchsorted(np.cumsum(left), u[i, -1] * np.cumsum(left)[-1], side="right")
    return accepted, out
