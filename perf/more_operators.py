"""Performance cases of the decoding loop's operators: rotary positions, the append of keys and values to the paged
cache, accumulation of attention weights, eviction by them, and log probabilities of given tokens.

A case is a dict of plain values.  ``op`` says which operator one pass runs:

  rotary    queries and keys are turned by their positions' angles (or back: the gradient)
  append    new tokens: queries are turned, keys are turned and written into the pages, values are written
  weigh     attention weights that the cached positions receive from the sessions' newest tokens are added up
  evict     sessions give up their lightest positions, head by head; the kept ones move together
  logprobs  log probabilities of given tokens, the entropy of their rows and the likeliest alternatives

With ``own`` false, ``run`` computes the operators in elementary torch operations; with ``own`` true it
calls the library.  Pools are indexed [layer][key or value][page][head][slot][component].
"""
import math
import random

import numpy as np
import torch

own = False

_TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # One token of a two-stream model: latency counts.
        _case("rotary-single", "rotary", N=1, heads=1, kheads=1, d=64, dim=64, far=4096, dtype="f16"),
        # A prefill of 16384 tokens, grouped heads, slices of one projection, a long context.
        _case("rotary-prefill", "rotary", N=16384, heads=32, kheads=8, d=128, dim=128, far=131072, ramp="turns", dtype="bf16", fused=True),
        # One decoding step of a full batch.
        _case("append-step", "append", S=256, n=1, H=8, G=4, d=128, dim=128, ctx=512, page=32, dtype="bf16"),
        # Chunks of prompts, a key head for each head, half of the head turned, neighbours paired.
        _case("append-chunk", "append", S=4, n=1024, H=32, G=1, d=128, dim=64, ctx=4096, page=64, dtype="f16", inter=True, slots_first=True),
        # One token of one short session.
        _case("weigh-single", "weigh", S=1, H=1, G=1, d=64, ctx=333, n=1, page=16, dtype="f16"),
        # A decoding step of a batch at prefill length, ragged, grouped heads.
        _case("weigh-batch", "weigh", S=64, H=8, G=4, d=128, ctx=4096, n=1, page=32, dtype="bf16"),
        # A chunk of a prompt behind a long one: products and exponentials.
        _case("weigh-chunk", "weigh", S=1, H=8, G=4, d=128, ctx=8192, n=2048, page=64, dtype="f16", slots_first=True),
        # One session of a few layers gives up half of its positions.
        _case("evict-single", "evict", S=1, L=4, H=8, d=128, ctx=1000, budget=512, recent=32, page=16, dtype="f16"),
        # Beams that share their prompt's pages, an odd page size, a budget for each row.
        _case("evict-beams", "evict", S=4, W=4, L=4, H=4, d=64, ctx=700, budget=333, recent=50, page=24, dtype="f32", per_row=True),
        # A batch of long sessions over several layers.
        _case("evict-batch", "evict", S=16, L=8, H=8, d=128, ctx=2048, budget=1024, recent=64, page=32, dtype="bf16", slots_first=True),
        # The token of one decoding step.
        _case("logprobs-single", "logprobs", N=1, V=32000, m=1, top=5, dtype="f16"),
        # Scoring of a batch of sequences over the large vocabulary.
        _case("logprobs-batch", "logprobs", N=1024, V=128256, m=1, top=8, dtype="bf16"),
    ]


def _case(name, op, **over):
    base = {"rotary": {"N": 1, "heads": 8, "kheads": 8, "d": 128, "dim": 128, "inter": False, "far": 4096, "ramp": "none", "dtype": "f16", "fused": False,
                       "back": False},
            "append": {"S": 1, "n": 1, "H": 8, "G": 1, "d": 128, "dim": 128, "inter": False, "ctx": 512, "page": 16, "ramp": "none", "dtype": "f16",
                       "tree": False, "slots_first": False},
            "weigh": {"S": 1, "H": 8, "G": 1, "d": 128, "ctx": 512, "n": 1, "page": 16, "dtype": "f16", "picked": False, "slots_first": False},
            "evict": {"S": 1, "W": 1, "L": 1, "H": 8, "d": 128, "ctx": 512, "budget": 256, "recent": 16, "page": 16, "dtype": "f16", "per_row": False,
                      "slots_first": False},
            "logprobs": {"N": 1, "V": 32000, "m": 1, "top": 0, "dtype": "f16"}}[op]
    c = dict(base, op=op)
    c.update(over)
    return dict(c, name=name) if name else c


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(max(lo, hi))))))))


def draw(rng):
    """One more case: the operators above over the sizes, types and layouts that the listed ones stand for."""
    op = rng.choice(["rotary", "rotary", "append", "append", "weigh", "weigh", "weigh", "evict", "evict", "logprobs", "logprobs"])
    if op == "logprobs":
        V = _log_int(rng, 256, 131072)
        return _case("", op, N=_log_int(rng, 1, min(8192, 60_000_000 // V)), V=V, m=rng.choice([1, 1, 1, 2, 7]), top=rng.choice([0, 1, 5, 8, 20, 64]),
                     dtype=rng.choice(["f16", "bf16", "f32"]))
    ramp = rng.choice(["none", "none", "all", "base", "turns", "index"])
    if op == "rotary":
        d = rng.choice([32, 64, 80, 96, 128, 128, 256])
        kheads = rng.choice([1, 2, 3, 8, 8, 32])
        heads = kheads * rng.choice([1, 1, 4, 5, 8])
        return _case("", op, N=_log_int(rng, 1, 80_000_000 // ((heads + kheads) * d * 2)), heads=heads, kheads=kheads, d=d,
                     dim=rng.choice([d, d, d // 2, d // 4]), inter=rng.random() < 0.5, far=_log_int(rng, 16, 1 << 30), ramp=ramp,
                     dtype=rng.choice(["f16", "bf16", "f32"]), fused=rng.random() < 0.5, back=rng.random() < 0.3)
    c = {"H": rng.choice([1, 2, 3, 4, 8, 8, 32]), "d": rng.choice([32, 64, 128, 128, 128, 256]),
         "page": rng.choice([1, 8, 16, 16, 24, 32, 64, 100, 128, 256]), "slots_first": rng.random() < 0.5}
    vec, size = c["H"] * c["d"], 2
    if op in ("append", "evict"):
        c["dtype"] = rng.choice(["f16", "bf16", "f32"])
        size = 4 if c["dtype"] == "f32" else 2
    if op == "append":
        c["G"] = rng.choice([1, 1, 2, 4, 5, 8])
        c["n"] = rng.choice([1, 1, 1, 2, 5, _log_int(rng, 2, 64), _log_int(rng, 64, 1024)])
        c["n"] = min(c["n"], 90_000_000 // size // (vec * (c["G"] + 2)))
        c["S"] = _log_int(rng, 1, max(1, min(256, 90_000_000 // size // (c["n"] * vec * (c["G"] + 2)))))
        c["ctx"] = _log_int(rng, 1, max(1, min(4096, 60_000_000 // (c["S"] * vec) - c["n"])))
        return _case("", op, **dict(c, dim=rng.choice([c["d"], c["d"], c["d"] // 2]), inter=rng.random() < 0.5, ramp=ramp,
                                    tree=c["n"] > 1 and rng.random() < 0.5))
    if op == "weigh":
        c["G"] = rng.choice([1, 2, 4, 5, 7, 8, 16])
        c["n"] = rng.choice([1, 1, 1, 2, 5, _log_int(rng, 2, 64), _log_int(rng, 64, 2048)])
        c["n"] = min(c["n"], 16_000_000 // (vec * c["G"]))
        c["S"] = _log_int(rng, 1, max(1, min(256, 16_000_000 // (c["n"] * vec * c["G"]))))
        most = min(130_000_000 // (c["S"] * vec) - c["n"], 300_000_000 // (c["S"] * c["H"] * c["G"] * c["n"]) - c["n"],
                   60_000_000_000 // (c["S"] * vec * c["G"] * c["n"]) - c["n"], 131072)
        return _case("", op, **dict(c, ctx=_log_int(rng, 1, max(1, most)), dtype=rng.choice(["f16", "bf16"]), picked=rng.random() < 0.4))
    c["L"], c["S"], c["W"] = _log_int(rng, 1, 32), _log_int(rng, 1, 64), rng.choice([1, 1, 1, 2, 4])
    per = c["S"] * c["W"] * c["L"] * vec * 2
    most = 330_000_000 // size // per
    if most < 4 * c["page"] + 64:
        c.update(L=2, H=2, d=64, page=16)
        most = 330_000_000 // size // (c["S"] * c["W"] * c["L"] * 256)
    c["ctx"] = _log_int(rng, 8, min(16384, most - 2 * c["page"]))
    c["budget"] = max(1, int(c["ctx"] * rng.choice([0.1, 0.25, 0.5, 0.5, 0.75, 0.9])))
    c["recent"] = int(c["budget"] * rng.choice([0.0, 0.1, 0.3]))
    return _case("", op, **dict(c, per_row=rng.random() < 0.4))


# ---------------------------------------------------------------------------------------------- inputs

def _ragged(case, count):
    """Lengths of `count` sessions: the case's own first, the others ragged; now and then one that has just begun."""
    rng = random.Random("%s %d %d" % (case["op"], count, case["ctx"]))
    ctx = case["ctx"]
    out = [ctx] + [int(ctx * (0.3 + 0.7 * rng.random())) for _ in range(count - 1)]
    return [0 if count > 8 and i % 37 == 5 else x for i, x in enumerate(out)]


def _news(case):
    """New tokens of each session: the case's n; sessions that have ended have none."""
    return [0 if case["S"] > 8 and i % 29 == 7 else case["n"] for i in range(case["S"])]


def _cdiv(a, b):
    return -(-a // b)


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _pool(case, pages, gen, layers=1):
    """Key and value pages, indexed [L][2][P][H][page][d]; in memory heads or slots come first."""
    H, d, page, dt = case["H"], case["d"], case["page"], _TYPES[case["dtype"]]
    kv = torch.empty((layers, 2, pages, page, H, d) if case["slots_first"] else (layers, 2, pages, H, page, d), dtype=dt, device="cuda")
    kv.normal_(generator=gen)
    return kv.transpose(3, 4) if case["slots_first"] else kv


def _plain_pool(kv):
    """The pool's memory as one plain tensor (the layout that it was made in)."""
    return kv if kv.is_contiguous() else kv.transpose(3, 4)


def _book(rows, cols, n_pages):
    """Table and counts of a page book from lists of page numbers."""
    table = np.full((len(rows), cols), -1, np.int32)
    ref = np.zeros(n_pages, np.int32)
    for r, p in enumerate(rows):
        table[r, :len(p)] = p
        np.add.at(ref, np.asarray(p, np.int64), 1)
    return torch.from_numpy(table).cuda(), torch.from_numpy(ref).cuda()


def _scattered(rng, held, spare):
    """Rows that hold so many pages each, in no order -> lists of page numbers, number of pages."""
    order = rng.permutation(sum(held) + spare)
    ends = np.cumsum([0] + held)
    return [order[ends[i]:ends[i + 1]] for i in range(len(held))], len(order)


_RAMP = {"none": {}, "all": {"factor": 4.0}, "base": {"factor": 4.0}, "turns": {"factor": 8.0, "context": 8192, "slow": 1.0, "fast": 4.0},
         "index": {"factor": 16.0, "context": 4096, "slow": 1.0, "fast": 32.0}}
_BASE = 500000.0


def _rotary(case):
    """What turns: the plain form's frequencies (radians a position, 64 bits) and magnitude, or the library's object."""
    dim, ramp = case["dim"], case["ramp"]
    scale = 0.1 * math.log(16.0) + 1.0 if ramp == "index" else 1.0
    if own:
        import paper_2604_15356_b200 as plc
        return {"rotary": plc.Rotary(dim, base=_BASE, interleaved=case["inter"], ramp=ramp, scale=scale, **_RAMP[ramp])}
    return {"freq": torch.tensor(_frequencies(dim, ramp), dtype=torch.float64, device="cuda"), "dim": dim, "inter": case["inter"], "scale": scale}


def _frequencies(dim, ramp):
    a = _RAMP[ramp]
    base = _BASE * a["factor"] ** (dim / (dim - 2)) if ramp == "base" else _BASE
    out = []
    for i in range(dim // 2):
        f = base ** (-2.0 * i / dim)
        if ramp == "all":
            f /= a["factor"]
        elif ramp in ("turns", "index"):
            if ramp == "turns":                         # how often the pair turns over the trained context
                g = (a["context"] * f / (2 * math.pi) - a["slow"]) / (a["fast"] - a["slow"])
            else:                                       # the pairs' numbers at which that is fast and slow
                lo, hi = (dim * math.log(a["context"] / (2 * math.pi * x)) / (2 * math.log(base)) for x in (a["fast"], a["slow"]))
                lo, hi = max(math.floor(lo), 0), min(math.ceil(hi), dim - 1)
                g = 1 - (i - lo) / max(hi - lo, 0.001)
            g = min(max(g, 0.0), 1.0)
            f = g * f + (1 - g) * f / a["factor"]
        out.append(f)
    return out


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 31))
    st = {"rotary": _prepare_rotary, "append": _prepare_append, "weigh": _prepare_weigh, "evict": _prepare_evict,
          "logprobs": _prepare_logprobs}[case["op"]](case, gen, rng)
    st["op"] = case["op"]
    if own and "kv" in st:                              # what a program keeps: the pool and the book as the library's objects
        import paper_2604_15356_b200 as plc
        st["pool"] = plc.PagePool(st["kv"])
        st["book"] = plc.PageBook(st["table"], st["len"], st["ref"])
    return st


def _normal(gen, dtype, *shape):
    return torch.empty(shape, dtype=_TYPES[dtype], device="cuda").normal_(generator=gen)


def _prepare_rotary(case, gen, rng):
    N, h, k, d = case["N"], case["heads"], case["kheads"], case["d"]
    if case["fused"]:                                   # slices of a projection's output, values behind them
        both = _normal(gen, case["dtype"], N, h + 2 * k, d)
        x = [both[:, :h], both[:, h:h + k]]
    else:
        x = [_normal(gen, case["dtype"], N, h, d), _normal(gen, case["dtype"], N, k, d)]
    first = max(0, case["far"] - N)                     # a run of positions that ends far, or scattered ones
    pos = torch.arange(first, first + N, device="cuda", dtype=torch.int64)
    if N % 2:
        pos = torch.randint(0, case["far"], (N,), generator=gen, device="cuda")
    return dict(_rotary(case), x=x, pos=pos.int(), back=case["back"])


def _prepare_append(case, gen, rng):
    S, H, G, d, page, n = case["S"], case["H"], case["G"], case["d"], case["page"], _news(case)
    lens = _ragged(case, S)
    rows, pages = _scattered(rng, [_cdiv(a + b, page) for a, b in zip(lens, n)], 3)
    table, ref = _book(rows, max(len(r) for r in rows) + 1, pages)
    begin = np.cumsum([0] + n)
    N = int(begin[-1])
    both = _normal(gen, case["dtype"], N, H * (G + 2), d)
    pos = None
    if case["tree"]:                                    # drafted trees: a token's position is its depth behind the session
        pos = _ints([lens[s] + int(x) for s in range(S) for x in np.minimum(rng.randint(0, 6, n[s]), np.arange(n[s]))])
    whose = np.repeat(np.arange(S), n)
    return dict(_rotary(case), kv=_pool(case, pages, gen), table=table, len=_ints(lens), ref=ref, begin=_ints(begin), q=both[:, :H * G],
                k=both[:, H * G:H * G + H], v=both[:, H * G + H:], pos=pos, whose=torch.from_numpy(whose).cuda())


def _prepare_weigh(case, gen, rng):
    S, H, G, d, page, n = case["S"], case["H"], case["G"], case["d"], case["page"], _news(case)
    lens = [a + b for a, b in zip(_ragged(case, S), n)]
    rows, pages = _scattered(rng, [_cdiv(x, page) for x in lens], 3)
    table, ref = _book(rows, max(max(len(r) for r in rows), 1) + 1, pages)
    begin = np.cumsum([0] + n)
    M = int(begin[-1])
    N = M + M // 2 + 1 if case["picked"] else M         # of the drafted rows some have been accepted
    picked = torch.from_numpy(np.sort(rng.permutation(N)[:M]).astype(np.int32)).cuda() if case["picked"] else None
    kv, q = _pool(case, pages, gen), _normal(gen, case["dtype"], N, H * G, d)
    cap = max(lens) + 5
    w = torch.empty(S, 1, H, cap, device="cuda").exponential_(generator=gen)
    st = {"kv": kv, "table": table, "len": _ints(lens), "ref": ref, "begin": _ints(begin), "q": q, "rows": picked, "weight": w, "decay": 0.875,
          "lens": lens, "news": n, "lse": torch.zeros(N, H * G, device="cuda")}
    at = torch.arange(N, device="cuda") if picked is None else picked.long()
    for s in range(S):                                  # the log-sum-exp that the attention before has left
        if n[s]:
            mine = at[begin[s]:begin[s + 1]]
            for h in range(H):
                z = _scores(st, s, h, q[mine, h * G:(h + 1) * G].float(), torch.float32)
                st["lse"][mine, h * G:(h + 1) * G] = torch.logsumexp(z, -1)
    return st


def _scores(st, s, h, q, dtype):
    """Scores [n][G][T] of one session's newest rows q [n][G][d] and one head, -inf where a row does not see."""
    kv, T, n = st["kv"], st["lens"][s], st["news"][s]
    t = torch.arange(T, device="cuda")
    K = kv[0, 0, st["table"][s].long()[t // kv.shape[4]], h, t % kv.shape[4]].to(dtype)
    z = torch.matmul(q, K.t()) / math.sqrt(q.shape[-1])
    return z.masked_fill_((t > (T - n + torch.arange(n, device="cuda"))[:, None])[:, None], -math.inf)


def _prepare_evict(case, gen, rng):
    S, W, L, H, page = case["S"], case["W"], case["L"], case["H"], case["page"]
    lens = [x for x in _ragged(case, S) for _ in range(W)]
    rows, used = [], 0
    for s in range(S):                                  # the beams of a session share three quarters of its full pages
        n = lens[s * W]
        shared = n // page * 3 // 4 if W > 1 else 0
        each = _cdiv(n, page) - shared
        for w in range(W):
            at = used + shared + w * each
            rows.append(np.array(list(range(used, used + shared)) + list(range(at, at + each)), np.int64))
        used += shared + W * each
    R = S * W
    spare = (R * _cdiv(case["budget"], page) if W > 1 else 0) + 3
    order = rng.permutation(used + spare)
    table, ref = _book([order[r] for r in rows], max(len(r) for r in rows) + 1, used + spare)
    cap = max(lens) + 3
    w = torch.empty(R, L, H, cap, device="cuda").exponential_(generator=gen).pow_(3)        # few heavy ones, and the first positions
    w[..., :4] *= 500.0
    w[w < 1e-3] = 0.0                                   # weights that have underflowed are alike
    budget = [case["budget"]] * R
    if case["per_row"]:
        budget = [-1 if R > 8 and i % 13 == 3 else int(case["budget"] * (0.3 + 0.7 * rng.rand())) for i in range(R)]
    return {"kv": _pool(case, used + spare, gen, L), "table": table, "len": _ints(lens), "ref": ref, "weight": w,
            "budget": _ints(budget) if case["per_row"] else case["budget"], "recent": case["recent"],
            "most": max([b if 0 <= b < n else n for b, n in zip(budget, lens)] + [1])}


def _prepare_logprobs(case, gen, rng):
    N, V, m = case["N"], case["V"], case["m"]
    x = torch.empty(N, V, dtype=torch.float32, device="cuda").normal_(generator=gen).mul_(2.5)
    tokens = torch.randint(0, V, (N, m), generator=gen, device="cuda", dtype=torch.int32)
    likely = torch.rand(N, m, generator=gen, device="cuda") < 0.7   # most tokens are likely ones
    tokens = torch.where(likely, x.argmax(1, keepdim=True).int(), tokens)
    if N > 8:
        tokens[3::17] = -1                              # padding
    return {"x": x.to(_TYPES[case["dtype"]]), "tokens": tokens, "top": case["top"]}


# ---------------------------------------------------------------------------------------------- the operators

def run(state):
    return {"rotary": _run_rotary, "append": _append, "weigh": _weigh, "evict": _evict, "logprobs": _logprobs}[state["op"]](state)


def _turned(st, x, pos, back=False):
    """x [N][heads][d] turned by pos [N], in 32 bits; the angles are products of 64 bits."""
    angle = pos.double()[:, None] * st["freq"]
    angle = torch.remainder(angle, 2 * math.pi)
    cos, sin = (angle.cos() * st["scale"]).float()[:, None], (angle.sin() * st["scale"]).float()[:, None]
    if back:
        sin = -sin
    dim, y = st["dim"], x.float()
    a, b = (y[..., 0:dim:2], y[..., 1:dim:2]) if st["inter"] else (y[..., :dim // 2], y[..., dim // 2:dim])
    a, b = a * cos - b * sin, b * cos + a * sin
    part = torch.stack((a, b), -1).flatten(-2) if st["inter"] else torch.cat((a, b), -1)
    return torch.cat((part, y[..., dim:]), -1).to(x.dtype)


def _run_rotary(st):
    if own:
        q, k = st["rotary"].apply((st["x"][0], st["x"][1]), st["pos"], back=st["back"])
        return {"q": q, "k": k}
    return {"q": _turned(st, st["x"][0], st["pos"], st["back"]), "k": _turned(st, st["x"][1], st["pos"], st["back"])}


def _append(st):
    if own:
        q = st["pool"].append(0, st["book"], st["q"], st["k"], st["v"], st["begin"], rotary=st["rotary"], pos=st["pos"])
        return {"q": q, "kv": _plain_pool(st["kv"])}
    kv, whose = st["kv"], st["whose"]
    page = kv.shape[4]
    stands = st["len"][whose] + torch.arange(len(whose), device=whose.device, dtype=torch.int32) - st["begin"][whose]
    pos = stands if st["pos"] is None else st["pos"]
    at, slot = st["table"][whose, stands.long() // page].long(), stands.long() % page
    kv[0, 0, at, :, slot] = _turned(st, st["k"], pos)
    kv[0, 1, at, :, slot] = st["v"]
    return {"q": _turned(st, st["q"], pos), "kv": _plain_pool(kv)}


def _weigh(st):
    if own:
        return {"weight": st["pool"].attention_weights(0, st["book"], st["q"], st["lse"], st["begin"], st["weight"], rows=st["rows"], decay=st["decay"])}
    kv, table, w, lens, n = st["kv"], st["table"].long(), st["weight"], st["lens"], st["news"]
    H, page, d = kv.shape[3:]
    (S, _), G, cap, dev = table.shape, st["q"].shape[1] // H, w.shape[3], w.device
    at = torch.arange(st["q"].shape[0], device=dev) if st["rows"] is None else st["rows"].long()
    t = torch.arange(cap, device=dev)
    ln, most = st["len"].long(), max(n)
    if most == 0:
        return {"weight": w}
    count = st["begin"].long().diff()
    mine = at[(st["begin"].long()[:-1, None] + torch.arange(most, device=dev)).clamp(max=len(at) - 1)]          # [S][n]
    there = torch.arange(most, device=dev) < count[:, None]
    for s0, s1 in _runs(S, most * H * G * cap):
        page_at = table[s0:s1, (t // page).clamp(max=table.shape[1] - 1)].clamp(min=0)
        k = kv[0, 0][page_at, :, (t % page).expand(s1 - s0, -1)].permute(0, 2, 3, 1).float()                    # [s][H][d][T]
        r = mine[s0:s1]
        q = st["q"][r].float().unflatten(2, (H, G)).permute(0, 2, 3, 1, 4).reshape(s1 - s0, H, G * most, d)
        z = (q @ k).unflatten(2, (G, most)).div_(math.sqrt(d))
        z -= st["lse"][r].unflatten(2, (H, G)).permute(0, 2, 3, 1)[..., None]
        sees = (t <= ((ln - count)[s0:s1, None] + torch.arange(most, device=dev))[..., None]) & there[s0:s1, :, None]
        z = z.exp_().masked_fill_(~sees[:, None, None], 0.0).sum((2, 3))                                        # [s][H][T]
        old = torch.where(t < (ln - count)[s0:s1, None], w[s0:s1, 0].transpose(0, 1), 0.0).transpose(0, 1)
        now = (t < ln[s0:s1, None]) & (count[s0:s1, None] > 0)
        w[s0:s1, 0] = torch.where(now[:, None], old * st["decay"] + z, w[s0:s1, 0])
    return {"weight": w}


def _runs(S, each):
    """Sessions in runs whose scores take a few gigabytes."""
    step = max(1, 1_000_000_000 // max(each, 1))
    return [(s, min(S, s + step)) for s in range(0, S, step)]


def _taken(table, n_pages):
    """How many entries of a table name each page."""
    flat = table.flatten().long()
    return torch.zeros(n_pages + 1, dtype=torch.int32, device=table.device).scatter_add_(
        0, torch.where(flat < 0, n_pages, flat), torch.ones_like(flat, dtype=torch.int32))[:n_pages]


def _evict(st):
    if own:
        b, w = st["pool"].evict(st["book"], st["weight"], st["budget"], recent=st["recent"])
        return {"table": b.table, "len": b.len, "ref": b.ref, "weight": w, "kv": _plain_pool(st["kv"])}
    kv, table, ln, ref, w, most = st["kv"], st["table"].long(), st["len"].long(), st["ref"], st["weight"], st["most"]
    (L, _, P, H, page, d), (R, cols), cap, dev = kv.shape, table.shape, w.shape[3], w.device
    budget = st["budget"].long() if torch.is_tensor(st["budget"]) else torch.full((R,), st["budget"], device=dev)
    goes = (budget >= 0) & (ln > budget)
    n = torch.where(goes, budget, ln)                                                               # the new lengths
    t, i = torch.arange(cap, device=dev), torch.arange(most, device=dev)
    recent = t >= (ln - n.clamp(max=st["recent"]))[:, None]
    f = torch.where((t < ln[:, None])[:, None, None], torch.where(recent[:, None, None], math.inf, w), -math.inf)
    kept = torch.sort(f, dim=-1, descending=True, stable=True).indices[..., :most]                  # ties: the lower position
    here = (i < n[:, None])[:, None, None]
    kept = torch.where(here, kept, cap).sort(-1).values                                             # [R][L][H][most], rising
    weight = torch.zeros_like(w)
    weight[..., :most] = torch.where(here, w.gather(3, kept.clamp(max=cap - 1)), 0.0)
    j = torch.arange(cols, device=dev)
    held = goes[:, None] & (j < _cdiv(n, page)[:, None])
    fresh = held & (ref[table.clamp(min=0)] != 1)
    free = torch.argsort((ref != 0).int(), stable=True)
    rank = (fresh.flatten().cumsum(0) - 1).view(R, cols)
    new = torch.where(fresh, free[rank.clamp(0, P - 1)], table)
    new = torch.where(goes[:, None] & ~held, -1, new)
    r = goes.nonzero()[:, 0]
    src, l, h = kept[r].clamp(max=cols * page - 1), torch.arange(L, device=dev)[:, None, None], torch.arange(H, device=dev)[:, None]
    a = table[r[:, None, None, None], src // page]
    b = new[r][:, (i // page)][:, None, None].expand_as(a)
    x = kv.permute(0, 2, 3, 4, 1, 5)[l, a, h, src % page]                        # [r][L][H][most][2][d]
    at = here[r].expand_as(a)
    full = [y.expand_as(a)[at] for y in (l, b, h, i % page)]
    kv.permute(0, 2, 3, 4, 1, 5)[full[0], full[1], full[2], full[3]] = x[at]
    return {"table": new.int(), "len": n.int(), "ref": ref - _taken(st["table"], P) + _taken(new, P), "weight": weight, "kv": _plain_pool(kv)}


def _logprobs(st):
    if own:
        import paper_2604_15356_b200 as plc
        logp, entropy, top_logp, top_token = plc.token_logprobs(st["x"], st["tokens"], n_top=st["top"])
        return {"logp": logp, "entropy": entropy, "top_logp": top_logp, "top_token": top_token}
    x, tokens, n = st["x"].float(), st["tokens"].long(), st["top"]
    V = x.shape[1]
    there = tokens >= 0
    picked = x.gather(1, tokens.clamp(min=0))
    top = x.amax(1, keepdim=True)
    y = x - top
    e = y.exp()
    total = e.sum(1, keepdim=True)
    log_total = total.log()
    entropy = log_total[:, 0] - (e * y).sum(1) / total[:, 0]
    out = {"logp": torch.where(there, picked - top - log_total, 0.0), "entropy": entropy}
    bits = (x + 0.0).view(torch.int32)                                                              # order of the values, then of the tokens
    key = (torch.where(bits < 0, bits ^ 0x7fffffff, bits).long() << 32) + (V - 1 - torch.arange(V, device=x.device))
    token = V - 1 - (key.topk(n, dim=1).values & 0xffffffff)
    return dict(out, top_logp=x.gather(1, token) - top - log_total, top_token=token.int())


# ---------------------------------------------------------------------------------------------- work and exact values

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    op, d = case["op"], case.get("d")
    if op == "rotary":
        x = case["N"] * (case["heads"] + case["kheads"])
        return {"bytes": 2 * x * d * size + case["N"] * 4, "flops": 3 * x * case["dim"]}
    if op == "logprobs":
        x = case["N"] * case["V"]
        return {"bytes": x * size + case["N"] * (case["m"] * 8 + 4 + case["top"] * 8), "flops": 4 * x}
    H, page = case["H"], case["page"]
    if op == "append":
        N, heads = sum(_news(case)), H * (case["G"] + 1)
        return {"bytes": N * 2 * (heads + H) * d * size + N * 8 + case["S"] * 8, "flops": 3 * N * heads * case["dim"]}
    if op == "weigh":
        G, n = case["G"], _news(case)
        lens = [(a + b, b) for a, b in zip(_ragged(case, case["S"]), n)]
        pairs = sum(b * (a - (b - 1) / 2) for a, b in lens)
        held = sum(a for a, b in lens if b)
        return {"bytes": held * H * (d * size + 8) + sum(n) * H * G * (d * size + 4) + sum(_cdiv(a, page) for a, b in lens if b) * 4,
                "flops": (2 * d + 2) * H * G * pairs}
    lens = [x for x in _ragged(case, case["S"]) for _ in range(case["W"])]
    share = 0.65 if case["per_row"] else 1.0            # the mean of the rows' budgets
    kept = sum(min(x, int(case["budget"] * share)) for x in lens if x > case["budget"] * share)
    lanes = case["L"] * H
    return {"bytes": lanes * (2 * 2 * kept * d * size + sum(lens) * 4 + kept * 4), "flops": 0}


def exact(case, seed):
    if case["op"] == "evict":
        return None                                     # whole numbers and copies: nothing is rounded
    st = prepare(case, seed)
    return {"rotary": _exact_rotary, "append": _exact_append, "weigh": _exact_weigh, "logprobs": _exact_logprobs}[case["op"]](case, st)


def _exact_turn(case, x, pos, back=False):
    """Each pair as a complex number times s exp(i angle)."""
    f = torch.tensor(_frequencies(case["dim"], case["ramp"]), dtype=torch.float64, device=x.device)
    s = 0.1 * math.log(16.0) + 1.0 if case["ramp"] == "index" else 1.0
    turn = torch.polar(torch.full_like(f, s).expand(len(pos), -1), torch.outer(pos.double(), f * (-1.0 if back else 1.0)))[:, None]
    y, dim = x.double().clone(), case["dim"]
    if case["inter"]:
        y[..., :dim] = torch.view_as_real(torch.view_as_complex(y[..., :dim].unflatten(-1, (dim // 2, 2)).contiguous()) * turn).flatten(-2)
    else:
        z = torch.complex(y[..., :dim // 2].contiguous(), y[..., dim // 2:dim].contiguous()) * turn
        y[..., :dim // 2], y[..., dim // 2:dim] = z.real, z.imag
    return y


def _exact_rotary(case, st):
    return {"q": _exact_turn(case, st["x"][0], st["pos"], case["back"]), "k": _exact_turn(case, st["x"][1], st["pos"], case["back"])}


def _exact_append(case, st):
    kv, begin, lens = st["kv"], st["begin"].tolist(), st["len"].tolist()
    page = kv.shape[4]
    stands = torch.tensor([lens[s] + i for s in range(len(lens)) for i in range(begin[s + 1] - begin[s])], dtype=torch.int64, device="cuda")
    rows = torch.tensor([s for s in range(len(lens)) for _ in range(begin[s + 1] - begin[s])], dtype=torch.int64, device="cuda")
    pos = stands if st["pos"] is None else st["pos"]
    out = kv.double()
    where = st["table"].long()[rows, torch.div(stands, page, rounding_mode="floor")]
    out[0, 0, where, :, stands % page] = _exact_turn(case, st["k"], pos)
    out[0, 1, where, :, stands % page] = st["v"].double()
    return {"q": _exact_turn(case, st["q"], pos), "kv": _plain_pool(out)}


def _exact_weigh(case, st):
    H, G, begin = case["H"], case["G"], st["begin"].tolist()
    out = st["weight"].double()
    at = st["rows"].long() if st["rows"] is not None else torch.arange(st["q"].shape[0], device="cuda")
    for s in range(case["S"]):
        T, n = st["lens"][s], st["news"][s]
        if not n:
            continue
        mine = at[begin[s]:begin[s + 1]]
        out[s, 0, :, :T - n] *= st["decay"]
        out[s, 0, :, T - n:T] = 0.0
        for h in range(H):
            z = _scores(st, s, h, st["q"][mine, h * G:(h + 1) * G].double(), torch.float64)
            z -= st["lse"][mine, h * G:(h + 1) * G].double()[..., None]
            out[s, 0, h, :T] += z.exp_().sum((0, 1))
    return {"weight": out}


def _exact_logprobs(case, st):
    N, n = case["N"], st["top"]
    out = {"logp": torch.empty(N, case["m"], dtype=torch.float64, device="cuda"), "entropy": torch.empty(N, dtype=torch.float64, device="cuda"),
           "top_logp": torch.empty(N, n, dtype=torch.float64, device="cuda"), "top_token": None}
    for r in range(0, N, 256):
        z = torch.log_softmax(st["x"][r:r + 256].double(), 1)
        tok = st["tokens"][r:r + 256].long()
        out["logp"][r:r + 256] = torch.where(tok < 0, 0.0, z.gather(1, tok.clamp(min=0)))
        out["entropy"][r:r + 256] = -(z.exp() * z).sum(1)
        out["top_logp"][r:r + 256] = z.topk(n, dim=1).values
    return out
