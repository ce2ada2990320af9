"""Performance cases of the serving operators: the paged KV cache, attention over it, and beam search.

A case is a dict of plain values.  ``op`` says which operator one pass runs:

  attend   attention of each session's drafted tokens (a tree, a chain, a single token) over its pages
  fork     rows of a page book continue rows of another one: full pages shared, partly filled ones copied
  keep     the accepted path of each session's drafts is moved together, pages behind it are released
  compact  pages in use move to the lowest page numbers
  beam     selection over beams and vocabulary, then reordering of the beams' state tensors

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
        # One token of one short session on a two-stream model: latency counts.
        _case("attend-single-token", "attend", S=1, H=1, G=1, d=64, ctx=333, n=1, page=16, dtype="f16"),
        # One decoding step of a full batch (ragged lengths, some sessions have just begun), grouped heads.
        _case("attend-batch-step", "attend", S=256, H=8, G=4, d=128, ctx=512, n=1, page=32, dtype="bf16"),
        # Verification of token trees of a small batch at prefill length, a key head for each head.
        _case("attend-trees", "attend", S=4, H=32, G=1, d=128, ctx=4096, n=26, page=64, dtype="f16", tree=True, slots_first=True),
        # Verification of a wide tree over one very long context, eight heads a key head.
        _case("attend-tree-longctx", "attend", S=1, H=8, G=8, d=128, ctx=131072, n=64, page=256, dtype="bf16", tree=True, full=True),
        # Beam search on one session of the tiny configuration: four beams fork, one more position each.
        _case("fork-single", "fork", S=1, W=4, L=1, H=1, d=64, ctx=333, page=16, dtype="f16"),
        # A beam step of 64 sessions: prompts shared between the beams, over a third of the rows copied.
        _case("fork-batch", "fork", S=64, W=4, L=8, H=8, d=128, ctx=512, page=32, dtype="f16"),
        # One session accepts a path of its drafted tree, odd page size.
        _case("keep-single", "keep", S=1, L=4, H=8, d=128, ctx=1000, n=13, page=24, dtype="f32"),
        # A batch accepts paths in every layer.
        _case("keep-batch", "keep", S=64, L=32, H=8, d=128, ctx=200, n=26, page=32, dtype="bf16", slots_first=True),
        # A small pool of the tiny configuration gives its upper pages back.
        _case("compact-small", "compact", S=4, L=1, H=1, d=64, ctx=512, page=16, dtype="f16"),
        # A pool of a gigabyte, 40 % of it free.
        _case("compact-pool", "compact", S=64, L=8, H=8, d=128, ctx=512, page=32, dtype="f16", slots_first=True),
        # A beam step of one session.
        _case("beam-single", "beam", S=1, W=4, V=32000, n_out=4, hist=4096, dtype="f16"),
        # A beam step of a batch over the large vocabulary.
        _case("beam-batch", "beam", S=64, W=8, V=128256, n_out=8, hist=8192, dtype="bf16"),
    ]


def _case(name, op, **over):
    base = {"attend": {"S": 1, "H": 8, "G": 1, "d": 128, "ctx": 512, "n": 1, "page": 16, "dtype": "f16", "tree": False, "full": False,
                       "slots_first": False},
            "fork": {"S": 1, "W": 4, "L": 1, "H": 8, "d": 128, "ctx": 512, "page": 16, "dtype": "f16", "slots_first": False},
            "keep": {"S": 1, "L": 1, "H": 8, "d": 128, "ctx": 512, "n": 8, "page": 16, "dtype": "f16", "slots_first": False},
            "compact": {"S": 1, "L": 1, "H": 8, "d": 128, "ctx": 512, "page": 16, "dtype": "f16", "slots_first": False},
            "beam": {"S": 1, "W": 4, "V": 32000, "n_out": 4, "hist": 512, "dtype": "f16"}}[op]
    c = dict(base, op=op)
    c.update(over)
    return dict(c, name=name) if name else c


def _log_int(rng, lo, hi):
    return max(lo, min(hi, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more case: the operators above over the sizes, types and layouts that the listed ones stand for."""
    op = rng.choice(["attend", "attend", "attend", "attend", "fork", "keep", "compact", "beam", "beam"])
    if op == "beam":
        W = _log_int(rng, 1, 32)
        V = _log_int(rng, 256, 131072)
        S = _log_int(rng, 1, max(1, min(128, 60_000_000 // (W * V))))
        n_out = rng.choice([W, W, 2 * W])
        return _case("", op, S=S, W=W, V=V, n_out=n_out, hist=_log_int(rng, 1, min(8192, 8_000_000 // (S * n_out))),
                     dtype=rng.choice(["f16", "bf16", "f32"]))
    page = rng.choice([1, 8, 16, 16, 24, 32, 64, 100, 128, 256])
    c = {"H": rng.choice([1, 2, 3, 4, 8, 8, 32]), "d": rng.choice([32, 64, 128, 128, 128, 256]), "page": page,
         "slots_first": rng.random() < 0.5}
    if op == "attend":
        c["G"] = rng.choice([1, 2, 4, 5, 7, 8, 8, 16])
        c["n"] = rng.choice([1, 1, 1, 2, 5, _log_int(rng, 2, 64), _log_int(rng, 2, 64), _log_int(rng, 64, 300)])
        c["S"] = _log_int(rng, 1, max(1, min(256, 65_000_000 // (c["n"] * c["H"] * c["G"] * c["d"]))))
        most = min(130_000_000 // (c["S"] * c["H"] * c["d"]) - c["n"], 500_000_000 // (c["S"] * c["H"] * c["G"] * c["n"]),
                   65_000_000_000 // (c["S"] * c["H"] * c["G"] * c["n"] * c["d"]), 131072)
        c["ctx"] = _log_int(rng, 1, max(1, most))
        return _case("", op, **dict(c, dtype=rng.choice(["f16", "bf16"]), tree=rng.random() < 0.6, full=rng.random() < 0.3))
    c["dtype"] = rng.choice(["f16", "bf16", "f32"])
    size = 4 if c["dtype"] == "f32" else 2
    c["L"] = _log_int(rng, 1, 32)
    c["S"] = _log_int(rng, 1, 128)
    if op == "fork":
        c["W"] = _log_int(rng, 1, 8)
    if op == "keep":
        c["n"] = _log_int(rng, 1, 64)
    rows = c["S"] * c.get("W", 1)
    position = c["L"] * 2 * c["H"] * c["d"] * size
    room = 900_000_000 // (rows * position) - 2 * page - c.get("n", 0)
    if room < page:                                     # the pool of the largest listed case is the limit
        c["L"], c["H"], c["d"], c["page"], page = 1, 1, 64, 16, 16
        position = 128 * size
        room = 900_000_000 // (rows * position) - 2 * page - c.get("n", 0)
    c["ctx"] = _log_int(rng, 1, max(1, min(4096, room)))
    return _case("", op, **c)


# ---------------------------------------------------------------------------------------------- inputs

def _lens(case):
    """Committed positions of the sessions: the case's own, ragged unless it says ``full``."""
    rng = random.Random("%s %d %d" % (case["op"], case["S"], case["ctx"]))
    S, ctx = case["S"], case["ctx"]
    if case.get("full"):
        return [ctx] * S
    out = [ctx] + [int(ctx * (0.3 + 0.7 * rng.random())) for _ in range(S - 1)]
    return [0 if S > 8 and i % 37 == 5 else x for i, x in enumerate(out)]


def _drafts(case):
    """Drafted tokens of each session: the case's n; sessions that have ended have none."""
    return [0 if case["S"] > 8 and i % 29 == 7 else case["n"] for i in range(case["S"])]


def _pool(case, pages, gen, layers=1):
    """Key and value pages, indexed [L][2][P][H][page][d]; in memory heads or slots come first."""
    H, d, page, dt = case["H"], case["d"], case["page"], _TYPES[case["dtype"]]
    kv = torch.empty((layers, 2, pages, page, H, d) if case["slots_first"] else (layers, 2, pages, H, page, d), dtype=dt, device="cuda")
    kv.normal_(generator=gen)
    if case["op"] == "attend":
        kv[:, 1] *= 0.5
    return kv.transpose(3, 4) if case["slots_first"] else kv


def _plain_pool(kv):
    """The pool's memory as one plain tensor (the layout that it was made in)."""
    return kv if kv.is_contiguous() else kv.transpose(3, 4)


def _cdiv(a, b):
    return -(-a // b)


def _book(rows_pages, max_pages, n_pages):
    """table, len-less parts of a page book from lists of page numbers."""
    table = np.full((len(rows_pages), max_pages), -1, np.int32)
    ref = np.zeros(n_pages, np.int32)
    for r, p in enumerate(rows_pages):
        table[r, :len(p)] = p
        np.add.at(ref, np.asarray(p, np.int64), 1)
    return torch.from_numpy(table).cuda(), torch.from_numpy(ref).cuda()


def _ints(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    rng = np.random.RandomState(seed % (1 << 31))
    return {"attend": _prepare_attend, "fork": _prepare_fork, "keep": _prepare_keep, "compact": _prepare_compact,
            "beam": _prepare_beam}[case["op"]](case, gen, rng)


def _with_calls(state, case):
    """What a program keeps: the pool and the book as the library's objects."""
    if own:
        import paper_2604_15356_b200 as plc
        state["pool"] = plc.PagePool(state["kv"])
        state["book"] = plc.PageBook(state["table"], state["len"], state["ref"])
    return state


def _prepare_attend(case, gen, rng):
    S, page, lens, n = case["S"], case["page"], _lens(case), _drafts(case)
    held = [_cdiv(a + b, page) for a, b in zip(lens, n)]
    n_pages = sum(held) + 3
    order = rng.permutation(n_pages)
    ends = np.cumsum([0] + held)
    table, ref = _book([order[ends[i]:ends[i + 1]] for i in range(S)], max(held) + 1, n_pages)
    begin = np.cumsum([0] + n)
    N, m = int(begin[-1]), case["n"]
    mask = None
    if case["tree"]:                                    # a node's parent is the root or an earlier node, ancestors see-able
        up = torch.from_numpy((rng.rand(S, m) * (np.arange(m) + 1)).astype(np.int64) - 1).cuda()
        seen = torch.zeros(S, m + 1, _cdiv(m, 32) * 32, dtype=torch.bool, device="cuda")   # row m: the root sees nothing
        rows = torch.arange(S, device="cuda")
        for i in range(m):
            seen[:, i] = seen[rows, torch.where(up[:, i] < 0, m, up[:, i])]
            seen[:, i, i] = True
        bits = seen[:, :m].view(S, m, -1, 32).long() << torch.arange(32, device="cuda")
        words = bits.sum(-1)
        words = torch.where(words >= 1 << 31, words - (1 << 32), words).int()
        mask = words[torch.tensor([x > 0 for x in n], device="cuda")].reshape(N, -1).contiguous()
    q = torch.empty(N, case["H"] * case["G"], case["d"], dtype=_TYPES[case["dtype"]], device="cuda").normal_(generator=gen)
    return _with_calls({"op": "attend", "kv": _pool(case, n_pages, gen), "table": table, "len": _ints(lens), "ref": ref, "begin": _ints(begin),
                        "mask": mask, "q": q, "most": max(a + b for a, b in zip(lens, n)), "n": m}, case)


def _prepare_fork(case, gen, rng):
    S, W, page = case["S"], case["W"], case["page"]
    lens = [x for x in _lens(case) for _ in range(W)]
    rows, used = [], 0
    for s in range(S):                                  # the beams of a session share three quarters of its full pages
        full, part = lens[s * W] // page, lens[s * W] % page > 0
        shared = full * 3 // 4
        first = used
        for w in range(W):
            at = first + shared + w * (full - shared + part)
            rows.append(list(range(first, first + shared)) + list(range(at, at + full - shared + part)))
        used = first + shared + W * (full - shared + part)
    n_pages = used + 2 * S * W + 8
    order = rng.permutation(n_pages)
    table, ref = _book([order[np.asarray(r, np.int64)] for r in rows], max(len(r) for r in rows) + 2, n_pages)
    # where the beams of a step come from: mostly a few good parents; now and then a session has ended
    parent = np.repeat(np.arange(S) * W, W) + (rng.rand(S * W) ** 2 * W).astype(np.int64)
    parent[np.repeat((np.arange(S) % 23 == 11), W)] = -1
    return _with_calls({"op": "fork", "kv": _pool(case, n_pages, gen, case["L"]), "table": table, "len": _ints(lens), "ref": ref,
                        "parent": _ints(parent), "room": torch.ones(S * W, dtype=torch.int32, device="cuda")}, case)


def _prepare_keep(case, gen, rng):
    S, page, m, lens = case["S"], case["page"], case["n"], _lens(case)
    held = [_cdiv(x + m, page) for x in lens]
    n_pages = sum(held) + 3
    order = rng.permutation(n_pages)
    ends = np.cumsum([0] + held)
    table, ref = _book([order[ends[i]:ends[i + 1]] for i in range(S)], max(held), n_pages)
    most = min(m, 8)
    path, count = np.zeros((S, most), np.int32), rng.randint(0 if S > 1 else most, most + 1, S)
    for s in range(S):
        path[s, :count[s]] = np.sort(rng.choice(m, count[s], replace=False))
    return _with_calls({"op": "keep", "kv": _pool(case, n_pages, gen, case["L"]), "table": table, "len": _ints(lens), "ref": ref,
                        "path": torch.from_numpy(path).cuda(), "n_path": _ints(count)}, case)


def _prepare_compact(case, gen, rng):
    S, page, lens = case["S"], case["page"], _lens(case)
    held = [_cdiv(x, page) for x in lens]
    n_pages = int(sum(held) / 0.6) + 4
    order = rng.permutation(n_pages)
    ends = np.cumsum([0] + held)
    table, ref = _book([order[ends[i]:ends[i + 1]] for i in range(S)], max(held) + 1, n_pages)
    return _with_calls({"op": "compact", "kv": _pool(case, n_pages, gen, case["L"]), "table": table, "len": _ints(lens), "ref": ref}, case)


def _prepare_beam(case, gen, rng):
    S, W, V, dt = case["S"], case["W"], case["V"], _TYPES[case["dtype"]]
    x = torch.empty(S, W, V, dtype=torch.float32, device="cuda").normal_(generator=gen)
    x = (x * 2.5).to(dt)
    cum = torch.empty(S, W, dtype=torch.float32, device="cuda").normal_(generator=gen).mul_(0.7).sub_(20.0)
    s = torch.arange(S, device="cuda")[:, None]
    w = torch.arange(W, device="cuda")[None]
    if S > 1:
        cum[((s % 5 == 3) & (w > 0)).expand(S, W)] = -math.inf    # sessions at their first step: one beam lives
    done = ((s * 7 + w * 3) % 11 == 4) & (w > 0)                  # beams that have reached the end token
    tokens = torch.randint(0, V, (S * W, case["hist"]), generator=gen, device="cuda", dtype=torch.int32)
    logp2 = -torch.empty(S * W, case["hist"], dtype=torch.float32, device="cuda").exponential_(generator=gen)
    return {"op": "beam", "x": x, "cum": cum, "done": done, "eos": 2, "n_out": case["n_out"], "states": [tokens, logp2]}


# ---------------------------------------------------------------------------------------------- the operators

def run(state):
    return {"attend": _attend, "fork": _fork, "keep": _keep, "compact": _compact, "beam": _beam}[state["op"]](state)


def _unpack_bits(words, n):
    """[..., words] int32 -> [..., n] truth values, bit j of the row."""
    b = (words.long()[..., None] >> torch.arange(32, device=words.device)) & 1
    return b.flatten(-2)[..., :n].bool()


def _attend(st):
    if own:
        out, lse = st["pool"].tree_attention(0, st["book"], st["q"], st["begin"], mask=st["mask"])
        return {"out": out, "lse": lse}
    kv, table, ln, begin, q, n = st["kv"], st["table"], st["len"].long(), st["begin"].long(), st["q"], st["n"]
    dev, (S, _), (_, _, _, H, page, d) = q.device, table.shape, kv.shape
    N, Hq, G = q.shape[0], q.shape[1], q.shape[1] // H
    count = begin[1:] - begin[:-1]
    pos, i = torch.arange(st["most"], device=dev), torch.arange(n, device=dev)
    at, slot = table[:, pos // page].long().clamp(min=0), (pos % page).expand(S, -1)
    held = pos < (ln + count)[:, None]
    k, v = (kv[0, j][at, :, slot].transpose(1, 2).float() for j in (0, 1))                         # [S][H][T][d]
    v = torch.where(held[:, None, :, None], v, 0.0)
    row = (begin[:-1, None] + i).clamp(max=max(N - 1, 0))                                           # [S][n] rows of q
    qs = q[row].float().view(S, n, H, G, d).permute(0, 2, 3, 1, 4).reshape(S, H, G * n, d)
    s = (qs @ k.transpose(2, 3)).view(S, H, G, n, -1) / math.sqrt(d)
    drafted = pos - ln[:, None]                                                                     # [S][T]
    if st["mask"] is None:
        sees = drafted[:, None] <= i[:, None]
    else:
        bits = _unpack_bits(st["mask"], n)[row]                                                     # [S][n][n]
        sees = (drafted < 0)[:, None] | bits.gather(2, drafted.clamp(0, n - 1)[:, None].expand(S, n, -1))
    s = s.masked_fill(~(sees & held[:, None])[:, None, None], -math.inf)
    top = s.amax(-1, keepdim=True)
    p = (s - torch.where(top == -math.inf, 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    o = (p.view(S, H, G * n, -1) @ v).view(S, H, G, n, d) / torch.where(total == 0, 1.0, total)
    lse = (top + total.log())[..., 0]
    whose = torch.repeat_interleave(torch.arange(S, device=dev), count, output_size=N)
    mine = torch.arange(N, device=dev) - begin[whose]
    return {"out": o.permute(0, 3, 1, 2, 4).reshape(S, n, Hq, d)[whose, mine].to(q.dtype),
            "lse": lse.permute(0, 3, 1, 2).reshape(S, n, Hq)[whose, mine]}


def _taken(table, n_pages):
    """How many entries of a table name each page."""
    flat = table.flatten().long()
    return torch.zeros(n_pages + 1, dtype=torch.int32, device=table.device).scatter_add_(
        0, torch.where(flat < 0, n_pages, flat), torch.ones_like(flat, dtype=torch.int32))[:n_pages]


def _fork(st):
    if own:
        b = st["pool"].fork(st["book"], st["parent"], st["room"])
        return {"table": b.table, "len": b.len, "ref": b.ref, "kv": _plain_pool(st["kv"])}
    kv, table, ln, ref = st["kv"], st["table"].long(), st["len"].long(), st["ref"].long()
    n_pages, page, (R, cols) = kv.shape[2], kv.shape[4], table.shape
    live, p = st["parent"] >= 0, st["parent"].long().clamp(min=0)
    s, j = torch.arange(len(p), device=p.device), torch.arange(cols, device=p.device)
    n = torch.where(live, ln[p], 0)
    full, part = n // page, n % page > 0
    last = table[p].gather(1, full[:, None].clamp(max=cols - 1))[:, 0]                              # the partly filled page
    first = torch.full((R + 1,), len(p), device=p.device).scatter_reduce_(0, torch.where(live, p, R), s, "amin")[p] == s
    copy = live & part & ~(first & (ref[last.clamp(min=0)] == 1))
    has, wants = _cdiv(n, page), torch.where(live, _cdiv(n + st["room"], page), 0)
    base = (copy + wants - has).cumsum(0) - (copy + wants - has)
    free = torch.argsort((ref != 0).int(), stable=True)
    fresh = base[:, None] + copy[:, None] + j - has[:, None]
    new = torch.where(j < has[:, None], table[p], free[fresh.clamp(0, n_pages - 1)])
    new = torch.where((j == full[:, None]) & copy[:, None], free[base.clamp(max=n_pages - 1)][:, None], new)
    new = torch.where(j < wants[:, None], new, -1).int()
    which = copy.nonzero()[:, 0]
    src, dst, used = last[which], free[base[which]], (n % page)[which]
    inside = (torch.arange(page, device=p.device) < used[:, None])[:, None, :, None]
    kv[:, :, dst] = torch.where(inside, kv[:, :, src], kv[:, :, dst])
    return {"table": new, "len": n.int(), "ref": st["ref"] - _taken(st["table"], n_pages) + _taken(new, n_pages), "kv": _plain_pool(kv)}


def _keep(st):
    if own:
        b = st["pool"].keep(st["book"], st["path"], st["n_path"])
        return {"table": b.table, "len": b.len, "ref": b.ref, "kv": _plain_pool(st["kv"])}
    kv, table, ln, path, count = st["kv"], st["table"].long(), st["len"].long(), st["path"].long(), st["n_path"].long()
    n_pages, page, cols = kv.shape[2], kv.shape[4], table.shape[1]
    i = torch.arange(path.shape[1], device=path.device)
    s, i = (i < count[:, None]).nonzero(as_tuple=True)
    a, b = ln[s] + path[s, i], ln[s] + i
    kv.permute(2, 4, 0, 1, 3, 5)[table[s, b // page], b % page] = kv.permute(2, 4, 0, 1, 3, 5)[table[s, a // page], a % page]
    n = ln + count
    new = torch.where(torch.arange(cols, device=path.device) < _cdiv(n, page)[:, None], table, -1).int()
    return {"table": new, "len": n.int(), "ref": st["ref"] - _taken(st["table"], n_pages) + _taken(new, n_pages), "kv": _plain_pool(kv)}


def _compact(st):
    if own:
        b, moved = st["pool"].compact(st["book"])
        return {"table": b.table, "len": b.len, "ref": b.ref, "moved": moved, "kv": _plain_pool(st["kv"])}
    kv, table, ref = st["kv"], st["table"].long(), st["ref"]
    ids = torch.arange(len(ref), device=ref.device)
    used = ref > 0
    live = used.sum()
    goes = used & (ids >= live)
    hole = torch.argsort((used | (ids >= live)).int(), stable=True)                                 # the holes come first, rising
    rank = goes.cumsum(0) - 1
    moved = torch.where(used, torch.where(goes, hole[rank.clamp(min=0)], ids), -1)
    src = goes.nonzero()[:, 0]
    kv[:, :, moved[src]] = kv[:, :, src]
    new_ref = torch.zeros(len(ref) + 1, dtype=torch.int32, device=ref.device).scatter_(0, torch.where(used, moved, len(ref)), ref)[:-1]
    return {"table": torch.where(table >= 0, moved[table.clamp(min=0)], -1).int(), "len": st["len"].clone(), "ref": new_ref,
            "moved": moved.int(), "kv": _plain_pool(kv)}


def _beam(st):
    if own:
        import paper_2604_15356_b200 as plc
        score, parent, token = plc.beam_select(st["x"], st["cum"], st["n_out"], done=st["done"], eos=st["eos"])
        tokens, logp2 = plc.beam_reorder(parent, st["states"])
        return {"score": score, "parent": parent, "token": token, "tokens": tokens, "logp2": logp2}
    S, W, V = st["x"].shape
    n, cum = st["n_out"], st["cum"].double()
    x = st["x"].double()
    top = x.amax(-1, keepdim=True)
    x -= top
    f = x.sub_(x.exp().sum(-1, keepdim=True).log_()).add_(cum[..., None])                           # [S][W][V] scores
    f.masked_fill_(st["done"][..., None], -math.inf)
    f[..., st["eos"]] = torch.where(st["done"], cum, f[..., st["eos"]])
    f = f.view(S, W * V).nan_to_num_(nan=-math.inf, posinf=math.inf, neginf=-math.inf)
    best, at = f.topk(n, dim=1)
    # ties at the border go to the lowest index: the r-th candidate that has the last value taken
    last = best[:, -1:]
    tie = (f == last).int().cumsum(1, dtype=torch.int32)
    r = (best == last).int().cumsum(1, dtype=torch.int32)
    at = torch.where(best == last, torch.searchsorted(tie, r.clamp(min=1)), at)
    at, o = at.sort(1)
    best, o = best.gather(1, o).sort(dim=1, descending=True, stable=True)
    at = at.gather(1, o)
    parent = (at // V + torch.arange(S, device=at.device)[:, None] * W).int()
    rows = parent.flatten().long()
    return {"score": best.float(), "parent": parent, "token": (at % V).int(), "tokens": st["states"][0][rows], "logp2": st["states"][1][rows]}


# ---------------------------------------------------------------------------------------------- work and exact values

def work(case):
    size = 4 if case["dtype"] == "f32" else 2
    if case["op"] == "beam":
        rows = case["S"] * case["n_out"]
        logits = case["S"] * case["W"] * case["V"]
        return {"bytes": logits * size + case["S"] * case["W"] * 5 + rows * 12 + 2 * rows * case["hist"] * 8, "flops": 4 * logits}
    lens, page, vec = _lens(case), case["page"], case["H"] * case["d"] * size * 2
    if case["op"] == "attend":
        n, G, m = _drafts(case), case["G"], case["n"]
        sees = (m + 1) / 2 if not case["tree"] else 1 + math.log(m)                                 # drafted positions a row sees
        held, N, Hq = sum(a + b for a, b in zip(lens, n)), sum(n), case["H"] * G
        pairs = sum(b * (a + sees) for a, b in zip(lens, n))
        return {"bytes": held * vec + 2 * N * Hq * case["d"] * size + N * Hq * 4 + (N * _cdiv(m, 32) * 4 if case["tree"] else 0)
                + sum(_cdiv(a + b, page) for a, b in zip(lens, n)) * 4, "flops": 4 * case["d"] * Hq * pairs}
    vec *= case["L"]
    pages = sum(_cdiv(x, page) for x in lens)
    if case["op"] == "fork":                            # what is copied: the children that are not their parent's first
        W = case["W"]
        odds = [((k + 1) / W) ** 0.5 - (k / W) ** 0.5 for k in range(W)]
        copied = sum(x % page for x in lens) * (W - sum(1 - (1 - p) ** W for p in odds))
        return {"bytes": 2 * copied * vec + pages * case["W"] * 4 * 4, "flops": 0}
    if case["op"] == "keep":
        each = min(case["n"], 8) * (1.0 if case["S"] == 1 else 0.5) * case["n"] / (case["n"] + 1.0)  # one of n + 1 stays in place
        return {"bytes": 2 * case["S"] * each * vec + pages * 4 * 4, "flops": 0}
    return {"bytes": 2 * pages * 0.4 * page * vec + pages * 4 * 4, "flops": 0}


def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] == "attend":
        return _exact_attend(st)
    if case["op"] == "beam":
        return _exact_beam(st)
    return None                                         # whole numbers and copies: nothing is rounded


def _exact_attend(st):
    kv, q, begin, lens, table = st["kv"], st["q"], st["begin"].tolist(), st["len"].tolist(), st["table"].long()
    H, page, d = kv.shape[3:]
    N, Hq = q.shape[:2]
    out = torch.zeros(N, Hq, d, dtype=torch.float64, device=q.device)
    lse = torch.zeros(N, Hq, dtype=torch.float64, device=q.device)
    for s in range(table.shape[0]):
        b, e = begin[s], begin[s + 1]
        if b == e:
            continue
        total = lens[s] + e - b
        t = torch.arange(total, device=q.device)
        at = table[s, torch.div(t, page, rounding_mode="floor")]
        hidden = torch.zeros(e - b, total, dtype=torch.bool, device=q.device)
        if st["mask"] is None:
            hidden[:, lens[s]:] = torch.triu(torch.ones(e - b, e - b, dtype=torch.bool, device=q.device), 1)
        else:
            w = st["mask"][b:e].cpu().numpy().view(np.uint8)
            hidden[:, lens[s]:] = torch.from_numpy(np.unpackbits(w, axis=1, bitorder="little")[:, :e - b] == 0).to(q.device)
        for h in range(H):
            K, V = (kv[0, j, at, h, t % page].double() for j in (0, 1))
            mine = q[b:e, h * (Hq // H):(h + 1) * (Hq // H)].double()
            z = torch.matmul(mine.transpose(0, 1), K.t()).mul_(d ** -0.5)                           # [G][n][T]
            z[:, hidden] = -math.inf
            l = torch.logsumexp(z, 2)
            lse[b:e, h * (Hq // H):(h + 1) * (Hq // H)] = l.t()
            out[b:e, h * (Hq // H):(h + 1) * (Hq // H)] = torch.matmul(torch.exp_(z.sub_(l[..., None])), V).transpose(0, 1)
    return {"out": out, "lse": lse}


def _exact_beam(st):
    S, W, V = st["x"].shape
    score = torch.empty(S, st["n_out"], dtype=torch.float64, device=st["x"].device)
    for s in range(S):
        z = torch.log_softmax(st["x"][s].double(), 1) + st["cum"][s].double()[:, None]
        for w in st["done"][s].nonzero()[:, 0].tolist():
            z[w] = -math.inf
            z[w, st["eos"]] = st["cum"][s, w].double()
        z = torch.where(z.isnan(), -math.inf, z).flatten()
        score[s] = torch.topk(z, st["n_out"]).values
    return {"score": score, "parent": None, "token": None, "tokens": None, "logp2": None}
