"""Oracle of the paged cache, the attention over it and beam search: literal definitions in numpy binary64 and Python
integers, one row, page and continuation after the other.  Test infrastructure only; shares nothing with the kernels."""
import math

import numpy as np

CAPACITY, RANGE = 1, 32


def _pages(n, page_pos):
    return -(-n // page_pos)


def fork(table, length, ref, parent, room, page_pos):
    """-> table, length, ref of the new book, copies [(source page, fresh page, slots)], status bits."""
    rows_in, cols = table.shape
    n_pages = len(ref)
    rows, bits = [], 0
    for s, f in enumerate(parent):
        more = 0 if room is None else int(room[s])
        if f == -1:
            rows.append(None)
        elif not 0 <= f < rows_in or not 0 <= length[f] <= cols * page_pos or more < 0:
            bits |= RANGE
            rows.append(None)
        else:
            rows.append((int(f), int(length[f]), more))
    new_ref = ref.astype(np.int64).copy()
    free = [p for p in range(n_pages) if ref[p] == 0]
    new = np.full((len(rows), cols), -1, np.int32)
    new_len = np.zeros(len(rows), np.int32)
    copies, continued, short = [], set(), False
    for p in table.flatten():                                   # the old book's names go ...
        if 0 <= p < n_pages:
            new_ref[p] -= 1
        elif p != -1:
            bits |= RANGE
    for s, r in enumerate(rows):                                # ... and the new one's come
        if r is None:
            continue
        f, n, more = r
        if _pages(n + more, page_pos) > cols:
            short = True
            continue
        new_len[s] = n
        for j in range(n // page_pos):
            new[s, j] = table[f, j]
        j = n // page_pos
        if n % page_pos:
            p = table[f, j]
            if 0 <= p < n_pages and (f in continued or ref[p] != 1):
                if not free:
                    short = True
                    continue
                new[s, j] = free.pop(0)
                copies.append((int(p), int(new[s, j]), n % page_pos))
            else:
                new[s, j] = p
            j += 1
        continued.add(f)
        while j < _pages(n + more, page_pos):
            if not free:
                short = True
                break
            new[s, j] = free.pop(0)
            j += 1
        for j in range(cols):
            if new[s, j] != -1 and not 0 <= new[s, j] < n_pages:
                bits |= RANGE
                new[s, j] = -1
            elif new[s, j] != -1:
                new_ref[new[s, j]] += 1
    if short:
        return np.full_like(new, -1), np.zeros_like(new_len), ref.copy(), [], bits | CAPACITY
    return new, new_len, new_ref.astype(np.int32), copies, bits


def keep(table, length, ref, path, n_path, page_pos):
    """-> table, length, ref, moves [(row, from position, to position)], status bits."""
    rows, cols = table.shape
    n_pages = len(ref)
    new, new_len, new_ref, moves, bits = table.copy(), length.copy(), ref.copy(), [], 0
    for s in range(rows):
        n, base = int(n_path[s]), int(length[s])
        ok = 0 <= n <= path.shape[1] and 0 <= base <= cols * page_pos
        mine = []
        for i in range(n if ok else 0):
            at = int(path[s, i])
            if at < 0 or (i and at <= path[s, i - 1]) or base + at >= cols * page_pos:
                ok = False
                break
            a, b = table[s, (base + at) // page_pos], table[s, (base + i) // page_pos]
            if not (0 <= a < n_pages and 0 <= b < n_pages) or (at != i and ref[b] != 1):
                ok = False
                break
            if at != i:
                mine.append((s, base + at, base + i))
        if not ok:
            bits |= RANGE
            continue
        moves += mine
        new_len[s] = base + n
        for j in range(_pages(base + n, page_pos), cols):
            if 0 <= table[s, j] < n_pages:
                new_ref[table[s, j]] -= 1
            elif table[s, j] != -1:
                bits |= RANGE
            new[s, j] = -1
    return new, new_len, new_ref, moves, bits


def compact(table, ref):
    """-> table, ref, moved."""
    live = int((ref > 0).sum())
    holes = [p for p in range(live) if ref[p] == 0]
    moved = np.where(ref > 0, np.arange(len(ref)), -1).astype(np.int32)
    new_ref = ref.copy()
    for p in range(live, len(ref)):
        if ref[p] > 0:
            moved[p] = holes.pop(0)
            new_ref[moved[p]], new_ref[p] = ref[p], 0
    new = np.full_like(table, -1)
    for i, p in np.ndenumerate(table):
        if p >= 0:
            new[i] = moved[p]
    return new, new_ref, moved


def attention(q, k_of, v_of, length, begin, mask, scale):
    """q [N][Hq][d]; k_of / v_of (session, kv head, position) -> vector (None: no page); mask [N][bits] of truth values or
    None -> out, lse, and per output the sum of |p v| and per (row, head) the largest sum of |q k| scale."""
    N, Hq, d = q.shape
    out, lse = np.zeros((N, Hq, d)), np.full((N, Hq), -math.inf)
    mag, big = np.zeros((N, Hq, d)), np.zeros((N, Hq))
    H = k_of.heads
    for s in range(len(begin) - 1):
        for row in range(begin[s], begin[s + 1]):
            i = row - begin[s]
            sees = [t for t in range(length[s])]
            for j in range(begin[s + 1] - begin[s]):
                if j <= i if mask is None else (j < mask.shape[1] and mask[row, j]):
                    sees.append(length[s] + j)
            for h in range(Hq):
                g = h // (Hq // H)
                t_ = [t for t in sees if k_of(s, g, t) is not None]
                if not t_:
                    continue
                K = np.stack([k_of(s, g, t) for t in t_]).astype(np.float64)
                V = np.stack([v_of(s, g, t) for t in t_]).astype(np.float64)
                x = K @ q[row, h].astype(np.float64) * scale
                m = x.max()
                p = np.exp(x - m)
                lse[row, h] = m + math.log(p.sum())
                p /= p.sum()
                out[row, h] = p @ V
                mag[row, h] = p @ np.abs(V)
                big[row, h] = (np.abs(K) @ np.abs(q[row, h].astype(np.float64))).max() * scale
    return out, lse, mag, big


def beam_select(logits, score, n_out, done=None, eos=-1):
    """logits [S][W][V], score [S][W] -> score, parent, token [S][n_out]."""
    S, W, V = logits.shape
    out = np.full((S, n_out), -math.inf)
    parent, token = np.full((S, n_out), -1, np.int32), np.full((S, n_out), -1, np.int32)
    for s in range(S):
        c = []
        for w in range(W):
            own = float(score[s, w])
            if not math.isfinite(own):
                continue
            if done is not None and done[s, w]:
                c.append((-own, w, eos))
                continue
            x = logits[s, w].astype(np.float64)
            if np.isnan(x).any() or x.max() == math.inf or x.max() == -math.inf:
                continue
            rest = own - math.log(np.exp(x - x.max()).sum())     # the maximum stays with x: at -3e38 it would swallow all else
            order = np.lexsort((np.arange(V), -x))[:n_out]
            c += [(-((x[v] - x.max()) + rest), w, int(v)) for v in order if x[v] > -math.inf]
        for i, (f, w, v) in enumerate(sorted(c)[:n_out]):
            out[s, i], parent[s, i], token[s, i] = -f, s * W + w, v
    return out, parent, token
