"""A search over the paged cache on the host, from its definitions, in numpy: the position rotation in
binary32 (as the library's interface names each rounding), a beam step in 64 bits, and the reordering."""
import numpy as np


def turn(x, cos_sin, rot, pairs):
    """Rows [rows][heads][D] float32 by their rows [rows][rot] of the table; every operation rounded by itself."""
    x = np.asarray(x, np.float32)
    j = np.arange(rot // 2)
    a, b = (2 * j, 2 * j + 1) if pairs else (j, j + rot // 2)
    c, s = cos_sin[:, None, :rot // 2], cos_sin[:, None, rot // 2:]
    out = x.copy()
    with np.errstate(all="ignore"):
        out[..., a] = x[..., a] * c - x[..., b] * s
        out[..., b] = x[..., b] * c + x[..., a] * s
    assert out.dtype == np.float32
    return out


def table_of(rows, rot, base=1e4):
    angle = np.arange(rows)[:, None] * base ** (-np.arange(rot // 2) * 2.0 / rot)
    return np.concatenate([np.cos(angle), np.sin(angle)], 1).astype(np.float32)


def select(logits, scores, k, done=None, end=0):
    """parent, token, score [groups][k] (64 bits).  logits [groups * beams][vocab], scores [groups][beams]."""
    logits, scores = np.asarray(logits, np.float64), np.asarray(scores, np.float64)
    groups, beams = scores.shape
    parent, token = np.full((groups, k), -1), np.full((groups, k), -1)
    best = np.full((groups, k), -np.inf)
    for g in range(groups):
        rows, tokens, values, order = [], [], [], []
        for b in range(beams):
            r, s = g * beams + b, scores[g, b]
            if not np.isfinite(s):
                continue
            if done is not None and done[r]:
                rows.append([r]), tokens.append([end]), values.append([s]), order.append([0.0])
                continue
            x = np.where(logits[r] < np.inf, logits[r], -np.inf)  # (a NaN is not)
            t = np.flatnonzero(x > -np.inf)
            if not len(t):
                continue
            # the k best and the ties of the last are enough
            top = x[t].max()
            norm = np.log(np.exp(x[t] - top).sum())
            if len(t) > k:
                t = t[x[t] >= np.partition(x[t], len(t) - k)[len(t) - k]]
            rows.append(np.full(len(t), r)), tokens.append(t), values.append((x[t] - top) - norm + s), order.append(x[t])
        if not rows:
            continue
        rows, tokens, values, order = [np.concatenate(z) for z in (rows, tokens, values, order)]
        # (equal scores of one row are told apart by its logits: 64 bits can hide what these say)
        take = np.lexsort((tokens, -order, rows, -values))[:k]
        n = len(take)
        parent[g, :n], token[g, :n], best[g, :n] = rows[take], tokens[take], values[take]
    return parent, token, best


def reorder(plain, seqs, parent):
    """The sequences of a Plain cache, as semkv_kv4_reorder says."""
    n, top = len(parent), len(plain.length)
    seqs = list(range(n)) if seqs is None else [int(s) for s in seqs]
    inside = [0 <= s < top for s in seqs]
    old = [(plain.table[s].copy(), int(plain.length[s])) if ok else None for s, ok in zip(seqs, inside)]
    for i, (s, p) in enumerate(zip(seqs, parent)):
        if not inside[i] or s in seqs[:i] or not -1 <= p < n or (p >= 0 and not inside[p]):
            continue
        table, tokens = old[p] if p >= 0 else (None, 0)
        for page in old[i][0][:plain.used(old[i][1])]:
            plain.refs[page] -= 1
        for j in range(plain.used(tokens)):
            plain.table[s, j] = table[j]
            plain.refs[table[j]] += 1
        plain.length[s] = tokens
