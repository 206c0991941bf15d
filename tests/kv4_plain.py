"""The paged 4-bit cache on the host: its format, attention and page operations from their
definitions, in numpy (64 bits where a number is rounded, binary32 where the format names it)."""
import numpy as np
import torch

LEVELS = np.array([0, 0.5, 1, 1.5, 2, 3, 4, 6])
GRID = np.concatenate([LEVELS, -LEVELS])


def e4m3_value(b):
    b = np.asarray(b, np.uint8).astype(np.int64)
    e, m = b >> 3 & 15, b & 7
    v = np.where(e > 0, np.exp2(e - 7.0) * (1 + m / 8), m * 2.0 ** -9)
    return np.where(b & 0x7F == 0x7F, np.nan, v) * np.where(b & 128, -1, 1)


E4M3 = e4m3_value(np.arange(127))  # the numbers from 0 up, 448 last


def nearest(grid, x):
    """Index of the nearest of an ascending grid, ties to the even index (e4m3 and e2m1 codes count
    up with their values, so an even index is an even significand); past the end: the last."""
    x = np.asarray(x, np.float64)
    hi = np.clip(np.searchsorted(grid, x), 1, len(grid) - 1)
    lo = hi - 1
    mid = (grid[lo] + grid[hi]) / 2
    return np.where(x > mid, hi, np.where(x < mid, lo, np.where(lo % 2 == 0, lo, hi)))


def quantize(x, g):
    """Rows [..., D] float32 with a scale g each [...] float32 -> codes [..., D] and scales [..., D/16]."""
    x = np.asarray(x, np.float32)
    b = x.reshape(*x.shape[:-1], -1, 16)
    g = np.asarray(g, np.float32)[..., None]
    with np.errstate(all="ignore"):
        clean = np.where(np.isnan(b), np.float32(0), b)
        a = np.abs(clean).max(-1)
        t = a / (np.float32(6) * g)
        s = nearest(E4M3, np.minimum(t, np.float32(448)))
        d = E4M3[s].astype(np.float32) * g
        y = np.where(d[..., None] > 0, clean / d[..., None], np.float32(0))
    assert y.dtype == np.float32
    code = nearest(LEVELS, np.abs(y.astype(np.float64))) + 8 * (y < 0)
    code = np.where(s[..., None] > 0, code, 0)
    return code.reshape(x.shape).astype(np.uint8), s.astype(np.uint8)


def values(codes, scales):
    """float64 values without the head's scale."""
    v = GRID[codes].reshape(*codes.shape[:-1], -1, 16) * e4m3_value(scales)[..., None]
    return v.reshape(codes.shape)


class Plain:
    """A cache's arrays on the host.  pages [layers][pages][H][P/16][tile]."""

    def __init__(self, cache):
        self.P, self.D, self.H = cache.s.page_tokens, cache.s.head_dim, cache.s.kv_heads
        self.layers, self.num_pages = cache.s.layers, cache.s.num_pages
        self.pages = cache.pages.cpu().numpy().copy()
        self.table, self.length, self.refs = [t.cpu().numpy().copy() for t in (cache.table, cache.length, cache.refs)]
        one = np.ones((self.layers, self.H), np.float32)
        self.kg = one if cache.k_scale is None else cache.k_scale.cpu().numpy()
        self.vg = one if cache.v_scale is None else cache.v_scale.cpu().numpy()

    def same_state(self, cache, pages=True):
        assert np.array_equal(self.length, cache.length.cpu().numpy())
        assert np.array_equal(self.refs, cache.refs.cpu().numpy())
        assert np.array_equal(self.table, cache.table.cpu().numpy())
        if pages:
            assert np.array_equal(self.pages, cache.pages.cpu().numpy())

    def _row(self, layer, seq, pos, kv):
        """Views of the code bytes [H][D/2] and scales [H][D/16] of a token."""
        D = self.D
        tile = self.pages[layer, self.table[seq, pos // self.P], :, pos % self.P // 16]
        r = pos % 16
        codes = tile[:, kv * 8 * D:(kv + 1) * 8 * D].reshape(self.H, 16, D // 2)[:, r]
        at = 16 * D + kv * D
        return codes, tile[:, at:at + D].reshape(self.H, 16, D // 16)[:, r]

    def write(self, layer, seq, pos, k, v):
        """k, v [H][D] float32."""
        for kv, x, g in ((0, k, self.kg), (1, v, self.vg)):
            c, s = quantize(x, g[layer])
            codes, scales = self._row(layer, seq, pos, kv)
            codes[:] = c[:, 0::2] | c[:, 1::2] << 4
            scales[:] = s

    def rows(self, layer, seq, kv, positions):
        """[positions][H][D] float64, with the head's scale as the last factor given apart."""
        out = np.empty((len(positions), self.H, self.D))
        for j, pos in enumerate(positions):
            codes, scales = self._row(layer, seq, pos, kv)
            nib = np.stack([codes & 15, codes >> 4], -1).reshape(self.H, self.D)
            out[j] = values(nib, scales)
        return out

    # ------------------------------------------------------ page operations ------
    def used(self, tokens):
        return -(-int(tokens) // self.P)

    def free(self, seqs):
        for s in seqs:
            if 0 <= s < len(self.length):
                for p in self.table[s, :self.used(self.length[s])]:
                    self.refs[p] -= 1
                self.length[s] = 0

    def fork(self, src, dst):
        for i, (a, b) in enumerate(zip(src, dst)):
            n = len(self.length)
            if not (0 <= a < n and 0 <= b < n) or b in src or a in dst or list(dst).count(b) > 1:
                continue
            if self.length[b]:
                continue
            u = self.used(self.length[a])
            self.table[b, :u] = self.table[a, :u]
            self.refs[self.table[a, :u]] += 1
            self.length[b] = self.length[a]

    def reserve(self, seqs, counts):
        """Starts, or None if there is no room."""
        shared, need, seen = [], [], set()
        for s, m in zip(seqs, counts):
            ok = 0 <= s < len(self.length) and s not in seen
            seen.add(s)
            if not ok:
                need.append(-1)
                shared.append(False)
                continue
            t = self.length[s]
            c = bool(m > 0 and t % self.P and self.refs[self.table[s, t // self.P]] > 1)
            shared.append(c)
            need.append(self.used(t + m) - self.used(t) + c)
            if self.used(t + m) > self.table.shape[1]:
                return None
        free = [p for p in range(self.num_pages) if self.refs[p] == 0]
        if sum(max(0, x) for x in need) > len(free):
            return None
        start = []
        for s, m, c, x in zip(seqs, counts, shared, need):
            if x < 0:
                start.append(-1)
                continue
            t = self.length[s]
            column = self.used(t) - c
            for j in range(x):
                page = free.pop(0)
                if c and j == 0:
                    old = self.table[s, column]
                    self.pages[:, page] = self.pages[:, old]
                    self.refs[old] -= 1
                self.table[s, column + j] = page
                self.refs[page] = 1
            self.length[s] = t + m
            start.append(t)
        return start

    def compact(self, seqs, keep):
        seen, plan = set(), []
        for s, flags in zip(seqs, keep):
            if not 0 <= s < len(self.length) or s in seen:
                continue
            seen.add(s)
            t = int(self.length[s])
            plan.append((s, [p for p in range(t) if p >= len(flags) or flags[p]]))
        free = [p for p in range(self.num_pages) if self.refs[p] == 0]
        if sum(self.used(len(k)) for _, k in plan) > len(free):
            return False
        new = {}
        for s, kept in plan:
            pages = [free.pop(0) for _ in range(self.used(len(kept)))]
            new[s] = pages
            for j, pos in enumerate(kept):
                for layer in range(self.layers):
                    for kv in (0, 1):
                        a = self._row(layer, s, pos, kv)
                        tile = self.pages[layer, pages[j // self.P], :, j % self.P // 16]
                        D, r = self.D, j % 16
                        tile[:, kv * 8 * D:(kv + 1) * 8 * D].reshape(self.H, 16, D // 2)[:, r] = a[0]
                        at = 16 * D + kv * D
                        tile[:, at:at + D].reshape(self.H, 16, D // 16)[:, r] = a[1]
        for s, kept in plan:
            for p in self.table[s, :self.used(self.length[s])]:
                self.refs[p] -= 1
            for j, p in enumerate(new[s]):
                self.table[s, j] = p
                self.refs[p] = 1
            self.length[s] = len(kept)
        return True

    # ------------------------------------------------------------ attention ------
    def attend(self, layer, seq, q, scale, window=0):
        """One sequence's rows q [m][Hq][D] float64 -> (out, lse, weight, size): weight =
        sum p |v| for each element of out, size = |scale| * max_t sum |q k| for each row."""
        m, Hq, D = q.shape
        G, t = Hq // self.H, int(self.length[seq])
        out, weight = np.zeros((m, Hq, D)), np.zeros((m, Hq, D))
        lse, size = np.full((m, Hq), -np.inf), np.zeros((m, Hq))
        if t == 0:
            return out, lse, weight, size
        k, v = self.rows(layer, seq, 0, range(t)), self.rows(layer, seq, 1, range(t))
        pos = np.arange(t)
        for j in range(m):
            p = t - m + j
            see = (pos <= p) & (pos > p - window if window else True)
            if not see.any():
                continue
            for h in range(Hq):
                kk, vv = k[see, h // G], v[see, h // G]
                z = kk @ q[j, h] * (scale * float(self.kg[layer, h // G]))
                size[j, h] = (np.abs(kk) @ np.abs(q[j, h])).max() * abs(scale) * float(self.kg[layer, h // G])
                e = np.exp(z - z.max())
                lse[j, h] = z.max() + np.log(e.sum())
                g = float(self.vg[layer, h // G])
                out[j, h] = e @ vv / e.sum() * g
                weight[j, h] = e @ np.abs(vv) / e.sum() * g
        return out, lse, weight, size


def attention_bounds(out, lse, weight, size, dtype, D, tokens, v_most):
    """How far the kernel's results may be from the definition's.

    A logit is D/16 chained matrix instructions; each loses less than one unit in the last place of
    its largest addend for each of 17 addends: 17 D/16 2^-23 size.  A weight is off by that
    (relative), by 2^-21 of the exponential and its argument's rounding (arguments stay below 2^7 or
    the weight below fp16's reach), and by half a step of fp16, 2^-11, where it meets V; below
    fp16's normal numbers by 2^-25 against a largest weight of at least 2^8.  Sums of products on
    the matrix unit lose 17 2^-23 of their size for each 16 tokens, the joining of parts
    2^-20.  The result's own rounding is half a step of its type; the smallest step of
    fp16 is 2^-24."""
    logit = 17 * D / 16 * 2.0 ** -23 * size + 2.0 ** -18
    rel = (2.0 ** -11 + 2 * logit + 17 * 2.0 ** -23 * np.ceil(tokens / 16) + 2.0 ** -19)[..., None]
    u = torch.finfo(dtype).eps / 2
    tol = u * np.abs(out) + (1 + u) * (rel * weight + tokens * 2.0 ** -33 * v_most) + 2.0 ** -25
    return tol, logit + 2.0 ** -19 + 2.0 ** -22 * np.abs(np.where(np.isfinite(lse), lse, 0))
