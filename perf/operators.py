"""The work of the paged 4-bit KV cache, as measured cases.

Four kinds of passes:

  write    the rows of new tokens into one layer's pages, and the same rows read back
  attend   attention of one layer: single tokens, a few tokens, chunks of prompts
  beams    a step of sampling with shared prefixes: free the old branches, fork the parents
           again, reserve room for the next tokens (a shared partial page is copied)
  compact  a branch of a long sequence is pruned to the tokens that a selection keeps

A cache is a pool of pages [layers][pages][kv heads][page tokens / 16][tile]; a tile holds 16
tokens of one head: K codes, V codes (two e2m1 values to a byte, the lower dim in the lower
half), K scales, V scales (one e4m3 number for 16 dims).  A value is code * scale * the head's
float32 scale.
"""
import math
import random

import torch

own = False

LEVELS = (0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0)
TYPES = {"f16": torch.float16, "bf16": torch.bfloat16}


def _write(name, n, lo, hi, H=8, D=128, P=64, dtype="bf16"):
    return {"name": name, "kind": "write", "n": n, "lo": lo, "hi": hi, "kv_heads": H, "head_dim": D, "page": P, "type": dtype}


def _attend(name, n, lo, hi, queries, H=8, G=4, D=128, P=64, dtype="bf16", window=0):
    return {"name": name, "kind": "attend", "n": n, "lo": lo, "hi": hi, "queries": queries, "kv_heads": H, "group": G,
            "head_dim": D, "page": P, "type": dtype, "window": window}


def _beams(name, parents, branches, lo, hi, layers, add=1, H=8, D=128, P=64):
    return {"name": name, "kind": "beams", "n": parents, "branches": branches, "lo": lo, "hi": hi, "layers": layers,
            "add": add, "kv_heads": H, "head_dim": D, "page": P}


def _compact(name, n, lo, hi, layers, keep, H=8, D=128, P=64):
    return {"name": name, "kind": "compact", "n": n, "lo": lo, "hi": hi, "layers": layers, "keep": keep, "kv_heads": H,
            "head_dim": D, "page": P}


def listed():
    return [
        # a decode step of 64 sessions: one new token each
        _write("write-64x1", 64, 1, 1),
        # prompts of a batch, ragged, as they come out of the projections
        _write("write-5x12k", 5, 9000, 16384, dtype="f16"),
        # one chat session early on: launches and latency
        _attend("attend-1x4k", 1, 4096, 4096, 1, dtype="f16"),
        # a serving batch at long context, one layer: the throughput case
        _attend("attend-16x64k", 16, 65536, 65536, 1),
        # sessions of very different lengths, eight query heads to a KV head, small pages
        _attend("attend-61-ragged", 61, 1, 16384, 1, G=8, P=16),
        # four drafted tokens checked with the last one, on a model with a window and a head dim of 64
        _attend("attend-8x20k-draft", 8, 9000, 32768, 5, H=4, G=8, D=64, P=32, window=8192),
        # a chunk of a prompt over what is cached of it
        _attend("attend-chunk-2k-30k", 1, 30011, 30011, 2048),
        # prompts of a batch, ragged: every token attends to its past
        _attend("attend-prompts-6", 6, 300, 4500, 4500, dtype="f16"),
        # four beams of a short chat: the branches move to new parents, one token each
        _beams("beams-4x2k", 1, 4, 2011, 2011, 32, P=32),
        # sixteen samples of each of four long prompts, a few tokens each
        _beams("samples-4x16", 4, 16, 12000, 16384, 8, add=3),
        # half of a chat's tokens kept
        _compact("compact-1x6k", 1, 6001, 6001, 4, 0.5, P=16),
        # the quarter of each long sequence that a selection keeps
        _compact("compact-4x32k", 4, 24000, 32768, 4, 0.25),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["write", "attend", "attend", "attend", "attend", "beams", "compact"])
    H, D, P = rng.choice([1, 2, 4, 8, 8]), rng.choice([64, 128, 128]), rng.choice([16, 32, 64, 128])
    dtype = rng.choice(["f16", "bf16"])
    if kind == "write":
        n = _log_int(rng, 1, 128)
        hi = rng.choice([1, _log_int(rng, 1, 16384)])
        hi = min(hi, 60000 // n + 1)
        c = _write("", n, max(1, hi // 3), hi, H, D, P, dtype)
    elif kind == "attend":
        G = rng.choice([1, 2, 3, 4, 4, 5, 8, 16])
        queries = rng.choice([1, 1, 1, rng.randint(2, 9), _log_int(rng, 10, 2048)])
        n, hi = _log_int(rng, 1, 128), _log_int(rng, 16, 65536)
        while n > 1 and n * hi * H * D > 16 * 65536 * 8 * 128 // 2:
            n = (n + 1) // 2
        while n > 1 and n * hi * H * G * D * queries > 2048 * 30000 * 32 * 128 // 2:
            n = (n + 1) // 2
        while hi * H * G * D * queries > 2048 * 30000 * 32 * 128:
            hi = (hi + 1) // 2
        window = rng.choice([0, 0, 0, _log_int(rng, 16, hi + 16)])
        c = _attend("", n, rng.choice([1, hi, max(1, hi // 4)]), hi, queries, H, G, D, P, dtype, window)
    elif kind == "beams":
        parents, branches = _log_int(rng, 1, 8), _log_int(rng, 1, 16)
        hi = _log_int(rng, 16, 16384)
        c = _beams("", parents, branches, max(1, hi // 2), hi, rng.choice([1, 2, 4, 8]), rng.randint(1, 9), H, D, P)
    else:
        n, hi = _log_int(rng, 1, 8), _log_int(rng, 16, 32768)
        while n > 1 and n * hi > 4 * 32768:
            n = (n + 1) // 2
        c = _compact("", n, max(1, hi // 2), hi, rng.choice([1, 2, 4]), rng.choice([0.1, 0.25, 0.35, 0.5, 0.9]), H, D, P)
    del c["name"]
    return c


# ------------------------------------------------------------------ shapes ------

def _lens(c):
    """The sequences' lengths: spread evenly over the logarithm of [lo, hi], in a fixed shuffle."""
    n, lo, hi = c["n"], c["lo"], c["hi"]
    got = [int(round(lo * (hi / lo) ** ((i + 0.5) / n))) for i in range(n)]
    random.Random(n * 7919 + hi).shuffle(got)
    return got


def _pages_of(c, tokens):
    return -(-tokens // c["page"])


def _tile_bytes(c):
    return 18 * c["head_dim"]


def _page_bytes(c):
    return c["kv_heads"] * c["page"] // 16 * _tile_bytes(c)


def _queries_of(c):
    return [min(c["queries"], t) for t in _lens(c)]


def _kept(c):
    return [max(1, int(c["keep"] * t)) for t in _lens(c)]


def work(c):
    H, D, kind = c["kv_heads"], c["head_dim"], c["kind"]
    if kind == "write":
        rows = sum(_lens(c)) * H
        return {"bytes": rows * 2 * (4 * D + 18 * D // 16), "flops": rows * D * 8}
    if kind == "attend":
        seen = rows = 0
        read = 0
        for t, m in zip(_lens(c), _queries_of(c)):
            w = c["window"] or t
            first = max(0, t - m + 1 - w)
            read += t - first
            rows += m
            # position p sees min(p + 1, w) tokens
            whole = max(0, min(m, t - max(t - m, w - 1)))  # queries that see w tokens
            part = m - whole
            seen += whole * w + part * (t - m + 1) + part * (part - 1) // 2
        Hq = H * c["group"]
        return {"bytes": read * H * 18 * D // 16 + rows * Hq * (4 * D + 4), "flops": 4 * D * seen * Hq}
    if kind == "beams":
        tables = sum(_pages_of(c, t) for t in _lens(c)) * c["branches"] * 4
        copied = sum(t % c["page"] > 0 for t in _lens(c)) * c["branches"] * c["layers"] * _page_bytes(c)
        return {"bytes": 4 * tables + 2 * copied, "flops": 0}
    row = 18 * D // 16
    return {"bytes": 2 * sum(_kept(c)) * c["layers"] * H * row + sum(_lens(c)), "flops": 0}


# ------------------------------------------------------------------ inputs ------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1009 + stream)
    return g


def _scales(c, layers, seed):
    """Calibrated scales of the heads: what puts the largest value seen near the top of the grid."""
    g = _gen(seed, 1)
    u = torch.rand((2, layers, c["kv_heads"]), generator=g, device="cuda") * 0.4 + 0.9
    return (u[0] * (40.0 / 2688)).contiguous(), (u[1] * (5.0 / 2688)).contiguous()


def _rows(c, tokens, g):
    """K and V rows [tokens][H][D]: N(0,1), K with four outlier channels to a head."""
    H, D = c["kv_heads"], c["head_dim"]
    gain = torch.ones((H, D), device="cuda")
    idx = torch.rand((H, D), generator=g, device="cuda").argsort(dim=1)[:, :4]
    gain.scatter_(1, idx, 8.0)
    k = torch.randn((tokens, H, D), generator=g, device="cuda") * gain
    return k, torch.randn((tokens, H, D), generator=g, device="cuda")


def _pool(c, layers, num_pages, seed, k_scale, v_scale):
    """A pool of quantized rows."""
    H, D, P = c["kv_heads"], c["head_dim"], c["page"]
    pages = torch.empty((layers, num_pages, H, P // 16, _tile_bytes(c)), dtype=torch.uint8, device="cuda")
    g = _gen(seed, 2)
    step = max(1, (1 << 26) // (P * H * D))
    for layer in range(layers):
        kc, vc, ks, vs = _views(c, pages[layer])
        for p in range(0, num_pages, step):
            n = min(step, num_pages - p)
            k, v = _rows(c, n * P, g)
            for x, gs, codes, scales in ((k, k_scale, kc, ks), (v, v_scale, vc, vs)):
                q, s = _quantize(x, gs[layer])
                codes[p:p + n] = q.view(n, P // 16, 16, H, D // 2).permute(0, 3, 1, 2, 4)
                scales[p:p + n] = s.view(n, P // 16, 16, H, D // 16).permute(0, 3, 1, 2, 4)
    return pages


def _tables(c, lens, spare, max_seqs, max_pages, seed):
    """Pages of the first sequences, in no order, and the reference counts."""
    need = [_pages_of(c, t) for t in lens]
    num = sum(need) + spare
    order = torch.randperm(num, generator=_gen(seed, 3), device="cuda").int()
    table = torch.full((max_seqs, max_pages), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(num, dtype=torch.int32, device="cuda")
    at = 0
    for i, m in enumerate(need):
        table[i, :m] = order[at:at + m]
        refs[order[at:at + m].long()] = 1
        at += m
    length = torch.zeros(max_seqs, dtype=torch.int32, device="cuda")
    length[:len(lens)] = torch.tensor(lens, dtype=torch.int32, device="cuda")
    return table, length, refs


def _cu(counts):
    cu = torch.zeros(len(counts) + 1, dtype=torch.int32, device="cuda")
    cu[1:] = torch.tensor(counts, device="cuda").cumsum(0).int()
    return cu


def prepare(c, seed):
    kind, D, H = c["kind"], c["head_dim"], c["kv_heads"]
    lens = _lens(c)
    s = {"case": c, "lens": lens}
    layers = c.get("layers", 1)
    s["k_scale"], s["v_scale"] = _scales(c, layers, seed)
    n, counts, seqs, branches = c["n"], None, None, 0
    if kind == "write":
        counts = lens
        spare, max_seqs, max_pages = 3, n, _pages_of(c, max(lens))
        k, v = _rows(c, sum(lens), _gen(seed, 4))
        # as a projection leaves them: K and V side by side in one row for each token
        s["kv"] = torch.stack((k, v), dim=1).to(TYPES[c["type"]])
        s["k_out"] = torch.empty_like(s["kv"][:, 0], memory_format=torch.contiguous_format)
        s["v_out"] = torch.empty_like(s["k_out"])
    elif kind == "attend":
        counts = _queries_of(c)
        spare, max_seqs, max_pages = 3, n, _pages_of(c, max(lens))
        q = torch.randn((sum(counts), H * c["group"], D), generator=_gen(seed, 5), device="cuda")
        s["q"] = q.to(TYPES[c["type"]])
        s["out"], s["lse"] = torch.empty_like(s["q"]), torch.empty(q.shape[:2], device="cuda")
    elif kind == "beams":
        branches = n * c["branches"]
        counts = [c["add"]] * branches
        spare = branches * (1 + _pages_of(c, c["add"])) + 5
        max_seqs, max_pages = n + branches, _pages_of(c, max(lens) + c["add"])
        seqs = torch.arange(n, n + branches, dtype=torch.int32, device="cuda")
        s["src"] = (seqs - n).div(c["branches"], rounding_mode="floor").int()
    else:
        branches = n
        kept = _kept(c)
        spare = sum(_pages_of(c, t) for t in kept) + 2
        max_seqs, max_pages = 2 * n, _pages_of(c, max(lens))
        seqs = torch.arange(n, 2 * n, dtype=torch.int32, device="cuda")
        s["src"] = seqs - n
        s["keep"] = torch.zeros((n, max(lens)), dtype=torch.uint8, device="cuda")
        g = _gen(seed, 6)
        for i, (t, m) in enumerate(zip(lens, kept)):
            s["keep"][i, torch.randperm(t, generator=g, device="cuda")[:m]] = 1
    s["table"], s["length"], s["refs"] = _tables(c, lens, spare, max_seqs, max_pages, seed)
    s["pages"] = _pool(c, layers, s["refs"].numel(), seed, s["k_scale"], s["v_scale"])
    s["seqs"], s["n"] = seqs, branches or n
    if counts is not None:
        s["counts"], s["cu"] = counts, _cu(counts)
        s["start"] = torch.zeros(len(counts), dtype=torch.int32, device="cuda")
    if own:
        _handles(s)
    return s


# ------------------------------------------------- the framework's operators ------

def _handles(s):
    from paper_2608_28911_gb300 import semkv
    c, kind = s["case"], s["case"]["kind"]
    s["cache"] = semkv.KV4Cache.over(s["pages"], s["table"], s["length"], s["refs"], c["head_dim"], s["k_scale"], s["v_scale"])
    if kind != "compact":
        s["batch"] = semkv.KV4Batch(s["n"], cu=s["cu"], seqs=s["seqs"], start=s["start"], total=sum(s["counts"]), max_count=max(s["counts"]))
    if kind == "attend":
        s["ws"] = s["cache"].attention_workspace(s["batch"], s["q"].shape[1])
    elif kind in ("beams", "compact"):
        s["ws"] = s["cache"].pages_workspace(s["n"], max(s["lens"]))


def _run_own(s):
    from paper_2608_28911_gb300 import semkv
    c, kind = s["case"], s["case"]["kind"]
    if kind == "write":
        semkv.semkv_kv4_write(s["cache"], s["batch"], 0, s["kv"][:, 0], s["kv"][:, 1])
        semkv.semkv_kv4_read(s["cache"], s["batch"], 0, s["k_out"], s["v_out"])
        return {"k": s["k_out"], "v": s["v_out"]}
    if kind == "attend":
        semkv.semkv_kv4_attention(s["cache"], s["batch"], 0, s["q"], s["out"], c["head_dim"] ** -0.5, s["ws"], lse=s["lse"], window=c["window"])
        return {"out": s["out"], "lse": s["lse"]}
    semkv.semkv_kv4_free(s["cache"], s["seqs"])
    semkv.semkv_kv4_fork(s["cache"], s["src"], s["seqs"])
    if kind == "beams":
        semkv.semkv_kv4_reserve(s["cache"], s["batch"], s["ws"])
    else:
        semkv.semkv_kv4_compact(s["cache"], s["seqs"], s["keep"], s["ws"])
    return _state(s)


def _state(s):
    got = {k: s[k] for k in ("table", "length", "refs", "pages")}
    if s["case"]["kind"] == "beams":
        got["start"] = s["start"]
    return got


# ------------------------------------------------------------ the plain form ------

def _views(c, pages):
    """K codes, V codes, K scales, V scales of pages [...][H][P / 16][tile], each [...][H][P / 16][16][bytes]."""
    D = c["head_dim"]
    a, b = 8 * D, 16 * D
    cut = (pages[..., :a], pages[..., a:b], pages[..., b:b + D], pages[..., b + D:])
    return [x.unflatten(-1, (16, -1)) for x in cut]


def _quantize(x, g):
    """Rows [tokens][H][D] to codes [tokens][H][D / 2] and scales [tokens][H][D / 16], as bytes."""
    x = x.float().unflatten(-1, (-1, 16))
    g = g.view(-1, 1)
    x = torch.where(x.isnan(), 0.0, x)
    scale = (x.abs().amax(-1) / (6 * g)).clamp(max=448.0).to(torch.float8_e4m3fn)
    step = scale.float() * g
    y = torch.where(step[..., None] > 0, x / step[..., None], 0.0)
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte()
    code = code + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5.0).byte() + 8 * (y < 0).byte()
    code = code.flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scale.view(torch.uint8)


def _values(codes, scales):
    """float32 values, without the head's scale, of codes [...][D / 2] and scales [...][D / 16]."""
    half = torch.tensor(LEVELS, device="cuda")
    grid = torch.cat((half, -half))
    b = torch.arange(256, device="cuda")
    pair = torch.stack((grid[b % 16], grid[b // 16]), dim=1)
    x = pair[codes.int()].flatten(-2)
    return (x.unflatten(-1, (-1, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]).flatten(-2)


def _places(s):
    """Page, tile, row and sequence of each new token."""
    c, P = s["case"], s["case"]["page"]
    counts = s["cu"][1:] - s["cu"][:-1]
    i = torch.repeat_interleave(torch.arange(s["n"], device="cuda"), counts, output_size=sum(s["counts"]))
    pos = s["start"][i] + torch.arange(i.numel(), device="cuda") - s["cu"][i]
    page = s["table"][i, pos // P].long()
    return page, pos % P // 16, pos % 16


def _plain_write(s):
    c = s["case"]
    page, tile, row = _places(s)
    kc, vc, ks, vs = _views(c, s["pages"][0])
    got = {}
    for name, x, codes, scales, g in (("k", s["kv"][:, 0], kc, ks, s["k_scale"][0]), ("v", s["kv"][:, 1], vc, vs, s["v_scale"][0])):
        codes[page, :, tile, row], scales[page, :, tile, row] = _quantize(x, g)
        back = _values(codes[page, :, tile, row], scales[page, :, tile, row]) * g[:, None]
        got[name] = back.to(x.dtype)
    return got


def _seen(c, length, count, T, queries):
    """Which positions [n][queries][T] each query sees; queries past a sequence's own see nothing."""
    j = torch.arange(queries, device="cuda")
    p = length[:, None] - count[:, None] + j
    t = torch.arange(T, device="cuda")
    seen = (t <= p[..., None]) & (j < count[:, None])[..., None]
    return seen & (t > p[..., None] - c["window"]) if c["window"] else seen


def _plain_attend(s):
    c = s["case"]
    n, H, G, D = c["n"], c["kv_heads"], c["group"], c["head_dim"]
    m, total, T = max(s["counts"]), sum(s["counts"]), max(s["lens"])
    pages = s["pages"][0][s["table"].long().clamp(min=0)]  # [n][pages][H][tiles][tile]
    kc, vc, ks, vs = _views(c, pages)
    rows = [_values(a, b).transpose(1, 2).flatten(2, 4)[:, :, :T] for a, b in ((kc, ks), (vc, vs))]  # [n][H][T][D]
    count = s["cu"][1:] - s["cu"][:-1]
    j = torch.arange(m, device="cuda")
    at = (s["cu"][:-1, None] + j).clamp(max=total - 1)
    q = s["q"].float()[at].view(n, m, H, G, D).permute(0, 2, 3, 1, 4).reshape(n, H, G * m, D)
    logit = torch.matmul(q, rows[0].transpose(-1, -2)) * (s["k_scale"][0].view(H, 1, 1) * D ** -0.5)
    seen = _seen(c, s["length"], count, T, m)[:, None, None].expand(n, H, G, m, T).reshape(n, H, G * m, T)
    logit.masked_fill_(~seen, -math.inf)
    top = logit.amax(-1, keepdim=True)
    top = torch.where(top == -math.inf, 0.0, top)
    p = logit.sub_(top).exp_()
    total_p = p.sum(-1, keepdim=True)
    out = torch.matmul(p, rows[1]) / torch.where(total_p > 0, total_p, 1.0) * s["v_scale"][0].view(H, 1, 1)
    lse = total_p.log() + top
    own_rows = (j < count[:, None])
    out = out.view(n, H, G, m, D).permute(0, 3, 1, 2, 4).reshape(n, m, H * G, D)[own_rows]
    lse = lse.view(n, H, G, m).permute(0, 3, 1, 2).reshape(n, m, H * G)[own_rows]
    return {"out": out.to(s["q"].dtype), "lse": lse}


def _held(s, seqs):
    """Which table entries of these sequences [len(seqs)][max_pages] hold a page."""
    P = s["case"]["page"]
    used = (s["length"][seqs] + P - 1) // P
    return torch.arange(s["table"].shape[1], device="cuda") < used[:, None]


def _count(s, pages, by):
    s["refs"].index_add_(0, pages.long(), torch.full_like(pages, by))


def _plain_free(s, seqs):
    _count(s, s["table"][seqs][_held(s, seqs)], -1)
    s["length"][seqs] = 0


def _plain_fork(s, src, dst):
    held = _held(s, src)
    s["table"][dst] = torch.where(held, s["table"][src], s["table"][dst])
    s["length"][dst] = s["length"][src]
    _count(s, s["table"][src][held], 1)


def _take(s, need):
    """The lowest free pages, need[i] of them for sequence i: [n][max need] and which are meant."""
    free = (s["refs"] == 0).nonzero().view(-1).int()
    most = torch.arange(int(need.max()), device="cuda")
    mine = most < need[:, None]
    at = (need.cumsum(0) - need)[:, None] + most
    return free[at.clamp(max=free.numel() - 1)], mine


def _plain_reserve(s, seqs):
    P = s["case"]["page"]
    old = s["length"][seqs]
    count = s["cu"][1:] - s["cu"][:-1]
    last = (old - 1).clamp(min=0) // P
    shared = (count > 0) & (old % P > 0) & (s["refs"][s["table"][seqs, last.long()].long()] > 1)
    had = (old + P - 1) // P
    need = (old + count + P - 1) // P - had + shared.int()
    got, mine = _take(s, need)
    i, k = mine.nonzero(as_tuple=True)
    page = got[i, k]
    column = (had[i] - shared[i].int() + k).long()
    copied = (shared[i] & (k == 0)).nonzero().view(-1)
    source = s["table"][seqs[i[copied]], column[copied]].long()
    s["pages"][:, page[copied].long()] = s["pages"][:, source]
    _count(s, source.int(), -1)
    s["table"][seqs[i], column] = page
    s["refs"][page.long()] = 1
    s["length"][seqs] = old + count
    s["start"].copy_(old)


def _plain_compact(s, seqs):
    P, n, T = s["case"]["page"], s["n"], s["keep"].shape[1]
    t = torch.arange(T, device="cuda")
    keep = (s["keep"] != 0) & (t < s["length"][seqs][:, None])
    kept = keep.sum(1).int()
    need = (kept + P - 1) // P
    got, mine = _take(s, need)
    i, old = keep.nonzero(as_tuple=True)
    new = (keep.cumsum(1) - 1)[i, old]
    source, to = s["table"][seqs][i, old // P].long(), got[i, new // P].long()
    for layer in s["pages"]:
        for x in _views(s["case"], layer):
            x[to, :, new % P // 16, new % 16] = x[source, :, old % P // 16, old % 16]
    _count(s, s["table"][seqs][_held(s, seqs)], -1)
    width = got.shape[1]
    s["table"][seqs, :width] = torch.where(mine, got, s["table"][seqs, :width])
    s["refs"][got[mine].long()] = 1
    s["length"][seqs] = kept


def _run_plain(s):
    kind = s["case"]["kind"]
    if kind == "write":
        return _plain_write(s)
    if kind == "attend":
        return _plain_attend(s)
    seqs = s["seqs"].long()
    _plain_free(s, seqs)
    _plain_fork(s, s["src"].long(), seqs)
    if kind == "beams":
        _plain_reserve(s, seqs)
    else:
        _plain_compact(s, seqs)
    return _state(s)


def run(s):
    return _run_own(s) if own else _run_plain(s)


# ------------------------------------------------ the definition, in 64 bits ------

def _exact_quantized(x, g):
    """What a row [tokens][H][D] is stored as: block by block, each number the nearest of its grid."""
    x = x.double()
    x = torch.where(x.isnan(), torch.zeros_like(x), x).reshape(*x.shape[:-1], -1, 16)
    g = g.double()[:, None, None]
    t = x.abs().max(-1, keepdim=True).values / (6 * g)
    ulp = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6, max=448.0))) - 3)
    scale = (torch.round(t / ulp) * ulp).clamp(max=448.0)
    y = x / torch.where(scale > 0, scale * g, torch.ones_like(scale))
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    v = (torch.round(a / step) * step).clamp(max=6.0) * torch.sign(y)
    return torch.where(scale > 0, v * scale * g, torch.zeros_like(v)).flatten(-2)


def _exact_row(s, i, base):
    """Sequence i's K (base 0) or V (base 1) rows [H][T][D], without the head's scale."""
    c, D = s["case"], s["case"]["head_dim"]
    t = s["lens"][i]
    pages = s["pages"][0, s["table"][i, :_pages_of(c, t)].long()]
    tiles = pages.transpose(0, 1).flatten(1, 2)  # [H][tiles][bytes]
    codes = tiles[..., base * 8 * D:(base + 1) * 8 * D].reshape(c["kv_heads"], -1, D // 2)[:, :t]
    scale = tiles[..., 16 * D + base * D:16 * D + (base + 1) * D].reshape(c["kv_heads"], -1, D // 16)[:, :t]
    nibble = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    e, m = (nibble >> 1 & 3).double(), (nibble & 1).double()
    size = torch.where(e > 0, torch.exp2(e - 1) * (1 + m / 2), m / 2)
    e, m = (scale >> 3 & 15).double(), (scale & 7).double()
    s4 = torch.where(e > 0, torch.exp2(e - 7) * (1 + m / 8), m * 2.0 ** -9)
    return torch.where(nibble > 7, -size, size) * s4.repeat_interleave(16, dim=-1)


def exact(c, seed):
    if c["kind"] in ("beams", "compact"):
        return None
    s = prepare(c, seed)
    if c["kind"] == "write":
        return {"k": _exact_quantized(s["kv"][:, 0], s["k_scale"][0]), "v": _exact_quantized(s["kv"][:, 1], s["v_scale"][0])}
    H, G, D = c["kv_heads"], c["group"], c["head_dim"]
    out = torch.empty(s["q"].shape, dtype=torch.float64, device="cuda")
    lse = torch.empty(s["lse"].shape, dtype=torch.float64, device="cuda")
    at = 0
    for i, (t, m) in enumerate(zip(s["lens"], s["counts"])):
        k, v = _exact_row(s, i, 0), _exact_row(s, i, 1)
        for j in range(0, m, 512):
            p = torch.arange(j, min(j + 512, m), device="cuda")
            rows = slice(at + j, at + j + p.numel())
            position = t - m + p
            place = torch.arange(t, device="cuda")
            hidden = place > position[:, None]
            if c["window"]:
                hidden |= place <= position[:, None] - c["window"]
            for h in range(H):
                heads = slice(h * G, (h + 1) * G)
                z = torch.einsum("jgd,td->jgt", s["q"][rows, heads].double(), k[h])
                z = (z * s["k_scale"][0, h].double() / math.sqrt(D)).masked_fill(hidden[:, None], -math.inf)
                lse[rows, heads] = torch.logsumexp(z, -1)
                out[rows, heads] = torch.einsum("jgt,td->jgd", torch.softmax(z, -1), v[h]) * s["v_scale"][0, h].double()
        at += m
    return {"out": out, "lse": lse}
