"""The work of a step of search over the paged 4-bit KV cache, as measured cases.

Three kinds of passes:

  append   new tokens of a step: queries and keys turned by their positions, keys and values
           into one layer's pages; the rows are read back
  select   one step of beam search: the best continuations over a group's beams and the vocabulary
  reorder  two steps of a search's bookkeeping: sequences become branches of others of the same list

An append turns the first `rot` dims of each head of Q and K by the position's angles, given as a
table of cosines and sines; pairs are the dims (j, j + rot / 2), or with `pairs` (2 j, 2 j + 1).  K's
turned rows and V's rows go into blocks of 16 values, e2m1 codes and one e4m3 scale each, beside the
head's float32 scale.  A tile holds 16 tokens of one head: K codes, V codes, K scales, V scales.

A selection scores token t of beam b with score[b] + logit[b][t] - ln sum exp logit[b] and takes the
k best of the group, the lower beam and token first where scores are equal.  A beam that is done offers
one candidate, the end token at the beam's own score.
"""
import math
import random

import torch

own = False

TYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}


def _append(name, n, lo, hi, past, H=8, G=4, D=128, P=64, rot=128, pairs=False, dtype="bf16", moved=False):
    return {"name": name, "kind": "append", "n": n, "lo": lo, "hi": hi, "past": past, "kv_heads": H, "group": G, "head_dim": D,
            "page": P, "rot": rot, "pairs": pairs, "type": dtype, "moved": moved}


def _select(name, groups, beams, vocab, k, dtype="bf16", pad=0, done=0.0, banned=0.0, first=False, width=3.0):
    return {"name": name, "kind": "select", "groups": groups, "beams": beams, "vocab": vocab, "k": k, "type": dtype, "pad": pad,
            "done": done, "banned": banned, "first": first, "width": width}


def _reorder(name, groups, beams, past, tail, P=64, saved=True):
    return {"name": name, "kind": "reorder", "groups": groups, "beams": beams, "past": past, "tail": tail, "page": P, "saved": saved}


def listed():
    return [
        # one chat session's next token: launches and latency
        _append("append-1x1", 1, 1, 1, 4096, dtype="f16"),
        # a decode step of 64 sessions
        _append("append-64x1", 64, 1, 1, 16384),
        # drafted tokens of a model that turns half of each head, in neighbouring pairs, over pruned caches:
        # positions are the tokens' own, not their places
        _append("append-9x5-half", 9, 5, 5, 20000, H=4, G=8, P=32, rot=64, pairs=True, moved=True),
        # prompts of a batch, ragged, as they come out of the projections
        _append("append-prompts-5x12k", 5, 9000, 16384, 0),
        # beams of one chat
        _select("select-1x4x32k", 1, 4, 32768, 8),
        # odd vocabulary, logits in 32 bits, some beams done, some tokens banned
        _select("select-5x5x50003", 5, 5, 50003, 10, dtype="f32", done=0.2, banned=0.3),
        # the first step of a batch's searches: one beam of each group is alive; a padded vocabulary
        _select("select-32x4-first", 32, 4, 131001, 8, dtype="f16", pad=71, first=True),
        # wide beams of a batch: the throughput case
        _select("select-64x16x128k", 64, 16, 131072, 32),
        # four beams of a chat trade places
        _reorder("reorder-1x4", 1, 4, 2011, 90, P=32, saved=False),
        # sixteen branches of each of four prompts begin again from saved ones, twice
        _reorder("reorder-4x16", 4, 16, 14000, 700),
        # a large batch of searches at long context, small pages
        _reorder("reorder-64x8", 64, 8, 30000, 2500, P=16),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def draw(rng):
    kind = rng.choice(["append", "append", "select", "select", "reorder"])
    if kind == "append":
        H, G, D = rng.choice([1, 2, 4, 8, 8]), rng.choice([1, 2, 3, 4, 4, 5, 8, 16]), rng.choice([64, 128, 128])
        n, hi = _log_int(rng, 1, 128), rng.choice([1, 1, rng.randint(2, 9), _log_int(rng, 10, 16384)])
        while n * hi * (2 * G + 2) * H * D > 61000 * 10 * 8 * 128:
            hi = (hi + 1) // 2
            n = (n + 1) // 2
        c = _append("", n, max(1, hi // 3), hi, rng.choice([0, _log_int(rng, 1, 30000)]), H, G, D, rng.choice([16, 32, 64, 128]),
                    rng.choice([D, D, D // 2, D // 4, 16 * rng.randint(1, D // 16)]), rng.random() < 0.4, rng.choice(["f16", "bf16"]), rng.random() < 0.3)
    elif kind == "select":
        beams = _log_int(rng, 1, 64)
        groups, vocab = _log_int(rng, 1, 128), _log_int(rng, 100, 262144)
        while groups * beams * vocab > 64 * 16 * 131072 // 2:
            groups, beams = (groups + 1) // 2, (beams + 1) // 2
        k = rng.choice([1, beams, min(128, 2 * beams), _log_int(rng, 1, 128)])
        c = _select("", groups, beams, vocab, k, rng.choice(["f16", "bf16", "f32"]), rng.choice([0, 0, rng.randint(1, 200)]), rng.choice([0.0, 0.0, 0.3]),
                    rng.choice([0.0, 0.0, 0.5]), rng.random() < 0.2, rng.choice([0.5, 3.0, 8.0]))
    else:
        beams, groups = _log_int(rng, 2, 64), _log_int(rng, 1, 64)
        past, P = _log_int(rng, 1, 65536), rng.choice([16, 32, 64, 128])
        while groups > 1 and groups * beams * past // P > 64 * 8 * 30000 // 16 // 2:
            groups = (groups + 1) // 2
        c = _reorder("", groups, beams, past, _log_int(rng, 1, 2000), P, rng.random() < 0.7)
    del c["name"]
    return c


# ------------------------------------------------------------------ shapes ------

def _counts(c):
    """The sequences' new rows: spread evenly over the logarithm of [lo, hi], in a fixed shuffle."""
    n, lo, hi = c["n"], c["lo"], c["hi"]
    got = [int(round(lo * (hi / lo) ** ((i + 0.5) / n))) for i in range(n)]
    random.Random(n * 7919 + hi).shuffle(got)
    return got


def _pasts(c):
    """What the sequences hold before the new rows."""
    rng = random.Random(c["n"] * 31 + c["past"])
    return [rng.randint(c["past"] // 2, c["past"]) for _ in range(c["n"])]


def _tails(c):
    """Tokens of each saved branch (or of each beam) behind its group's prompt."""
    rng = random.Random(c["groups"] * 131 + c["tail"])
    return [rng.randint(c["tail"] // 2, c["tail"]) for _ in range(c["groups"] * c["beams"])]


def _pages(c, tokens):
    return -(-tokens // c["page"])


def work(c):
    if c["kind"] == "append":
        rows, H, D = sum(_counts(c)), c["kv_heads"], c["head_dim"]
        q = rows * H * c["group"] * D * 4
        kv = rows * H * 2 * (2 * D + 2 * (18 * D // 16) + 2 * D)  # written into the pages, and read back
        return {"bytes": q + kv + rows * 4 * c["rot"], "flops": rows * H * (3 * c["rot"] * (c["group"] + 1) + 2 * 8 * D)}
    if c["kind"] == "select":
        rows = c["groups"] * c["beams"]
        read = rows
        if c["first"]:
            read = c["groups"]
        elif c["done"]:
            read = sum(not d for d in _done(c))
        size = 4 if c["type"] == "f32" else 2
        return {"bytes": read * c["vocab"] * size + rows * 5 + c["groups"] * c["k"] * 12, "flops": read * c["vocab"] * 4}
    # for each step: the list's tables and the beams' new ones
    held = sum(_pages(c, c["past"] + t) for t in _tails(c))
    return {"bytes": 2 * 4 * held * (3 if c["saved"] else 2), "flops": 0}


# ------------------------------------------------------------------ inputs ------

def _gen(seed, stream):
    g = torch.Generator(device="cuda")
    g.manual_seed(int(seed) * 1009 + stream)
    return g


def _ints(values):
    return torch.tensor(values, dtype=torch.int32, device="cuda")


def _tile(c):
    return 18 * c["head_dim"]


def _prepare_append(c, seed):
    H, G, D, P = c["kv_heads"], c["group"], c["head_dim"], c["page"]
    counts, past = _counts(c), _pasts(c)
    n, total = c["n"], sum(counts)
    need = [_pages(c, a + b) for a, b in zip(past, counts)]
    s = {"case": c, "total": total, "counts": counts}
    # a projection's rows: Q, K and V of a token side by side; K has four outlier channels to a head
    g = _gen(seed, 1)
    gain = torch.ones((H, D), device="cuda")
    gain.scatter_(1, torch.rand((H, D), generator=g, device="cuda").argsort(dim=1)[:, :4], 8.0)
    rows = torch.randn((total, H * (G + 2), D), generator=g, device="cuda")
    rows[:, H * G:H * (G + 1)] *= gain
    rows = rows.to(TYPES[c["type"]])
    s["q"], s["k"], s["v"] = rows[:, :H * G], rows[:, H * G:H * (G + 1)], rows[:, H * (G + 1):]
    s["q_out"] = torch.empty((total, H * G, D), dtype=rows.dtype, device="cuda")
    s["k_out"], s["v_out"] = (torch.empty((total, H, D), dtype=rows.dtype, device="cuda") for _ in range(2))
    u = torch.rand((2, 1, H), generator=g, device="cuda") * 0.4 + 0.9
    s["k_scale"], s["v_scale"] = (u[0] * (40.0 / 2688)).contiguous(), (u[1] * (5.0 / 2688)).contiguous()
    # sequences' pages, in no order
    order = torch.randperm(sum(need) + 3, generator=g, device="cuda").int()
    s["table"] = torch.full((n, max(need)), -1, dtype=torch.int32, device="cuda")
    at = 0
    for i, m in enumerate(need):
        s["table"][i, :m] = order[at:at + m]
        at += m
    s["refs"] = torch.zeros(order.numel(), dtype=torch.int32, device="cuda")
    s["refs"][order[:at].long()] = 1
    s["pages"] = torch.zeros((1, order.numel(), H, P // 16, _tile(c)), dtype=torch.uint8, device="cuda")
    s["length"] = _ints([a + b for a, b in zip(past, counts)])
    s["start"] = _ints(past)
    s["cu"] = torch.zeros(n + 1, dtype=torch.int32, device="cuda")
    s["cu"][1:] = torch.tensor(counts, device="cuda").cumsum(0).int()
    # cosines and sines of the positions that can occur
    top = max(a + b for a, b in zip(past, counts)) + 1
    s["positions"] = None
    if c["moved"]:
        j = torch.arange(total, device="cuda") - s["cu"][:-1].repeat_interleave(torch.tensor(counts, device="cuda")).long()
        ahead = torch.randint(0, 5000, (n,), generator=g, device="cuda") + s["start"]
        s["positions"] = (ahead.repeat_interleave(torch.tensor(counts, device="cuda")) + j).int()
        top += 5000
    half = c["rot"] // 2
    angle = torch.arange(top, device="cuda", dtype=torch.float64)[:, None] * 5e5 ** (-torch.arange(half, device="cuda", dtype=torch.float64) / half)
    s["cos_sin"] = torch.cat((angle.cos(), angle.sin()), dim=1).float()
    if own:
        from paper_2608_28911_gb300 import semkv
        s["cache"] = semkv.KV4Cache.over(s["pages"], s["table"], s["length"], s["refs"], D, s["k_scale"], s["v_scale"])
        s["batch"] = semkv.KV4Batch(n, cu=s["cu"], start=s["start"], total=total, max_count=max(counts))
        s["rotation"] = semkv.KV4Rotation(s["cos_sin"], pairs=c["pairs"])
    return s


def _done(c):
    rng = random.Random(c["vocab"] * 17 + c["beams"])
    return [rng.random() < c["done"] for _ in range(c["groups"] * c["beams"])]


def _prepare_select(c, seed):
    rows, V = c["groups"] * c["beams"], c["vocab"]
    g = _gen(seed, 2)
    s = {"case": c, "end": V // 3}
    # a projection onto a padded vocabulary; some tokens are far likelier than the others, the same
    # for all beams of a group in part
    store = torch.empty((rows, V + c["pad"]), dtype=TYPES[c["type"]], device="cuda")
    shared = torch.randn((c["groups"], V + c["pad"]), generator=g, device="cuda")
    for i in range(c["groups"]):
        x = torch.randn((c["beams"], V + c["pad"]), generator=g, device="cuda") + shared[i]
        store[i * c["beams"]:(i + 1) * c["beams"]] = x * (c["width"] / math.sqrt(2))
    s["logits"] = store[:, :V]
    if c["banned"]:
        ban = torch.rand(V, generator=g, device="cuda") < c["banned"]
        s["logits"][:, ban] = -math.inf
    s["scores"] = torch.rand((c["groups"], c["beams"]), generator=g, device="cuda") * -6.0 - 2.0
    if c["first"]:
        s["scores"][:, 1:] = -math.inf
        s["scores"][:, 0] = 0.0
    s["done"] = torch.tensor(_done(c), device="cuda").byte() if c["done"] else None
    for name, dtype in (("parent", torch.int32), ("token", torch.int32), ("score", torch.float32)):
        s[name] = torch.empty((c["groups"], c["k"]), dtype=dtype, device="cuda")
    if own:
        from paper_2608_28911_gb300 import semkv
        s["ws"] = semkv.beam_select_workspace(s["logits"], s["scores"], c["k"])
    return s


def _prepare_reorder(c, seed):
    g = _gen(seed, 3)
    B, groups, tails = c["beams"], c["groups"], _tails(c)
    m = B * groups  # saved branches (or the beams themselves), then, with saved ones, the beams
    n = 2 * m if c["saved"] else m
    shared = c["past"] // c["page"]  # whole pages of a prompt, which its branches share
    need = [_pages(c, c["past"] + t) - shared for t in tails]
    pages = groups * shared + sum(need) + 3
    order = torch.randperm(pages, generator=g, device="cuda").int()
    wide = shared + max(need)
    table = torch.full((n, wide), -1, dtype=torch.int32, device="cuda")
    refs = torch.zeros(pages, dtype=torch.int32, device="cuda")
    prompt = order[:groups * shared].view(groups, shared)
    table[:m, :shared] = prompt.repeat_interleave(B, dim=0)
    refs[prompt.reshape(-1).long()] = B
    at = groups * shared
    for i, k in enumerate(need):
        table[i, shared:shared + k] = order[at:at + k]
        at += k
    refs[order[groups * shared:at].long()] = 1
    length = torch.zeros(n, dtype=torch.int32, device="cuda")
    length[:m] = _ints([c["past"] + t for t in tails])
    s = {"case": c, "table": table, "length": length, "refs": refs}
    s["seqs"] = torch.randperm(n, generator=g, device="cuda").int() if c["saved"] else torch.arange(n, dtype=torch.int32, device="cuda")
    place = s["seqs"].argsort()  # where a sequence stands in the list
    first = torch.arange(m, device="cuda") // B * B
    s["parent"] = []
    for _ in range(2):
        parent = torch.arange(n, dtype=torch.int32, device="cuda")
        if c["saved"]:
            pick = first + torch.randint(0, B, (m,), generator=g, device="cuda")
            parent[place[m:]] = place[pick].int()
        else:
            by = torch.randint(1, B, (groups,), generator=g, device="cuda").repeat_interleave(B)
            parent = (first + (torch.arange(m, device="cuda") - first + by) % B).int()
        s["parent"].append(parent)
    if own:
        from paper_2608_28911_gb300 import semkv
        pool = torch.zeros((1, pages, 1, c["page"] // 16, 1152), dtype=torch.uint8, device="cuda")
        s["cache"] = semkv.KV4Cache.over(pool, table, length, refs, 64)
        s["ws"] = s["cache"].pages_workspace(n, 0)
    return s


def prepare(c, seed):
    return {"append": _prepare_append, "select": _prepare_select, "reorder": _prepare_reorder}[c["kind"]](c, seed)


# ------------------------------------------------- the framework's operators ------

def _run_own(s):
    from paper_2608_28911_gb300 import semkv
    kind = s["case"]["kind"]
    if kind == "append":
        semkv.semkv_kv4_write_rotated(s["cache"], s["batch"], 0, s["rotation"], s["k"], s["v"], s["q"], s["q_out"], positions=s["positions"])
        semkv.semkv_kv4_read(s["cache"], s["batch"], 0, s["k_out"], s["v_out"])
        return {"q": s["q_out"], "k": s["k_out"], "v": s["v_out"]}
    if kind == "select":
        semkv.semkv_beam_select(s["logits"], s["scores"], s["parent"], s["token"], s["score"], s["ws"], done=s["done"], end_token=s["end"])
        return {"parent": s["parent"], "token": s["token"], "score": s["score"]}
    for parent in s["parent"]:
        semkv.semkv_kv4_reorder(s["cache"], s["seqs"], parent, s["ws"])
    return {k: s[k] for k in ("table", "length", "refs")}


# ------------------------------------------------------------ the plain form ------

def _turn(x, cos, sin, c):
    """x [rows][heads][D] in 32 bits, its first dims turned by the rows' angles."""
    rot = c["rot"]
    y = x.float()
    if c["pairs"]:
        a, b = y[..., 0:rot:2], y[..., 1:rot:2]
    else:
        a, b = y[..., :rot // 2], y[..., rot // 2:rot]
    c1, s1 = cos[:, None], sin[:, None]
    first, second = a * c1 - b * s1, b * c1 + a * s1
    head = torch.stack((first, second), dim=-1).flatten(-2) if c["pairs"] else torch.cat((first, second), dim=-1)
    return torch.cat((head, y[..., rot:]), dim=-1)


def _grid_codes(y):
    """e2m1 codes of quotients: nearest, ties to the even code."""
    a = y.abs()
    code = (a > 0.25).byte() + (a >= 0.75).byte() + (a > 1.25).byte() + (a >= 1.75).byte()
    code = code + (a > 2.5).byte() + (a >= 3.5).byte() + (a > 5.0).byte()
    return code + 8 * (y < 0).byte()


def _pack(x, g):
    """Rows [rows][H][D] in 32 bits to codes [rows][H][D / 2] and scales [rows][H][D / 16], as bytes."""
    x = x.unflatten(-1, (-1, 16))
    g = g.view(-1, 1)
    scale = (x.abs().amax(-1) / (6 * g)).clamp(max=448.0).to(torch.float8_e4m3fn)
    step = scale.float() * g
    code = _grid_codes(torch.where(step[..., None] > 0, x / step[..., None], 0.0)).flatten(-2)
    return code[..., 0::2] + 16 * code[..., 1::2], scale.view(torch.uint8)


def _unpack(codes, scales, g):
    half = torch.tensor((0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0), device="cuda")
    grid = torch.cat((half, -half))
    code = torch.stack((codes & 15, codes >> 4), dim=-1).flatten(-2)
    x = grid[code.int()].unflatten(-1, (-1, 16)) * scales.view(torch.float8_e4m3fn).float()[..., None]
    return x.flatten(-2) * g[:, None]


def _plain_append(s):
    c = s["case"]
    D, P = c["head_dim"], c["page"]
    counts = s["cu"][1:] - s["cu"][:-1]
    i = torch.repeat_interleave(torch.arange(c["n"], device="cuda"), counts, output_size=s["total"])
    place = s["start"][i] + torch.arange(s["total"], device="cuda") - s["cu"][i]
    position = place if s["positions"] is None else s["positions"]
    cos, sin = s["cos_sin"][position.long()].chunk(2, dim=1)
    page, tile, row = s["table"][i, place // P].long(), place % P // 16, place % 16
    a, b = 8 * D, 16 * D
    parts = [x.unflatten(-1, (16, -1)) for x in (s["pages"][0][..., :a], s["pages"][0][..., a:b], s["pages"][0][..., b:b + D], s["pages"][0][..., b + D:])]
    got = {"q": _turn(s["q"], cos, sin, c).to(s["q"].dtype)}
    rows = {"k": _turn(s["k"], cos, sin, c), "v": s["v"].float()}
    for name, codes, scales, g in (("k", parts[0], parts[2], s["k_scale"][0]), ("v", parts[1], parts[3], s["v_scale"][0])):
        codes[page, :, tile, row], scales[page, :, tile, row] = _pack(rows[name], g)
        got[name] = _unpack(codes[page, :, tile, row], scales[page, :, tile, row], g).to(s["k"].dtype)
    return got


def _plain_select(s):
    c = s["case"]
    groups, beams, k = c["groups"], c["beams"], c["k"]
    x = s["logits"].double()
    if s["done"] is not None:
        over = s["done"].bool()[:, None]
        x = torch.where(over, torch.where(torch.arange(c["vocab"], device="cuda") == s["end"], 0.0, -math.inf), x)
    top = x.amax(1, keepdim=True)
    x = x - (x - top).exp_().sum(1, keepdim=True).log_().add_(top)
    x = (x.view(groups, beams, -1) + s["scores"].double()[..., None]).flatten(1)
    best, at = x.sort(dim=1, descending=True, stable=True)
    want = min(k, x.shape[1])
    best, at = best[:, :want], at[:, :want]
    none = best == -math.inf
    beam = at // c["vocab"] + torch.arange(groups, device="cuda")[:, None] * beams
    s["parent"].fill_(-1)[:, :want] = torch.where(none, -1, beam).int()
    s["token"].fill_(-1)[:, :want] = torch.where(none, -1, at % c["vocab"]).int()
    s["score"].fill_(-math.inf)[:, :want] = best.float()
    return {"parent": s["parent"], "token": s["token"], "score": s["score"]}


def _count(s, table, length, by):
    used = (length + s["case"]["page"] - 1) // s["case"]["page"]
    held = torch.arange(table.shape[1], device="cuda") < used[:, None]
    pages = table[held].long()
    s["refs"].index_add_(0, pages, torch.full_like(table[held], by))
    return held


def _plain_reorder(s):
    rows = s["seqs"].long()
    for parent in s["parent"]:
        table, length = s["table"][rows], s["length"][rows]
        _count(s, table, length, -1)
        after, tokens = table[parent.long()], length[parent.long()]
        held = _count(s, after, tokens, 1)
        s["table"][rows] = torch.where(held, after, table)
        s["length"][rows] = tokens
    return {k: s[k] for k in ("table", "length", "refs")}


def run(s):
    if own:
        return _run_own(s)
    return {"append": _plain_append, "select": _plain_select, "reorder": _plain_reorder}[s["case"]["kind"]](s)


# ------------------------------------------------ the definition, in 64 bits ------

def _exact_grid(x, g):
    """What turned rows [rows][H][D] in 64 bits are stored as: each number the nearest of its grid."""
    x = x.reshape(*x.shape[:-1], -1, 16)
    g = g.double()[:, None, None]
    t = x.abs().max(-1, keepdim=True).values / (6 * g)
    ulp = torch.exp2(torch.floor(torch.log2(t.clamp(min=2.0 ** -6, max=448.0))) - 3)
    scale = (torch.round(t / ulp) * ulp).clamp(max=448.0)
    y = x / torch.where(scale > 0, scale * g, torch.ones_like(scale))
    a = y.abs()
    step = torch.where(a < 2, 0.5, torch.where(a < 4, 1.0, 2.0)).double()
    v = (torch.round(a / step) * step).clamp(max=6.0) * torch.sign(y)
    return torch.where(scale > 0, v * scale * g, torch.zeros_like(v)).flatten(-2)


def _exact_append(c, s):
    rot, where = c["rot"], s["positions"]
    if where is None:
        where = torch.cat([torch.arange(b, device="cuda") + a for a, b in zip(s["start"].tolist(), s["counts"])])
    angle = torch.view_as_complex(s["cos_sin"].double()[where.long()].unflatten(1, (2, -1)).transpose(1, 2).contiguous())[:, None]
    order = torch.arange(rot, device="cuda")
    order = order.view(-1, 2) if c["pairs"] else order.view(2, -1).t()  # the dims of each pair

    def turned(x):
        y = x.double()
        y[..., order] = torch.view_as_real(torch.view_as_complex(y[..., order].contiguous()) * angle)
        return y

    return {"q": turned(s["q"]), "k": _exact_grid(turned(s["k"]), s["k_scale"][0]), "v": _exact_grid(s["v"].double(), s["v_scale"][0])}


def exact(c, seed):
    if c["kind"] == "reorder":
        return None
    s = prepare(c, seed)
    if c["kind"] == "append":
        return _exact_append(c, s)
    best = torch.full((c["groups"], c["k"]), -math.inf, dtype=torch.float64, device="cuda")
    over = None if s["done"] is None else s["done"].view(c["groups"], c["beams"]).bool()
    for i in range(c["groups"]):
        rows = s["logits"][i * c["beams"]:(i + 1) * c["beams"]].double()
        x = torch.log_softmax(rows, dim=1) + s["scores"][i].double()[:, None]
        if over is not None:
            x = torch.cat((x[~over[i]].reshape(-1), s["scores"][i].double()[over[i]]))
        x = x.reshape(-1)
        x = torch.where(x.isnan(), -math.inf, x)
        want = min(c["k"], x.numel())
        best[i, :want] = x.topk(want).values
    return {"parent": None, "token": None, "score": best}
