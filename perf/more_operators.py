"""Cases of the operators around a KV cache's attention that its speed is judged by.

Each case is one pass through an operator, as a serving loop makes it next to
the cache's other ones: norms of queries and keys with the rotation of their
positions, attention of trees of drafted tokens, keeping a tree's accepted
path, adding up the attention weight of every cached token, and pruning
contexts by it. Where ``own`` is false, ``run`` computes the operators in
elementary torch operations on the same buffers.

The cache: ``data`` holds num_pages pages; a page holds, for every layer, K
then V, for every KV head, page tokens of 8-bit codes in tiles of 16 tokens (a
K tile as [dim / 16][16 tokens][16 channels], a V tile as [dim][16 tokens]);
``scale`` [num_pages, layers, 2, kv_heads] float32 is what a code is multiplied
by. ``book`` is one int32 buffer of four parts, each padded to 64 entries: the
live bits of the pages, their reference counts, the sequences' lengths and
their page tables.
"""

import json
import math
import random

import torch

own = False

DEV = "cuda"
TOP = {"int8": 127.0, "fp8": 448.0}
EPS = 1e-6


def listed():
    """The cases; each states what in real use it is."""
    return [
        # The next token of one user, far into a context: latency counts.
        dict(name="rotate_tick", kind="rotate", tokens=1, heads=32, kv_heads=8, dim=128, rot=128,
             pairs=False, norm=True, dtype="bf16", far=100000),
        # A decode step: a token of each request; half of each head's channels rotate, in
        # neighbouring pairs, without norms.
        dict(name="rotate_step", kind="rotate", tokens=251, heads=16, kv_heads=16, dim=64, rot=32,
             pairs=True, norm=False, dtype="f16", far=8192),
        # The prompts of a prefill step.
        dict(name="rotate_prompt", kind="rotate", tokens=16384, heads=32, kv_heads=8, dim=128,
             rot=128, pairs=False, norm=True, dtype="bf16", far=32768),
        # One user's tree of a dozen drafted tokens over a short context.
        dict(name="tree_tick", kind="tree", seqs=1, new_low=13, new_high=13, len_low=777,
             len_high=777, heads=32, kv_heads=8, dim=128, page=64, layers=2, format="int8",
             dtype="bf16"),
        # A batch of requests with small trees over contexts of very different lengths.
        dict(name="tree_batch", kind="tree", seqs=64, new_low=5, new_high=24, len_low=64,
             len_high=8192, heads=32, kv_heads=8, dim=128, page=32, layers=1, format="fp8",
             dtype="f16"),
        # Wide trees over long contexts.
        dict(name="tree_wide", kind="tree", seqs=8, new_low=57, new_high=64, len_low=8192,
             len_high=32768, heads=32, kv_heads=8, dim=128, page=64, layers=1, format="int8",
             dtype="bf16"),
        # The accepted paths of a few trees.
        dict(name="accept_small", kind="accept", seqs=4, new_low=13, new_high=13, len_low=100,
             len_high=2000, kv_heads=8, dim=128, page=64, layers=2, format="int8"),
        # Those of a batch, in all layers of a model.
        dict(name="accept_batch", kind="accept", seqs=64, new_low=16, new_high=64, len_low=64,
             len_high=2048, kv_heads=8, dim=128, page=64, layers=32, format="fp8"),
        # What a decode step of ragged requests looks at.
        dict(name="weigh_step", kind="weigh", seqs=251, new_low=1, new_high=1, len_low=16,
             len_high=4096, heads=32, kv_heads=8, dim=128, page=64, layers=1, format="fp8",
             dtype="f16"),
        # What the last queries of long prompts look at.
        dict(name="weigh_window", kind="weigh", seqs=4, new_low=32, new_high=32, len_low=8192,
             len_high=32768, heads=32, kv_heads=8, dim=128, page=64, layers=1, format="int8",
             dtype="bf16"),
        # A few requests are held to a small context.
        dict(name="prune_small", kind="prune", seqs=8, len_low=200, len_high=1200, budget=256,
             sinks=4, recent=32, kv_heads=8, dim=128, page=64, layers=2, format="fp8"),
        # Long contexts give up most of their tokens to make room for others.
        dict(name="prune_large", kind="prune", seqs=32, len_low=2048, len_high=16384, budget=2000,
             sinks=4, recent=512, kv_heads=8, dim=128, page=64, layers=4, format="int8"),
    ]


def _log(rng, low, high):
    """An integer spread over the logarithm of [low, high]."""
    x = low * (high / low) ** rng.random()
    return max(low, min(high, int(round(x))))


def draw(rng):
    """One more case of the same ranges."""
    kind = rng.choice(["rotate", "tree", "tree", "accept", "weigh", "weigh", "prune"])
    kvh, dim = rng.choice([1, 2, 4, 5, 8]), rng.choice([64, 128, 128, 256])
    heads = kvh * rng.choice([1, 2, 3, 4, 6, 8])
    c = dict(kind=kind, kv_heads=kvh, dim=dim)
    if kind == "rotate":
        most = 16384 * 40 * 128 // ((heads + kvh) * dim)
        c.update(tokens=_log(rng, 1, min(most, 65536)), heads=heads,
                 rot=rng.choice([dim, dim, dim // 2, 16 * rng.randint(1, dim // 16)]),
                 pairs=rng.random() < 0.3, norm=rng.random() < 0.7,
                 dtype=rng.choice(["bf16", "f16"]), far=_log(rng, 1, 1 << 30))
        return c
    c.update(page=rng.choice([16, 32, 64, 64, 128, 256]), format=rng.choice(["int8", "fp8"]))
    if kind in ("tree", "weigh"):
        c.update(heads=heads, dtype=rng.choice(["bf16", "f16"]), layers=rng.randint(1, 2))
    if kind == "tree":
        c.update(new_high=_log(rng, 1, 96), len_high=_log(rng, 64, 65536))
        c["new_low"] = rng.randint(1, c["new_high"])
        c["len_high"] = max(c["len_high"], c["new_high"])
        room = (1 << 17) * 8 // (kvh * dim // 128 + 1) // max(1, c["new_high"] * heads // 512)
        c["len_high"] = max(c["new_high"], min(c["len_high"], room // 2))
        c["seqs"] = _log(rng, 1, max(1, min(128, room // c["len_high"])))
        c["len_low"] = max(c["new_high"], c["len_high"] // rng.choice([1, 2, 16]))
    elif kind == "weigh":
        new = rng.choice([1, 1, _log(rng, 2, 64)])
        c.update(new_low=max(1, new // 2), new_high=new, len_high=_log(rng, 64, 131072))
        room = (1 << 17) * 8 // (kvh * dim // 128 + 1) // max(1, new * heads // 256)
        c["len_high"] = max(new, min(c["len_high"], room // 2))
        c["seqs"] = _log(rng, 1, max(1, min(256, room // c["len_high"])))
        c["len_low"] = max(new, c["len_high"] // rng.choice([1, 2, 16]))
    elif kind == "accept":
        c.update(new_high=_log(rng, 2, 96), layers=_log(rng, 1, 32), len_high=_log(rng, 100, 8192))
        c["new_low"] = rng.randint(1, c["new_high"])
        c["len_low"] = c["new_high"]
        size = 2 * kvh * dim * c["layers"]
        c["seqs"] = _log(rng, 1, max(1, min(96, (1 << 31) // (size * c["len_high"]))))
    else:
        c.update(layers=rng.randint(1, 4), len_high=_log(rng, 32, 32768),
                 sinks=rng.choice([0, 1, 4, 16]))
        c["len_low"] = max(1, c["len_high"] // rng.choice([1, 4, 16]))
        c["budget"] = _log(rng, 1, max(1, min(c["len_high"], 4096)))
        c["recent"] = rng.choice([0, 1, c["budget"] // 4, c["budget"] // 2])
        size = 2 * kvh * dim * c["layers"]
        most = min((1 << 31) // (size * c["len_high"]), (1 << 29) // (size * c["budget"]))
        c["seqs"] = _log(rng, 1, max(1, min(128, most)))
    return c


def _plan(case):
    """The lengths and trees of a case (one rng per case, so that its work is known)."""
    rng = random.Random(json.dumps({k: v for k, v in case.items() if k != "name"}, sort_keys=True))
    n, pt = case["seqs"], case["page"]
    p = dict(lens=[_log(rng, case["len_low"], case["len_high"]) for _ in range(n)])
    if "new_high" in case:
        p["new"] = [min(rng.randint(case["new_low"], case["new_high"]), m) for m in p["lens"]]
    if case["kind"] in ("tree", "accept"):
        # a drafted token continues one of the few before it, or the context
        p["parents"] = [[-1 if j == 0 or rng.random() < 0.15 else rng.randint(max(0, j - 4), j - 1)
                         for j in range(m)] for m in p["new"]]
    if case["kind"] == "accept":  # the path to one of the tokens, or none of them
        p["path"] = []
        for m, parent in zip(p["new"], p["parents"]):
            j, path = rng.randint(-1, m - 1), []
            while j >= 0:
                path.append(j)
                j = parent[j]
            p["path"].append(path[::-1])
    p["max_blocks"] = -(-max(p["lens"]) // pt) + 1
    p["pages"] = sum(-(-m // pt) for m in p["lens"]) + 3
    return p


def _pad(n):
    return -(-n // 64) * 64


def _parts(book, pages, slots, max_blocks):
    """(live, refs, lens, tables) views of the flat book."""
    words = -(-pages // 32)
    a = _pad(words)
    b = a + _pad(pages)
    c = b + _pad(slots)
    return (book[:words], book[a:a + pages], book[b:b + slots],
            book[c:c + slots * max_blocks].view(slots, max_blocks))


def _set_live(live, refs):
    """The live bits of the pages, 32 to a word."""
    bits = torch.zeros(live.numel() * 32, dtype=torch.int64, device=refs.device)
    bits[:refs.numel()] = (refs > 0).to(torch.int64)
    live.copy_(_words(bits.view(-1, 32)))


def _words(bits):
    """int32 words of [..., 32] bits."""
    word = (bits.to(torch.int64) << torch.arange(32, device=bits.device)).sum(-1)
    return torch.where(word >= 1 << 31, word - (1 << 32), word).to(torch.int32)


def _codes(n, fmt, gen):
    """n codes as bytes, of values spread like keys and values are."""
    out = torch.empty(n, dtype=torch.uint8, device=DEV)
    for part in out.split(1 << 28):
        x = torch.randn(part.numel(), generator=gen, device=DEV)
        if fmt == "int8":
            part.copy_(x.mul_(32).round_().clamp_(-127, 127).to(torch.int8).view(torch.uint8))
        else:
            part.copy_(x.mul_(110).clamp_(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8))
    return out


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device=DEV)


def _type(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float16


def prepare(case, seed):
    gen = torch.Generator(device=DEV)
    gen.manual_seed(seed * 2 + 1)
    kvh, dim = case["kv_heads"], case["dim"]
    if case["kind"] == "rotate":
        t, heads, rot = case["tokens"], case["heads"], case["rot"]
        # the projections' output: queries, keys and values are slices of its rows
        x = torch.randn(t, (heads + 2 * kvh) * dim, generator=gen, device=DEV)
        x[:, ::29] *= 5  # a few channels are much larger than the others
        x = x.to(_type(case))
        s = dict(case=case, q=x[:, :heads * dim].view(t, heads, dim),
                 k=x[:, heads * dim:(heads + kvh) * dim].view(t, kvh, dim))
        s["positions"] = torch.randint(0, case["far"], (t,), generator=gen, device=DEV,
                                       dtype=torch.int32)
        i = torch.arange(rot // 2, device=DEV, dtype=torch.float64)
        s["inv_freq"] = (1e6 ** (-2 * i / rot)).float()
        w = torch.randn(2, dim, generator=gen, device=DEV) * 0.2 + 1
        s["q_weight"], s["k_weight"] = (w[0], w[1]) if case["norm"] else (None, None)
        s["q_out"] = torch.empty(t, heads, dim, dtype=x.dtype, device=DEV)
        s["k_out"] = torch.empty(t, kvh, dim, dtype=x.dtype, device=DEV)
        return s
    p = _plan(case)
    pages, mb, pt, n = p["pages"], p["max_blocks"], case["page"], case["seqs"]
    layers, fmt = case["layers"], case["format"]
    s = dict(case=case, plan=p, layer=layers - 1)
    s["data"] = _codes(pages * layers * 2 * kvh * pt * dim, fmt, gen).view(pages, -1)
    s["scale"] = torch.exp(torch.randn(pages, layers, 2, kvh, generator=gen, device=DEV) * 0.3)
    s["scale"] /= 32 if fmt == "int8" else 110
    # a pool in use: the sequences' pages lie anywhere in it
    book = torch.zeros(_pad(-(-pages // 32)) + _pad(pages) + _pad(n) + n * mb, dtype=torch.int32,
                       device=DEV)
    live, refs, lens, tables = _parts(book, pages, n, mb)
    host = torch.full((n, mb), -1, dtype=torch.int32)
    perm = torch.randperm(pages, generator=gen, device=DEV).to(torch.int32).cpu()
    at = 0
    for i, m in enumerate(p["lens"]):
        nb = -(-m // pt)
        host[i, :nb] = perm[at:at + nb]
        at += nb
    tables.copy_(host)
    lens.copy_(_i32(p["lens"]))
    refs[perm[:at].long().to(DEV)] = 1
    _set_live(live, refs)
    s["book"], s["seqs"] = book, _i32(list(range(n)))
    if case["kind"] in ("accept", "prune"):
        s["work"] = book.clone()  # the step can be taken back: it works on a copy
    if "new" in p:
        cu = [0]
        for m in p["new"]:
            cu.append(cu[-1] + m)
        s["cu"] = None if case["new_high"] == 1 and case["kind"] != "tree" else _i32(cu)
        s["new"] = _i32(p["new"])
        s["tokens"] = cu[-1]
        if case["kind"] != "accept":
            x = torch.randn(cu[-1], case["heads"] * dim + 64, generator=gen, device=DEV)
            s["q"] = x.to(_type(case))[:, :case["heads"] * dim].view(cu[-1], case["heads"], dim)
    if case["kind"] == "tree":
        s["parents"] = _i32([j for tree in p["parents"] for j in tree])
        s["out"] = torch.empty(layers, cu[-1], case["heads"], dim, dtype=_type(case), device=DEV)
        s["lse"] = torch.empty(layers, cu[-1], case["heads"], device=DEV)
    elif case["kind"] == "accept":
        at = [0]
        for path in p["path"]:
            at.append(at[-1] + len(path))
        s["index"], s["at"] = _i32([j for path in p["path"] for j in path]), _i32(at)
    else:
        # what earlier steps added up: most weight on few tokens
        s["mass"] = torch.exp(2 * torch.randn(n, mb * pt, generator=gen, device=DEV)) / 1000
        s["mass"][torch.arange(mb * pt, device=DEV) >= lens[:, None]] = 0
        s["sums"] = s["mass"].clone()
    if case["kind"] == "weigh":
        x, hide = _scores(s, s["layer"])
        x = x.masked_fill_(hide[:, None, None], -math.inf).double()
        s["lse"] = _unpad(s, torch.logsumexp(x, -1).float().flatten(1, 2).transpose(1, 2))
    if own:
        import paper_2506_12204_amd as ss
        s["cache"] = ss.KVCache(pages, n, mb, layers=layers, kv_heads=kvh, head_dim=dim,
                                page_tokens=pt, format=ss.KV_INT8 if fmt == "int8" else ss.KV_FP8,
                                data=s["data"], scale=s["scale"], book=s.get("work", book))
    return s


# ---- the plain forms, over all sequences at once ---------------------------


def _plain_rotate(s):
    c = s["case"]
    rot = c["rot"]
    angle = s["positions"].double()[:, None] * s["inv_freq"].double()
    cos, sin = torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]
    out = []
    for x, w in ((s["q"], s["q_weight"]), (s["k"], s["k_weight"])):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + EPS) * w
        if c["pairs"]:
            a, b = y[..., 0:rot:2], y[..., 1:rot:2]
            turned = torch.stack((a * cos - b * sin, b * cos + a * sin), -1).flatten(-2)
        else:
            a, b = y[..., :rot // 2], y[..., rot // 2:rot]
            turned = torch.cat((a * cos - b * sin, b * cos + a * sin), -1)
        out.append(torch.cat((turned, y[..., rot:]), -1).to(x.dtype))
    return dict(q=out[0], k=out[1])


def _number(codes, fmt):
    return codes.view(torch.int8 if fmt == "int8" else torch.float8_e4m3fn).float()


def _views(s):
    p = s["plan"]
    return _parts(s.get("work", s["book"]), p["pages"], s["case"]["seqs"], p["max_blocks"])


def _held(s, layer, which):
    """[seqs, kv_heads, longest, dim] keys or values of all sequences (float32)."""
    c = s["case"]
    pt, dim, kvh = c["page"], c["dim"], c["kv_heads"]
    pages = _views(s)[3].clamp(min=0).long()
    raw = s["data"].view(-1, c["layers"], 2, kvh, pt * dim)[pages, layer, which]
    n, nb = pages.shape
    if which == 0:
        x = _number(raw, c["format"]).view(n, nb, kvh, pt // 16, dim // 16, 16, 16)
        x = x.transpose(4, 5).reshape(n, nb, kvh, pt, dim)
    else:
        x = _number(raw, c["format"]).view(n, nb, kvh, pt // 16, dim, 16)
        x = x.transpose(4, 5).reshape(n, nb, kvh, pt, dim)
    x = x * s["scale"][pages, layer, which][..., None, None]
    return x.transpose(1, 2).reshape(n, kvh, nb * pt, dim)


def _row(s):
    """([seqs, most] row of q of each sequence's new tokens, whether there is one)."""
    new = s["new"].long()
    j = torch.arange(s["case"]["new_high"], device=DEV)
    there = j < new[:, None]
    return torch.where(there, (new.cumsum(0) - new)[:, None] + j, 0), there


def _unpad(s, x):
    """[seqs, most, ...] as rows of q."""
    return x[_row(s)[1]].contiguous()


def _scores(s, layer):
    """([seqs, kv_heads, group, most, longest] scores, which of them are hidden [seqs, most,
    longest] where each new token sees those up to its own)."""
    c = s["case"]
    n, kvh, dim, group = c["seqs"], c["kv_heads"], c["dim"], c["heads"] // c["kv_heads"]
    row, there = _row(s)
    q = s["q"][row].float().view(n, -1, kvh, group, dim).permute(0, 2, 3, 1, 4)
    k = _held(s, layer, 0).transpose(2, 3).contiguous()
    x = torch.matmul(q.reshape(n, kvh, -1, dim), k).mul_(dim ** -0.5)
    lens = _views(s)[2].long()
    pos = (lens - s["new"])[:, None] + torch.arange(row.shape[1], device=DEV)
    hide = torch.arange(k.shape[3], device=DEV) > pos[..., None]
    return x.view(n, kvh, group, row.shape[1], -1), hide | ~there[..., None]


def _ancestors(s):
    """[seqs, most, most]: whether token j is token i or one that it continues."""
    row, there = _row(s)
    parent = s["parents"].long()[row]
    m = row.shape[1]
    step = torch.eye(m, device=DEV) + ((parent[..., None] == torch.arange(m, device=DEV))
                                       & there[..., None]).float()
    far = 1
    while far < m:  # paths of twice the length
        step = (torch.matmul(step, step) > 0).float()
        far *= 2
    return step > 0


def _plain_tree(s):
    c = s["case"]
    seen = _ancestors(s)
    n, m, _ = seen.shape
    lens, new = _views(s)[2].long(), s["new"].long()
    words = -(-c["new_high"] // 32)
    bits = torch.zeros(n, m, words * 32, dtype=torch.bool, device=DEV)
    bits[..., :m] = seen
    mask = _unpad(s, _words(bits.view(n, m, words, 32)))
    positions = _unpad(s, (lens - new)[:, None] + seen.sum(-1) - 1).to(torch.int32)
    for layer in range(c["layers"]):
        x, hide = _scores(s, layer)
        first = (lens - new)[:, None]  # of the drafted keys
        local = torch.arange(x.shape[-1], device=DEV) - first
        drafted = (local >= 0) & (local < new[:, None])
        other = torch.gather(~seen, 2, local.clamp(0, m - 1)[:, None].expand(-1, m, -1))
        hide = torch.where(drafted[:, None], other, (local >= 0)[:, None])
        x.masked_fill_(hide[:, None, None], -math.inf)
        top = x.amax(-1, keepdim=True)
        x = torch.exp(x.sub_(top))
        total = x.sum(-1, keepdim=True)
        v = _held(s, layer, 1)
        o = torch.matmul(x.flatten(2, 3), v).view(*x.shape[:-1], -1) / total
        s["out"][layer] = _unpad(s, o.flatten(1, 2).transpose(1, 2)).to(s["out"].dtype)
        lse = (top + torch.log(total))[..., 0].flatten(1, 2).transpose(1, 2)
        s["lse"][layer] = _unpad(s, lse)
    return dict(mask=mask, positions=positions, out=s["out"], lse=s["lse"])


def _plain_weigh(s):
    x, hide = _scores(s, s["layer"])
    row, _ = _row(s)
    n, kvh, group, m, keys = x.shape
    lse = s["lse"][row].view(n, m, kvh, group).permute(0, 2, 3, 1)[..., None]
    x = torch.exp(x.sub_(lse)).masked_fill_(hide[:, None, None], 0)
    s["sums"].copy_(s["mass"])
    s["sums"][:, :keys] += x.sum((1, 2, 3))
    return s["sums"]


def _round(x, fmt):
    if fmt == "int8":
        return x.round().clamp(-127, 127).to(torch.int8).view(torch.uint8)
    return x.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)


def _move(s, src, count):
    """Token t < count[i] of sequence i becomes its token src[i, t]; the rest leaves."""
    c, p = s["case"], s["plan"]
    pt, dim, kvh, fmt = c["page"], c["dim"], c["kv_heads"], c["format"]
    live, refs, lens, tables = _views(s)
    t = torch.arange(src.shape[1], device=DEV)
    first = torch.where((src != t) & (t < count[:, None]), t, src.shape[1]).amin(1)
    moved = (t >= (first // pt * pt)[:, None]) & (t < count[:, None])
    i, to = moved.nonzero(as_tuple=True)
    at = src[i, to]
    page_from, page_to = tables[i, at // pt].long(), tables[i, to // pt].long()
    old = s["scale"][page_from]  # [rows, layers, 2, kv_heads]
    scale = torch.zeros_like(s["scale"])
    scale.scatter_reduce_(0, page_to.view(-1, 1, 1, 1).expand_as(old), old, "amax")
    new = scale[page_to]
    d = s["data"].view(-1, c["layers"], 2, kvh, pt * dim)
    ch = torch.arange(dim, device=DEV)
    for which in (0, 1):
        def place(x):
            x = (x % pt)[:, None]
            inside = ch // 16 * 256 + x % 16 * 16 + ch % 16 if which == 0 else ch * 16 + x % 16
            return x // 16 * 16 * dim + inside
        codes = d[page_from[:, None], :, which, :, place(at)]  # [rows, dim, layers, kv_heads]
        by = new[:, None, :, which]
        by = torch.where(by > 0, by, torch.ones_like(by))
        codes = _round(_number(codes, fmt) * old[:, None, :, which] / by, fmt)
        d[page_to[:, None], :, which, :, place(to)] = codes
    s["scale"][page_to] = new
    # the pages beyond
    have, want = (lens.long() + pt - 1) // pt, (count + pt - 1) // pt
    col = torch.arange(tables.shape[1], device=DEV)
    gone = (col >= want[:, None]) & (col < have[:, None])
    refs.index_add_(0, tables[gone].long(), torch.full_like(tables[gone], -1))
    tables[gone] = -1
    lens.copy_(count)
    _set_live(live, refs)
    number = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    return dict(book=s["work"], codes=s["data"].view(number), scale=s["scale"])


def _plain_accept(s):
    s["work"].copy_(s["book"])
    lens, new = _views(s)[2].long(), s["new"].long()
    at = s["at"].long()
    kept = at[1:] - at[:-1]
    count = lens - new + kept
    t = torch.arange(int(lens.max()), device=DEV).expand(lens.numel(), -1)
    k = t - (lens - new)[:, None]  # the place among those kept
    drafted = (k >= 0) & (k < kept[:, None])
    where = torch.where(drafted, at[:-1, None] + k, 0)
    index = torch.cat((s["index"].long(), torch.zeros(1, dtype=torch.long, device=DEV)))
    return _move(s, torch.where(drafted, (lens - new)[:, None] + index[where], t), count)


def _plain_prune(s):
    c = s["case"]
    s["work"].copy_(s["book"])
    lens = _views(s)[2].long()
    longest, budget = s["mass"].shape[1], c["budget"]
    t = torch.arange(longest, device=DEV).expand(lens.numel(), -1)
    there = t < lens[:, None]
    a = min(c["sinks"], budget)
    r = min(c["recent"], budget - a)
    always = (t < a) | (t >= (lens - r)[:, None])
    order = torch.where(always, math.inf, s["mass"]).masked_fill(~there, -math.inf)
    order = torch.sort(order, dim=1, descending=True, stable=True)[1]
    kept = torch.zeros_like(there).scatter_(1, order[:, :budget], True)
    kept = torch.where((lens <= budget)[:, None], there, kept & there)
    count = kept.sum(1)
    src = torch.sort((~kept).to(torch.uint8), dim=1, stable=True)[1]
    inside = t < count[:, None]
    s["sums"].copy_(torch.where(inside, torch.gather(s["mass"], 1, src), 0))
    return dict(_move(s, torch.where(inside, src, t), count), mass=s["sums"])


def run(s):
    c = s["case"]
    if not own:
        return {"rotate": _plain_rotate, "tree": _plain_tree, "accept": _plain_accept,
                "weigh": _plain_weigh, "prune": _plain_prune}[c["kind"]](s)
    if c["kind"] == "rotate":
        import paper_2506_12204_amd as ss
        q, k = ss.qk_rotate(s["q"], s["k"], s["positions"], s["inv_freq"], q_weight=s["q_weight"],
                            k_weight=s["k_weight"], eps=EPS, interleaved=c["pairs"],
                            q_out=s["q_out"], k_out=s["k_out"])
        return dict(q=q, k=k)
    cache = s["cache"]
    if c["kind"] == "tree":
        mask, positions = cache.tree(s["parents"], s["seqs"], s["cu"], max_new=c["new_high"])
        for layer in range(c["layers"]):
            cache.attend(layer, s["q"], s["seqs"], s["cu"], tree=mask, max_new=c["new_high"],
                         max_len=c["len_high"], out=s["out"][layer], lse=s["lse"][layer])
        return dict(mask=mask, positions=positions, out=s["out"], lse=s["lse"])
    if c["kind"] == "weigh":
        s["sums"].copy_(s["mass"])
        cache.weigh(s["layer"], s["q"], s["lse"], s["sums"], s["seqs"], s["cu"],
                    max_new=c["new_high"], max_len=c["len_high"])
        return s["sums"]
    s["work"].copy_(s["book"])
    number = torch.int8 if c["format"] == "int8" else torch.float8_e4m3fn
    out = dict(book=s["work"], codes=s["data"].view(number), scale=s["scale"])
    if c["kind"] == "accept":
        cache.keep(s["seqs"], s["new"], s["index"], s["at"])
        return out
    s["sums"].copy_(s["mass"])
    cache.prune(s["sums"], s["seqs"], c["budget"], sinks=c["sinks"], recent=c["recent"])
    return dict(out, mass=s["sums"])


def work(case):
    """What a pass cannot do without: inputs read once, outputs written once."""
    kvh, dim = case["kv_heads"], case["dim"]
    if case["kind"] == "rotate":
        size = case["tokens"] * (case["heads"] + kvh) * dim
        return {"bytes": 4 * size + 4 * case["tokens"], "flops": 8 * size}
    p = _plan(case)
    pt, layers = case["page"], case["layers"]
    if case["kind"] in ("tree", "weigh"):
        heads, size, pairs = case["heads"], 0, 0
        sides = 2 if case["kind"] == "tree" else 1  # keys and values, or keys alone
        for i, (n, m) in enumerate(zip(p["lens"], p["new"])):
            size += sides * kvh * (n * dim + 4 * -(-n // pt)) + (sides * 2 * dim + 4) * heads * m
            if case["kind"] == "weigh":
                size += 8 * n
                pairs += sum(n - m + j + 1 for j in range(m))
                continue
            depth = []
            for j in p["parents"][i]:
                depth.append(1 if j < 0 else depth[j] + 1)
            pairs += m * (n - m) + sum(depth)
        times = layers if case["kind"] == "tree" else 1
        return {"bytes": size * times, "flops": 2 * sides * heads * dim * pairs * times}
    token = 2 * kvh * dim * layers
    if case["kind"] == "accept":
        moved = sum(j != at for path in p["path"] for at, j in enumerate(path))
        return {"bytes": 2 * moved * token + 4 * sum(map(len, p["path"])) + 12 * case["seqs"],
                "flops": 0}
    gone = [n for n in p["lens"] if n > case["budget"]]
    moved = len(gone) * max(0, case["budget"] - case["sinks"])
    return {"bytes": 2 * moved * token + 8 * sum(gone) + 4 * case["seqs"], "flops": 0}


# ---- the definitions in 64 bits --------------------------------------------


def _exact_rotate(case, seed):
    s = prepare(case, seed)
    half = case["rot"] // 2
    turn = torch.polar(torch.ones(case["tokens"], half, dtype=torch.float64, device=DEV),
                       torch.outer(s["positions"].double(), s["inv_freq"].double()))
    out = {}
    for name in ("q", "k"):
        x = s[name].double()
        if case["norm"]:
            length = torch.linalg.vector_norm(x, dim=-1, keepdim=True) ** 2 / case["dim"]
            x = x / torch.sqrt(length + EPS) * s[name + "_weight"].double()
        z = x[..., :2 * half]
        z = z.unflatten(-1, (half, 2)) if case["pairs"] else z.unflatten(-1, (2, half)).mT
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn[:, None])
        z = z if case["pairs"] else z.mT
        out[name] = torch.cat((z.flatten(-2), x[..., 2 * half:]), -1)
    return out


def _values(s, i, layer, which, head):
    """[length, dim] keys or values of one sequence by the layout's arithmetic."""
    c = s["case"]
    pt, dim, kvh = c["page"], c["dim"], c["kv_heads"]
    token = torch.arange(s["plan"]["lens"][i], device=DEV)
    page = _views(s)[3][i].long()[token // pt]
    t, d = (token % pt)[:, None], torch.arange(dim, device=DEV)
    base = ((layer * 2 + which) * kvh + head) * pt * dim + t // 16 * 16 * dim
    inside = d // 16 * 256 + t % 16 * 16 + d % 16 if which == 0 else d * 16 + t % 16
    raw = s["data"].view(-1)[page[:, None] * s["data"].shape[1] + base + inside]
    number = raw.view(torch.int8) if c["format"] == "int8" else raw.view(torch.float8_e4m3fn)
    return number.double() * s["scale"][page, layer, which, head].double()[:, None]


def _exact_tree(case, seed):
    s = prepare(case, seed)
    p, group, layers = s["plan"], case["heads"] // case["kv_heads"], case["layers"]
    out = torch.zeros(layers, s["tokens"], case["heads"], case["dim"], dtype=torch.float64,
                      device=DEV)
    lse = torch.zeros(layers, s["tokens"], case["heads"], dtype=torch.float64, device=DEV)
    lo = 0
    for i, (n, m) in enumerate(zip(p["lens"], p["new"])):
        see = torch.ones(m, n, dtype=torch.bool)
        see[:, n - m:] = False
        for t, j in enumerate(p["parents"][i]):
            if j >= 0:
                see[t, n - m:] = see[j, n - m:]
            see[t, n - m + t] = True
        see = see.to(DEV)
        for layer in range(layers):
            for kh in range(case["kv_heads"]):
                k, v = (_values(s, i, layer, w, kh) for w in (0, 1))
                for h in range(kh * group, (kh + 1) * group):
                    x = s["q"][lo:lo + m, h].double() @ k.T / math.sqrt(case["dim"])
                    x[~see] = -math.inf
                    sums = torch.logsumexp(x, 1)
                    lse[layer, lo:lo + m, h] = sums
                    out[layer, lo:lo + m, h] = (x - sums[:, None]).exp() @ v
        lo += m
    return dict(mask=None, positions=None, out=out, lse=lse)


def _exact_weigh(case, seed):
    s = prepare(case, seed)
    p, group = s["plan"], case["heads"] // case["kv_heads"]
    sums = s["mass"].double()
    lo = 0
    for i, (n, m) in enumerate(zip(p["lens"], p["new"])):
        see = torch.ones(m, n, dtype=torch.bool, device=DEV).tril(n - m)
        for kh in range(case["kv_heads"]):
            k = _values(s, i, s["layer"], 0, kh)
            for h in range(kh * group, (kh + 1) * group):
                x = s["q"][lo:lo + m, h].double() @ k.T / math.sqrt(case["dim"])
                x = torch.where(see, x - s["lse"][lo:lo + m, h, None].double(), -math.inf)
                sums[i, :n] += x.exp().sum(0)
        lo += m
    return sums


def _grid(x, fmt):
    """The nearest value an 8-bit code stands for, ties to the even code."""
    if fmt == "int8":
        return x.round().clamp(-127, 127)
    x = x.clamp(-448, 448)
    step = torch.exp2(torch.floor(torch.log2(x.abs().clamp(min=2.0 ** -6))) - 3)
    return (x / step).round() * step


def _exact_kept(case, s, chosen):
    """The codes (fp8 ones, as numbers) and scales of sequences that keep the tokens
    chosen[i], in order, block by block."""
    kvh, dim, pt, layers, fmt = (case[k] for k in ("kv_heads", "dim", "page", "layers", "format"))
    number = torch.int8 if fmt == "int8" else torch.float8_e4m3fn
    held = s["data"].view(number).double().view(-1, layers, 2, kvh, pt * dim)
    scale = s["scale"].double()
    tables = _views(s)[3].tolist()
    ch = torch.arange(dim, device=DEV)
    for i, tokens in enumerate(chosen):
        first = next((t for t, at in enumerate(tokens) if at != t), len(tokens))
        for b in range(first // pt if first < len(tokens) else 1 << 30, -(-len(tokens) // pt)):
            at = torch.tensor(tokens[b * pt:(b + 1) * pt], device=DEV)
            page = torch.tensor([tables[i][t // pt] for t in tokens[b * pt:(b + 1) * pt]],
                                device=DEV)
            to = scale[page].amax(0)
            for which in (0, 1):
                def inside(t):
                    t = (t % pt)[:, None]
                    k = ch // 16 * 256 + t % 16 * 16 + ch % 16
                    return t // 16 * 16 * dim + (k if which == 0 else ch * 16 + t % 16)
                old = held[page[:, None], :, which, :, inside(at)]
                by = to[:, which]
                x = old * scale[page][:, None, :, which] / torch.where(by > 0, by, 1.0)
                held[tables[i][b], :, which][:, :, inside(torch.arange(at.numel(), device=DEV))] \
                    = _grid(x, fmt).permute(2, 3, 0, 1)
            scale[tables[i][b]] = to
    held = held.view(s["data"].shape)
    return dict(book=None, codes=held if fmt == "fp8" else None, scale=scale)


def _exact_accept(case, seed):
    s = prepare(case, seed)
    p = s["plan"]
    return _exact_kept(case, s, [list(range(n - m)) + [n - m + j for j in path]
                                 for n, m, path in zip(p["lens"], p["new"], p["path"])])


def _exact_prune(case, seed):
    s = prepare(case, seed)
    budget, chosen = case["budget"], []
    mass = s["mass"].tolist()
    for n, row in zip(s["plan"]["lens"], mass):
        if n <= budget:
            chosen.append(list(range(n)))
            continue
        a = min(case["sinks"], budget)
        r = min(case["recent"], budget - a)
        rest = sorted(range(a, n - r), key=lambda t: (-row[t], t))[:budget - a - r]
        chosen.append(sorted([*range(a), *rest, *range(n - r, n)]))
    sums = torch.zeros_like(s["mass"], dtype=torch.float64)
    for i, tokens in enumerate(chosen):
        sums[i, :len(tokens)] = torch.tensor([mass[i][t] for t in tokens], dtype=torch.float64,
                                             device=DEV)
    return dict(_exact_kept(case, s, chosen), mass=sums)


def exact(case, seed):
    """None for pools whose codes would take too long."""
    if case["kind"] in ("accept", "prune"):
        kept = sum(min(n, case.get("budget", n)) for n in _plan(case)["lens"])
        pages = _plan(case)["pages"] * case["page"] * 2 * case["layers"]
        if pages * case["kv_heads"] * case["dim"] > 6 << 30 or kept > 1 << 17:
            return None
    return {"rotate": _exact_rotate, "tree": _exact_tree, "accept": _exact_accept,
            "weigh": _exact_weigh, "prune": _exact_prune}[case["kind"]](case, seed)
