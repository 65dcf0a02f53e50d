"""Operators of a decode step around its attention and its logits, as a serving program calls them.

A layer's projection gives q, k and v; q and k are normalised and turned by their positions; K and V of tokens that stay
are kept in 8 bits, attention reads them there, and a program that moves or keeps a request reads them back; the step ends with tokens
drawn from the logits.  A case is a dict of plain values; its ``op`` says which entry point one pass goes through:

  rope    binding.qk_rope: norms of each head of q and k, and the rotation by the row's position
  store   binding.kv_commit into a cache of 8 bits: K and V of new tokens of every layer, quantised as they are written
  load    binding.kv_read: K and V of tokens of every layer back as rows
  attn    binding.tree_attn over a cache of 8 bits: one token, or a tree of tokens, of each request
  sample  binding.sample: a token for each row of logits; binding.tree_sample: and the branch of each drafted tree that agrees

Layouts: K pages ``[layers][pages][heads][page][dim]``, V pages ``[layers][pages][heads][page / e][dim][e]``, e tokens of one
channel side by side: 8 in 8 and 16 bits, 4 in 32.  In 8 bits (e4m3) an element stands for its value times a power of two, one
for each token and head of K and of V: ``[layers][pages][heads][page]``, as biased exponents (e8m0).  It is the least one at
which no element of the token's head is above 448, but not below 2^-96.  Requests' lengths and trees follow from the case (``mix``),
values from the seed.
"""
from __future__ import annotations

import random

import torch

own = False

DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32, "e4m3": torch.float8_e4m3fn}
# query heads, K/V heads and width of a head of the layers whose shapes the decode step is built for
HEADS = {"7b": (32, 32, 128), "13b": (40, 40, 128), "mistral": (32, 8, 128), "qwen": (28, 4, 128), "tiny": (4, 2, 64)}
UNIT = 2.0 ** 44        # of the weights that tokens are drawn by: the largest one has so many


def listed():
    return [
        # one token of one request, far into a document: the smallest call of every layer, bound by latency
        dict(name="rope one token", op="rope", shape="7b", dtype="bf16", T=1, far=100000, rot=128, inter=0, norm=1, each=0, mix=1),
        # the rows of several prompts, K and V shared by query heads: bound by reading and writing
        dict(name="rope prompts", op="rope", shape="mistral", dtype="bf16", T=19001, far=32768, rot=128, inter=0, norm=1, each=0, mix=2),
        # the accepted branch of one tree, in every layer
        dict(name="store a branch", op="store", shape="7b", layers=32, R=1, nodes=8, page=64, prompt=0, mix=3),
        # a prompt, in every layer
        dict(name="store a prompt", op="store", shape="mistral", layers=32, R=1, nodes=1, page=64, prompt=2357, mix=4),
        # a short prefix that another request shares
        dict(name="load a prefix", op="load", shape="qwen", dtype="e4m3", layers=28, R=1, lo=77, hi=77, page=32, mix=5),
        # two requests that leave the card for a while
        dict(name="load two requests", op="load", shape="mistral", dtype="e4m3", layers=32, R=2, lo=900, hi=2501, page=64, mix=6),
        # one new token, a short conversation
        dict(name="attn8 one token", op="attn", shape="7b", R=1, nodes=1, lo=777, hi=777, page=64, mix=7),
        # one new token each of many requests of very different lengths: what a server does most of the time, bound by reading
        dict(name="attn8 batch ragged", op="attn", shape="mistral", R=24, nodes=1, lo=500, hi=16384, page=64, mix=8),
        # wide trees of several requests over long contexts: bound by the products
        dict(name="attn8 trees of 64", op="attn", shape="qwen", R=4, nodes=64, lo=20000, hi=32768, page=128, mix=9),
        # the next token of one request
        dict(name="sample one token", op="sample", V=32000, dtype="f32", R=1, nodes=0, mix=10),
        # the answers to one drafted tree
        dict(name="sample tree of 8", op="sample", V=32000, dtype="bf16", R=1, nodes=8, mix=11),
        # wide trees of many requests, each with its own settings, over a large vocabulary
        dict(name="sample 16 trees", op="sample", V=152064, dtype="bf16", R=16, nodes=64, mix=12),
    ]


def _log(rng, lo, hi):
    return int(round(lo * (hi / lo) ** rng.random()))


def draw(rng):
    """One more case: any operator, sizes over the whole range of the listed ones, odd ones as a rule."""
    op = rng.choice(["rope", "store", "load", "attn", "attn", "sample", "sample"])
    mix = rng.randrange(1 << 30)
    shape = rng.choice(["7b", "13b", "mistral", "qwen", "tiny"])
    hq, hkv, dim = HEADS[shape]
    page = rng.choice([32, 64, 64, 128, 256])
    if op == "rope":
        dtype = rng.choice(["bf16", "bf16", "f32"])
        most = 19001 * 40 * 128 // ((hq + hkv) * dim) // (2 if dtype == "f32" else 1)
        return dict(op=op, shape=shape, dtype=dtype, T=_log(rng, 1, most), far=_log(rng, 100, 1 << 20), rot=dim // rng.choice([1, 1, 2, 4]),
                    inter=rng.randrange(2), norm=rng.randrange(2), each=rng.randrange(2), mix=mix)
    if op == "store":
        layers = rng.randint(1, 32)
        prompt = rng.choice([0, _log(rng, 30, 2357 * 8 * 128 // (hkv * dim))])
        return dict(op=op, shape=shape, layers=layers, R=1 if prompt else _log(rng, 1, 40), nodes=_log(rng, 1, 48), page=page, prompt=prompt,
                    mix=mix)
    if op == "load":
        dtype, layers, R = rng.choice(["e4m3", "e4m3", "bf16", "f32"]), rng.randint(1, 32), _log(rng, 1, 24)
        hi = _log(rng, 1, max(2, 3500 * 8 * 128 * 32 // (layers * R * hkv * dim * {"e4m3": 1, "bf16": 2, "f32": 4}[dtype])))
        return dict(op=op, shape=shape, dtype=dtype, layers=layers, R=R, lo=rng.choice([0, hi // 2, hi]), hi=hi, page=page, mix=mix)
    if op == "attn":
        nodes, R = rng.choice([1, 1, _log(rng, 1, 64)]), _log(rng, 1, 24)
        # what the largest listed cases read and compute
        most = min(32768, (1 << 27) // (R * hkv * dim), int(1.0e11 / (4 * R * nodes * hq * dim)))
        hi = _log(rng, 16, max(most, 17))
        return dict(op=op, shape=shape, R=R, nodes=nodes, lo=rng.choice([0, hi // 8, hi // 2, hi]), hi=hi, page=page, mix=mix)
    V, dtype = _log(rng, 1000, 152064), rng.choice(["bf16", "f32"])
    nodes = rng.choice([0, _log(rng, 1, 64)])
    return dict(op=op, V=V, dtype=dtype, R=_log(rng, 1, max(2, min(16 if nodes else 700, 75_000_000 // (V * max(nodes, 1))))), nodes=nodes, mix=mix)


# ---- what a case says about lengths and trees (no values) -----------------------------------------------------------------


def _parents(rng, n):
    """A drafted tree: node 0 is the newest certain token, every other node hangs below an earlier one, near the end as a rule."""
    return [-1] + [max(0, j - 1 - int(rng.expovariate(0.4))) for j in range(1, n)]


def _masks(parents):
    """Sets of ancestors and self, as the 64-bit words that hold them (signed)."""
    m = []
    for j, p in enumerate(parents):
        m.append((1 << j) | (m[p] if p >= 0 else 0))
    return [v - (1 << 64) if v >> 63 else v for v in m]


def _lengths(rng, R, lo, hi):
    """R lengths from lo to hi, spread over their logarithm; the first is the longest."""
    return [hi] + [min(hi, max(lo, int((lo + 1) * ((hi + 1) / (lo + 1)) ** rng.random()) - 1)) for _ in range(R - 1)]


def _trees(rng, R, nodes):
    n = [nodes] + [rng.randint(max(1, nodes // 2), nodes) for _ in range(R - 1)]
    return [_parents(rng, k) for k in n]


def _starts(counts):
    at = [0]
    for c in counts:
        at.append(at[-1] + c)
    return at


def _facts(case):
    """Lengths, and trees where the case has any."""
    rng = random.Random(case["mix"])
    lens = _lengths(rng, case["R"], case.get("lo", 0), case.get("hi", 0))
    return lens, _trees(rng, case["R"], case["nodes"]) if case.get("nodes") else []


def _store_facts(case):
    """The cache position of each row of a step (request, position), -1 for a rejected row; and lengths after it."""
    rng = random.Random(case["mix"])
    if case["prompt"]:
        return [(0, i) for i in range(case["prompt"])], [case["prompt"]]
    where, ends = [], []
    for r in range(case["R"]):
        n = rng.randint(max(1, case["nodes"] // 2), case["nodes"])
        a, at = rng.randint(1, n), rng.randint(0, 300)
        kept = set([0] + sorted(rng.sample(range(1, n), a - 1)))
        for j in range(n):
            where.append((r, at) if j in kept else -1)
            at += j in kept
        ends.append(at)
    return where, ends


def _settings(case, rows):
    """Per row: temperature, top_k, top_p, min_p, as the requests of a server ask for them (one request, one setting)."""
    rng = random.Random(case["mix"] + 1)
    each = [rng.choice([(0.8, 0, 0.95, 0.0), (1.0, 0, 1.0, 0.0), (0.7, 50, 0.9, 0.0), (1.2, 0, 1.0, 0.05), (0.6, 20, 0.95, 0.0), (0.0, 0, 1.0, 0.0),
                        (1.0, 1000, 0.99, 0.01)]) for _ in rows]
    each[0] = (0.8, 0, 0.95, 0.0)
    return [s for s, n in zip(each, rows) for _ in range(n)]


# ---- inputs ---------------------------------------------------------------------------------------------------------------


def _gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def _i32(v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


def _f32(v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


def _normal(g, shape, dtype):
    return torch.empty(shape, device="cuda", dtype=dtype).normal_(generator=g)


def _pages(g, layers, pages, page, hkv, dim, name):
    """K and V of a cache, and their scales in 8 bits: elements of about 1, as they are after projections."""
    dtype, e = DTYPES[name], 4 if name == "f32" else 8
    shapes = ((layers, pages, hkv, page, dim), (layers, pages, hkv, page // e, dim, e))
    if name != "e4m3":
        return [_normal(g, s, dtype) for s in shapes] + [None, None]
    values = [_normal(g, s, torch.bfloat16).mul_(110).clamp_(-448, 448).to(dtype) for s in shapes]
    scales = [torch.randint(118, 122, shapes[0][:4], device="cuda", generator=g, dtype=torch.uint8).view(torch.float8_e8m0fnu) for _ in shapes]
    return values + scales


def _table(g, lens, page, spare):
    """Pages of the requests in no order, as they are after a while; entries that no token needs are -1.  (table, pages)"""
    need = [-(-n // page) for n in lens]
    total, width = sum(need), max(max(need), 1)
    pages = total + spare
    ids = torch.randperm(pages, device="cuda", generator=g).to(torch.int32)
    table = torch.full((len(lens), width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for r, n in enumerate(need):
        table[r, :n] = ids[at:at + n]
        at += n
    return table, pages


def _slots(table, where, page):
    """Slots of (request, position) pairs, -1 stays -1."""
    held = table.tolist()
    slots = [-1 if w == -1 else held[w[0]][w[1] // page] * page + w[1] % page for w in where]
    return torch.tensor(slots, dtype=torch.int64, device="cuda")


def prepare(case, seed):
    g = _gen(seed)
    return dict({"rope": _prepare_rope, "store": _prepare_store, "load": _prepare_load, "attn": _prepare_attn,
                 "sample": _prepare_sample}[case["op"]](case, g), op=case["op"])


def _cache(s):
    """The framework's handle of the pages: kept by the program beside them."""
    if "cache" not in s:
        from paper_2603_14110_amd import binding

        s["cache"] = binding.KVCache(s["K"], s["V"], s["K_scale"], s["V_scale"])
    return s["cache"]


def _prepare_rope(case, g):
    hq, hkv, dim = HEADS[case["shape"]]
    T, rot = case["T"], case["rot"]
    # the rows of the projection that makes q, k and v of a token at once
    qkv = _normal(g, (T, hq + 2 * hkv, dim), DTYPES[case["dtype"]])
    last = torch.randint(case["far"], (1,), device="cuda", generator=g)
    places = (last + torch.arange(T, device="cuda") % 4099).to(torch.int32)
    shape = lambda heads: (heads, dim) if case["each"] else (dim,)
    weights = [torch.rand(shape(n), device="cuda", generator=g) + 0.5 if case["norm"] else None for n in (hq, hkv)]
    inv_freq = (10000.0 ** (torch.arange(0, rot, 2, device="cuda", dtype=torch.float64) / -rot)).float()
    return dict(q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], places=places, inv_freq=inv_freq, q_weight=weights[0], k_weight=weights[1],
                eps=1e-6 if case["norm"] else None, inter=bool(case["inter"]))


def _prepare_store(case, g):
    _, hkv, dim = HEADS[case["shape"]]
    where, ends = _store_facts(case)
    table, pages = _table(g, ends, case["page"], 2)
    K, V, K_scale, V_scale = _pages(g, case["layers"], pages, case["page"], hkv, dim, "e4m3")
    shape = (case["layers"], len(where), hkv, dim)
    # keys have a few channels that are much larger than the others
    k = _normal(g, shape, torch.bfloat16) * (1 + 7 * (torch.rand(dim, device="cuda", generator=g) < 0.05)).bfloat16()
    return dict(K=K, V=V, K_scale=K_scale, V_scale=V_scale, k=k, v=_normal(g, shape, torch.bfloat16), slots=_slots(table, where, case["page"]))


def _prepare_load(case, g):
    _, hkv, dim = HEADS[case["shape"]]
    lens, _ = _facts(case)
    table, pages = _table(g, lens, case["page"], 3)
    K, V, K_scale, V_scale = _pages(g, case["layers"], pages, case["page"], hkv, dim, case["dtype"])
    return dict(K=K, V=V, K_scale=K_scale, V_scale=V_scale, slots=_slots(table, [(r, i) for r, n in enumerate(lens) for i in range(n)], case["page"]))


def _prepare_attn(case, g):
    hq, hkv, dim = HEADS[case["shape"]]
    lens, trees = _facts(case)
    table, pages = _table(g, lens, case["page"], 3)
    K, V, K_scale, V_scale = _pages(g, 1, pages, case["page"], hkv, dim, "e4m3")
    starts = _starts([len(t) for t in trees])
    qkv = _normal(g, (starts[-1], hq + 2 * hkv, dim), torch.bfloat16)
    qkv[:, :hq] *= 1.5          # answers that attend to some tokens more than to others
    return dict(K=K, V=V, K_scale=K_scale, V_scale=V_scale, table=table, lens=_i32(lens), starts=_i32(starts),
                tree=torch.tensor(sum((_masks(t) for t in trees), []), dtype=torch.int64, device="cuda"),
                q=qkv[:, :hq], k=qkv[:, hq:hq + hkv], v=qkv[:, hq + hkv:], nodes=case["nodes"], scale=dim ** -0.5)


def _prepare_sample(case, g):
    _, trees = _facts(case)
    rows = [len(t) for t in trees] if trees else [1] * case["R"]
    T, V = sum(rows), case["V"]
    # a wide body, and some tokens that the model thinks likely
    logits = _normal(g, (T, V), DTYPES[case["dtype"]]).mul_(2)
    likely = torch.randint(V // 24, (T, 24), device="cuda", generator=g) + torch.arange(24, device="cuda") * (V // 24)
    logits.scatter_(1, likely, (torch.rand((T, 24), device="cuda", generator=g) * 8 + 6).to(logits.dtype))
    t, k, p, m = zip(*_settings(case, rows))
    s = dict(logits=logits, u=torch.rand(T, device="cuda", generator=g), temperature=_f32(t), top_k=_i32(k), top_p=_f32(p), min_p=_f32(m))
    if not trees:
        return s
    starts = _starts(rows)
    # drafts that are among what the model thinks likely
    flat = torch.tensor([a + max(p, 0) for a, t in zip(starts, trees) for p in t], device="cuda")
    pick = torch.randint(3, (T,), device="cuda", generator=g)
    tokens = logits[flat].gather(1, likely[flat]).float().argsort(1, descending=True).gather(1, pick[:, None])
    return dict(s, tokens=likely[flat].gather(1, tokens)[:, 0].to(torch.int32), starts=_i32(starts), nodes=case["nodes"],
                tree=torch.tensor(sum((_masks(t) for t in trees), []), dtype=torch.int64, device="cuda"))


# ---- one pass -------------------------------------------------------------------------------------------------------------


def run(state):
    return (_OWN if own else _PLAIN)[state["op"]](state)


def _own_rope(s):
    from paper_2603_14110_amd import binding

    q, k = binding.qk_rope(s["q"], s["k"], s["places"], s["inv_freq"], q_weight=s["q_weight"], k_weight=s["k_weight"], eps=s["eps"],
                           interleaved=s["inter"])
    return {"q": q, "k": k}


def _own_store(s):
    from paper_2603_14110_amd import binding

    binding.kv_commit(_cache(s), s["k"], s["v"], s["slots"])
    return {"K": s["K"], "V": s["V"], "K_scale": s["K_scale"], "V_scale": s["V_scale"]}


def _own_load(s):
    from paper_2603_14110_amd import binding

    k, v = binding.kv_read(_cache(s), s["slots"])
    return {"k": k, "v": v}


def _own_attn(s):
    from paper_2603_14110_amd import binding

    out, lse = binding.tree_attn(_cache(s), 0, s["q"], s["k"], s["v"], s["table"], s["lens"], s["starts"], tree=s["tree"],
                                 max_nodes=s["nodes"], scale=s["scale"], want_lse=True)
    return {"out": out, "lse": lse}


def _own_sample(s):
    from paper_2603_14110_amd import binding

    how = dict(temperature=s["temperature"], top_k=s["top_k"], top_p=s["top_p"], min_p=s["min_p"], want_logp=True)
    if "tree" not in s:
        answers, logp = binding.sample(s["logits"], s["u"], **how)
        return {"answers": answers, "logp": logp}
    keep, counts, following, answers, logp = binding.tree_sample(s["logits"], s["u"], s["tokens"], s["starts"], tree=s["tree"],
                                                                 max_nodes=s["nodes"], **how)
    return {"keep": keep, "counts": counts, "next": following, "answers": answers, "logp": logp}


_OWN = {"rope": _own_rope, "store": _own_store, "load": _own_load, "attn": _own_attn, "sample": _own_sample}


def _plain_rope(s):
    angle = s["places"].double()[:, None] * s["inv_freq"].double()
    cos, sin = angle.cos().float()[:, None], angle.sin().float()[:, None]
    half = s["inv_freq"].numel()

    def turned(x, weight):
        y = x.float()
        if s["eps"] is not None:
            y = y * torch.rsqrt(y.square().mean(-1, keepdim=True) + s["eps"])
        if weight is not None:
            y = y * weight
        front, rest = y[..., :2 * half], y[..., 2 * half:]
        if s["inter"]:
            a, b = front[..., 0::2], front[..., 1::2]
            front = torch.stack([a * cos - b * sin, b * cos + a * sin], -1).flatten(-2)
        else:
            a, b = front[..., :half], front[..., half:]
            front = torch.cat([a * cos - b * sin, b * cos + a * sin], -1)
        return torch.cat([front, rest], -1).to(x.dtype)

    return {"q": turned(s["q"], s["q_weight"]), "k": turned(s["k"], s["k_weight"])}


def _plain_quantised(x):
    """Codes and biased exponents of [..., dim]."""
    top = x.float().abs().amax(-1)
    m, e = torch.frexp(top)                             # top = m 2^e, m in [1/2, 1)
    by = torch.where(m > 0.875, e - 8, e - 9).clamp(min=-96)
    by = torch.where(top == 0, -96, by)
    return torch.ldexp(x.float(), -by[..., None]).to(torch.float8_e4m3fn), (by + 127).to(torch.uint8)


def _plain_store(s):
    slots, page, e = s["slots"], s["K"].shape[3], s["V"].shape[5]
    kept = (slots >= 0).nonzero()[:, 0]
    at = slots[kept]
    where, off = at // page, at % page
    as_bytes = lambda t: t.view(torch.uint8)
    k, k_by = _plain_quantised(s["k"][:, kept])
    v, v_by = _plain_quantised(s["v"][:, kept])
    as_bytes(s["K"])[:, where, :, off] = as_bytes(k).permute(1, 0, 2, 3)
    as_bytes(s["V"])[:, where, :, off // e, :, off % e] = as_bytes(v).permute(1, 0, 2, 3)
    as_bytes(s["K_scale"])[:, where, :, off] = k_by.permute(1, 0, 2)
    as_bytes(s["V_scale"])[:, where, :, off] = v_by.permute(1, 0, 2)
    return {"K": s["K"], "V": s["V"], "K_scale": s["K_scale"], "V_scale": s["V_scale"]}


def _power(scale):
    """2^(byte - 127) of e8m0 bytes, none of which is 0 or 255."""
    return torch.ldexp(torch.ones((), device="cuda"), scale.view(torch.uint8).to(torch.int32) - 127)


def _gathered(K, V, K_scale, V_scale, where, off, wide=torch.float32):
    """Rows [tokens][layers][heads][dim] of K and V at places of pages."""
    e, raw = V.shape[5], K.element_size() == 1
    bits = (lambda t: t.view(torch.uint8)) if raw else (lambda t: t)
    k, v = bits(K)[:, where, :, off], bits(V)[:, where, :, off // e, :, off % e]
    if not raw:
        return k.to(wide), v.to(wide)
    k, v = k.view(K.dtype).to(wide), v.view(V.dtype).to(wide)
    return k * _power(bits(K_scale)[:, where, :, off])[..., None].to(wide), v * _power(bits(V_scale)[:, where, :, off])[..., None].to(wide)


def _plain_load(s):
    page = s["K"].shape[3]
    k, v = _gathered(s["K"], s["V"], s["K_scale"], s["V_scale"], s["slots"] // page, s["slots"] % page)
    to = torch.bfloat16 if s["K"].element_size() == 1 else s["K"].dtype
    return {"k": k.transpose(0, 1).to(to).contiguous(), "v": v.transpose(0, 1).to(to).contiguous()}


def _padded(starts, nodes, rows):
    """[R][nodes] row of each node, and whether the request has it."""
    j = torch.arange(nodes, device="cuda")
    n = (starts[1:] - starts[:-1])[:, None]
    return (starts[:-1, None].long() + j).clamp(max=rows - 1), j < n


def _owners(starts, rows):
    """Request and node of each row."""
    t = torch.arange(rows, device="cuda")
    r = torch.searchsorted(starts[1:].contiguous(), t.to(torch.int32), right=True)
    return r, t - starts[r].long()


def _bits(tree, rows, real):
    """[R][nodes][nodes]: node i of a request sees its node j."""
    j = torch.arange(rows.shape[1], device="cuda")
    return ((tree[rows][:, :, None] >> j) & 1).bool() & real[:, None, :] & real[:, :, None]


def _plain_attn(s):
    q, k, v, N = s["q"], s["k"], s["v"], s["nodes"]
    T, hq, dim = q.shape
    hkv, R = k.shape[1], s["lens"].numel()
    at = s["table"].clamp(min=0).long()
    rows, real = _padded(s["starts"], N, T)
    # pages of the requests, token by token
    K = (s["K"][0].view(torch.uint8)[at].view(s["K"].dtype).float() * _power(s["K_scale"])[0][at][..., None]).permute(0, 1, 3, 2, 4)
    V = s["V"][0].view(torch.uint8)[at].view(s["V"].dtype).float().permute(0, 1, 3, 5, 2, 4)
    V = V.flatten(2, 3) * _power(s["V_scale"])[0][at].permute(0, 1, 3, 2)[..., None]
    keys, values = (torch.cat([c.reshape(R, -1, hkv, dim), x[rows].float()], 1) for c, x in ((K, k), (V, v)))
    cached = torch.arange(keys.shape[1] - N, device="cuda") < s["lens"][:, None]
    values = values * torch.cat([cached, real], 1)[:, :, None, None]
    sees = torch.cat([cached[:, None, :] & real[:, :, None], _bits(s["tree"], rows, real)], 2)          # [R][N][L]
    qr = q[rows].float().reshape(R, N, hkv, hq // hkv, dim).permute(0, 2, 1, 3, 4).reshape(R, hkv, -1, dim)
    score = (qr @ keys.permute(0, 2, 3, 1).contiguous()) * s["scale"]
    score = score.reshape(R, hkv, N, hq // hkv, -1).masked_fill_(~sees[:, None, :, None, :], float("-inf"))
    top = score.amax(-1, keepdim=True)
    p = (score - torch.where(top == float("-inf"), 0.0, top)).exp_()
    total = p.sum(-1, keepdim=True)
    out = (p.reshape(R, hkv, -1, p.shape[-1]) @ values.permute(0, 2, 1, 3).contiguous()).reshape(R, hkv, N, hq // hkv, dim)
    out = out / torch.where(total == 0, 1.0, total)
    lse = torch.where(total > 0, top + total.log(), float("-inf"))[..., 0]
    r, i = _owners(s["starts"], T)
    out = out.permute(0, 2, 1, 3, 4).reshape(R, N, hq, dim)[r, i]
    return {"out": out.to(q.dtype), "lse": lse.permute(0, 2, 1, 3).reshape(R, N, hq)[r, i]}


def _plain_sample(s):
    T, V = s["logits"].shape
    x, order = s["logits"].float().sort(dim=1, descending=True, stable=True)
    col = lambda name: s[name].double()[:, None]
    greedy = col("temperature") <= 0
    z = (x.double() - x[:, :1].double()) / torch.where(greedy, 1.0, col("temperature"))
    rank = torch.arange(V, device="cuda")
    top_k = torch.where(greedy, 1, torch.where(s["top_k"][:, None] <= 0, V, s["top_k"][:, None]))
    weight = torch.where(rank < top_k, (z.exp() * UNIT).round(), 0.0).long()
    upto = weight.cumsum(1)
    need = torch.where(col("top_p") < 1, (col("top_p") * upto[:, -1:].double()).ceil().long(), upto[:, -1:])
    weight = torch.where(((upto - weight < need) & (weight >= (col("min_p") * UNIT).ceil().long())) | (rank == 0), weight, 0)
    upto = weight.cumsum(1)
    total = upto[:, -1:]
    goal = (col("u") * total.double()).floor().long().minimum(total - 1)
    place = torch.searchsorted(upto, goal, right=True)
    answers = order.gather(1, place)[:, 0].to(torch.int32)
    logp = (z.gather(1, place) - (total.double() / UNIT).log())[:, 0].float()
    if "tree" not in s:
        return {"answers": answers, "logp": logp}
    N = s["nodes"]
    rows, real = _padded(s["starts"], N, T)
    sees = _bits(s["tree"], rows, real)
    j = torch.arange(N, device="cuda")
    parent = torch.where(sees & (j[None, None, :] < j[None, :, None]), j, -1).amax(2)                    # [R][N]
    agrees = (s["tokens"][rows] == answers[rows].gather(1, parent.clamp(min=0))) & (parent >= 0) & real
    earlier = (parent[:, :, None] == parent[:, None, :]) & agrees[:, None, :] & (j[None, None, :] < j[None, :, None])
    good = (agrees & ~earlier.any(2)) | ((j == 0) & real)
    kept = (good[:, None, :] | ~sees).all(2) & real & sees[:, :, 0]
    last = torch.where(kept, j, -1).amax(1)
    r, i = _owners(s["starts"], T)
    return {"keep": torch.where(kept, sees.sum(2) - 1, -1)[r, i].to(torch.int32), "counts": kept.sum(1).to(torch.int32),
            "next": answers[rows].gather(1, last[:, None])[:, 0], "answers": answers, "logp": logp}


_PLAIN = {"rope": _plain_rope, "store": _plain_store, "load": _plain_load, "attn": _plain_attn, "sample": _plain_sample}


# ---- what a pass cannot do without ----------------------------------------------------------------------------------------


def work(case):
    size = {"bf16": 2, "f32": 4, "e4m3": 1}.get(case.get("dtype"), 2)
    if case["op"] == "sample":
        lens, trees = _facts(case)
        rows = sum(len(t) for t in trees) if trees else case["R"]
        return {"bytes": rows * (case["V"] * size + 28) + (rows * 16 + case["R"] * 12 if trees else 0), "flops": rows * case["V"]}
    hq, hkv, dim = HEADS[case["shape"]]
    if case["op"] == "rope":
        heads = case["T"] * (hq + hkv)
        return {"bytes": 2 * heads * dim * size + case["T"] * 4, "flops": heads * (dim * 4 * case["norm"] + case["rot"] * 3)}
    if case["op"] == "store":
        where, _ = _store_facts(case)
        kept = 2 * sum(w != -1 for w in where) * case["layers"] * hkv
        return {"bytes": kept * (3 * dim + 1) + 8 * len(where), "flops": 2 * kept * dim}
    lens, trees = _facts(case)
    if case["op"] == "load":
        rows = 2 * sum(lens) * case["layers"] * hkv
        return {"bytes": rows * (3 * dim + 1 if size == 1 else 2 * dim * size) + 8 * sum(lens), "flops": rows * dim if size == 1 else 0}
    rows = sum(len(t) for t in trees)
    pages = sum(-(-n // case["page"]) for n in lens)
    read = 2 * sum(lens) * hkv * (dim + 1) + 2 * rows * hkv * dim * 2 + rows * hq * dim * 2 + rows * 8 + pages * 4
    pairs = sum(n * len(t) + sum(bin(m & (1 << 64) - 1).count("1") for m in _masks(t)) for n, t in zip(lens, trees))
    return {"bytes": read + rows * hq * (dim * 2 + 4), "flops": 4 * pairs * hq * dim}


# ---- the same outputs from the definitions, in 64 bits --------------------------------------------------------------------


def exact(case, seed):
    s = prepare(case, seed)
    return {"rope": _exact_rope, "store": _exact_store, "load": _exact_load, "attn": _exact_attn, "sample": _exact_sample}[case["op"]](s)


def _exact_rope(s):
    half, out = s["inv_freq"].numel(), {}
    turn = torch.polar(torch.ones((), dtype=torch.float64, device="cuda"), s["places"].double()[:, None, None] * s["inv_freq"].double())
    for name in ("q", "k"):
        y, w = s[name].double(), s[name + "_weight"]
        if s["eps"] is not None:
            y = y / (y.pow(2).sum(-1, keepdim=True) / y.shape[-1] + s["eps"]).sqrt()
        y = (y if w is None else y * w.double()).contiguous()
        pairs = y[..., :2 * half].unflatten(-1, (half, 2) if s["inter"] else (2, half))
        pairs = pairs if s["inter"] else pairs.transpose(-1, -2)
        z = torch.view_as_real(torch.view_as_complex(pairs.contiguous()) * turn)
        y[..., :2 * half] = (z if s["inter"] else z.transpose(-1, -2)).flatten(-2)
        out[name] = y
    return out


def _exact_codes(x):
    """x = [layers][heads][dim] of one token: the values of its codes, and of its scales."""
    top = x.double().abs().amax(-1)
    by = torch.ceil(torch.log2(top.clamp(min=1e-300) / 448.0)).clamp(min=-96.0)
    by = torch.where(top > 448.0 * torch.exp2(by), by + 1, by)          # a logarithm next to a whole number
    by = torch.where((top <= 448.0 * torch.exp2(by - 1)) & (by > -96), by - 1, by)
    y = x.double() / torch.exp2(by)[..., None]
    step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(-6, 8) - 3)
    return torch.round(y / step) * step, torch.exp2(by)


def _exact_store(s):
    page, e = s["K"].shape[3], s["V"].shape[5]
    out = {n: s[n].float().double() for n in ("K", "V")}
    out.update({n: _power(s[n]).double() for n in ("K_scale", "V_scale")})
    for t, slot in enumerate(s["slots"].tolist()):
        if slot >= 0:
            p, o = divmod(slot, page)
            out["K"][:, p, :, o], out["K_scale"][:, p, :, o] = _exact_codes(s["k"][:, t])
            out["V"][:, p, :, o // e, :, o % e], out["V_scale"][:, p, :, o] = _exact_codes(s["v"][:, t])
    return out


def _exact_load(s):
    page = s["K"].shape[3]
    k, v = _gathered(s["K"], s["V"], s["K_scale"], s["V_scale"], s["slots"] // page, s["slots"] % page, torch.float64)
    return {"k": k.transpose(0, 1), "v": v.transpose(0, 1)}


def _exact_attn(s):
    q, page = s["q"], s["K"].shape[3]
    T, hq, dim = q.shape
    hkv = s["K"].shape[2]
    out = torch.zeros((T, hq, dim), dtype=torch.float64, device="cuda")
    lse = torch.full((T, hq), float("-inf"), dtype=torch.float64, device="cuda")
    starts, tree = s["starts"].tolist(), s["tree"].tolist()
    for r, length in enumerate(s["lens"].tolist()):
        a, b = starts[r], starts[r + 1]
        i = torch.arange(length, device="cuda")
        kr, vr = _gathered(s["K"], s["V"], s["K_scale"], s["V_scale"], s["table"][r].long()[i // page], i % page, torch.float64)
        sees = torch.tensor([[(tree[t] >> j) & 1 for j in range(b - a)] for t in range(a, b)], device="cuda").bool()
        sees = torch.cat([torch.ones((b - a, length), dtype=torch.bool, device="cuda"), sees], 1)
        for h in range(hkv):
            kh = torch.cat([kr[:, 0, h], s["k"][a:b, h].double()])
            vh = torch.cat([vr[:, 0, h], s["v"][a:b, h].double()])
            for g in range(h * (hq // hkv), (h + 1) * (hq // hkv)):
                z = (q[a:b, g].double() @ kh.t() * s["scale"]).masked_fill(~sees, float("-inf"))
                lse[a:b, g] = torch.logsumexp(z, 1)
                out[a:b, g] = torch.softmax(z, 1) @ vh
    return {"out": out, "lse": lse}


def _exact_sample(s):
    """The logarithms of the drawn tokens' probabilities, row by row, from real weights; tokens and branches are whole numbers."""
    logp = []
    how = zip(*(s[n].tolist() for n in ("temperature", "top_k", "top_p", "min_p", "u")))
    for row, (t, k, p, m, u) in zip(s["logits"], how):
        x = row.double().sort(descending=True, stable=True).values
        if t <= 0:
            logp.append(x.new_zeros(()))
            continue
        z = ((x - x[0]) / t)[:k if k > 0 else None]
        w = z.exp()
        upto = w.cumsum(0)
        n = 1 + int((upto[:-1] < p * upto[-1]).sum()) if p < 1 else w.numel()
        kept = w[:n] * (w[:n] >= m)
        upto = kept.cumsum(0)
        i = min(int((upto <= u * upto[-1]).sum()), n - 1)
        logp.append(z[i] - upto[-1].log())
    return {"answers": None, "logp": torch.stack(logp), **({"keep": None, "counts": None, "next": None} if "tree" in s else {})}
