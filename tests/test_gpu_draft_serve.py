"""Block tables and slots, acceptance, and the commit of K and V, against the oracle: whole numbers and copies, so everything is equal."""
import random

import numpy as np
import pytest

from draft_cases import parents, signed, words

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from oracle import draft
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding, draft


def i32(torch, v):
    return torch.tensor(v, dtype=torch.int32, device="cuda")


# ---- plan ------------------------------------------------------------------------------------------------------------------


def make_plan(seed, R, page, width, pages, rows, free=None, ends=0.1, padded=0):
    """Requests of random lengths in a pool: some grow, some end, the ring anywhere in its cycle."""
    rng = random.Random(seed)
    ids = list(range(pages))
    rng.shuffle(ids)
    table, lens, add, starts, keep = [], [], [], [0], []
    for _ in range(R):
        held = rng.randint(0, min(width, max(0, len(ids) // 2)))
        n = max(0, held * page - rng.choice([0, 0, 1, page - 1, rng.randrange(page)])) if held else 0
        held = -(-n // page)
        table.append([ids.pop() for _ in range(held)] + [-1] * (width - held))
        lens.append(n)
        a = -1 if rng.random() < ends else rng.choice([0, 1, 2, rng.randint(0, rows)])
        add.append(a)
        r = max(a, 0) + rng.randint(0, 3)
        places = sorted(rng.sample(range(r), max(a, 0)))
        keep += [places.index(i) if i in places else -1 for i in range(r)]
        starts.append(starts[-1] + r)
    free = len(ids) if free is None else min(free, len(ids))
    head = rng.randrange(pages)
    ring = [-7] * pages
    for i in range(free):
        ring[(head + i) % pages] = ids[i]
    return dict(table=table, ring=ring, pool=[head, free], lens=lens, add=add, starts=starts, keep=keep + [0] * padded, page=page)


def run_plan(torch, binding, c, keep=True):
    d = {k: i32(torch, v) for k, v in c.items() if k != "page"}
    got = binding.kv_plan(d["table"], d["ring"], d["pool"], d["lens"], d["add"], d["starts"], c["page"],
                          keep=d["keep"] if keep else None, rows=None if keep else c["starts"][-1])
    for name in ("pool", "lens", "add", "starts", "keep"):
        assert d[name].tolist() == c[name]                      # the inputs stay
    slots, lens, pool, refused = got
    return slots.tolist(), lens.tolist(), pool.tolist(), refused.tolist(), d["table"].tolist(), d["ring"].tolist()


@pytest.mark.parametrize("R,page,width,pages,rows,free", [
    (1, 64, 4, 7, 8, None), (1, 32, 1, 1, 40, None), (3, 32, 5, 30, 70, None), (8, 64, 9, 90, 64, None), (63, 32, 6, 400, 9, None),
    (64, 128, 3, 200, 64, None), (65, 256, 7, 500, 500, None), (257, 32, 4, 900, 33, None), (700, 64, 12, 9000, 200, None),
    (9, 32, 8, 80, 100, 0), (9, 32, 8, 80, 100, 3), (40, 32, 8, 300, 60, 20), (300, 64, 5, 900, 130, 50),
])
def test_plan_against_the_oracle(env, R, page, width, pages, rows, free):
    torch, binding, draft = env
    refusals = 0
    for seed in range(4):
        c = make_plan(seed, R, page, width, pages, rows, free, padded=(0, 5)[seed % 2])
        want = draft.plan(**c, rows=len(c["keep"]))
        got = run_plan(torch, binding, c)
        assert got == tuple(want)
        refusals += sum(got[3])
        c["keep"] = None
        want = draft.plan(**c, rows=c["starts"][-1])
        c["keep"] = []
        assert run_plan(torch, binding, c, keep=False) == tuple(want)
    assert refusals > 0 or free is None                         # some do not fit


def test_plan_of_the_most_requests(env):
    torch, binding, draft = env
    c = make_plan(5, 4096, 32, 3, 9000, 20)
    assert run_plan(torch, binding, c) == tuple(draft.plan(**c, rows=len(c["keep"])))


def test_plan_with_long_prompts(env):
    """Rows by the ten thousand: many blocks, each with its own sums."""
    torch, binding, draft = env
    c = make_plan(6, 20, 32, 200, 4200, 5000)
    assert run_plan(torch, binding, c) == tuple(draft.plan(**c, rows=len(c["keep"])))


def test_plan_again_with_the_same_inputs(env):
    """What a call writes depends on its inputs alone: the second call finds table and ring as the first one left them."""
    torch, binding, draft = env
    c = make_plan(9, 30, 64, 6, 200, 90)
    want = draft.plan(**c, rows=len(c["keep"]))
    d = {k: i32(torch, v) for k, v in c.items() if k != "page"}
    for _ in range(3):
        slots, lens, pool, refused = binding.kv_plan(d["table"], d["ring"], d["pool"], d["lens"], d["add"], d["starts"], 64, keep=d["keep"])
        assert (slots.tolist(), lens.tolist(), pool.tolist(), refused.tolist(), d["table"].tolist(), d["ring"].tolist()) == tuple(want)


def test_plans_in_a_row_hand_every_page_to_one_request(env):
    """Two hundred steps of requests that grow and end: no page is ever held twice, none is lost."""
    torch, binding, draft = env
    rng = random.Random(1)
    R, page, width, pages = 12, 32, 6, 40
    table, ring = i32(torch, [[-1] * width] * R), i32(torch, list(range(pages)))
    pool, lens = i32(torch, [0, pages]), i32(torch, [0] * R)
    grants = refusals = 0
    for step in range(200):
        add = [-1 if rng.random() < 0.1 else rng.choice([0, 1, 5, 40]) for _ in range(R)]
        starts = [0]
        for a in add:
            starts.append(starts[-1] + max(a, 0))
        slots, lens, pool, refused = binding.kv_plan(table, ring, pool, lens, i32(torch, add), i32(torch, starts), page, rows=starts[-1])
        n, t, rg, (head, free) = lens.tolist(), table.tolist(), ring.tolist(), pool.tolist()
        held = [p for r in range(R) for p in t[r][:-(-n[r] // page)]]
        spare = [rg[(head + i) % pages] for i in range(free)]
        assert sorted(held + spare) == list(range(pages))
        s = slots.tolist()
        real = [v for v in s if v >= 0]
        assert len(set(real)) == len(real)
        refusals += sum(refused.tolist())
        grants += len(real)
    assert grants > 200 and refusals > 5


def test_plan_in_a_graph(env):
    torch, binding, draft = env
    c = make_plan(3, 20, 32, 6, 200, 60)
    d = {k: i32(torch, v) for k, v in c.items() if k != "page"}
    call = lambda: binding.kv_plan(d["table"], d["ring"], d["pool"], d["lens"], d["add"], d["starts"], 32, keep=d["keep"])
    first = {k: d[k].clone() for k in d}
    call()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = call()
    for seed in (3, 4, 5):
        c = make_plan(3, 20, 32, 6, 200, 60)
        rng = random.Random(seed)
        c["add"] = [a if rng.random() < 0.5 else min(a, 1) for a in c["add"]]
        for k in ("table", "ring"):
            d[k].copy_(first[k])
        d["add"].copy_(i32(torch, c["add"]))
        graph.replay()
        torch.cuda.synchronize()
        want = draft.plan(**c, rows=len(c["keep"]))
        assert (*(o.tolist() for o in out), d["table"].tolist(), d["ring"].tolist()) == tuple(want)


def test_plan_keeps_to_its_buffers(env):
    """Lengths, places and counts that make no sense change nothing outside the arrays."""
    torch, binding, draft = env
    guard = torch.full((3, 64), 99, dtype=torch.int32, device="cuda")
    table, ring = guard[1, :12].view(3, 4), guard[1, 16:22]
    table.fill_(-5)
    ring.copy_(i32(torch, [900, -4, 3, 1, 1 << 30, 2]))
    slots, lens, pool, refused = binding.kv_plan(table, ring, i32(torch, [-9, 1 << 30]), i32(torch, [-40, 1 << 30, 5]),
                                                 i32(torch, [(1 << 31) - 1, -1, 60]), i32(torch, [0, 40, 90, 150]), 32,
                                                 keep=i32(torch, [i - 40 for i in range(170)]))
    torch.cuda.synchronize()
    assert bool((guard[[0, 2]] == 99).all()) and bool((guard[1, 22:] == 99).all()) and bool((guard[1, 12:16] == 99).all())
    assert refused.tolist()[0] == 1 and int(slots.max()) < 6 * 32 and int(slots.min()) >= -1


def test_plan_refusals(env):
    torch, binding, draft = env
    c = make_plan(0, 4, 32, 5, 40, 20)
    d = {k: i32(torch, v) for k, v in c.items() if k != "page"}
    ok = dict(table=d["table"], ring=d["ring"], pool=d["pool"], lens=d["lens"], add=d["add"], starts=d["starts"], page=32, keep=d["keep"])
    for bad in (dict(page=48), dict(page=16), dict(page=0), dict(lens=d["lens"].long()), dict(add=d["add"][:3]), dict(starts=d["starts"][:4]),
                dict(pool=d["pool"][:1]), dict(ring=d["ring"][:0]), dict(table=d["table"].t()), dict(keep=None), dict(keep=d["keep"].cpu())):
        with pytest.raises(binding.SvdpError):
            binding.kv_plan(**{**ok, **bad})
    many = torch.zeros((4097, 2), dtype=torch.int32, device="cuda")
    row = torch.zeros(4098, dtype=torch.int32, device="cuda")
    with pytest.raises(binding.SvdpError, match="unsupported"):
        binding.kv_plan(many, d["ring"], d["pool"], row[:4097], row[:4097], row, 32, rows=1)


# ---- accept ----------------------------------------------------------------------------------------------------------------


def make_accept(torch, seed, R, nodes, V, dtype, chain=False, right=0.7, empty=False):
    g = torch.Generator(device="cuda").manual_seed(seed)
    rng = random.Random(seed)
    n = [0 if empty and rng.random() < 0.3 else rng.randint(1, nodes) for _ in range(R)]
    par = [([-1] + list(range(k - 1)) if chain else parents(rng, k))[:k] for k in n]
    starts = [0]
    for k in n:
        starts.append(starts[-1] + k)
    logits = torch.randn((starts[-1], V), device="cuda", generator=g).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    answer = [int(np.flatnonzero(r == r.max())[0]) for r in logits.float().cpu().numpy()]
    tokens = [answer[starts[r] + max(p, 0)] if rng.random() < right else rng.randrange(V) for r in range(R) for p in par[r]]
    return logits, tokens, None if chain else sum((words(p) for p in par), []), starts


def run_accept(torch, binding, logits, tokens, tree, starts, **over):
    d = None if tree is None else torch.tensor(signed(tree), dtype=torch.int64, device="cuda")
    got = binding.tree_accept(logits, i32(torch, tokens), i32(torch, starts), tree=d, **over)
    return tuple(g.tolist() for g in got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("R,nodes,V", [(1, 1, 1), (1, 8, 2), (3, 8, 7), (2, 64, 1000), (70, 9, 129), (5, 20, 32000), (1, 3, 152064), (1, 2, 50257),
                                       (300, 64, 65)])
def test_accept_against_the_oracle(env, dtype, R, nodes, V):
    torch, binding, draft = env
    for seed, chain in ((1, False), (2, True)):
        logits, tokens, tree, starts = make_accept(torch, seed, R, nodes, V, dtype, chain, empty=R > 2)
        want = draft.accept(logits.float().cpu().numpy(), tokens, tree, starts)
        got = run_accept(torch, binding, logits, tokens, tree, starts)
        assert got == tuple(want)
    if R * nodes > 500:
        assert max(got[1]) > 2


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accept_of_rows_at_any_address(env, dtype):
    """Rows whose width and stride are no multiple of a vector, down to rows that share none of their 16 bytes with a boundary."""
    torch, binding, draft = env
    e = 8 if dtype == "bf16" else 4
    for V in (1, 3, e - 1, e, e + 1, 5 * e - 1, 3001):
        for shift in range(e):
            wide = torch.randn((4, V + 13), device="cuda", generator=torch.Generator(device="cuda").manual_seed(V)).to(
                torch.bfloat16 if dtype == "bf16" else torch.float32)
            wide[:, :shift] = 1e9                        # neighbours that must not win
            wide[:, shift + V:] = 1e9
            logits = wide[:, shift:shift + V]
            got = run_accept(torch, binding, logits, [0, 0, 1, 2], None, [0, 4])
            assert got == tuple(draft.accept(logits.float().cpu().numpy(), [0, 0, 1, 2], None, [0, 4]))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_accept_ties_infinities_and_nan(env, dtype):
    torch, binding, draft = env
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    V, inf, nan = 9001, float("inf"), float("nan")
    x = torch.full((9, V), -1.0)
    x[0, [77, 78, 8999]] = 2.0                           # equal: the lowest
    x[1, 5000] = -0.0
    x[1, 5001] = 0.0                                     # -0 equals 0
    x[2, 8192] = inf
    x[2, 17] = 3e38
    x[3, :] = -inf                                       # all equal, nothing finite
    x[4, 6000] = nan                                     # NaN above infinity
    x[4, 12] = inf
    x[5, [9000, 8998]] = nan
    x[6, :] = nan
    x[7, :] = -inf
    x[7, 4444] = -3e38
    x[8, 3] = 1.0
    x = x.to(td).cuda()
    if dtype == "f32":
        x[5].view(torch.int32)[8998] = -1                # a NaN with its sign set
    else:
        x[5].view(torch.int16)[8998] = -1
    got = run_accept(torch, binding, x, [0] * 9, None, [0, 9])
    assert got[3] == [77, 5000, 8192, 0, 6000, 8998, 0, 4444, 3]
    assert got == tuple(draft.accept(x.float().cpu().numpy(), [0] * 9, None, [0, 9]))


def test_accept_walks_to_the_lowest_child_that_agrees(env):
    torch, binding, draft = env
    par = [-1, 0, 0, 0, 2, 2, 4, 1]                      # node 1 and its child agree with nothing; 2 and 3 are equal
    logits = torch.zeros((8, 10), device="cuda")
    for row, t in ((0, 5), (2, 7), (4, 7), (5, 1), (6, 9)):
        logits[row, t] = 1.0
    tokens = [3, 4, 5, 5, 7, 7, 7, 4]
    keep, counts, following, best = run_accept(torch, binding, logits, tokens, words(par), [0, 8])
    assert keep == [0, -1, 1, -1, 2, -1, 3, -1] and counts == [4] and following == [9] and best[0] == 5


def test_accept_padding_and_limit(env):
    """Rows of no request and nodes past the limit are answered but in no branch."""
    torch, binding, draft = env
    logits, tokens, tree, starts = make_accept(torch, 5, 1, 30, 333, "f32", chain=True, right=1.0)
    n = starts[-1]
    assert n > 8
    keep, counts, following, best = run_accept(torch, binding, logits, tokens, None, [0, n - 3], max_nodes=4)
    assert keep == [0, 1, 2, 3] + [-1] * (n - 4) and counts == [4]
    assert best == [draft.best_token(r) for r in logits.cpu().numpy()] and following == [best[3]]
    none = binding.tree_accept(logits[:0], i32(torch, []), i32(torch, [0, 0, 0]))
    assert none[1].tolist() == [0, 0] and none[2].tolist() == [-1, -1]


def test_accept_in_a_graph(env):
    torch, binding, draft = env
    logits, tokens, tree, starts = make_accept(torch, 6, 4, 8, 5000, "bf16")
    d = torch.tensor(signed(tree), dtype=torch.int64, device="cuda")
    tk, st = i32(torch, tokens), i32(torch, starts)
    binding.tree_accept(logits, tk, st, tree=d)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        out = binding.tree_accept(logits, tk, st, tree=d)
    for seed in (6, 7, 8):
        logits.copy_(torch.randn(logits.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(seed)))
        graph.replay()
        torch.cuda.synchronize()
        assert tuple(o.tolist() for o in out) == tuple(draft.accept(logits.float().cpu().numpy(), tokens, tree, starts))


def test_accept_refusals(env):
    torch, binding, draft = env
    logits, tokens, tree, starts = make_accept(torch, 6, 2, 8, 50, "bf16")
    tk, st = i32(torch, tokens), i32(torch, starts)
    for bad in (dict(logits=logits.half()), dict(logits=logits.t().contiguous().t()), dict(logits=logits[0]), dict(tokens=tk[:1]),
                dict(tokens=tk.long()), dict(starts=st[:1]), dict(max_nodes=65), dict(max_nodes=0), dict(tree=tk), dict(logits=logits[:, :0]),
                dict(ws=torch.empty(0, dtype=torch.uint8, device="cuda"))):
        with pytest.raises(binding.SvdpError):
            binding.tree_accept(**{**dict(logits=logits, tokens=tk, starts=st), **bad})


# ---- commit ----------------------------------------------------------------------------------------------------------------


def run_commit(torch, binding, draft, dtype, layers, heads, dim, page, pages, slots, strided, seed=0):
    td = torch.bfloat16 if dtype == "bf16" else torch.float32
    g = torch.Generator(device="cuda").manual_seed(seed)
    cache = binding.KVCache.empty(layers, pages, page, heads, dim, dtype=td)
    cache.K.normal_(generator=g)
    cache.V.normal_(generator=g)
    T = len(slots)
    kv = torch.randn((layers, T, 3 if strided else 2, heads, dim), device="cuda", generator=g).to(td)
    k, v = (kv[:, :, 0], kv[:, :, 2]) if strided else (kv[:, :, 0].contiguous(), kv[:, :, 1].contiguous())
    n = lambda t: t.float().cpu().numpy()
    K, V = n(cache.K), n(cache.V)
    draft.commit(K, V, n(k), n(v), slots)
    binding.kv_commit(cache, k, v, torch.tensor(slots, dtype=torch.int64, device="cuda"))
    assert np.array_equal(n(cache.K), K) and np.array_equal(n(cache.V), V)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,dim,page,strided", [(1, 64, 32, False), (3, 128, 64, True), (8, 128, 32, False), (2, 256, 128, True), (5, 64, 256, True)])
def test_commit_against_the_oracle(env, dtype, heads, dim, page, strided):
    torch, binding, draft = env
    pages, rng = 5, random.Random(heads)
    every = list(range(pages * page))
    cases = [[0], [pages * page - 1], [-1], every[3:4], every[0:8], every[1:10], every[5:45], every[:page],
             every[page - 5:page + 3], [-1] * 3 + every[8:24] + [-1], rng.sample(every, 21), every[16:24][::-1],
             every[8:16] + every[40:48] + every[7:8],
             # a prompt in pages of no order, and slots that do not exist
             sum((every[p * page:(p + 1) * page] for p in (3, 0, 4)), [])[:2 * page + 13],
             [pages * page, -(1 << 40), 1 << 40, 2, -8, -7, -6, -5, -4, -3, -2, -1]]
    for i, slots in enumerate(cases):
        run_commit(torch, binding, draft, dtype, 1 + i % 3, heads, dim, page, pages, slots, strided, seed=i)


def test_commit_of_nothing_and_refusals(env):
    torch, binding, draft = env
    cache = binding.KVCache.empty(2, 3, 32, 2, 64)
    new = torch.zeros((2, 4, 2, 64), dtype=torch.bfloat16, device="cuda")
    slots = torch.tensor([1, 2, 3, 4], dtype=torch.int64, device="cuda")
    binding.kv_commit(cache, new[:, :0], new[:, :0], slots[:0])
    binding.kv_commit(cache, new, new, slots)
    for k, v, s in ((new[:1], new, slots), (new, new.float(), slots), (new, new[:, :3], slots), (new, new, slots.int()), (new, new, slots[:3]),
                    (new.transpose(2, 3), new, slots), (new.cpu(), new, slots), (new, new, slots.cpu())):
        with pytest.raises(binding.SvdpError):
            binding.kv_commit(cache, k, v, s)


def test_commit_in_a_graph(env):
    torch, binding, draft = env
    cache = binding.KVCache.empty(2, 3, 32, 2, 64, dtype=torch.float32)
    cache.K.zero_()
    cache.V.zero_()
    new = torch.randn((2, 9, 2, 64), device="cuda")
    slots = torch.arange(9, dtype=torch.int64, device="cuda")
    binding.kv_commit(cache, new, new, slots)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        binding.kv_commit(cache, new, new, slots)
    for first in (0, 3, 60):
        slots.copy_(torch.arange(first, first + 9))
        new.normal_()
        K, V = cache.K.cpu().numpy(), cache.V.cpu().numpy()
        draft.commit(K, V, new.cpu().numpy(), new.cpu().numpy(), slots.tolist())
        graph.replay()
        torch.cuda.synchronize()
        assert np.array_equal(cache.K.cpu().numpy(), K) and np.array_equal(cache.V.cpu().numpy(), V)


@pytest.mark.parametrize("R,page,width,pages,rows,free", [(1024, 32, 4, 5000, 700, None), (1025, 64, 4, 5000, 300, None), (2500, 32, 3, 9000, 2600, 1500),
                                                          (4096, 32, 2, 9000, 50, 700)])
def test_plan_of_more_requests_than_threads(env, R, page, width, pages, rows, free):
    torch, binding, draft = env
    c = make_plan(R, R, page, width, pages, rows, free, padded=3)
    assert run_plan(torch, binding, c) == tuple(draft.plan(**c, rows=len(c["keep"])))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [701, 40003])
def test_accept_of_few_and_of_many_logits(env, dtype, V):
    """A request's logits read by one block, and by many: rows at any address, ties, infinities and NaN, padding behind the requests."""
    torch, binding, draft = env
    td, e = (torch.bfloat16, 8) if dtype == "bf16" else (torch.float32, 4)
    inf, nan = float("inf"), float("nan")
    g = torch.Generator(device="cuda").manual_seed(V)
    for shift in range(e):
        wide = torch.randn((24, V + 13), device="cuda", generator=g).to(td)
        wide[:, :shift] = 1e9                                # neighbours that must not win
        wide[:, shift + V:] = inf
        x = wide[:, shift:shift + V]
        x[0, [5, V // 2, V - 1]] = 50.0
        x[1] = -inf
        x[2, V - 1] = nan
        x[3, 0] = nan
        x[3, 7] = inf
        x[4, [V - 2, V - 1]] = inf
        x[5] = 0.0
        x[5, 3] = -0.0
        rows = x.float().cpu().numpy()
        for starts in ([0, 8, 8, 15], [0, 1, 2, 3], [0, 0, 0, 0], [0, 8, 16, 24]):
            tokens = [draft.best_token(rows[max(t - 1, 0)]) for t in range(24)]
            got = run_accept(torch, binding, x, tokens, None, starts, max_nodes=8)
            assert got == tuple(draft.accept(rows, tokens, None, starts))
    best = got[3]
    assert best[0] == 5 and best[1] == 0 and best[2] == V - 1 and best[3] == 0 and best[4] == V - 2 and best[5] == 0


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [333, 152064])
@pytest.mark.parametrize("max_nodes", [None, 1, 64])
def test_accept_of_no_rows(env, dtype, V, max_nodes):
    """Requests without rows, whatever kernel their logits' number would ask for: lengths of zero and no next token."""
    torch, binding, draft = env
    logits = torch.empty((0, V), dtype=torch.bfloat16 if dtype == "bf16" else torch.float32, device="cuda")
    got = run_accept(torch, binding, logits, [], None, [0, 0, 0, 0], max_nodes=max_nodes)
    assert got == ([], [0, 0, 0], [-1, -1, -1], [])


@pytest.mark.parametrize("V", [701, 40003])
def test_accept_of_a_request_with_more_rows_than_nodes(env, V):
    """Rows past the limit are answered and in no branch, in one launch (few logits) and in two; the requests behind have none."""
    torch, binding, draft = env
    logits = torch.randn((24, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(torch.bfloat16)
    rows = logits.float().cpu().numpy()
    tokens = [draft.best_token(rows[max(t - 1, 0)]) for t in range(24)]
    tree = sum((words(parents(random.Random(k), 8)) for k in range(3)), [])
    for t in (None, tree):
        want = draft.accept(rows, tokens, t, [0, 8, 8, 8])
        for starts in ([0, 24, 24, 24], [0, 17, 17, 17], [0, 9, 9, 9]):
            assert run_accept(torch, binding, logits, tokens, t, starts, max_nodes=8) == tuple(want)


def test_accept_of_the_most_rows(env):
    """As many rows as a call takes, all but 64 of them padding: more threads than one grid can have."""
    torch, binding, draft = env
    T, V = 1 << 24, 3
    x = torch.randn((T, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(8))
    best = torch.where(x == x.amax(1, keepdim=True), torch.arange(V, device="cuda", dtype=torch.int32), V).amin(1)
    tokens = torch.cat([best[:1], best[:-1]])
    keep, counts, following, got = binding.tree_accept(x, tokens, i32(torch, [0, 64]))
    assert torch.equal(got, best) and counts.tolist() == [64] and following.tolist() == best[63:64].tolist()
    assert keep[:64].tolist() == list(range(64)) and bool((keep[64:] == -1).all())


def test_plan_refuses_for_two_reasons(env):
    """Too wide for the table: nobody else is touched.  Too few pages: nor does any later request get one."""
    torch, binding, draft = env
    c = dict(table=[[0, 1], [-1, -1], [-1, -1], [2, -1], [3, -1], [-1, -1]], ring=[4, 5, 6, 7, 8, 9, 10, 11], pool=[0, 3],
             lens=[64, 0, 0, 10, 32, 0], add=[1, 64, 40, 5, 1, 0], starts=[0, 1, 65, 105, 110, 111, 111], keep=None, page=32)
    want = draft.plan(**c, rows=111)
    assert want[1] == [64, 64, 0, 15, 32, 0] and want[3] == [1, 0, 1, 0, 1, 0] and want[2] == [2, 1]
    c["keep"] = []
    assert run_plan(torch, binding, c, keep=False) == tuple(want)


def test_accept_keeps_no_scratch_alive(env):
    """What a caller keeps of the outputs holds the outputs' memory and not the call's scratch."""
    torch, binding, draft = env
    logits, tokens, tree, starts = make_accept(torch, 6, 4, 8, 152064, "bf16")
    out = binding.tree_accept(logits, i32(torch, tokens), i32(torch, starts))
    assert binding.tree_accept_workspace_bytes(len(tokens), 152064, binding.SVDP_BF16) > 2048
    assert all(o.untyped_storage().nbytes() <= 4 * (2 * len(tokens) + 2 * 4) for o in out)
    want = draft.accept(logits.float().cpu().numpy(), tokens, None, starts)
    assert tuple(o.tolist() for o in out) == tuple(want)


@pytest.mark.parametrize("R", [4064, 4095])
def test_plan_at_the_end_of_the_memory_that_needs_no_grant(env, R):
    """Sums of just below 64 KB, with what every block has besides above it."""
    torch, binding, draft = env
    c = make_plan(R, R, 32, 2, 9000, 30)
    assert run_plan(torch, binding, c) == tuple(draft.plan(**c, rows=len(c["keep"])))
