"""Attention of drafted tokens over paged K and V and over their own tree, against the 64-bit oracle."""
import numpy as np
import pytest

from draft_cases import Attn

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from oracle import draft
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding, draft


SHAPES = [
    # dtype, dim, heads, group, page, lens, nodes
    ("bf16", 128, 2, 1, 64, [1], [1]),
    ("bf16", 128, 3, 1, 64, [777], [1]),
    ("bf16", 128, 2, 4, 64, [0, 1, 31, 32, 33, 63, 64, 65], [1, 2, 3, 4, 5, 6, 7, 8]),
    ("bf16", 128, 1, 7, 128, [127, 128, 129, 1000], [64, 33, 17, 1]),
    ("bf16", 128, 1, 8, 256, [255, 700], [64, 64]),
    ("bf16", 128, 2, 5, 32, [95, 96, 97, 411], [13, 32, 0, 47]),
    ("bf16", 64, 2, 2, 32, [2, 0, 500], [31, 9, 16]),
    ("bf16", 64, 1, 16, 64, [300, 4], [40, 64]),
    ("bf16", 256, 2, 1, 64, [200, 0, 65], [1, 40, 3]),
    ("bf16", 256, 1, 6, 32, [100, 33], [64, 11]),
    ("f32", 64, 2, 2, 32, [0, 1, 31, 32, 33, 400], [13, 1, 2, 16, 17, 5]),
    ("f32", 128, 2, 4, 64, [65, 300], [8, 64]),
    ("f32", 128, 1, 1, 128, [1], [1]),
    ("f32", 256, 1, 3, 256, [257, 5], [30, 2]),
]


@pytest.mark.parametrize("tree", ["tree", "random", None])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:5])))
def test_attention_against_the_oracle(env, shape, tree):
    torch, binding, draft = env
    dtype, dim, heads, group, page, lens, nodes = shape
    c = Attn(torch, binding, dtype=dtype, dim=dim, heads=heads, group=group, page=page, lens=lens, nodes=nodes, tree=tree,
             seed=len(lens) * 100 + dim, strided=dim != 64)
    out, lse = c.call(binding)
    c.check(draft, out, lse)


@pytest.mark.parametrize("dtype,heads,group,lens,nodes", [
    ("bf16", 4, 1, [6001, 3, 900], [1, 2, 1]),          # cut into many parts
    ("bf16", 1, 4, [9001], [8]),
    ("bf16", 1, 7, [5000, 5100], [64, 50]),
    ("f32", 2, 2, [4100, 17], [7, 13]),
])
def test_long_contexts(env, dtype, heads, group, lens, nodes):
    torch, binding, draft = env
    c = Attn(torch, binding, dtype=dtype, dim=128 if dtype == "bf16" else 64, heads=heads, group=group, page=64, lens=lens,
             nodes=nodes, seed=7, spread=2.0)
    out, lse = c.call(binding)
    c.check(draft, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_requests(env, dtype):
    """More requests than a wave has lanes, requests without rows and without tokens among them."""
    torch, binding, draft = env
    rng = np.random.default_rng(3)
    lens = [int(v) for v in rng.integers(0, 90, 150)]
    nodes = [int(v) for v in rng.integers(0, 4, 150)]
    c = Attn(torch, binding, dtype=dtype, dim=64, heads=1, group=2, page=32, lens=lens, nodes=nodes, tree="random", seed=5)
    out, lse = c.call(binding)
    c.check(draft, out, lse)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_what_a_row_does_not_see_has_no_influence(env, dtype, bad):
    """Bits of the output stay the same when everything outside a row's sight is NaN or infinite: the places of a page behind the
    length, pages of no request, nodes of the tree that it does not see."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype=dtype, dim=128, heads=2, group=3, page=64, lens=[70, 0, 33], nodes=[7, 40, 5], seed=11)
    out, lse = c.call(binding)
    c.check(draft, out, lse)
    e = 8 if dtype == "bf16" else 4
    K, V = c.cache.K, c.cache.V
    used = torch.zeros(c.cache.pages, c.page, dtype=torch.bool)
    for r, n in enumerate(c.lens):
        for j in range(n):
            used[c.table[r][j // c.page], j % c.page] = True
    used = used.cuda()
    K[1].masked_fill_(~used[:, None, :, None], bad)
    V[1].masked_fill_(~used.reshape(c.cache.pages, 1, c.page // e, 1, e), bad)
    K[0].fill_(bad)
    V[0].fill_(bad)
    out2, lse2 = c.call(binding)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    # one node at a time: rows that do not see it keep their values (to the last bit but for the order of a sum)
    for r, node in ((0, 3), (1, 20), (1, 39), (2, 1)):
        t = c.starts[r] + node
        k, v = c.k[t].clone(), c.v[t].clone()
        c.k[t] = bad
        c.v[t] = bad
        out3, lse3 = c.call(binding)
        c.k[t], c.v[t] = k, v
        blind = torch.tensor([not (i in range(c.starts[r], c.starts[r + 1]) and (c.words[i] >> node) & 1)
                              for i in range(c.starts[-1])], device="cuda")
        assert bool(blind.any()) and not bool(blind.all())
        scale = out.float().abs().amax()
        assert float((out3.float() - out.float()).abs()[blind].amax()) <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * scale
        assert float((lse3 - lse).abs()[blind].amax()) <= 1e-5
        assert not bool(torch.isfinite(out3[~blind].float()).all(-1).all(-1).any())


def test_values_that_a_row_does_see_pass_through(env):
    """An infinite V of a token that a row sees: infinite where 64 bits say so; NaN in K: NaN in the whole row."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=64, heads=1, group=1, page=32, lens=[40], nodes=[3], tree=None, seed=2)
    c.cache.V[1, c.table[0][1], 0, 0, 5, 3] = float("inf")               # token 35, channel 5
    c.v[1, 0, 9] = float("-inf")                                         # node 1, channel 9
    out, lse = c.call(binding)
    o = out.float().cpu().numpy()[:, 0]
    assert np.isposinf(o[:, 5]).all() and np.isfinite(o[0, 9]) and np.isneginf(o[1:, 9]).all()
    assert np.isfinite(np.delete(o, [5, 9], 1)).all() and bool(torch.isfinite(lse).all())
    c.cache.K[1, c.table[0][0], 0, 7, 0] = float("nan")
    out, lse = c.call(binding)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


def test_scores_of_minus_infinity(env):
    """Weights that are all zero give zeros, as for a row that sees nothing; a single finite score is the whole answer."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="f32", dim=64, heads=1, group=1, page=32, lens=[33], nodes=[2], tree=None, seed=2)
    c.q.fill_(1.0)
    c.cache.K[1].fill_(1.0)
    c.cache.K[1, :, :, :, 0] = float("-inf")
    c.k[:, :, 0] = float("-inf")
    out, lse = c.call(binding)
    assert bool((out == 0).all()) and bool(torch.isneginf(lse).all())
    c.k[0, 0, 0] = 1.0
    out, lse = c.call(binding)
    assert torch.equal(out[0, 0], c.v[0, 0]) and torch.equal(out[1, 0], c.v[0, 0])
    assert float((lse - c.k[0, 0].sum() / 8).abs().max()) < 1e-5


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(env, dtype):
    """Scores of some hundreds: the running maximum moves by more than the exponent's range."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype=dtype, dim=128, heads=1, group=4, page=64, lens=[1500], nodes=[9], seed=21)
    out, lse = c.call(binding, scale=4.0)
    c.check(draft, out, lse, scale=4.0)
    out, lse = c.call(binding, scale=-4.0)
    c.check(draft, out, lse, scale=-4.0)
    out, lse = c.call(binding, scale=0.0)
    c.check(draft, out, lse, scale=0.0)


def test_padding_and_nodes_past_the_limit_are_left_alone(env):
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=64, heads=1, group=2, page=32, lens=[50, 20], nodes=[10, 4], pad=5, seed=4)
    out = torch.full((19, 2, 64), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((19, 2), 7.0, device="cuda")
    c.call(binding, out=out, lse=lse, max_nodes=6)
    c.check(draft, out, lse, max_nodes=6)
    for rows in (slice(6, 10), slice(14, 19)):
        assert bool((out[rows] == 7).all()) and bool((lse[rows] == 7).all())


def test_pages_that_do_not_exist_are_skipped(env):
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=128, heads=2, group=1, page=32, lens=[100, 300], nodes=[2, 3], seed=8)
    for r, i, bad in ((0, 1, -1), (0, 3, c.cache.pages), (1, 0, -(1 << 31)), (1, 5, (1 << 31) - 1)):
        c.table[r][i] = bad
    c.d_table = torch.tensor(c.table, dtype=torch.int32, device="cuda")
    out, lse = c.call(binding)
    c.check(draft, out, lse)


def test_lengths_past_the_table_are_cut_to_it(env):
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=64, heads=1, group=1, page=32, lens=[64, 32], nodes=[1, 1], seed=8)
    narrow = c.d_table[:, :2].contiguous()
    want = c.call(binding)
    c.d_table, c.d_lens = narrow, torch.tensor([5000, -3], dtype=torch.int32, device="cuda")
    out, lse = c.call(binding)
    assert torch.equal(out[0], want[0][0]) and torch.equal(lse[0], want[1][0])
    assert torch.equal(out[1], c.v[1])


def test_offsets_past_32_bits(env):
    """A layer of more than 2^31 elements, and a layer that begins behind 2^32 bytes."""
    torch, binding, draft = env
    page, heads, dim = 256, 32, 256
    per = page * heads * dim
    pages = (1 << 31) // per + 9
    K = torch.zeros((2, pages, heads, page, dim), dtype=torch.bfloat16, device="cuda")
    V = torch.zeros((2, pages, heads, page // 8, dim, 8), dtype=torch.bfloat16, device="cuda")
    cache = binding.KVCache(K, V)
    g = torch.Generator(device="cuda").manual_seed(1)
    q = torch.randn((2, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    table = torch.tensor([[pages - 1, 3], [5, pages - 2]], dtype=torch.int32, device="cuda")
    lens = torch.tensor([300, 290], dtype=torch.int32, device="cuda")
    starts = torch.tensor([0, 1, 2], dtype=torch.int32, device="cuda")
    small_k = torch.randn((2, 4, heads, page, dim), device="cuda", generator=g).to(torch.bfloat16)
    small_v = torch.randn((2, 4, heads, page // 8, dim, 8), device="cuda", generator=g).to(torch.bfloat16)
    for i, p in enumerate((pages - 1, 3, 5, pages - 2)):
        K[:, p], V[:, p] = small_k[:, i], small_v[:, i]
    small = binding.KVCache(small_k, small_v)
    near = torch.tensor([[0, 1], [2, 3]], dtype=torch.int32, device="cuda")
    for layer in (0, 1):
        a = binding.tree_attn(cache, layer, q, q, q, table, lens, starts, max_nodes=1)
        b = binding.tree_attn(small, layer, q, q, q, near, lens, starts, max_nodes=1)
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())
    # a commit to the far end
    new = torch.randn((2, 1, heads, dim), device="cuda", generator=g).to(torch.bfloat16)
    slot = torch.tensor([pages * page - 3], dtype=torch.int64, device="cuda")
    binding.kv_commit(cache, new, new, slot)
    assert torch.equal(K[:, pages - 1, :, page - 3], new[:, 0])
    assert torch.equal(V[:, pages - 1, :, page // 8 - 1, :, 5], new[:, 0])


def test_repeats_streams_and_graphs(env):
    """The same bits on every call, on another stream, and from a graph replayed on lengths that change in between."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=128, heads=2, group=4, page=64, lens=[900, 2100], nodes=[5, 8], seed=13)
    out, lse = c.call(binding)
    for _ in range(3):
        again = c.call(binding)
        assert torch.equal(again[0], out) and torch.equal(again[1], lse)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        other = c.call(binding)
    side.synchronize()
    assert torch.equal(other[0], out) and torch.equal(other[1], lse)
    o, z = torch.empty_like(out), torch.empty_like(lse)
    ws = torch.empty(binding.tree_attn_workspace_bytes(c.cache, 8, 2, c.d_table.shape[1], c.max_nodes), dtype=torch.uint8,
                     device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        c.call(binding, out=o, lse=z, ws=ws)
    for lens in ([900, 2100], [0, 77], [899, 1], [333, 2048]):
        c.d_lens.copy_(torch.tensor(lens, dtype=torch.int32))
        c.lens = lens
        graph.replay()
        torch.cuda.synchronize()
        c.check(draft, o, z)
        want = c.call(binding)
        assert torch.equal(want[0], o) and torch.equal(want[1], z)


def test_no_rows(env):
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=64, heads=1, group=2, page=32, lens=[50], nodes=[3], seed=4)
    out = binding.tree_attn(c.cache, 0, c.q[:0], c.k[:0], c.v[:0], c.d_table, c.d_lens, torch.zeros(2, dtype=torch.int32, device="cuda"))
    assert out.shape == (0, 2, 64)


def test_binding_refuses_what_does_not_go_together(env):
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=64, heads=2, group=2, page=32, lens=[50], nodes=[3], seed=4)
    E = binding.SvdpError
    ok = dict(cache=c.cache, layer=0, q=c.q, k=c.k, v=c.v, table=c.d_table, lens=c.d_lens, starts=c.d_starts)
    binding.tree_attn(**ok)
    for bad in (dict(q=c.q.float()), dict(k=c.k[:2]), dict(v=c.v[:, :1]), dict(q=c.q[:, :3]), dict(layer=2), dict(layer=-1),
                dict(max_nodes=65), dict(max_nodes=0), dict(lens=c.d_lens.long()), dict(starts=c.d_starts[:1]), dict(table=c.d_table.t()),
                dict(scale=float("nan")), dict(scale=float("inf")), dict(tree=c.d_starts), dict(q=c.q.transpose(0, 1).contiguous().transpose(0, 1)),
                dict(q=c.q.cpu()), dict(ws=torch.empty(0, dtype=torch.uint8, device="cuda")),
                dict(out=torch.empty((3, 4, 64), device="cuda")), dict(lse=torch.empty((3, 3), device="cuda"))):
        with pytest.raises(E):
            binding.tree_attn(**{**ok, **bad})
    with pytest.raises(E):
        binding.KVCache(c.cache.K, c.cache.V.float())
    with pytest.raises(E):
        binding.KVCache(c.cache.K, c.cache.V[:1])
    with pytest.raises(E):
        binding.KVCache.empty(1, 1, 64, 1, 64, dtype=torch.float16)
    odd = binding.KVCache.empty(1, 1, 48, 1, 64)
    with pytest.raises(E, match="unsupported"):
        binding.tree_attn_workspace_bytes(odd, 1, 1, 1, 1)


@pytest.mark.parametrize("dim", [64, 128])
def test_many_requests_of_many_rows(env, dim):
    """More requests than a wave has lanes, for the kernel whose waves take different rows."""
    torch, binding, draft = env
    rng = np.random.default_rng(4)
    lens = [int(v) for v in rng.integers(0, 200, 100)]
    nodes = [24] + [int(v) for v in rng.integers(0, 25, 99)]
    c = Attn(torch, binding, dtype="bf16", dim=dim, heads=2, group=3, page=32, lens=lens, nodes=nodes, tree="random", seed=6)
    out, lse = c.call(binding)
    c.check(draft, out, lse)


@pytest.mark.parametrize("dtype,dim,group", [("bf16", 64, 2), ("bf16", 128, 2), ("bf16", 128, 4), ("bf16", 256, 4), ("f32", 64, 2), ("f32", 128, 4)])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
def test_few_rows_do_not_see_what_is_hidden(env, dtype, dim, group, bad):
    """One and two row tiles: the places behind a length and a node that not every row sees."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype=dtype, dim=dim, heads=2, group=group, page=64, lens=[70, 0, 33], nodes=[7, 4, 5], seed=12)
    out, lse = c.call(binding)
    c.check(draft, out, lse)
    e = 8 if dtype == "bf16" else 4
    K, V = c.cache.K, c.cache.V
    for r, n in enumerate(c.lens):
        for j in range(n, -(-n // c.page) * c.page):
            K[1, c.table[r][j // c.page], :, j % c.page] = bad
            V[1, c.table[r][j // c.page], :, j % c.page // e, :, j % e] = bad
    out2, lse2 = c.call(binding)
    assert torch.equal(out, out2) and torch.equal(lse, lse2)
    t = c.starts[0] + 6
    c.k[t] = bad
    c.v[t] = bad
    out3, lse3 = c.call(binding)
    blind = torch.tensor([i >= c.starts[1] or not (c.words[i] >> 6) & 1 for i in range(c.starts[-1])], device="cuda")
    scale = out.float().abs().amax()
    assert float((out3.float() - out.float()).abs()[blind].amax()) <= (2.0 ** -7 if dtype == "bf16" else 1e-5) * scale
    assert float((lse3 - lse).abs()[blind].amax()) <= 1e-5
    assert not bool(torch.isfinite(out3[t].float()).any())


@pytest.mark.parametrize("tree", ["tree", None])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:5])))
def test_tables_wider_than_the_requests_are_long(env, shape, tree):
    """Room for long requests, of which the host knows nothing but the table's width: what is short is cut all the same."""
    torch, binding, draft = env
    dtype, dim, heads, group, page, lens, nodes = shape
    c = Attn(torch, binding, dtype=dtype, dim=dim, heads=heads, group=group, page=page, lens=lens, nodes=nodes, tree=tree, seed=len(lens) + dim)
    narrow = c.call(binding)
    wide = torch.full((c.d_table.shape[0], 4096 // page), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :c.d_table.shape[1]] = c.d_table
    c.d_table = wide
    out, lse = c.call(binding)
    c.check(draft, out, lse)
    assert float((out.float() - narrow[0].float()).abs().amax()) <= 2.0 ** -6 * float(out.float().abs().amax())


@pytest.mark.parametrize("dtype,dim,group", [("bf16", 128, 2), ("bf16", 128, 5), ("bf16", 128, 9), ("bf16", 64, 9), ("bf16", 256, 2), ("f32", 64, 2), ("f32", 128, 5)])
def test_cut_requests_with_padding_limits_and_missing_pages(env, dtype, dim, group):
    """Tables with room for much more: work is cut into parts, of rows that are no node, pages that do not exist, requests of nothing."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype=dtype, dim=dim, heads=2, group=group, page=32, lens=[700, 20, 0, 1500, 0], nodes=[10, 4, 3, 6, 0], pad=5, seed=21)
    for r, i, bad in ((0, 0, -1), (0, 21, c.cache.pages), (1, 0, -(1 << 31)), (3, 5, (1 << 31) - 1), (3, 6, 1 << 29)):
        c.table[r][i] = bad
    wide = torch.full((5, 128), 1 << 30, dtype=torch.int32, device="cuda")
    wide[:, :c.d_table.shape[1]] = torch.tensor(c.table, dtype=torch.int32)
    c.d_table = wide
    T, hq = c.starts[-1] + 5, 2 * group
    out = torch.full((T, hq, dim), 7.0, dtype=c.q.dtype, device="cuda")
    lse = torch.full((T, hq), 7.0, device="cuda")
    c.call(binding, out=out, lse=lse, max_nodes=6)
    c.check(draft, out, lse, max_nodes=6)
    for rows in (slice(6, 10), slice(c.starts[-1], T)):
        assert bool((out[rows] == 7).all()) and bool((lse[rows] == 7).all())
