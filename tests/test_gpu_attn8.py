"""Attention over a cache of 8 bits, against the 64-bit oracle on the values that its codes stand for."""
import numpy as np
import pytest

from serve_cases import Attn8, fill_cache

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
    # dim, heads, group, page, lens, nodes
    (128, 2, 1, 64, [1], [1]), (128, 3, 1, 64, [777], [1]), (128, 2, 4, 64, [0, 1, 31, 32, 33, 63, 64, 65], [1, 2, 3, 4, 5, 6, 7, 8]),
    (128, 2, 8, 32, [7, 8, 9, 500], [4, 1, 3, 2]), (128, 1, 7, 128, [127, 128, 129, 1000], [64, 33, 17, 1]), (128, 1, 8, 256, [255, 700], [64, 64]),
    (128, 2, 5, 32, [95, 96, 97, 411], [13, 32, 0, 47]), (64, 2, 2, 32, [2, 0, 500], [31, 9, 16]), (64, 1, 16, 64, [300, 4], [40, 64]),
    (64, 3, 1, 128, [129, 1], [1, 1]), (64, 2, 4, 64, [70, 300], [6, 8]), (256, 2, 1, 64, [200, 0, 65], [1, 40, 3]), (256, 1, 6, 32, [100, 33], [64, 11]),
]


@pytest.mark.parametrize("tree", ["tree", "random", None])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_attention_against_the_oracle(env, shape, tree):
    torch, binding, draft = env
    dim, heads, group, page, lens, nodes = shape
    c = Attn8(torch, binding, dim=dim, heads=heads, group=group, page=page, lens=lens, nodes=nodes, tree=tree, seed=len(lens) * 100 + dim,
              strided=dim != 64)
    c.check(draft, *c.call(binding))


@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "-".join(map(str, s[:4])))
def test_tables_wider_than_the_requests_are_long(env, shape):
    """Room for long requests: what is short is cut into parts all the same, and joined."""
    torch, binding, draft = env
    dim, heads, group, page, lens, nodes = shape
    c = Attn8(torch, binding, dim=dim, heads=heads, group=group, page=page, lens=lens, nodes=nodes, seed=len(lens) + dim)
    wide = torch.full((len(lens), 8000 // page), -1, dtype=torch.int32, device="cuda")
    wide[:, :c.d_table.shape[1]] = c.d_table
    c.d_table, c.table = wide, wide.tolist()
    c.check(draft, *c.call(binding))


@pytest.mark.parametrize("heads,group,lens,nodes", [(4, 1, [6001, 3, 900], [1, 2, 1]), (1, 4, [9001], [8]), (1, 7, [5000, 5100], [64, 50]),
                                                    (8, 4, [5001, 2300], [1, 1])])
def test_long_contexts(env, heads, group, lens, nodes):
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=128, heads=heads, group=group, page=64, lens=lens, nodes=nodes, seed=7, spread=2.0)
    c.check(draft, *c.call(binding))


@pytest.mark.parametrize("most", [3, 40])
def test_many_requests(env, most):
    """More requests than a wave has lanes, requests without rows and without tokens among them; few rows of each, and many."""
    torch, binding, draft = env
    rng = np.random.default_rng(most)
    lens = [int(v) for v in rng.integers(0, 90, 150)]
    nodes = [most] + [int(v) for v in rng.integers(0, most + 1, 149)]
    c = Attn8(torch, binding, dim=64, heads=1, group=2, page=32, lens=lens, nodes=nodes, tree="random", seed=5)
    c.check(draft, *c.call(binding))


@pytest.mark.parametrize("dim", [64, 128, 256])
@pytest.mark.parametrize("nodes", [[1, 1, 1], [7, 4, 5], [7, 40, 5]], ids=["one", "few", "many"])
def test_what_a_row_does_not_see_has_no_influence(env, dim, nodes):
    """NaN codes and scales of any kind behind a length, in pages of no request and in another layer: the output's bits stay the same."""
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=dim, heads=2, group=3, page=64, lens=[70, 0, 33], nodes=nodes, seed=11)
    out, lse = c.call(binding)
    c.check(draft, out, lse)
    cache = c.cache
    used = torch.zeros(cache.pages, c.page, dtype=torch.bool)
    for r, n in enumerate(c.lens):
        for j in range(n):
            used[c.table[r][j // c.page], j % c.page] = True
    used = used.cuda()
    raw = {n: getattr(cache, n).view(torch.uint8) for n in ("K", "V", "K_scale", "V_scale")}
    for code, scale in ((0x7f, 255), (0xff, 254), (0x7e, 0)):
        raw["K"][1].masked_fill_(~used[:, None, :, None], code)
        raw["V"][1].masked_fill_(~used.reshape(cache.pages, 1, c.page // 8, 1, 8), code)
        for n in ("K_scale", "V_scale"):
            raw[n][1].masked_fill_(~used[:, None, :], scale)
            raw[n][0].fill_(scale)
        raw["K"][0].fill_(code)
        raw["V"][0].fill_(code)
        again = c.call(binding)
        assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("bad", [float("nan"), float("inf"), float("-inf")])
@pytest.mark.parametrize("dim,group,nodes", [(64, 2, 7), (128, 2, 7), (128, 4, 7), (128, 7, 40), (256, 2, 7)])
def test_nodes_that_a_row_does_not_see(env, dim, group, nodes, bad):
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=dim, heads=2, group=group, page=64, lens=[70, 0], nodes=[nodes, nodes], seed=12)
    out, lse = c.call(binding)
    t = c.starts[0] + 5
    c.k[t] = bad
    c.v[t] = bad
    out3, lse3 = c.call(binding)
    blind = torch.tensor([i >= c.starts[1] or not (c.words[i] >> 5) & 1 for i in range(c.starts[-1])], device="cuda")
    scale = out.float().abs().amax()
    assert float((out3.float() - out.float()).abs()[blind].amax()) <= 2.0 ** -7 * scale
    assert float((lse3 - lse).abs()[blind].amax()) <= 1e-5
    assert not bool(torch.isfinite(out3[t].float()).any())


@pytest.mark.parametrize("nodes", [3, 40])
def test_nan_codes_that_a_row_does_see(env, nodes):
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=64, heads=1, group=1, page=32, lens=[40], nodes=[nodes], tree=None, seed=2)
    want, _ = c.call(binding)
    c.cache.V.view(torch.uint8)[1, c.table[0][1], 0, 0, 5, 3] = 0x7f     # token 35, channel 5
    out, lse = c.call(binding)
    assert bool(torch.isnan(out[:, 0, 5]).all()) and bool(torch.isfinite(lse).all())
    other = [i for i in range(64) if i != 5]
    assert torch.equal(out[:, 0, other], want[:, 0, other])
    c.cache.K.view(torch.uint8)[1, c.table[0][0], 0, 7, 0] = 0xff
    out, lse = c.call(binding)
    assert bool(torch.isnan(out).all()) and bool(torch.isnan(lse).all())


@pytest.mark.parametrize("nodes", [9, 64])
def test_large_scores_and_far_scales(env, nodes):
    """Scores of some hundreds; and tokens whose powers of two lie 2^60 apart."""
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=128, heads=1, group=4, page=64, lens=[1500], nodes=[nodes], seed=21)
    for scale in (4.0, -4.0, 0.0):
        c.check(draft, *c.call(binding, scale=scale), scale=scale)
    for t in (c.cache.K_scale, c.cache.V_scale):
        t.view(torch.uint8)[:, :, :, ::3] = 60
    c.cache.V_scale.view(torch.uint8)[:, :, :, 1::3] = 150
    c.v *= 2.0 ** 20
    c.check(draft, *c.call(binding))


def test_padding_missing_pages_and_lengths_past_the_table(env):
    torch, binding, draft = env
    for nodes in ([10, 4], [40, 33]):
        c = Attn8(torch, binding, dim=128, heads=1, group=2, page=32, lens=[100, 300], nodes=nodes, pad=5, seed=4)
        for r, i, bad in ((0, 1, -1), (0, 3, c.cache.pages), (1, 0, -(1 << 31)), (1, 5, (1 << 31) - 1)):
            c.table[r][i] = bad
        c.d_table = torch.tensor(c.table, dtype=torch.int32, device="cuda")
        T = sum(nodes) + 5
        out, lse = torch.full((T, 2, 128), 7.0, dtype=torch.bfloat16, device="cuda"), torch.full((T, 2), 7.0, device="cuda")
        c.call(binding, out=out, lse=lse, max_nodes=nodes[0] - 4)
        c.check(draft, out, lse, max_nodes=nodes[0] - 4)
        for rows in (slice(nodes[0] - 4, nodes[0]), slice(T - 5, T)):
            assert bool((out[rows] == 7).all()) and bool((lse[rows] == 7).all())
    c = Attn8(torch, binding, dim=64, heads=1, group=1, page=32, lens=[64, 32], nodes=[1, 1], seed=8)
    want = c.call(binding)
    c.d_table, c.d_lens = c.d_table[:, :2].contiguous(), torch.tensor([5000, -3], dtype=torch.int32, device="cuda")
    out, lse = c.call(binding)
    assert torch.equal(out[0], want[0][0]) and torch.equal(lse[0], want[1][0]) and torch.equal(out[1], c.v[1])


@pytest.mark.parametrize("nodes", [1, 40])
def test_offsets_past_32_bits(env, nodes):
    torch, binding, draft = env
    page, heads, dim = 256, 32, 128
    pages = (1 << 32) // (page * heads * dim) + 5
    cache = binding.KVCache.empty(2, pages, page, heads, dim, dtype=torch.float8_e4m3fn)
    small = binding.KVCache.empty(2, 4, page, heads, dim, dtype=torch.float8_e4m3fn)
    fill_cache(torch, small, 3)
    far = [pages - 1, 3, 5, pages - 2]
    for n in ("K", "V", "K_scale", "V_scale"):
        for i, p in enumerate(far):
            getattr(cache, n).view(torch.uint8)[:, p] = getattr(small, n).view(torch.uint8)[:, i]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    q = torch.randn((2 * nodes, heads, dim), device="cuda").bfloat16()
    lens, starts = i32([300, 290]), i32([0, nodes, 2 * nodes])
    for layer in (0, 1):
        a = binding.tree_attn(cache, layer, q, q, q, i32([far[:2], far[2:]]), lens, starts, max_nodes=nodes)
        b = binding.tree_attn(small, layer, q, q, q, i32([[0, 1], [2, 3]]), lens, starts, max_nodes=nodes)
        assert torch.equal(a, b) and bool(torch.isfinite(a.float()).all())


@pytest.mark.parametrize("nodes", [[5, 8], [40, 64]])
def test_repeats_streams_and_graphs(env, nodes):
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=128, heads=2, group=4, page=64, lens=[900, 2100], nodes=nodes, seed=13)
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
    ws = torch.empty(binding.tree_attn_workspace_bytes(c.cache, 8, 2, c.d_table.shape[1], c.max_nodes), dtype=torch.uint8, device="cuda")
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


def test_binding_refuses_rows_of_another_type(env):
    torch, binding, draft = env
    c = Attn8(torch, binding, dim=64, heads=2, group=2, page=32, lens=[50], nodes=[3], seed=4)
    ok = dict(cache=c.cache, layer=0, q=c.q, k=c.k, v=c.v, table=c.d_table, lens=c.d_lens, starts=c.d_starts)
    assert binding.tree_attn(**ok).dtype is torch.bfloat16
    for bad in (dict(q=c.q.float()), dict(q=c.q.to(torch.float8_e4m3fn)), dict(k=c.k.float()), dict(v=c.v.to(torch.float8_e4m3fn)),
                dict(out=torch.empty((3, 4, 64), dtype=torch.float8_e4m3fn, device="cuda"))):
        with pytest.raises(binding.SvdpError):
            binding.tree_attn(**{**ok, **bad})
