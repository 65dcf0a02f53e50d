"""How far the weights of the bf16 attention are off by themselves, in every kernel: less than the output's own rounding hides."""
import numpy as np
import pytest

from draft_cases import U16, Attn, attention_bound

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from oracle import draft
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding, draft


@pytest.mark.parametrize("lens", [[3, 0, 40], [500, 61, 1300]], ids=["whole", "cut"])
@pytest.mark.parametrize("dim,group,nodes", [(64, 1, [1, 2, 3]), (64, 2, [9, 12, 1]), (64, 3, [20, 7, 30]), (128, 1, [1, 4, 9]), (128, 4, [8, 5, 3]),
                                             (128, 7, [30, 64, 2]), (256, 2, [4, 20, 1])])
def test_weights_are_off_by_less_than_the_output(env, dim, group, nodes, lens):
    """V is zero but for one token of each request: an output is that token's weight times V, with the weight's error in full.

    The output is rounded once, to 2^-8 of itself, and a weight is kept in two terms, within 2^-15 of its value in fp32; what the fp32
    arithmetic adds is attention_bound's."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=dim, heads=2, group=group, page=32, lens=lens, nodes=nodes, seed=dim + group)
    first = c.v[torch.tensor(c.starts[:-1]).cuda()].clone()
    c.v.zero_()
    V = c.cache.V[c.layer]
    for r, n in enumerate(lens):
        t = n // 2                                                       # a token of the cache, or of the tree where there is none
        if n == 0:
            c.v[c.starts[r]] = first[r]
        for i in range(-(-n // 32)):
            keep = V[c.table[r][i], :, t % 32 // 8, :, t % 8].clone()
            V[c.table[r][i]] = 0
            if i == t // 32:
                V[c.table[r][i], :, t % 32 // 8, :, t % 8] = keep
    out, lse = c.call(binding)
    c.check(draft, out, lse)
    o, z, w, reach = c.expect(draft)
    b, _ = attention_bound(w, o, reach, z, max(lens) + 64, dim, bf16=False)
    b += w * 1.01 * 2.0 ** -15 + np.abs(o) * 1.01 * U16
    off = np.abs(out.float().cpu().numpy().astype(np.float64) - o) / b
    assert off.max() <= 1.0, off.max()


@pytest.mark.parametrize("lens", [[3, 1, 40], [500, 61, 1300]], ids=["whole", "cut"])
@pytest.mark.parametrize("dim,group,nodes", [(64, 1, [1, 2, 3]), (64, 2, [9, 12, 1]), (64, 3, [20, 7, 30]), (128, 1, [1, 4, 9]), (128, 4, [8, 5, 3]),
                                             (128, 7, [30, 64, 2]), (256, 2, [4, 20, 1])])
def test_infinities_of_the_cache_stay_infinities(env, dim, group, nodes, lens):
    """Neither term of a weight may be zero or negative: infinity times that would be NaN, or the other infinity.  Weights of one (a
    single token, the largest score) among them."""
    torch, binding, draft = env
    c = Attn(torch, binding, dtype="bf16", dim=dim, heads=2, group=group, page=32, lens=lens, nodes=nodes, tree="random", seed=dim + group)
    want, _ = c.call(binding)
    V = c.cache.V[c.layer]
    for r, n in enumerate(lens):
        for t, channel, bad in ((0, 7, "inf"), (n - 1, 30, "-inf"), (n // 2, dim - 1, "nan")):
            V[c.table[r][t // 32], :, t % 32 // 8, channel, t % 8] = float(bad)
    out, _ = c.call(binding)
    rows = slice(0, c.starts[-1])
    assert bool((out[rows, :, 7] == float("inf")).all()) and bool((out[rows, :, 30] == float("-inf")).all())
    assert bool(torch.isnan(out[rows, :, dim - 1]).all())
    other = [i for i in range(dim) if i not in (7, 30, dim - 1)]
    assert torch.equal(out[rows][:, :, other], want[rows][:, :, other])
