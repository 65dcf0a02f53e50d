"""Caches of 8 bits whose tokens have any power of two that a scale can say, near the ends of fp32's and bf16's range too."""
import math

import numpy as np
import pytest

from draft_cases import U16, attention_bound
from serve_cases import Attn8, decoded

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from oracle import draft, serve
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding, draft, serve


# dim, group, page, nodes: 16 and 32 rows at a time, and rows over the waves
KERNELS = [(64, 2, 32, 3), (128, 2, 32, 1), (128, 2, 64, 9), (128, 4, 32, 16), (256, 2, 64, 6), (128, 2, 32, 40), (64, 4, 64, 33)]


def check(c, draft, out, lse, scale):
    """As Attn8.check, but each element is held to what reaches its own channel: outputs may be of any size.  Below 2^-126 bf16's numbers lie 2^-133
    apart, and the output's rounding is off by half of that."""
    o, z, w, reach = c.expect(draft, scale)
    bound, zb = attention_bound(w, o, reach, z, max(c.lens) + 64, c.dim, bf16=False)
    bound += w * 1.01 * 2.0 ** -15 + np.abs(o) * 1.01 * U16 + 2.0 ** -134 - 1e-30
    out, lse = decoded(out), lse.cpu().numpy().astype(np.float64)
    assert np.isfinite(out).all() and (np.abs(lse - z) <= zb).all()
    assert (np.abs(out - o) <= bound).all(), (np.abs(out - o) / np.where(bound > 0, bound, 1e-300)).max()


def codes(torch, t, values, seed):
    """Random ones of the given values."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    pick = torch.tensor(values, device="cuda")[torch.randint(len(values), t.shape, device="cuda", generator=g)]
    t.copy_(pick.to(t.dtype))


def flat_scores(torch, c, above):
    """Scores of 0, and with a scale of ln 2 of 7 in base two for the cached tokens `above`."""
    K = c.cache.K
    K.copy_(torch.zeros(K.shape, device="cuda").to(K.dtype))
    c.cache.K_scale.view(torch.uint8).fill_(127)
    seven = torch.tensor(7.0, device="cuda").to(K.dtype).view(torch.uint8)
    for r in range(len(c.lens)):
        for j in above:
            K.view(torch.uint8)[c.layer, c.table[r][j // c.page], :, j % c.page, 0] = seven
    c.q.zero_()
    c.q[:, :, 0] = 1.0
    c.k.zero_()


@pytest.mark.parametrize("dim,group,page,nodes", KERNELS)
def test_high_powers_and_a_score_that_rises(env, dim, group, page, nodes):
    """Powers of 2^123 with codes of 0 and up to 2^-8 in magnitude, so that all values are finite; scores are 0 but for a few tokens behind a wave's
    first tile, where they are 7 in base two: weights of 2^7 beside a shift that stays.  Sums are below (300 + 3 2^7 + 64) 2^115, some 2^125."""
    torch, binding, draft, _ = env
    c = Attn8(torch, binding, dim=dim, heads=2, group=group, page=page, lens=[300, 290], nodes=[nodes, max(1, nodes - 2)], seed=dim + nodes)
    cache = c.cache
    codes(torch, cache.V, [0.0, 0.0, 2.0 ** -9, -2.0 ** -9, 2.0 ** -8], 1)
    cache.V_scale.view(torch.uint8).fill_(250)
    flat_scores(torch, c, (130, 200, 287))
    c.v *= 2.0 ** 112
    scale = math.log(2.0)
    out, lse = c.call(binding, scale=scale)
    check(c, draft, out, lse, scale)


@pytest.mark.parametrize("dim,group,page,nodes", KERNELS)
def test_low_powers(env, dim, group, page, nodes):
    """Powers of 2^-126 and 2^-125 with codes of 2 to 14 in magnitude, and weights of 2^-6.5 beside those of a few tokens whose codes are 0: values
    are normal numbers (2^-126 and more), a weight times such a power is not.  The numerators are sums of 300 products, each rounded to 2^-149 at the
    worst: below 2^-140 together, 2^-149 of an output after the division by some 2^9."""
    torch, binding, draft, _ = env
    c = Attn8(torch, binding, dim=dim, heads=1, group=group, page=page, lens=[300], nodes=[nodes], seed=dim + nodes)
    cache = c.cache
    codes(torch, cache.V, [2.0, 3.25, -2.5, 14.0, -5.0, -9.0], 2)
    cache.V_scale.view(torch.uint8).copy_(torch.randint(1, 3, cache.V_scale.shape, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)))
    flat_scores(torch, c, (5, 37, 69, 101))
    raw = cache.V.view(torch.uint8)
    for j in (5, 37, 69, 101):
        raw[c.layer, c.table[0][j // page], :, j % page // 8, :, j % 8] = 0
    c.v.copy_((c.v.abs() + 1) * 2.0 ** -122)
    scale = 0.93 * math.log(2.0)                # 6.51 in base two: no weight is a power of two
    out, lse = c.call(binding, scale=scale)
    check(c, draft, out, lse, scale)


@pytest.mark.parametrize("lens", [[300], [3000]])
@pytest.mark.parametrize("dim,group,page,nodes", KERNELS)
def test_powers_far_apart(env, dim, group, page, nodes, lens):
    """Tokens of small and of large powers beside each other, the large ones' codes 0 in half of the channels: there the small ones are all that counts."""
    torch, binding, draft, _ = env
    c = Attn8(torch, binding, dim=dim, heads=1, group=group, page=page, lens=lens, nodes=[nodes], seed=dim + nodes)
    g = torch.Generator(device="cuda").manual_seed(4)
    kinds = torch.tensor([40, 60, 95, 96, 127, 159, 160, 200], dtype=torch.uint8, device="cuda")
    by = kinds[torch.randint(len(kinds), c.cache.V_scale.shape, device="cuda", generator=g)]
    by[:, :, :, :page // 2] = by[:, :, :, :page // 2].clamp(96, 159)          # tiles without a far one, and with some
    c.cache.V_scale.view(torch.uint8).copy_(by)
    # V [layers][pages][heads][page / 8][dim][8]
    large = (by > 60).view(*by.shape[:3], page // 8, 1, 8).expand_as(c.cache.V).clone()
    large[:, :, :, :, dim // 2:] = False
    c.cache.V.view(torch.uint8).masked_fill_(large, 0)
    c.v[:, :, :dim // 2] *= 2.0 ** -80
    scale = c.dim ** -0.5
    out, lse = c.call(binding)
    check(c, draft, out, lse, scale)


@pytest.mark.parametrize("dim", [64, 128, 256])
def test_the_largest_numbers_stay_finite(env, dim):
    """Every bf16 number from 2^126 on, of either sign: what was finite is read back finite and within half a step of e4m3, and stored again it is the
    same; in whole packs, and for tokens on their own."""
    torch, binding, _, serve = env
    T = 24
    rng = np.random.default_rng(dim)
    bits = np.concatenate([np.arange(0x7e80, 0x7f80), rng.integers(0x7e80, 0x7f80, T * dim)])[:T * dim]
    bits[::3] |= 0x8000
    x = torch.from_numpy(rng.permutation(bits).astype(np.uint16).view(np.int16)).view(torch.bfloat16).view(1, T, 1, dim).cuda()
    x[0, 0, 0, 0], x[0, 0, 0, 1], x[0, 0, 0, 2] = float("nan"), float("inf"), 3.3895313892515355e38
    want, by = serve.quantise(decoded(x))
    assert by.max() == 120
    for slots in (list(range(8, 8 + T)), [2 * i for i in range(T)]):
        cache = binding.KVCache.empty(1, 2, 32, 1, dim, dtype=torch.float8_e4m3fn)
        d_slots = torch.tensor(slots, dtype=torch.int64, device="cuda")
        binding.kv_commit(cache, x, x, d_slots)
        first = binding.kv_read(cache, d_slots)
        binding.kv_commit(cache, *first, d_slots)
        for rows in (first, binding.kv_read(cache, d_slots)):
            for t in rows:
                got = decoded(t)
                assert np.array_equal(got, want * 2.0 ** by[..., None].astype(float), equal_nan=True)
                fin = np.isfinite(decoded(x))
                assert np.array_equal(np.isfinite(got), fin)
                assert (np.abs(got - decoded(x))[fin] <= 2.0 ** -4 * np.abs(decoded(x))[fin]).all()


def test_read_of_every_scale_and_code(env):
    """What the header says of an element: exact from 2^-126 on, infinite past bf16's largest number, below 2^-126 no further off than that."""
    torch, binding, _, serve = env
    cache = binding.KVCache.empty(1, 1, 256, 2, 256, dtype=torch.float8_e4m3fn)
    every = torch.arange(256, device="cuda", dtype=torch.uint8)
    cache.K.view(torch.uint8).copy_(every)
    cache.V.view(torch.uint8).copy_(every[:, None])
    for t in (cache.K_scale, cache.V_scale):
        t.view(torch.uint8).copy_(every)
    value = serve.e4m3_values() * 2.0 ** (np.arange(256)[:, None] - 127.0)
    for slots in (list(range(1, 255)), list(range(254, 0, -1))):         # packs, and tokens on their own
        for rows in binding.kv_read(cache, torch.tensor(slots, dtype=torch.int64, device="cuda")):
            got, want = decoded(rows)[0], np.repeat(value[slots][:, None], 2, 1)
            normal = np.abs(want) >= 2.0 ** -126
            assert np.array_equal(got[normal], np.where(np.abs(want) >= 2.0 ** 128, np.copysign(np.inf, want), want)[normal])
            assert np.array_equal(np.isnan(got), np.isnan(want))
            assert (np.abs(got - want)[np.abs(want) < 2.0 ** -126] <= 2.0 ** -126).all()
