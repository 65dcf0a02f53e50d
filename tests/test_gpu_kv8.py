"""K and V of a cache in 8 bits as they are written, and K and V of any cache read back: values and copies, so everything is equal."""
import numpy as np
import pytest

from serve_cases import decoded, exponents, fill_cache

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from oracle import serve
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding, serve


def i64(torch, v):
    return torch.tensor(v, dtype=torch.int64, device="cuda")


def arrays(torch, cache):
    by = (exponents(torch, cache.K_scale), exponents(torch, cache.V_scale)) if cache.K_scale is not None else (None, None)
    return decoded(cache.K), decoded(cache.V), *by


def same(torch, cache, want):
    got = arrays(torch, cache)
    for g, w in zip(got, want):
        assert np.array_equal(g, w, equal_nan=True)


def slots_of(rng, T, total):
    """Prompts and branches: runs of places that follow each other, places on their own, rows that are not stored, places that are not there."""
    free = [int(v) for v in rng.permutation(total // 8)]
    out = []
    while len(out) < T:
        kind = rng.integers(0, 5)
        if kind < 2 and len(free) > 4:
            start = free.pop() * 8 + int(rng.integers(0, 3)) * int(kind)
            out += list(range(start, start + 8 - start % 8))
        elif kind == 2 and free:
            out.append(free.pop() * 8 + int(rng.integers(0, 8)))
        else:
            out.append(int(rng.choice([-1, -(1 << 40), total, total + 5, 1 << 40])))
    return out[:T]


@pytest.mark.parametrize("dim,heads,page,layers,T", [(64, 2, 32, 3, 1), (64, 5, 64, 1, 29), (128, 8, 64, 2, 100), (128, 1, 128, 1, 8), (128, 32, 64, 4, 5),
                                                     (256, 3, 256, 2, 50), (128, 4, 32, 1, 1000)])
def test_commit_against_the_oracle(env, dim, heads, page, layers, T):
    torch, binding, serve = env
    rng = np.random.default_rng(T + dim)
    pages = 40 if T < 500 else 100
    cache = binding.KVCache.empty(layers, pages, page, heads, dim, dtype=torch.float8_e4m3fn)
    fill_cache(torch, cache, 3)
    g = torch.Generator(device="cuda").manual_seed(T)
    rows = torch.randn((layers, T, heads + 1, 2, dim), device="cuda", generator=g).bfloat16()
    rows *= 2.0 ** torch.randint(-20, 20, (layers, T, heads + 1, 2, 1), device="cuda", generator=g)
    wide = rows.transpose(2, 3).contiguous()                 # K's heads, one more, V's heads, one more
    k, v = wide[:, :, 0, :heads], wide[:, :, 1, :heads]
    slots = slots_of(rng, T, pages * page)
    want = arrays(torch, cache)
    serve.commit(*want, decoded(k), decoded(v), slots)
    binding.kv_commit(cache, k, v, i64(torch, slots))
    same(torch, cache, want)


def test_commit_of_values_at_the_borders(env):
    """Zeros, numbers at and right above 448 2^b, ties between codes, the largest and smallest numbers, infinities and NaN."""
    torch, binding, serve = env
    dim, T = 64, 24
    x = torch.randn((1, T, 1, dim), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)).bfloat16()
    x[0, 0] = 0
    x[0, 1] = -0.0
    x[0, 2, 0, :2] = torch.tensor([448.0, 17.0])                    # b = 0: 448 is a code
    x[0, 3, 0, :2] = torch.tensor([450.0, 17.0])                    # the next bf16 number: b = 1
    x[0, 4, 0, :4] = torch.tensor([224.0, 9.5, 10.5, 8.25])         # ties at b = -1
    x[0, 5, 0, 0] = 3.38e38
    x[0, 6] = 1e-38
    x[0, 7] = 9.2e-41                                               # a number below the normal ones
    x[0, 8, 0, 3] = float("inf")
    x[0, 9, 0, 4] = float("-inf")
    x[0, 10, 0, 5] = float("nan")
    x[0, 11] = float("inf")
    x[0, 12] = float("nan")
    x[0, 13] = 2.0 ** -96 * 448                                     # the least power of two, just in use
    x[0, 14] = 2.0 ** -96
    x[0, 15] = 2.0 ** -105                                          # the least code, then half of it: a tie, to zero
    x[0, 16] = 2.0 ** -106
    x[0, 17] = torch.linspace(-448, 448, dim).bfloat16()
    x[0, 18] = 2.0 ** -torch.arange(0, dim).float()                 # down to where codes end
    cache = binding.KVCache.empty(1, 2, 32, 1, dim, dtype=torch.float8_e4m3fn)
    for slots in (list(range(8, 8 + T)), [2 * i for i in range(T)]):          # whole packs, and tokens on their own
        fill_cache(torch, cache, 5)
        want = arrays(torch, cache)
        serve.commit(*want, decoded(x), decoded(x), slots)
        binding.kv_commit(cache, x, x, i64(torch, slots))
        same(torch, cache, want)


@pytest.mark.parametrize("dtype", ["e4m3", "bf16", "f32"])
@pytest.mark.parametrize("dim,heads,page,layers,T", [(64, 2, 32, 3, 1), (128, 8, 64, 2, 100), (256, 3, 256, 1, 50), (128, 2, 32, 1, 1001), (64, 33, 64, 2, 9)])
def test_read_against_the_oracle(env, dtype, dim, heads, page, layers, T):
    torch, binding, serve = env
    rng = np.random.default_rng(T + heads)
    td = {"e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    pages = 40 if T < 500 else 100
    cache = binding.KVCache.empty(layers, pages, page, heads, dim, dtype=td)
    if dtype == "e4m3":
        fill_cache(torch, cache, 4)
    else:
        cache.K.normal_()
        cache.V.normal_()
    slots = slots_of(rng, T, pages * page)
    if T > 8:
        slots[5] = slots[T - 1] = 17                           # the same one twice
    want = serve.read(*arrays(torch, cache), slots)
    before = [t.clone().view(torch.uint8) for t in (cache.K, cache.V)]
    k, v = binding.kv_read(cache, i64(torch, slots))
    assert k.dtype is (td if dtype != "e4m3" else torch.bfloat16)
    assert np.array_equal(decoded(k), want[0]) and np.array_equal(decoded(v), want[1])
    assert all(torch.equal(a, t.view(torch.uint8)) for a, t in zip(before, (cache.K, cache.V)))
    # into rows that are slices of something wider; what lies between stays
    wide = torch.full((layers, T + 2, 2 * heads + 1, dim), 7.0, dtype=cache.rows, device="cuda")
    binding.kv_read(cache, i64(torch, slots), k=wide[:, 1:-1, :heads], v=wide[:, 1:-1, heads + 1:])
    assert torch.equal(wide[:, 1:-1, :heads], k) and torch.equal(wide[:, 1:-1, heads + 1:], v)
    assert bool((wide[:, [0, -1]] == 7).all()) and bool((wide[:, :, heads] == 7).all())


@pytest.mark.parametrize("dtype", ["e4m3", "bf16", "f32"])
def test_what_is_read_and_stored_again_is_the_same(env, dtype):
    """A request that leaves and comes back, to other places: not a bit of its values is lost, in 8 bits either."""
    torch, binding, serve = env
    td = {"e4m3": torch.float8_e4m3fn, "bf16": torch.bfloat16, "f32": torch.float32}[dtype]
    cache = binding.KVCache.empty(3, 20, 32, 4, 128, dtype=td)
    new = [torch.randn((3, 250, 4, 128), device="cuda").to(cache.rows) for _ in range(2)]
    here, there = torch.randperm(320, device="cuda")[:250], 320 + torch.arange(250, device="cuda")
    binding.kv_commit(cache, *new, here)
    k, v = binding.kv_read(cache, here)
    if dtype != "e4m3":
        assert torch.equal(k, new[0]) and torch.equal(v, new[1])
    binding.kv_commit(cache, k, v, there)
    again = binding.kv_read(cache, there)
    assert torch.equal(again[0], k) and torch.equal(again[1], v)


def test_read_of_codes_that_are_not_finite_and_of_far_scales(env):
    """NaN codes are NaN; the least and the largest power of two that rows in bf16 hold."""
    torch, binding, serve = env
    cache = binding.KVCache.empty(1, 1, 32, 1, 64, dtype=torch.float8_e4m3fn)
    fill_cache(torch, cache, 2)
    cache.K.view(torch.uint8)[0, 0, 0, 3, 5] = 0x7f
    cache.V.view(torch.uint8)[0, 0, 0, 1, 9, 2] = 0xff        # token 10
    for t in (cache.K_scale, cache.V_scale):
        t.view(torch.uint8)[0, 0, 0, 4] = 31
        t.view(torch.uint8)[0, 0, 0, 6] = 246
    for slots in (list(range(32)), [7, 10, 3, 6, 4, 31]):
        want = serve.read(*arrays(torch, cache), slots)
        k, v = binding.kv_read(cache, i64(torch, slots))
        assert np.array_equal(decoded(k), want[0], equal_nan=True) and np.array_equal(decoded(v), want[1], equal_nan=True)


def test_offsets_past_32_bits(env):
    """Layers of more than 2^32 bytes: rows to and from the far end."""
    torch, binding, serve = env
    page, heads, dim = 256, 32, 256
    pages = (1 << 32) // (page * heads * dim) + 3
    cache = binding.KVCache.empty(2, pages, page, heads, dim, dtype=torch.float8_e4m3fn)
    new = [torch.randn((2, 11, heads, dim), device="cuda").bfloat16() for _ in range(2)]
    slots = torch.arange(pages * page - 11, pages * page, device="cuda")
    binding.kv_commit(cache, *new, slots)
    small = binding.KVCache.empty(2, 1, page, heads, dim, dtype=torch.float8_e4m3fn)
    near = torch.arange(page - 11, page, device="cuda")
    binding.kv_commit(small, *new, near)
    for a, b in ((cache.K, small.K), (cache.K_scale, small.K_scale)):
        assert torch.equal(a.view(torch.uint8)[:, -1, :, -11:], b.view(torch.uint8)[:, -1, :, -11:])
    for a, b in zip(binding.kv_read(cache, slots), binding.kv_read(small, near)):
        assert torch.equal(a, b)
    serve_k, _ = serve.read(*arrays(torch, small), near.tolist())
    assert np.array_equal(decoded(binding.kv_read(cache, slots)[0]), serve_k)


def test_no_rows_streams_and_graphs(env):
    torch, binding, serve = env
    cache, other = (binding.KVCache.empty(2, 9, 32, 2, 64, dtype=torch.float8_e4m3fn) for _ in range(2))
    none = i64(torch, [])
    k, v = binding.kv_read(cache, none)
    assert k.shape == v.shape == (2, 0, 2, 64)
    binding.kv_commit(cache, k, v, none)
    slots = torch.randperm(9 * 32, device="cuda")[:40]
    new = torch.randn((2, 40, 2, 64), device="cuda").bfloat16()
    out = [torch.empty_like(new) for _ in range(2)]
    for c in (cache, other):
        fill_cache(torch, c, 1)
    graph = torch.cuda.CUDAGraph()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        binding.kv_commit(cache, new, new, slots)
        binding.kv_read(cache, slots, k=out[0], v=out[1])
    side = torch.cuda.Stream()
    for step in range(3):
        slots.copy_(torch.randperm(9 * 32, device="cuda")[:40])
        new.normal_()
        graph.replay()
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            binding.kv_commit(other, new, new, slots)
            k, v = binding.kv_read(other, slots)
        side.synchronize()
        assert torch.equal(out[0], k) and torch.equal(out[1], v)
        for n in ("K", "V", "K_scale", "V_scale"):
            assert torch.equal(getattr(cache, n).view(torch.uint8), getattr(other, n).view(torch.uint8))


def test_binding_refuses_what_does_not_go_together(env):
    torch, binding, serve = env
    E = binding.SvdpError
    c = binding.KVCache.empty(2, 4, 32, 2, 64, dtype=torch.float8_e4m3fn)
    new, slots = torch.zeros((2, 3, 2, 64), dtype=torch.bfloat16, device="cuda"), i64(torch, [1, 2, 3])
    binding.kv_commit(c, new, new, slots)
    for k, v, s in ((new.float(), new, slots), (new, new.to(torch.float8_e4m3fn), slots), (new, new[:1], slots), (new[:, :2], new, slots), (new, new, slots.int()),
                    (new, new, slots.cpu()), (new.cpu(), new, slots), (new.transpose(1, 2).contiguous().transpose(1, 2), new, slots)):
        with pytest.raises(E):
            binding.kv_commit(c, k, v, s)
        with pytest.raises(E):
            binding.kv_read(c, s, k=k, v=v)
    for K, V, a, b in ((c.K, c.V, None, None), (c.K, c.V, c.K_scale, None), (c.K, c.V, c.K_scale.view(torch.uint8), c.V_scale), (c.K, c.V, c.K_scale[:1], c.V_scale),
                       (c.K, c.V[:, :1], c.K_scale, c.V_scale), (c.K, c.V.view(torch.uint8), c.K_scale, c.V_scale)):
        with pytest.raises(E):
            binding.KVCache(K, V, a, b)
    plain = binding.KVCache.empty(2, 4, 32, 2, 64)
    with pytest.raises(E):
        binding.KVCache(plain.K, plain.V, c.K_scale, c.V_scale)
