"""Rows that K and V are read into: every layout whose rows do not overlap, and the refusal of those that do."""
import pytest

pytestmark = pytest.mark.gpu

L, T, H, D = 3, 21, 2, 64


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    cache = binding.KVCache.empty(L, 4, 32, H, D, dtype=torch.float8_e4m3fn)
    new = [torch.randn((L, T, H, D), device="cuda").bfloat16() for _ in range(2)]
    slots = torch.randperm(4 * 32, device="cuda")[:T]
    binding.kv_commit(cache, *new, slots)
    return torch, binding, cache, slots, binding.kv_read(cache, slots)


@pytest.mark.parametrize("shape,order", [
    ((2, L, T, H, D), (0, 1, 2, 3, 4)), ((L, T, 2, H, D), (2, 0, 1, 3, 4)), ((L, 2, T, H, D), (1, 0, 2, 3, 4)), ((T, L, 2, H, D), (2, 1, 0, 3, 4)),
    ((T, 2, L, H, D), (1, 2, 0, 3, 4)), ((2, T, L, H, D), (0, 2, 1, 3, 4)),
])
def test_layers_rows_and_both_in_any_order(env, shape, order):
    torch, binding, cache, slots, want = env
    k, v = torch.zeros(shape, dtype=torch.bfloat16, device="cuda").permute(order)
    binding.kv_read(cache, slots, k=k, v=v)
    assert torch.equal(k, want[0]) and torch.equal(v, want[1])


def test_rows_that_overlap_are_refused(env):
    torch, binding, cache, slots, want = env
    empty = lambda *s: torch.zeros(s, dtype=torch.bfloat16, device="cuda")
    one, buf = empty(L, T, H, D), empty(L + 1, T, H, D)
    for k, v in ((one, one), (one[:1].expand(L, T, H, D), empty(L, T, H, D)), (empty(L, T, H, D), one[:1].expand(L, T, H, D)),
                 (buf[:-1], buf[1:]), (empty(L, 1, H, D).expand(L, T, H, D), empty(L, T, H, D))):
        with pytest.raises(binding.SvdpError):
            binding.kv_read(cache, slots, k=k, v=v)
    # rows that are stored may be the same ones
    binding.kv_commit(cache, one, one, slots)
    binding.kv_commit(cache, want[0][:1].expand(L, T, H, D), one, slots)
    k, v = binding.kv_read(cache, slots)
    assert torch.equal(k, want[0][:1].expand(L, T, H, D)) and bool((v == 0).all())
    # the last test of the cache: as it was
    binding.kv_commit(cache, *want, slots)
