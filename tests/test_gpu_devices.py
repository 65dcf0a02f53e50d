"""Operators of decoding with drafted tokens go to the current device's stream: tensors of another device are refused, whatever the cache's type."""
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding


def calls(torch, binding, dtype):
    """name -> (call, its tensors)."""
    i32 = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
    cache = binding.KVCache.empty(1, 4, 32, 1, 64, dtype=dtype)
    q = torch.ones((2, 1, 64), dtype=cache.rows, device="cuda")
    attn = dict(q=q, k=q.clone(), v=q.clone(), table=i32(0, 1)[None], lens=i32(3), starts=i32(0, 2), tree=torch.tensor([1, 3], device="cuda"),
                out=torch.empty_like(q), lse=torch.empty((2, 1), device="cuda"),
                ws=torch.empty(binding.tree_attn_workspace_bytes(cache, 1, 1, 2, 2), dtype=torch.uint8, device="cuda"))
    accept = dict(logits=torch.randn((2, 50), device="cuda"), tokens=i32(1, 2), starts=i32(0, 2), tree=torch.tensor([1, 3], device="cuda"),
                  ws=torch.empty(binding.tree_accept_workspace_bytes(2, 50, 0), dtype=torch.uint8, device="cuda"))
    plan = dict(table=i32(0, 0)[None], ring=i32(0, 1, 2, 3), pool=i32(0, 4), lens=i32(0), add=i32(2), starts=i32(0, 2), keep=i32(0, 1))
    commit = dict(k=q[None], v=q[None].clone(), slots=torch.tensor([1, 2], device="cuda"))
    return {"tree_attn": (lambda **a: binding.tree_attn(cache, 0, **a), attn), "tree_accept": (binding.tree_accept, accept),
            "kv_plan": (lambda **a: binding.kv_plan(page=32, **a), plan), "kv_commit": (lambda **a: binding.kv_commit(cache, **a), commit),
            "kv_read": (lambda **a: binding.kv_read(cache, **a), commit)}


@pytest.mark.parametrize("dtype", ["float32", "bfloat16", "float8_e4m3fn"])
@pytest.mark.parametrize("name", ["tree_attn", "tree_accept", "kv_plan", "kv_commit", "kv_read"])
def test_tensors_of_another_device_are_refused(env, monkeypatch, name, dtype):
    torch, binding = env
    call, tensors = calls(torch, binding, getattr(torch, dtype))[name]
    call(**{n: t.clone() for n, t in tensors.items()})
    for n in tensors:
        with pytest.raises(binding.SvdpError):
            call(**{**tensors, n: tensors[n].cpu()})
    torch.cuda.synchronize()
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    with pytest.raises(binding.SvdpError, match="current device"):
        call(**tensors)
