"""Operators around a decode step's attention and logits, without a GPU: the library's checks of arguments, and pins of the oracle."""
import ctypes
import os

import numpy as np
import pytest

from oracle import serve

P = 0x10000          # an address that is never followed: every call below is refused, or has nothing to do
OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.fixture(scope="module")
def svdp():
    from paper_2603_14110_amd import binding, build

    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    return binding


def cache8(svdp, layers=2, pages=100, page=64, heads=8, dim=128, dtype=8, K=P, V=P, K_scale=P, V_scale=P):
    return svdp.svdp_kv_cache(layers, pages, page, heads, dim, dtype, K, V, K_scale, V_scale)


def attn(svdp, c, **over):
    a = dict(layer=0, q=P, qs=4096, k=P, ks=1024, v=P, vs=1024, tree=P, table=P, max_pages=10, lens=P, starts=P, R=2, T=8,
             max_nodes=8, heads_q=32, scale=0.1, out=P, lse=P, ws=P, ws_bytes=1 << 40)
    a.update(over)
    return svdp.lib().svdp_tree_attn(ctypes.byref(c), *a.values(), None)


@pytest.mark.parametrize("over,status", [
    (dict(page=48), UNSUPPORTED), (dict(dim=96), UNSUPPORTED), (dict(dtype=2), UNSUPPORTED), (dict(dtype=9), UNSUPPORTED), (dict(layers=0), INVALID),
    (dict(K=None), INVALID), (dict(V=P + 8), INVALID), (dict(K_scale=None), INVALID), (dict(V_scale=None), INVALID), (dict(K_scale=P + 8), INVALID),
    (dict(V_scale=P + 1), INVALID), (dict(pages=1 << 26), UNSUPPORTED),
])
def test_an_8_bit_cache_is_checked_by_every_call(svdp, over, status):
    c = cache8(svdp, **over)
    assert attn(svdp, c) == status
    rows = (P, 1 << 20, 1024, P, 1 << 20, 1024)
    assert svdp.lib().svdp_kv_commit(ctypes.byref(c), *rows, P, 3, None) == status
    assert svdp.lib().svdp_kv_read(ctypes.byref(c), P, 3, *rows, None) == status
    if status == UNSUPPORTED:
        assert svdp.lib().svdp_tree_attn_workspace_bytes(ctypes.byref(c), 32, 2, 10, 8) == 0


@pytest.mark.parametrize("over,status", [
    (dict(T=0), OK), (dict(ws_bytes=0), WORKSPACE), (dict(q=P + 8), INVALID), (dict(qs=4095), INVALID), (dict(qs=4100), INVALID), (dict(ks=1028), INVALID),
    (dict(vs=1020), INVALID), (dict(layer=2), INVALID), (dict(max_nodes=65), UNSUPPORTED),
])
def test_attention_over_an_8_bit_cache_checks_its_arguments(svdp, over, status):
    """Rows are bf16: strides of whole 16 bytes are multiples of eight."""
    assert attn(svdp, cache8(svdp), **over) == status
    n = svdp.lib().svdp_tree_attn_workspace_bytes(ctypes.byref(cache8(svdp)), 32, 2, 1000, 64)
    assert n > 0 and attn(svdp, cache8(svdp), max_pages=1000, max_nodes=64, ws_bytes=n - 1) == WORKSPACE


@pytest.mark.parametrize("dtype", [0, 1, 8])
@pytest.mark.parametrize("over,status", [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID),
    (dict(k=P + 8), INVALID), (dict(v=P + 4), INVALID), (dict(slots=P + 4), INVALID), (dict(kr=1023), INVALID), (dict(vr=1016), INVALID),
    (dict(kr=1026), INVALID), (dict(kl=-8), INVALID), (dict(vl=2), INVALID),
])
def test_commit_and_read_check_their_arguments(svdp, dtype, over, status):
    a = dict(k=P, kl=1 << 20, kr=1024, v=P, vl=1 << 20, vr=1024, slots=P, T=3)
    a.update(over)
    c, rows = cache8(svdp, dtype=dtype), [a[n] for n in ("k", "kl", "kr", "v", "vl", "vr")]
    assert svdp.lib().svdp_kv_read(ctypes.byref(c), a["slots"], a["T"], *rows, None) == status
    assert svdp.lib().svdp_kv_commit(ctypes.byref(c), *rows, a["slots"], a["T"], None) == status


@pytest.mark.parametrize("over,status", [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(dtype=8), UNSUPPORTED), (dict(dtype=5), UNSUPPORTED),
    (dict(dim=96), UNSUPPORTED), (dict(dim=512), UNSUPPORTED), (dict(heads_q=0), INVALID), (dict(heads=-1), INVALID), (dict(heads_q=1 << 16), UNSUPPORTED),
    (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(q_out=None), INVALID), (dict(k_out=None), INVALID), (dict(q=P + 8), INVALID),
    (dict(k_out=P + 4), INVALID), (dict(qs=4095), INVALID), (dict(qs=4088), INVALID), (dict(ks=1028), INVALID), (dict(qos=4000), INVALID),
    (dict(places=None), INVALID), (dict(inv_freq=None), INVALID), (dict(places=P + 2), INVALID), (dict(inv_freq=P + 1), INVALID),
    (dict(rot=-8), INVALID), (dict(rot=136), INVALID), (dict(rot=12), UNSUPPORTED), (dict(flags=8), INVALID), (dict(eps=-1.0), INVALID),
    (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID), (dict(flags=0, q_weight=P), INVALID), (dict(flags=4), INVALID),
    (dict(q_weight=P + 4), INVALID), (dict(k_weight=P + 8), INVALID), (dict(q_out=P, qos=4104), INVALID),
])
def test_rotation_checks_its_arguments(svdp, over, status):
    a = dict(dtype=1, dim=128, T=8, q=P, qs=4096, heads_q=32, k=2 * P, ks=1024, heads=8, places=P, inv_freq=P, rot=128, flags=2, q_weight=None,
             k_weight=None, eps=1e-6, q_out=3 * P, qos=4096, k_out=4 * P, kos=1024)
    a.update(over)
    assert svdp.lib().svdp_qk_rope(*a.values(), None) == status


@pytest.mark.parametrize("over,status", [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(T=(1 << 24) + 1), UNSUPPORTED), (dict(V=0), INVALID), (dict(V=(1 << 19) + 1, stride=1 << 20), UNSUPPORTED),
    (dict(stride=99), INVALID), (dict(dtype=8), UNSUPPORTED), (dict(logits=None), INVALID), (dict(u=None), INVALID), (dict(answers=None), INVALID),
    (dict(logits=P + 1), INVALID), (dict(u=P + 2), INVALID), (dict(temperature=P + 1), INVALID), (dict(top_k=P + 2), INVALID), (dict(top_p=P + 3), INVALID),
    (dict(min_p=P + 1), INVALID), (dict(answers=P + 2), INVALID), (dict(logp=P + 2), INVALID),
])
def test_sampling_checks_its_arguments(svdp, over, status):
    a = dict(logits=P, stride=100, dtype=1, V=100, u=P, temperature=None, top_k=None, top_p=None, min_p=None, T=8, answers=P, logp=None)
    a.update(over)
    assert svdp.lib().svdp_sample(*a.values(), None) == status


@pytest.mark.parametrize("over,status", [
    (dict(R=0), INVALID), (dict(T=-1), INVALID), (dict(R=5000), UNSUPPORTED), (dict(max_nodes=65), UNSUPPORTED), (dict(answers=None), INVALID),
    (dict(tokens=None), INVALID), (dict(starts=None), INVALID), (dict(keep=None), INVALID), (dict(counts=None), INVALID), (dict(next=None), INVALID),
    (dict(tree=P + 4), INVALID), (dict(keep=P + 2), INVALID), (dict(answers=P + 1), INVALID),
])
def test_walk_checks_its_arguments(svdp, over, status):
    a = dict(answers=P, tokens=P, tree=P, starts=P, R=2, T=8, max_nodes=8, keep=P, counts=P, next=P)
    a.update(over)
    assert svdp.lib().svdp_tree_walk(*a.values(), None) == status


# ---- pins of the oracle ----------------------------------------------------------------------------------------------------


def test_e4m3_of_the_oracle_is_torchs():
    import torch

    v = serve.e4m3_values()
    t = torch.arange(256, dtype=torch.int32).to(torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(v, t, equal_nan=True) and np.nanmax(v) == serve.E4M3_MAX
    x = np.random.default_rng(1).standard_normal(20000) * 2.0 ** np.random.default_rng(2).integers(-12, 7, 20000)
    grid = np.sort(v[np.isfinite(v)])
    x = np.concatenate([np.clip(x, -448, 448), grid, (grid[1:] + grid[:-1]) / 2]).astype(np.float32)
    assert np.array_equal(serve.e4m3(x), torch.from_numpy(x).to(torch.float8_e4m3fn).double().numpy())


def test_quantised_rows_are_as_near_as_e4m3_gets():
    x = np.random.default_rng(3).standard_normal((50, 64)) * 2.0 ** np.arange(-25, 25)[:, None]
    x[7] = 0
    codes, by = serve.quantise(x)
    top = np.abs(x).max(-1)
    live = top > 0
    assert (top <= 448 * 2.0 ** by).all() and (top[live] > 224 * 2.0 ** by[live]).all() and by[7] == serve.LEAST
    # half a step: 2^-4 of the value, or of the least normal number 2^-6
    assert (np.abs(codes * (2.0 ** by)[:, None] - x) <= 2.0 ** -4 * np.maximum(np.abs(x), 2.0 ** (by - 6.0)[:, None])).all()
    # once more: the same values, though the power may be one less (448 for 224)
    again, by2 = serve.quantise(codes * (2.0 ** by)[:, None])
    assert np.array_equal(again * (2.0 ** by2)[:, None], codes * (2.0 ** by)[:, None]) and ((by - by2 == 0) | (by - by2 == 1)).all()


def test_drawn_tokens_follow_the_distribution():
    """As u goes through [0, 1) in equal steps each kept token comes as often as its share, to one step at each end."""
    rng = np.random.default_rng(4)
    row, n = rng.standard_normal(40) * 2, 2000
    for how in (dict(), dict(temperature=0.7), dict(top_k=5), dict(top_p=0.8), dict(min_p=0.1), dict(temperature=1.5, top_k=20, top_p=0.9, min_p=0.02)):
        kept = serve.draw(row, 0.0, **how)[2]
        p = np.exp(row[kept] / how.get("temperature", 1.0))
        p /= p.sum()
        got = [serve.draw(row, (i + 0.5) / n, **how)[0] for i in range(n)]
        for token, share in zip(kept, p):
            assert abs(got.count(token) - share * n) <= 1
        assert set(got) <= set(kept)
        logp = serve.draw(row, 0.3, **how)
        assert abs(logp[1] - np.log(p[kept.index(logp[0])])) < 1e-9


def test_what_is_kept():
    row = np.array([0.0, 3.0, 3.0, -np.inf, 2.0, 3.0])
    kept = lambda **how: serve.draw(row, 0.0, **how)[2]
    assert kept() == [1, 2, 5, 4, 0, 3] and kept(top_k=2) == [1, 2] and kept(top_k=4) == [1, 2, 5, 4] and kept(top_k=99) == kept()
    assert kept(top_p=0.0) == [1] and kept(top_p=0.3) == [1, 2] and kept(top_p=1.0) == kept() and kept(top_p=0.5, top_k=2) == [1]
    assert kept(min_p=1.0) == [1, 2, 5] and kept(min_p=0.3) == [1, 2, 5, 4] and kept(temperature=0.0) == [1]
    assert serve.draw(np.full(3, -np.inf), 0.5)[:2] == (-1, -np.inf)
    assert serve.draw(np.array([1.0, np.nan, np.inf]), 0.5)[0] == 1 and serve.draw(np.array([1.0, np.inf, np.inf]), 0.9)[0] == 1


def test_rotation_keeps_lengths_and_depends_on_distance_only():
    rng = np.random.default_rng(5)
    x, f = rng.standard_normal((2, 3, 64)), 100.0 ** (-np.arange(0, 32, 2) / 32)
    for inter in (False, True):
        y = serve.rope(x, [5, 5], f, interleaved=inter)
        assert np.allclose(np.linalg.norm(y, axis=-1), np.linalg.norm(x, axis=-1)) and np.array_equal(y[..., 32:], x[..., 32:])
        near, far = serve.rope(x, [3, 10], f, interleaved=inter), serve.rope(x, [1003, 1010], f, interleaved=inter)
        assert np.allclose((near[0] * near[1]).sum(-1), (far[0] * far[1]).sum(-1))


def test_quantised_rows_are_finite_in_bf16():
    """At the largest power, 2^120, codes end at 240: 256 2^120 is no bf16 number any more.  255 2^120, the largest one, is off by less than half a step."""
    x = np.array([255.0, 248.0, 247.0, 232.0, -255.0, 1.0, 100.0, 240.0]) * 2.0 ** 120
    codes, by = serve.quantise(x)
    assert by == 120 and codes.tolist() == [240.0, 240.0, 240.0, 224.0, -240.0, 1.0, 96.0, 240.0]
    assert (np.abs(codes * 2.0 ** 120 - x) <= 2.0 ** -4 * np.abs(x)).all()
    codes, by = serve.quantise(np.array([224.0, 223.0, 112.0]) * 2.0 ** 120)
    assert by == 119 and codes.tolist() == [448.0, 448.0, 224.0]


def _rows_meet(at_k, at_v, layers, T, k, v, row):
    """By looking at every element."""
    where = [at + l * s[0] + t * s[1] for at, s in ((at_k, k), (at_v, v)) for l in range(layers) for t in range(T)]
    return len({w + i for w in where for i in range(row)}) < len(where) * row


def test_read_refuses_rows_that_overlap(svdp):
    """A read writes its rows: layers on top of each other, one buffer for K and V, rows that run into each other's gaps.  Where K's strides are V's every
    such call is refused; with other strides where their first rows meet, or K's or V's rows each other.  What does not overlap is
    not refused (asked only where no GPU is there to follow the addresses)."""
    import torch

    rng, row, unit = np.random.default_rng(6), 128, 64
    refused = taken = 0
    for _ in range(3000):
        layers, T = int(rng.integers(1, 5)), int(rng.integers(1, 5))
        strides = lambda: (unit * int(rng.choice([0, 1, 2, 3, 4, 6, 8, 16, 20])), row + unit * int(rng.choice([0, 1, 2, 4, 6, 14])))
        k, alike = strides(), rng.random() < 0.7
        v = k if alike else strides()
        apart = unit * int(rng.choice([0, 1, 2, 3, 4, 8, 10, 100, -1, -2, -4, -40]))
        c = cache8(svdp, layers=layers, heads=2, dim=64, dtype=1)
        call = lambda: svdp.lib().svdp_kv_read(ctypes.byref(c), P, T, 1 << 20, k[0], k[1], (1 << 20) + 2 * apart, v[0], v[1], None)
        itself = _rows_meet(0, 1 << 30, layers, T, k, v, row)
        meet = _rows_meet(0, apart, layers, T, k, v, row)
        if itself or abs(apart) < row or (alike and meet):
            assert call() == INVALID, (layers, T, k, v, apart)
            refused += 1
        elif not meet and not torch.cuda.is_available():
            assert call() != INVALID, (layers, T, k, v, apart)
            taken += 1
    assert refused > 500 and (taken > 100 or torch.cuda.is_available())
    for over in (dict(kl=1 << 46), dict(vl=1 << 62), dict(kr=1 << 45), dict(vr=1 << 62)):
        a = {**dict(kl=1 << 20, kr=1024, vl=1 << 20, vr=1024), **over}
        assert svdp.lib().svdp_kv_read(ctypes.byref(cache8(svdp)), P, 3, P, a["kl"], a["kr"], 1 << 40, a["vl"], a["vr"], None) == INVALID



def test_rotation_refuses_rows_that_overlap(svdp):
    """One buffer for both outputs, an output over the other input, an output moved against its own input: every such call is refused where the strides are
    the same; what does not overlap is not (asked only where no GPU is there to follow the addresses)."""
    import torch

    rng, unit, dim = np.random.default_rng(7), 64, 64
    refused = taken = 0

    def elements(at, stride, heads, T):
        return {at + t * stride + i for t in range(T) for i in range(0, heads * dim, 8)}       # addresses are whole 16 bytes apart

    for _ in range(4000):
        T, hq, h = int(rng.integers(1, 5)), int(rng.integers(1, 4)), int(rng.integers(0, 4))
        stride = unit * int(rng.integers(max(hq, h), 9))
        place = lambda: 8 * int(rng.integers(0, 8 * 8 * 3)) if rng.random() < 0.3 else unit * int(rng.integers(0, 40))
        q, k, qo, ko = (place() for _ in range(4))
        qo, ko = q if rng.random() < 0.5 else qo, k if rng.random() < 0.5 else ko
        e = {n: elements(at, stride, heads, T) for n, at, heads in (("q", q, hq), ("k", k, h), ("qo", qo, hq), ("ko", ko, h))}
        meet = bool((q != qo and e["qo"] & e["q"]) or (k != ko and e["ko"] & e["k"]) or e["qo"] & e["ko"] or e["qo"] & e["k"] or e["ko"] & e["q"])
        at = lambda place: (1 << 20) + 2 * place
        call = lambda: svdp.lib().svdp_qk_rope(1, dim, T, at(q), stride, hq, at(k), stride, h, P, P, dim, 0, None, None, 0.0, at(qo), stride, at(ko), stride, None)
        if meet:
            assert call() == INVALID, (T, hq, h, stride, q, k, qo, ko)
            refused += 1
        elif not torch.cuda.is_available():
            assert call() != INVALID, (T, hq, h, stride, q, k, qo, ko)
            taken += 1
    assert refused > 500 and (taken > 500 or torch.cuda.is_available())
