"""Decoding with drafted tokens, without a GPU: the library's checks of arguments, and pins of the oracle."""
import ctypes
import os

import numpy as np
import pytest

from oracle import draft

P = 0x10000          # an address that is never followed: every call below is refused, or has nothing to do


@pytest.fixture(scope="module")
def svdp():
    from paper_2603_14110_amd import binding, build

    if not os.path.exists(binding.LIB_PATH):
        build.build_lib()
    return binding


def cache(svdp, layers=2, pages=100, page=64, heads=8, dim=128, dtype=1, K=P, V=P):
    return svdp.svdp_kv_cache(layers, pages, page, heads, dim, dtype, K, V)


def attn(svdp, c=None, **over):
    a = dict(layer=0, q=P, qs=4096, k=P, ks=1024, v=P, vs=1024, tree=P, table=P, max_pages=10, lens=P, starts=P, R=2, T=8,
             max_nodes=8, heads_q=32, scale=0.1, out=P, lse=P, ws=P, ws_bytes=1 << 40)
    a.update(over)
    c = cache(svdp) if c is None else c
    return svdp.lib().svdp_tree_attn(ctypes.byref(c), *a.values(), None)


OK, INVALID, UNSUPPORTED, WORKSPACE = 0, 1, 2, 3


@pytest.mark.parametrize("over,status", [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(R=0), INVALID), (dict(R=4097), UNSUPPORTED), (dict(layer=2), INVALID),
    (dict(layer=-1), INVALID), (dict(q=None), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(out=None), INVALID),
    (dict(table=None), INVALID), (dict(lens=None), INVALID), (dict(starts=None), INVALID), (dict(q=P + 8), INVALID),
    (dict(k=P + 2), INVALID), (dict(v=P + 4), INVALID), (dict(out=P + 8), INVALID), (dict(tree=P + 4), INVALID), (dict(lse=P + 2), INVALID),
    (dict(qs=4095), INVALID), (dict(qs=4088), INVALID), (dict(qs=4100), INVALID), (dict(ks=1020), INVALID), (dict(vs=1028), INVALID),
    (dict(max_pages=0), INVALID), (dict(max_pages=1 << 26), UNSUPPORTED), (dict(max_nodes=65), UNSUPPORTED), (dict(max_nodes=0), INVALID),
    (dict(heads_q=30), INVALID), (dict(heads_q=0), INVALID), (dict(scale=float("inf")), INVALID), (dict(scale=float("nan")), INVALID),
    (dict(ws=None), WORKSPACE), (dict(ws=P + 128), WORKSPACE), (dict(ws_bytes=0), WORKSPACE),
])
def test_attention_checks_its_arguments(svdp, over, status):
    assert attn(svdp, **over) == status


@pytest.mark.parametrize("over,status", [
    (dict(page=48), UNSUPPORTED), (dict(page=16), UNSUPPORTED), (dict(page=512), UNSUPPORTED), (dict(dim=96), UNSUPPORTED), (dict(dim=0), UNSUPPORTED),
    (dict(dtype=2), UNSUPPORTED), (dict(layers=0), INVALID), (dict(pages=0), INVALID), (dict(heads=0), INVALID), (dict(K=None), INVALID),
    (dict(V=None), INVALID), (dict(K=P + 8), INVALID), (dict(V=P + 8), INVALID), (dict(pages=1 << 26), UNSUPPORTED),
])
def test_a_cache_is_checked_by_every_call(svdp, over, status):
    c = cache(svdp, **over)
    assert attn(svdp, c) == status
    assert svdp.lib().svdp_kv_commit(ctypes.byref(c), P, 1 << 20, 1024, P, 1 << 20, 1024, P, 3, None) == status
    if status == UNSUPPORTED:
        assert svdp.lib().svdp_tree_attn_workspace_bytes(ctypes.byref(c), 32, 2, 10, 8) == 0


def test_attention_workspace(svdp):
    f = svdp.lib().svdp_tree_attn_workspace_bytes
    c = cache(svdp)
    n = f(ctypes.byref(c), 32, 8, 1000, 64)
    assert n > 0 and n % 256 == 0 and n < 1 << 30
    for bad in ((30, 8, 10, 8), (32, 0, 10, 8), (32, 4097, 10, 8), (32, 8, 0, 8), (32, 8, 10, 65), (32, 8, 10, 0)):
        assert f(ctypes.byref(c), *bad) == 0
    assert f(None, 32, 8, 10, 8) == 0
    assert attn(svdp, max_pages=1000, max_nodes=64, ws_bytes=f(ctypes.byref(c), 32, 2, 1000, 64) - 1) == WORKSPACE


@pytest.mark.parametrize("over,status", [
    (dict(V=0), INVALID), (dict(stride=99), INVALID), (dict(dtype=5), UNSUPPORTED), (dict(R=0), INVALID), (dict(T=-1), INVALID),
    (dict(R=5000), UNSUPPORTED), (dict(max_nodes=65), UNSUPPORTED), (dict(logits=None), INVALID), (dict(logits=P + 1), INVALID),
    (dict(tokens=None), INVALID), (dict(starts=None), INVALID), (dict(keep=None), INVALID), (dict(counts=None), INVALID), (dict(next=None), INVALID),
    (dict(best=None), INVALID), (dict(tree=P + 4), INVALID), (dict(keep=P + 2), INVALID), (dict(ws=None), WORKSPACE), (dict(ws_bytes=8), WORKSPACE),
    (dict(ws=P + 64), WORKSPACE),
])
def test_acceptance_checks_its_arguments(svdp, over, status):
    a = dict(logits=P, stride=100, dtype=1, V=100, tokens=P, tree=P, starts=P, R=2, T=8, max_nodes=8, keep=P, counts=P, next=P, best=P, ws=P,
             ws_bytes=1 << 30)
    a.update(over)
    assert svdp.lib().svdp_tree_accept(*a.values(), None) == status


def test_acceptance_workspace(svdp):
    f = svdp.lib().svdp_tree_accept_workspace_bytes
    assert f(8, 32000, 1) >= 64 and f(0, 32000, 1) > 0 and f(2048, 152064, 0) % 256 == 0
    assert f(-1, 10, 1) == 0 and f(1, 0, 1) == 0 and f(1, 10, 3) == 0


@pytest.mark.parametrize("over,status", [
    (dict(max_pages=0), INVALID), (dict(pages=0), INVALID), (dict(page=33), UNSUPPORTED), (dict(R=0), INVALID), (dict(R=4097), UNSUPPORTED),
    (dict(T=-1), INVALID), (dict(table=None), INVALID), (dict(ring=None), INVALID), (dict(pool=None), INVALID), (dict(lens=None), INVALID),
    (dict(add=None), INVALID), (dict(starts=None), INVALID), (dict(slots=None), INVALID), (dict(slots=P + 4), INVALID), (dict(lens_out=None), INVALID),
    (dict(pool_out=None), INVALID), (dict(refused=None), INVALID), (dict(keep=P + 1), INVALID), (dict(pages=1 << 26), UNSUPPORTED),
    (dict(max_pages=1 << 30), UNSUPPORTED),
    # outputs over inputs that other blocks still read
    (dict(lens_out=5 * P), INVALID), (dict(lens_out=5 * P + 4), INVALID), (dict(pool_out=4 * P), INVALID), (dict(refused=6 * P), INVALID),
])
def test_plan_checks_its_arguments(svdp, over, status):
    a = dict(table=2 * P, max_pages=4, ring=3 * P, pages=50, page=64, pool=4 * P, lens=5 * P, add=6 * P, starts=7 * P, keep=None, R=2, T=8,
             slots=8 * P, lens_out=9 * P, pool_out=10 * P, refused=11 * P)
    a.update(over)
    assert svdp.lib().svdp_kv_plan(*a.values(), None) == status


@pytest.mark.parametrize("over,status", [
    (dict(T=0), OK), (dict(T=-1), INVALID), (dict(k=None), INVALID), (dict(v=None), INVALID), (dict(slots=None), INVALID), (dict(k=P + 8), INVALID),
    (dict(v=P + 8), INVALID), (dict(slots=P + 4), INVALID), (dict(kr=1020), INVALID), (dict(kr=1025), INVALID), (dict(vr=512), INVALID),
    (dict(kl=-8), INVALID), (dict(vl=4), INVALID),
])
def test_commit_checks_its_arguments(svdp, over, status):
    a = dict(k=P, kl=8192, kr=1024, v=P, vl=8192, vr=1024, slots=P, T=8)
    a.update(over)
    c = cache(svdp)
    assert svdp.lib().svdp_kv_commit(ctypes.byref(c), *a.values(), None) == status


# ---- the oracle ------------------------------------------------------------------------------------------------------------


def test_oracle_attention_is_a_softmax_over_what_a_row_sees():
    rng = np.random.default_rng(0)
    page, dim, e = 32, 64, 4
    K, V = rng.normal(size=(3, 2, page, dim)), rng.normal(size=(3, 2, page // e, dim, e))
    q, k, v = rng.normal(size=(3, 4, dim)), rng.normal(size=(3, 2, dim)), rng.normal(size=(3, 2, dim))
    out, lse, _, _ = draft.attention(K, V, q, k, v, [0b001, 0b011, 0b101], [[2, 0]], [40], [0, 3], 0.125)
    # row 2, query head 3 (head 1 of K and V): 40 cached tokens, nodes 0 and 2
    ks = np.concatenate([K[2, 1], K[0, 1, :8], k[[0, 2], 1]])
    vs = np.concatenate([V[2, 1].transpose(0, 2, 1).reshape(page, dim), V[0, 1].transpose(0, 2, 1).reshape(page, dim)[:8], v[[0, 2], 1]])
    z = 0.125 * ks @ q[2, 3]
    w = np.exp(z) / np.exp(z).sum()
    assert np.allclose(out[2, 3], w @ vs, atol=1e-12) and np.isclose(lse[2, 3], np.log(np.exp(z).sum()))
    out, lse, _, _ = draft.attention(K, V, q, k, v, [0, 1, 2], [[2, 0]], [0], [0, 3], 0.125)
    assert (out[0] == 0).all() and np.isneginf(lse[0]).all() and np.allclose(out[1, 0], v[0, 0])


def test_oracle_acceptance_worked_example():
    """Root 0 with children 1, 2; 1 with child 3; 2 with child 4.  The answer at 0 is 7 = the token of 2; at 2 it is 9 = that of 4."""
    logits = np.zeros((5, 12))
    for row, t in enumerate((7, 1, 9, 2, 3)):
        logits[row, t] = 1
    keep, counts, following, best = draft.accept(logits, [0, 6, 7, 1, 9], [0b1, 0b11, 0b101, 0b1011, 0b10101], [0, 5])
    assert keep == [0, -1, 1, -1, 2] and counts == [3] and following == [3] and best == [7, 1, 9, 2, 3]


def test_oracle_plan_worked_example():
    """Pages of 32.  Request 0 grows from 30 to 70 tokens and takes two pages, 1 ends and gives two back, 2 asks for two where one is left."""
    slots, lens, pool, refused, table, ring = draft.plan(
        [[4, -1, -1], [0, 5, -1], [1, -1, -1]], [9, 9, 7, 8, 6, 3], [2, 3], [30, 50, 31], [40, -1, 34], [0, 41, 41, 75], 32, None, 75)
    assert lens == [70, 0, 31] and refused == [0, 0, 1] and pool == [4, 3]
    assert table == [[4, 7, 8], [0, 5, -1], [1, -1, -1]] and ring == [5, 9, 7, 8, 6, 0]
    assert slots[:4] == [4 * 32 + 30, 4 * 32 + 31, 7 * 32, 7 * 32 + 1] and slots[39] == 8 * 32 + 5 and slots[40:] == [-1] * 35


def test_oracle_commit_worked_example():
    K, V = np.zeros((1, 2, 1, 32, 64)), np.zeros((1, 2, 1, 4, 64, 8))
    k, v = np.ones((1, 2, 1, 64)), np.arange(128.0).reshape(1, 2, 1, 64) + 1
    draft.commit(K, V, k, v, [32 + 13, -1])
    assert K.sum() == 64 and (K[0, 1, 0, 13] == 1).all() and (V[0, 1, 0, 1, :, 5] == v[0, 0, 0]).all() and V.sum() == v[0, 0].sum()


def test_rows_beyond_a_grid_are_refused(svdp):
    most = 1 << 24
    assert attn(svdp, T=most + 1) == UNSUPPORTED and attn(svdp, T=1 << 21, heads_q=32) == UNSUPPORTED
    c = cache(svdp)
    assert svdp.lib().svdp_kv_commit(ctypes.byref(c), P, 1 << 20, 1024, P, 1 << 20, 1024, P, most + 1, None) == UNSUPPORTED
    assert svdp.lib().svdp_tree_accept(P, 100, 1, 100, P, P, P, 2, most + 1, 8, P, P, P, P, P, 1 << 40, None) == UNSUPPORTED
    assert svdp.lib().svdp_tree_accept_workspace_bytes(most + 1, 100, 1) == 0
    a = (2 * P, 4, 3 * P, 50, 64, 4 * P, 5 * P, 6 * P, 7 * P, None, 2, most + 1, 8 * P, 9 * P, 10 * P, 11 * P)
    assert svdp.lib().svdp_kv_plan(*a, None) == UNSUPPORTED


@pytest.mark.parametrize("dtype,dim,heads_q,nodes,parts", [(1, 128, 8, 1, 1024), (1, 128, 56, 1, 1024), (1, 64, 24, 5, 1024), (1, 128, 56, 3, 512),
                                                           (1, 256, 8, 13, 512), (0, 64, 8, 7, 1024), (0, 64, 24, 9, 512), (1, 128, 56, 33, 512)])
def test_parts_of_the_attention_begin_at_16_bytes(svdp, dtype, dim, heads_q, nodes, parts):
    """Parts are written and read 16 bytes at a time: with odd numbers of rows, too, each of them is whole 16 bytes long."""
    c = cache(svdp, dtype=dtype, dim=dim)
    n = svdp.lib().svdp_tree_attn_workspace_bytes(ctypes.byref(c), heads_q, 8, 1000, nodes)
    rows = min(nodes * heads_q // 8, 256 if nodes > 30 else 32 if parts == 512 and dim < 256 else 16)
    least = rows * (dim + 2) * 4
    assert rows % 2 == 1
    assert n % (16 * parts) == 0 and least <= n // parts < least + 16


@pytest.mark.parametrize("keep", [None, 12])
@pytest.mark.parametrize("name,at", [(o, i) for o in ("slots", "lens_out", "pool_out", "refused", "table", "ring")
                                     for i in ("table", "ring", "pool", "lens", "add", "starts", "keep", "slots", "lens_out", "pool_out", "refused")
                                     if o != i])
def test_plan_writes_over_nothing_it_has(svdp, name, at, keep):
    """Any two of its arrays of which one is written: from the same place on, and by the last eight bytes."""
    a = dict(table=2, max_pages=4, ring=3, pages=50, page=64, pool=4, lens=5, add=6, starts=7, keep=keep, R=2, T=8,
             slots=8, lens_out=9, pool_out=10, refused=11)
    size = dict(table=32, ring=200, pool=8, lens=8, add=8, starts=12, keep=32, slots=64, lens_out=8, pool_out=8, refused=8)
    if a[at] is None:
        return
    for back in (0, 8 - size[at]):
        b = {k: v * P if k in size and v is not None else v for k, v in a.items()}
        b[name] = b[at] - back
        if b[name] % 8 and name == "slots":
            continue
        assert svdp.lib().svdp_kv_plan(*b.values(), None) == INVALID
