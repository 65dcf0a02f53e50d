"""Inputs and bounds that the tests of decoding with drafted tokens share."""
import random

import numpy as np

U32 = 2.0 ** -24
U16 = 2.0 ** -8          # bf16: seven bits behind the leading one


def parents(rng, n):
    return ([-1] + [rng.randrange(max(0, j - 5), j) for j in range(1, n)])[:n]


def words(par):
    """Ancestors and self as 64-bit words (unsigned)."""
    m = []
    for j, p in enumerate(par):
        m.append((1 << j) | (m[p] if p >= 0 else 0))
    return m


def signed(ws):
    return [w - (1 << 64) if w >> 63 else w for w in ws]


def attention_bound(weight, out, reach, lse, tokens, dim, bf16):
    """Elementwise bounds on the error of out and of lse.

    A score is a product of `dim` terms summed in fp32, scaled, and taken relative to a maximum in base two: its error is below
    (dim + 8) u reach plus four roundings of numbers below 2 reach.  That is a relative error of the weight; the exponential
    has 2^-21 of its own, a sum of `tokens` weights and its partial sums at most (tokens + 64) u.  bf16: a weight is rounded
    once for its product with V, the output once."""
    score = (dim + 8) * U32 * reach + 16 * U32 * reach
    rel = 2 * score + 2.0 ** -20 + 2 * (tokens + 64) * U32
    b = weight * (rel[..., None] + (1.01 * U16 if bf16 else 0.0)) + np.abs(out) * (1.01 * U16 if bf16 else 2 * U32) + 1e-30
    return b, score + 2.0 ** -20 + (tokens + 64) * U32 + 4 * U32 * np.abs(np.where(np.isfinite(lse), lse, 0.0))


class Attn:
    """One call's inputs on the device and decoded on the host."""

    def __init__(self, torch, binding, *, dtype, dim, heads, group, page, lens, nodes, tree="tree", seed=0, layers=2, layer=1,
                 pad=0, extra_pages=3, strided=True, spread=1.0):
        g = torch.Generator(device="cuda").manual_seed(seed)
        rng = random.Random(seed)
        self.dtype, self.dim, self.heads, self.group, self.page = dtype, dim, heads, group, page
        self.lens, self.nodes, self.layer = list(lens), list(nodes), layer
        td = torch.bfloat16 if dtype == "bf16" else torch.float32
        e = 8 if dtype == "bf16" else 4
        R, hq = len(lens), heads * group
        self.starts = [0]
        for n in nodes:
            self.starts.append(self.starts[-1] + n)
        T = self.starts[-1] + pad
        need = [-(-n // page) for n in lens]
        pages = sum(need) + extra_pages
        ids = list(range(pages))
        rng.shuffle(ids)
        width = max(max(need), 1) + 1
        # entries past a request's length are not to be read: ids that no cache has
        self.table = [[ids.pop() for _ in range(k)] + [rng.choice([-1, pages, 1 << 30])] * (width - k) for k in need]
        normal = lambda *s: torch.randn(s, device="cuda", generator=g).to(td)
        K, V = normal(layers, pages, heads, page, dim), normal(layers, pages, heads, page // e, dim, e)
        self.cache = binding.KVCache(K, V)
        if strided:
            rows = normal(T, hq + 2 * heads + 1, dim)
            self.q, self.k, self.v = rows[:, :hq], rows[:, hq:hq + heads], rows[:, hq + heads:hq + 2 * heads]
            self.q *= spread
        else:
            self.q, self.k, self.v = normal(T, hq, dim) * spread, normal(T, heads, dim), normal(T, heads, dim)
        if tree == "tree":
            self.words = sum((words(parents(rng, n)) for n in nodes), [])
        elif tree == "random":                   # any sets of nodes, empty ones among them
            self.words = [rng.choice([0, rng.getrandbits(64), rng.getrandbits(64) & rng.getrandbits(64)]) for _ in range(T - pad)]
        else:
            self.words = None
        i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
        self.d_table, self.d_lens, self.d_starts = i32(self.table), i32(self.lens), i32(self.starts)
        self.d_tree = None if self.words is None else torch.tensor(signed(self.words + [0] * pad), dtype=torch.int64, device="cuda")
        self.max_nodes = max(max(nodes), 1)

    def call(self, binding, **over):
        a = dict(tree=self.d_tree, max_nodes=self.max_nodes, want_lse=True)
        a.update(over)
        return binding.tree_attn(self.cache, self.layer, self.q, self.k, self.v, self.d_table, self.d_lens, self.d_starts, **a)

    def expect(self, oracle_draft, scale=None, max_nodes=64):
        f = lambda t: t.float().cpu().numpy().astype(np.float64)
        return oracle_draft.attention(f(self.cache.K[self.layer]), f(self.cache.V[self.layer]), f(self.q), f(self.k), f(self.v),
                                      self.words, self.table, self.lens, self.starts, self.dim ** -0.5 if scale is None else scale,
                                      max_nodes)

    def check(self, oracle_draft, out, lse, scale=None, max_nodes=64):
        o, z, w, reach = self.expect(oracle_draft, scale, max_nodes)
        ob, zb = attention_bound(w, o, reach, z, max(self.lens) + 64, self.dim, self.dtype == "bf16")
        rows = ~np.isnan(z).all(1)
        out, lse = out.float().cpu().numpy().astype(np.float64), lse.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isneginf(z[rows]), np.isneginf(lse[rows]))
        fin = np.isfinite(z) & rows[:, None]
        off = np.abs(out - o)[rows] / ob[rows]
        assert np.isfinite(out[rows]).all() and off.max() <= 1.0, off.max()
        if fin.any():
            assert (np.abs(lse[fin] - z[fin]) <= zb[fin]).all(), (np.abs(lse[fin] - z[fin]) / zb[fin]).max()
        empty = np.isneginf(z) & rows[:, None]
        assert (out[empty] == 0).all()
        return float(off.max())
