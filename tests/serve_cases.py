"""Inputs and bounds that the tests of the operators around attention and logits share."""
import numpy as np

from draft_cases import U16, U32, Attn, attention_bound


def decoded(t):
    """A device tensor's values in 64 bits."""
    return t.float().cpu().numpy().astype(np.float64)


def fill_cache(torch, cache, seed):
    """Codes of about 1 times powers of two, token by token: as a commit leaves them."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    for t in (cache.K, cache.V):
        t.copy_((torch.randn(t.shape, device="cuda", generator=g) * 110).clamp_(-448, 448).to(t.dtype))
    for t in (cache.K_scale, cache.V_scale):
        t.view(torch.uint8).copy_(torch.randint(117, 122, t.shape, device="cuda", generator=g))


def exponents(torch, scale):
    return scale.view(torch.uint8).cpu().numpy().astype(np.int64) - 127


class Attn8(Attn):
    """A call of Attn whose cached tokens are kept in 8 bits."""

    def __init__(self, torch, binding, **how):
        super().__init__(torch, binding, dtype="bf16", **how)
        self.torch = torch
        c = self.cache
        self.cache = binding.KVCache.empty(c.layers, c.pages, c.page, c.heads, c.dim, dtype=torch.float8_e4m3fn)
        fill_cache(torch, self.cache, how.get("seed", 0) + 1)

    def expect(self, oracle_draft, scale=None, max_nodes=64):
        torch, c = self.torch, self.cache
        K = decoded(c.K[self.layer]) * 2.0 ** exponents(torch, c.K_scale[self.layer])[..., None]
        by = exponents(torch, c.V_scale[self.layer]).reshape(c.pages, c.heads, c.page // 8, 1, 8)
        V = decoded(c.V[self.layer]) * 2.0 ** by
        return oracle_draft.attention(K, V, decoded(self.q), decoded(self.k), decoded(self.v), self.words, self.table, self.lens, self.starts,
                                      self.dim ** -0.5 if scale is None else scale, max_nodes)

    def check(self, oracle_draft, out, lse, scale=None, max_nodes=64):
        """K and V are exact in bf16: what is off is the scores' and sums' fp32 (attention_bound), the weights' two bf16 terms (2^-15)
        and the output's rounding."""
        o, z, w, reach = self.expect(oracle_draft, scale, max_nodes)
        ob, zb = attention_bound(w, o, reach, z, max(self.lens) + 64, self.dim, bf16=False)
        ob += w * 1.01 * 2.0 ** -15 + np.abs(o) * 1.01 * U16
        rows = ~np.isnan(z).all(1)
        out, lse = decoded(out), lse.cpu().numpy().astype(np.float64)
        assert np.array_equal(np.isneginf(z[rows]), np.isneginf(lse[rows]))
        fin = np.isfinite(z) & rows[:, None]
        off = np.abs(out - o)[rows] / ob[rows]
        assert np.isfinite(out[rows]).all() and off.max() <= 1.0, off.max()
        if fin.any():
            assert (np.abs(lse[fin] - z[fin]) <= zb[fin]).all(), (np.abs(lse[fin] - z[fin]) / zb[fin]).max()
        empty = np.isneginf(z) & rows[:, None]
        assert (out[empty] == 0).all()
        return float(off.max())


def rope_bound(x, y, weight, eps, half, interleaved, dim, rounding):
    """Elementwise bound on the error of a turned row whose exact value is y.

    The norm: a sum of dim squares, each rounded, summed in any order: relative (dim + 1) u, halved by the root; the mean, the sum with
    eps, the root and the quotient four more, and two products: below (dim / 2 + 8) u of the element.  The angle: in turns it is off by 2^-50
    of itself (three roundings in 64 bits; up to 2^18 turns here: 2^-32) and, as a part of a turn, by u / 2 of up to a half: 2^-26 turns, with
    pi 2^-25 rad; the sine and the cosine are within 4 ulp, 4 2^-23 of 1: together below 2^-20 absolute.  The rotation's own three roundings: 3 u.
    All of it scales with |a| + |b| of the pair.  The output is rounded once."""
    n = np.abs(np.array(x, dtype=np.float64))
    if eps is not None:
        n = n / np.sqrt((n * n).mean(-1, keepdims=True) + eps)
    if weight is not None:
        n = n * np.abs(weight)
    pair = n.copy()
    if half:
        a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if interleaved else (slice(0, half), slice(half, 2 * half))
        s = n[..., a] + n[..., b]
        pair[..., a] = pair[..., b] = s
    turned = np.zeros(dim)
    turned[:2 * half] = 2.0 ** -20 + 3 * U32
    return pair * ((dim / 2 + 8) * U32 * (eps is not None) + turned) + np.abs(y) * 1.01 * rounding + 1e-30
