"""Greedy decoding with drafted tokens: a small decoder of attention and sparse FFN layers over a paged cache.

A step takes, for each request, a tree of drafted tokens whose first node is the newest certain token.  It runs

  binding.qk_rope      norms and rotation of a layer's queries and keys (a decoder with inv_freq),
  binding.tree_attn    every layer's attention of the trees over the cache (of the weights' type, or in 8 bits),
  binding.ffn_step     the layer's sparse FFN, up to ``rows`` tokens sharing one list of active neurons,
  binding.tree_accept  the model's own answers and the branch that agrees with them (or binding.tree_sample: answers drawn),
  binding.kv_plan      pages and slots for that branch (and pages back from requests that end),
  binding.kv_commit    K and V of that branch into the cache,

all enqueued on the current stream; the host reads the accepted tokens once a step.  With ``rows=1`` the tokens are those of
decoding one by one, up to rounding; more rows share the union of their lists, as a batch of the FFN step does.

``python -m paper_2603_14110_amd.draft`` decodes with random weights and drafts looked up in what a request has so far.
"""
from __future__ import annotations

from typing import Callable, List, Optional, Sequence, Tuple

import torch

from . import binding

Tree = Tuple[List[int], List[int]]          # tokens and parents of the drafted nodes; parent -1: the newest certain token


def lookup(history: Sequence[int], nodes: int, branches: int = 3) -> Tree:
    """Drafts from a request's own text: what followed earlier occurrences of its last token, newest first, as one tree."""
    tokens, parents, children = [], [], {}
    found = [i for i in range(len(history) - 2, -1, -1) if history[i] == history[-1]][:branches]
    for i in found:
        at = -1
        for t in history[i + 1:i + 1 + max(1, nodes // len(found))]:
            if (at, t) not in children:
                if len(tokens) == nodes:
                    return tokens, parents
                children[at, t] = len(tokens)
                tokens.append(t)
                parents.append(at)
            at = children[at, t]
    return tokens, parents


def _look_over(tree: Tree, vocabulary: float = float("inf")) -> None:
    tokens, parents = tree
    if len(tokens) != len(parents) or any(not -1 <= p < j for j, p in enumerate(parents)) or any(not 0 <= t < vocabulary for t in tokens):
        raise ValueError("a tree has tokens of the vocabulary and a parent for each, in front of it or -1")


def cut(tree: Tree, levels: int) -> Tree:
    """The first ``levels`` levels of a drafted tree."""
    _look_over(tree)
    tokens, parents, depth, place = [], [], {-1: 0}, {-1: -1}
    for j, (t, p) in enumerate(zip(*tree)):
        depth[j] = depth[p] + 1
        if depth[j] <= levels:
            place[j] = len(tokens)
            tokens.append(t)
            parents.append(place[p])
    return tokens, parents


class Decoder:
    """Weights: per layer a binding.DeviceLayer, Wqkv [d][(heads_q + 2 heads) dim] and Wo [heads_q dim][d]; embed and
    head [V][d].  The cache has ``pages`` pages of ``page`` tokens for ``requests`` requests of up to ``max_len``; cache_dtype: its
    type, e.g. torch.float8_e4m3fn (default: the weights').  Positions are added to the embedding, or with inv_freq [rot / 2] turn queries
    and keys; qk_norm: float32 weights ([layers][dim] for queries, for keys) of norms in front of that."""

    def __init__(self, ffn: List[binding.DeviceLayer], Wqkv: List[torch.Tensor], Wo: List[torch.Tensor], embed: torch.Tensor,
                 head: torch.Tensor, heads_q: int, heads: int, dim: int, requests: int, pages: int, page: int = 64, max_len: int = 4096, rows: int = 8,
                 cache_dtype=None, inv_freq: Optional[torch.Tensor] = None, qk_norm: Optional[Tuple[torch.Tensor, torch.Tensor]] = None):
        self.ffn, self.Wqkv, self.Wo, self.embed, self.head = ffn, Wqkv, Wo, embed, head
        self.heads_q, self.heads, self.dim, self.rows = heads_q, heads, dim, rows
        dev, i32 = embed.device, torch.int32
        self.cache = binding.KVCache.empty(len(ffn), pages, page, heads, dim, dtype=embed.dtype if cache_dtype is None else cache_dtype, device=dev)
        if inv_freq is None and qk_norm is not None:
            raise ValueError("qk_norm goes with inv_freq")
        self.inv_freq, self.qk_norm = inv_freq, qk_norm
        self.table = torch.zeros((requests, -(-max_len // page)), dtype=i32, device=dev)
        self.ring = torch.arange(pages, dtype=i32, device=dev)
        self.pool = torch.tensor([0, pages], dtype=i32, device=dev)
        self.lens = torch.zeros(requests, dtype=i32, device=dev)
        d = embed.shape[1]
        room = self.table.shape[1] * page + binding.MAX_NODES
        turn = torch.arange(room, device=dev)[:, None] / 10000 ** (torch.arange(0, d, 2, device=dev) / d)
        self.where = (torch.cat([turn.sin(), turn.cos()], 1) * embed.float().std()).to(embed.dtype)

    @staticmethod
    def _norm(x: torch.Tensor) -> torch.Tensor:
        return x * torch.rsqrt(x.square().mean(-1, keepdim=True) + 1e-6)

    def forward(self, tokens, starts, tree, places, max_nodes: int):
        """logits [T][V], and K and V [layers][T][heads][dim] of rows that the cache does not have yet."""
        T, hq, h, dim, wt = tokens.numel(), self.heads_q, self.heads, self.dim, self.embed.dtype
        x = self.embed[tokens].float()
        if self.inv_freq is None:
            x = x + self.where[places].float()
        new = torch.empty((2, len(self.ffn), T, h, dim), dtype=wt, device=x.device)
        for l, layer in enumerate(self.ffn):
            qkv = (self._norm(x).to(wt) @ self.Wqkv[l]).view(T, hq + 2 * h, dim)
            q, k, v = qkv.split((hq, h, h), dim=1)
            if self.inv_freq is not None:
                norm = dict(zip(("q_weight", "k_weight"), (w[l] for w in self.qk_norm)), eps=1e-6) if self.qk_norm is not None else {}
                q, k = binding.qk_rope(q, k, places, self.inv_freq, k_out=new[0, l], **norm)
            else:
                new[0, l] = k
            new[1, l] = v
            a = binding.tree_attn(self.cache, l, q, k, v, self.table, self.lens, starts, tree=tree, max_nodes=max_nodes)
            x = x + (a.view(T, hq * dim) @ self.Wo[l]).float()
            z = self._norm(x).to(wt)
            x = x + torch.cat([binding.ffn_step(layer, z[i:i + self.rows].contiguous()) for i in range(0, T, self.rows)])
        return self._norm(x).to(wt) @ self.head.t(), new[0], new[1]

    def _rows(self, trees: List[Tree]):
        """Device tensors of one step's rows from (tokens, parents) of each request, roots among them (parent -1)."""
        tokens, masks, depth, starts = [], [], [], [0]
        for toks, parents in trees:
            _look_over((toks, parents), self.embed.shape[0])
            first = len(tokens)
            for j, p in enumerate(parents):
                masks.append((masks[first + p] if p >= 0 else 0) | 1 << j)
                depth.append(depth[first + p] + 1 if p >= 0 else 0)
            tokens += toks
            starts.append(len(tokens))
        most = max(1, max(len(t) for t, _ in trees))
        signed = [m - (1 << 64) if m >> 63 else m for m in masks]
        dev, i32 = self.embed.device, torch.int32
        sizes = torch.tensor([len(t) for t, _ in trees], device=dev)
        places = torch.repeat_interleave(self.lens, sizes, output_size=len(tokens)) + torch.tensor(depth, dtype=i32, device=dev)
        return (torch.tensor(tokens, dtype=i32, device=dev), torch.tensor(starts, dtype=i32, device=dev),
                torch.tensor(signed, dtype=torch.int64, device=dev), places, most)

    def _store(self, k, v, add, starts, keep=None, rows=None):
        slots, self.lens, self.pool, refused = binding.kv_plan(self.table, self.ring, self.pool, self.lens, add, starts,
                                                               self.cache.page, keep=keep, rows=rows)
        binding.kv_commit(self.cache, k, v, slots)
        return refused

    def release(self) -> None:
        """Every request ends: all pages are free again.  What prefill() or step() stored before they raised is given back by it too."""
        ends = torch.full_like(self.lens, -1)
        none = torch.zeros(ends.numel() + 1, dtype=torch.int32, device=ends.device)
        _, self.lens, self.pool, _ = binding.kv_plan(self.table, self.ring, self.pool, self.lens, ends, none, self.cache.page, rows=0)

    def prefill(self, prompts: List[List[int]]) -> None:
        """All but the last token of each prompt into the cache, up to 64 tokens of each request at a time."""
        done, ends = 0, [len(p) - 1 for p in prompts]
        while done < max(ends):
            part = [p[done:min(e, done + binding.MAX_NODES)] for p, e in zip(prompts, ends)]
            tokens, starts, tree, places, most = self._rows([(t, list(range(-1, len(t) - 1))) for t in part])
            _, k, v = self.forward(tokens, starts, tree, places, most)
            if self._store(k, v, starts.diff(), starts, rows=tokens.numel()).any():
                raise RuntimeError("the cache has too few pages for these prompts")
            done += binding.MAX_NODES

    def save(self):
        """The cached tokens of all requests, to bring back with load(): (lengths, k, v [layers][tokens][heads][dim]).  All pages are free
        afterwards."""
        lens, page = self.lens.tolist(), self.cache.page
        i = torch.cat([torch.arange(n, device=self.lens.device) for n in lens])
        r = torch.repeat_interleave(torch.arange(len(lens), device=i.device), self.lens, output_size=sum(lens))
        k, v = binding.kv_read(self.cache, self.table[r, i // page].long() * page + i % page)
        self.release()
        return lens, k, v

    def load(self, saved) -> None:
        """What save() gave, into pages of a decoder without tokens (of the same layers; its cache may be of another size)."""
        lens, k, v = saved
        c, shape = self.cache, (self.cache.layers, sum(lens), self.heads, self.dim)
        if (len(lens) != self.lens.numel() or any(n < 0 for n in lens)
                or any(t.shape != shape or t.dtype is not c.rows or t.device != c.K.device for t in (k, v))):
            raise ValueError(f"a length for each request and K and V {shape} of {c.rows} on {c.K.device} go with this decoder, "
                             f"got {len(lens)} lengths, {tuple(k.shape)} {k.dtype} on {k.device} and {tuple(v.shape)} {v.dtype} on {v.device}")
        if bool(self.lens.any()):
            raise RuntimeError("the cache holds tokens of other requests: release() them first")
        starts = torch.tensor([0] + lens, dtype=torch.int32, device=self.lens.device).cumsum(0, dtype=torch.int32)
        if self._store(k, v, starts.diff(), starts, rows=sum(lens)).any():
            self.release()
            raise RuntimeError("the cache has too few pages for these requests")

    def step(self, trees: List[Tree], live: List[bool], drawn: Optional[dict] = None) -> List[List[int]]:
        """One step; trees[r] starts with the newest certain token.  live[r] False: the request ends, its pages are free again.
        drawn: settings of binding.sample as numbers, and ``generator`` of its random numbers; None: the largest logits.
        Returns the new certain tokens of each request, one at least."""
        tokens, starts, tree, places, most = self._rows([t if on else ([], []) for t, on in zip(trees, live)])
        logits, k, v = self.forward(tokens, starts, tree, places, most)
        if drawn is None:
            keep, counts, following, _ = binding.tree_accept(logits, tokens, starts, tree=tree, max_nodes=most)
        else:
            keep, counts, following, _ = self._drawn(logits, tokens, starts, tree, most, **drawn)
        add = torch.where(torch.tensor(live, device=counts.device), counts, -1)
        refused = self._store(k, v, add, starts, keep=keep)
        R, T = len(trees), tokens.numel()
        got = torch.cat([refused, following, starts, keep]).tolist()        # the step's one read-back
        if any(got[:R]):
            raise RuntimeError("the cache has too few pages for these requests")
        following, starts, keep = got[R:2 * R], got[2 * R:3 * R + 1], got[3 * R + 1:]
        out = []
        for r, (toks, _) in enumerate(trees):
            ranks = keep[starts[r]:starts[r + 1]]
            branch = [t for rank, t in sorted((n, t) for n, t in zip(ranks, toks) if n > 0)]
            out.append(branch + [following[r]] if live[r] else [])
        return out

    @staticmethod
    def _drawn(logits, tokens, starts, tree, most, generator=None, **how):
        dev, T = logits.device, tokens.numel()
        each = {n: torch.full((T,), v, dtype=torch.int32 if n == "top_k" else torch.float32, device=dev) for n, v in how.items()}
        return binding.tree_sample(logits, torch.rand(T, device=dev, generator=generator), tokens, starts, tree=tree, max_nodes=most, **each)

    def generate(self, prompts: List[List[int]], new: int, nodes: int = 8, draft: Callable[[Sequence[int], int], Tree] = lookup,
                 drawn: Optional[dict] = None) -> Tuple[List[List[int]], int]:
        """``new`` tokens after each prompt (one for each of the cache's requests), and the number of steps that took.  draft
        proposes up to nodes - 1 tokens from what a request has (none are taken that would lead past ``new``, so a request never needs
        room for more than its prompt and those); nodes=1 decodes one by one.  drawn: as in step(), e.g. dict(temperature=0.8,
        top_p=0.95).  All pages are free afterwards, after an error too."""
        assert len(prompts) == self.lens.numel() and min(map(len, prompts)) > 0
        if bool(self.lens.any()):
            raise RuntimeError("the cache holds tokens of other requests: release() them first")
        try:
            return self._generate(prompts, new, nodes, draft, drawn)
        finally:
            self.release()

    def _generate(self, prompts, new, nodes, draft, drawn):
        self.prefill(prompts)
        text, steps = [list(p) for p in prompts], 0
        live = [new > 0] * len(prompts)
        while any(live):
            trees = []
            for t, p in zip(text, prompts):
                levels = len(p) + new - len(t) - 1          # a step's answers are one more than the drafts it keeps
                toks, parents = cut(draft(t, nodes - 1), levels) if nodes > 1 and levels > 0 else ([], [])
                trees.append(([t[-1]] + toks, [-1] + [p + 1 for p in parents]))
            for t, more in zip(text, self.step(trees, live, drawn)):
                t += more
            steps += 1
            live = [on and len(t) < len(p) + new for on, t, p in zip(live, text, prompts)]
        return [t[len(p):len(p) + new] for t, p in zip(text, prompts)], steps


def random_decoder(layers: int = 2, d: int = 512, D: int = 2048, r: int = 64, V: int = 1000, heads_q: int = 8, heads: int = 2, dim: int = 64,
                   dtype=torch.bfloat16, bias: float = -1.3, seed: int = 0, device="cuda", **cache) -> Decoder:
    """A decoder of random weights, but for its head: as a rule it answers a token with the next one of twelve in a circle.  bias:
    of the FFN's predictor; a large one makes every neuron active."""
    g = torch.Generator().manual_seed(seed)

    def made(rows, cols, scale=None):
        return (torch.randn(rows, cols, generator=g) * (rows ** -0.5 if scale is None else scale)).to(dtype).to(device)

    ffn = [binding.DeviceLayer(made(d, r), made(D, r, 1.0), torch.full((D,), bias, device=device), made(D, d, d ** -0.5),
                               made(D, d, d ** -0.5), made(D, d, D ** -0.5)) for _ in range(layers)]
    Wqkv = [made(d, (heads_q + 2 * heads) * dim) for _ in range(layers)]
    Wo = [made(heads_q * dim, d) for _ in range(layers)]
    embed, t = made(V, d, 1.0), torch.arange(V)
    first = t - t % 12
    head = torch.empty_like(embed)
    head[first + (t - first + 1) % (V - first).clamp(max=12)] = embed
    return Decoder(ffn, Wqkv, Wo, embed, head, heads_q, heads, dim, **cache)


def main() -> None:
    g = torch.Generator().manual_seed(1)
    prompts = [torch.randint(0, 1000, (n,), generator=g).tolist() * 2 for n in (5, 40, 100)]
    decoder = random_decoder(requests=len(prompts), pages=64, max_len=1024)
    for nodes in (1, 8, 24):
        out, steps = decoder.generate(prompts, 100, nodes=nodes)
        print(f"trees of {nodes}: {steps} steps for 100 tokens of {len(prompts)} requests; the first of each: {[o[:3] for o in out]}")
    inv_freq = (10000.0 ** (-torch.arange(0, 64, 2, device="cuda").double() / 64)).float()
    weights = torch.ones((2, 64), device="cuda")
    decoder = random_decoder(requests=len(prompts), pages=64, max_len=1024, cache_dtype=torch.float8_e4m3fn, inv_freq=inv_freq, qk_norm=(weights, weights))
    out, steps = decoder.generate(prompts, 100, nodes=8, drawn=dict(temperature=0.8, top_k=50, top_p=0.95))
    print(f"rotary positions, a cache in 8 bits, drawn tokens: {steps} steps; the first of each: {[o[:3] for o in out]}")


if __name__ == "__main__":
    main()
