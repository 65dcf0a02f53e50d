"""Tokens from logits and given random numbers, against the oracle's whole weights: the same tokens.

The kernel's exponentials may be off by an ulp of 64 bits, so that a weight of up to 2^44 units is now and then another one by a unit, and
a sum of V weights by some sqrt(V) units of 2^44 or more: a token is another one where u lies within 1e-11 of a border, which random numbers
of 24 bits on rows of random logits do not do here."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def env():
    import torch
    from oracle import draft, serve
    from paper_2603_14110_amd import binding

    assert torch.cuda.is_available(), "this test needs a GPU"
    binding.lib()
    return torch, binding, serve, draft


DEFAULTS = dict(temperature=1.0, top_k=0, top_p=1.0, min_p=0.0)
SETTINGS = [dict(), dict(temperature=0.7), dict(top_k=1), dict(top_k=5), dict(top_k=50, top_p=0.9), dict(top_p=0.95), dict(top_p=0.3, temperature=2.5),
            dict(min_p=0.05), dict(min_p=0.5, top_k=20), dict(temperature=0.6, top_k=40, top_p=0.95, min_p=0.02), dict(temperature=0.0), dict(top_p=0.999),
            dict(temperature=30.0), dict(temperature=30.0, top_k=300, top_p=0.7), dict(temperature=0.02)]


def f32(torch, v):
    return torch.tensor(v, dtype=torch.float32, device="cuda")


def run(torch, binding, logits, u, hows, **more):
    hows = [{**DEFAULTS, **h} for h in hows]
    col = lambda n: [h[n] for h in hows]
    return binding.sample(logits, f32(torch, u), temperature=f32(torch, col("temperature")), top_k=torch.tensor(col("top_k"), dtype=torch.int32, device="cuda"),
                          top_p=f32(torch, col("top_p")), min_p=f32(torch, col("min_p")), want_logp=True, **more)


def as_f32(how):
    """Settings as the device has them."""
    return {n: v if n == "top_k" else float(np.float32(v)) for n, v in how.items()}


def check(torch, binding, serve, logits, u, hows):
    answers, logp = run(torch, binding, logits, u, hows)
    rows = logits.float().cpu().numpy()
    for t, (a, p) in enumerate(zip(answers.tolist(), logp.tolist())):
        want = serve.draw(rows[t], float(np.float32(u[t])), **as_f32(hows[t]))
        assert a == want[0], (t, hows[t], u[t], a, want[:2])
        # fp32's rounding, and sums that are off by 1e-11
        assert p == want[1] or abs(p - want[1]) <= 2.0 ** -24 * abs(want[1]) + 1e-10, (t, hows[t], p, want[1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("V", [1, 2, 7, 64, 1000, 1023, 32000, 40003])
def test_tokens_against_the_oracle(env, dtype, V):
    torch, binding, serve, _ = env
    rng = np.random.default_rng(V)
    T = 2 * len(SETTINGS)
    for shift, spread in ((0, 2.0), (3, 0.1), (1, 8.0)):         # rows at any address
        g = torch.Generator(device="cuda").manual_seed(V + shift)
        wide = (torch.randn((T, V + 5), device="cuda", generator=g) * spread).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
        wide[:, :shift] = 1e9                                    # neighbours that must not win
        wide[:, shift + V:] = float("nan")
        u = [float(v) for v in rng.random(T, dtype=np.float32)]
        u[0], u[-1] = 0.0, float(np.nextafter(np.float32(1), np.float32(0)))
        check(torch, binding, serve, wide[:, shift:shift + V], u, SETTINGS + SETTINGS[::-1])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_ties_masks_and_values_that_are_not_finite(env, dtype):
    torch, binding, serve, _ = env
    td, V, inf = torch.bfloat16 if dtype == "bf16" else torch.float32, 3001, float("inf")
    g = torch.Generator(device="cuda").manual_seed(2)
    least = float(torch.finfo(td).min)
    rows = []

    def row(f):
        x = torch.randn(V, device="cuda", generator=g).to(td)
        f(x)
        rows.append(x)

    def half_masked(value):
        def f(x):
            x[torch.rand(V, device="cuda", generator=g) < 0.7] = value
        return f

    row(lambda x: x.fill_(0.25))                                 # all equal
    row(lambda x: x.fill_(-0.0))
    row(lambda x: x.copy_((x * 2).round() / 2))                  # a few values, each many times
    row(lambda x: x[::2].fill_(1.0))
    row(half_masked(-inf))
    row(half_masked(least))
    row(half_masked(-1e9))
    row(half_masked(-1e4))
    row(lambda x: x.fill_(-inf))                                 # nothing is left
    row(lambda x: (x.fill_(-inf), x[17].fill_(-3.0)))            # one token is
    row(lambda x: (x.fill_(-inf), x[V - 1].fill_(least)))
    row(lambda x: x.fill_(least))
    row(lambda x: x.index_fill_(0, torch.tensor([5, 2000], device="cuda"), inf))
    row(lambda x: x.index_fill_(0, torch.tensor([9, 2], device="cuda"), float("nan")))
    row(lambda x: (x[100].fill_(inf), x[2999].fill_(float("nan"))))
    row(lambda x: x.mul_(1e30))
    row(lambda x: x.mul_(1e-30))
    row(lambda x: (x[::3].fill_(-0.0), x[1::3].fill_(0.0), x[2::3].fill_(0.0)))
    row(lambda x: (x.fill_(-200.0), x[0].fill_(float(torch.finfo(td).max))))
    x = torch.stack(rows)
    for k, how in enumerate(SETTINGS):
        for u in (0.0, 0.37, 0.999999):
            check(torch, binding, serve, x, [u] * len(rows), [how] * len(rows))


def test_settings_at_their_ends(env):
    torch, binding, serve, _ = env
    nan, inf = float("nan"), float("inf")
    x = torch.randn((1, 500), device="cuda", generator=torch.Generator(device="cuda").manual_seed(3))
    first = int(x[0].argmax())
    ask = lambda u=0.7, **how: int(run(torch, binding, x, [u], [how])[0])
    plain = ask()
    row = x[0].cpu().numpy()
    assert plain == serve.draw(row, float(np.float32(0.7)))[0]
    for how in (dict(top_k=-3), dict(top_k=500), dict(top_k=1 << 30), dict(top_p=1.5), dict(top_p=nan), dict(top_p=inf), dict(min_p=-1.0), dict(min_p=nan)):
        assert ask(**how) == plain, how
    for how in (dict(temperature=0.0), dict(temperature=-1.0), dict(temperature=nan), dict(temperature=1e-38), dict(temperature=1e-42), dict(top_k=1), dict(top_p=0.0), dict(top_p=-1.0),
                dict(top_p=1e-30), dict(min_p=1.0), dict(min_p=7.0)):
        assert ask(u=0.99, **how) == first, how
    assert ask(u=nan) == ask(u=-1.0) == ask(u=0.0) == first
    last = ask(u=1.0)
    assert last == ask(u=5.0) == ask(u=inf) == int(np.argsort(-row, kind="stable")[-1])
    for u in (0.0, 0.25, 0.9):                                    # all tokens alike; 0.9 is 0.89999998 in fp32, 449.99999 tokens
        assert ask(u=u, temperature=inf) == int(np.argsort(-row, kind="stable")[int(float(np.float32(u)) * 500)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_shares_of_drawn_tokens(env, dtype):
    """4096 equal steps of u on one row: each kept token comes as often as its share says, to one step."""
    torch, binding, serve, _ = env
    n = 4096
    row = (torch.randn(3000, device="cuda", generator=torch.Generator(device="cuda").manual_seed(5)) * 3).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    for how in (dict(), dict(temperature=0.8, top_p=0.9), dict(top_k=30)):
        how = as_f32({**DEFAULTS, **how})
        answers, _ = run(torch, binding, row.expand(n, -1), [(i + 0.5) / n for i in range(n)], [how] * n)
        kept = serve.draw(row.float().cpu().numpy(), 0.0, **how)[2]
        z = row.double()[kept] / how["temperature"]
        count = torch.bincount(answers.long(), minlength=3000)[kept]
        assert int(count.sum()) == n and float((count - z.softmax(0) * n).abs().max()) <= 1.0 + 1e-6


@pytest.mark.parametrize("dtype,V", [("bf16", 152064), ("f32", 152064), ("bf16", 1 << 19), ("f32", (1 << 19) - 1)])
def test_large_vocabularies(env, dtype, V):
    torch, binding, serve, _ = env
    g = torch.Generator(device="cuda").manual_seed(7)
    x = (torch.randn((6, V), device="cuda", generator=g) * 2.5).to(torch.bfloat16 if dtype == "bf16" else torch.float32)
    x[4] = 1.0                                                    # the largest sum there is
    check(torch, binding, serve, x, [0.3, 0.91, 0.5, 0.77, 0.9999, 0.2], [dict(top_p=0.95), dict(), dict(top_k=1000, top_p=0.99), dict(min_p=0.01), dict(), dict(top_p=0.9999)])


def test_no_rows_repeats_streams_and_graphs(env):
    torch, binding, serve, _ = env
    none = binding.sample(torch.empty((0, 50), device="cuda"), torch.empty(0, device="cuda"))
    assert none.shape == (0,)
    x = torch.randn((30, 5000), device="cuda").bfloat16()
    how = dict(temperature=f32(torch, [0.9] * 30), top_p=f32(torch, [0.8] * 30), want_logp=True)
    u = torch.rand(30, device="cuda")
    graph, out = torch.cuda.CUDAGraph(), None
    torch.cuda.synchronize()
    with torch.cuda.graph(graph):
        out = binding.sample(x, u, **how)
    side = torch.cuda.Stream()
    for step in range(4):
        u.uniform_()
        x.normal_()
        graph.replay()
        torch.cuda.synchronize()
        got = [o.clone() for o in out]
        with torch.cuda.stream(side):
            want = binding.sample(x, u, **how)
        side.synchronize()
        again = binding.sample(x, u, **how)
        assert all(torch.equal(a, b) and torch.equal(a, c) for a, b, c in zip(got, want, again))


def test_trees_of_drawn_answers(env):
    """The walk is tree_accept's, with drawn answers in the place of the largest logits'; padding and rows past the limit are in no branch."""
    torch, binding, serve, draft = env
    from draft_cases import parents, signed, words
    import random

    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")
    rng = random.Random(3)
    sizes, V = [1, 8, 0, 64, 17], 40
    starts = np.cumsum([0] + sizes).tolist()
    tree = sum((words(parents(rng, n)) for n in sizes), [])
    T = starts[-1] + 4
    x = torch.randn((T, V), device="cuda", generator=torch.Generator(device="cuda").manual_seed(1)) * 3
    u = torch.rand(T, device="cuda")
    answers = binding.sample(x, u)
    rows = x.cpu().numpy()
    # a draft that is right as a rule: the answer at its parent
    up = [s + max(draft.parent(tree, s + j, j), 0) for s, n in zip(starts, sizes) for j in range(n)]
    tokens = [answers.tolist()[p] if rng.random() < 0.8 else rng.randrange(V) for p in up] + [0] * 4
    marked = np.full((T, V), -1.0)
    marked[np.arange(T), answers.tolist()] = 1.0                 # rows whose largest logit is the answer
    for t, w in ((None, None), (torch.tensor(signed(tree + [0] * 4), dtype=torch.int64, device="cuda"), tree + [0] * 4)):
        want = draft.accept(marked, tokens, w, starts)
        got = binding.tree_sample(x, u, i32(tokens), i32(starts), tree=t, max_nodes=64)
        assert [g.tolist() for g in got] == [list(v) for v in want]
        walked = binding.tree_walk(answers, i32(tokens), i32(starts), tree=t, max_nodes=64)
        assert all(torch.equal(a, b) for a, b in zip(walked, got))
        full = binding.tree_sample(x, u, i32(tokens), i32(starts), tree=t, max_nodes=64, want_logp=True, temperature=torch.zeros(T, device="cuda"))
        best = binding.tree_accept(x, i32(tokens), i32(starts), tree=t, max_nodes=64)
        assert all(torch.equal(a, b) for a, b in zip(full[:4], best)) and bool((full[4] == 0).all())
    keep, counts, following = binding.tree_walk(answers, i32(tokens), i32(starts), max_nodes=8)
    assert bool((keep[starts[3] + 8:starts[4]] == -1).all()) and int(counts.max()) <= 8 and counts[2] == 0 and following[2] == -1
    # an answer of -1 agrees with no token
    keep, counts, following = binding.tree_walk(i32([-1, 3]), i32([5, 3]), i32([0, 2]))
    assert keep.tolist() == [0, -1] and counts.tolist() == [1] and following.tolist() == [-1]


def test_binding_refuses_what_does_not_go_together(env):
    torch, binding, serve, _ = env
    x, u = torch.randn((4, 100), device="cuda"), torch.rand(4, device="cuda")
    binding.sample(x, u)
    for bad in (dict(logits=x.half()), dict(logits=x.t()), dict(logits=x[0]), dict(u=u[:2]), dict(u=u.double()), dict(temperature=u[:1]), dict(top_k=u),
                dict(top_p=u.bfloat16()), dict(min_p=u.cpu()),
                dict(logits=torch.empty((4, (1 << 19) + 1), device="cuda"))):
        with pytest.raises(binding.SvdpError):
            binding.sample(**{**dict(logits=x, u=u), **bad})
    i32 = torch.zeros(4, dtype=torch.int32, device="cuda")
    for a, b, c in ((i32.long(), i32, i32[:2]), (i32, i32[:3], i32[:2]), (i32, i32, i32[:2].long())):
        with pytest.raises(binding.SvdpError):
            binding.tree_walk(a, b, c)


@pytest.mark.parametrize("T", [256, 257, 700])
def test_many_rows_of_every_kind(env, T):
    """More rows than there are compute units: rows with values that have no bin, masked ones and ordinary ones between each other."""
    torch, binding, serve, _ = env
    rng, inf = np.random.default_rng(T), float("inf")
    x = torch.randn((T, 1201), device="cuda", generator=torch.Generator(device="cuda").manual_seed(T)).mul_(3).bfloat16()
    x[::7] *= 1e-20                                              # below the smallest bin
    x[3::11, ::2] = -inf
    x[5::13, 17] = 300.0
    x[6::17] = -inf
    x[8::19, 40:50] = 0.0
    x[2::23, 9] = float("nan")
    x[4::29] -= 270.0                                            # all far below, and near to each other
    u = [float(v) for v in rng.random(T, dtype=np.float32)]
    check(torch, binding, serve, x, u, [SETTINGS[i % len(SETTINGS)] for i in range(T)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_more_rows_than_a_launch_takes(env, dtype):
    torch, binding, serve, _ = env
    T = (1 << 21) + 7
    x = torch.tensor([[0.0, 1.0], [3.0, -1.0]], device="cuda").to(torch.bfloat16 if dtype == "bf16" else torch.float32).repeat(T // 2 + 1, 1)[:T]
    u = torch.rand(T, device="cuda", generator=torch.Generator(device="cuda").manual_seed(1))
    answers = binding.sample(x, u)
    share = x.double().softmax(1).amax(1)                        # of the larger one, which comes first in the order
    clear = (u.double() - share).abs() > 1e-6
    first = x.float().argmax(1).int()
    assert torch.equal(answers[clear], torch.where(u.double() < share, first, 1 - first)[clear]) and int((~clear).sum()) < 100


def test_tensors_of_another_device_are_refused(env, monkeypatch):
    """Kernels go to the current device's stream."""
    torch, binding, serve, _ = env
    x, u = torch.randn((2, 50), device="cuda"), torch.rand(2, device="cuda")
    cache = binding.KVCache.empty(1, 1, 32, 1, 64)
    i32 = torch.zeros(2, dtype=torch.int32, device="cuda")
    q = torch.zeros((2, 1, 64), device="cuda")
    monkeypatch.setattr(binding, "_current_device", lambda: 1)
    coded = binding.KVCache.empty(1, 1, 32, 1, 64, dtype=torch.float8_e4m3fn)
    h, slots = q.bfloat16(), torch.zeros(2, dtype=torch.int64, device="cuda")
    for call in (lambda: binding.sample(x, u), lambda: binding.tree_walk(i32, i32, i32), lambda: binding.kv_read(cache, i32.long()),
                 lambda: binding.qk_rope(q, q, i32, torch.ones(4, device="cuda")), lambda: binding.kv_commit(coded, h[None], h[None], slots),
                 lambda: binding.tree_attn(coded, 0, h, h, h, i32[None], i32[:1], i32)):
        with pytest.raises(binding.SvdpError, match="current device"):
            call()
