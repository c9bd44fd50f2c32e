"""Filtered sampling (msd_sample) and tree acceptance on filtered distributions
(msd_accept_batch) against their definitions in 64 bits: settings alone and together, equal
logits at every border, masked and infinite logits, odd widths and strides, both types,
streams, graphs, repeated runs, and the calls that are refused."""
import math
import random

import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.tokens_support import check_accept, check_sample, settings

pytestmark = pytest.mark.gpu
INF = math.inf


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def logits(rows, vocab, seed=0, dtype=torch.float32, spread=2.5, peaks=60):
    g = gen(seed)
    x = spread * torch.randn(rows, vocab, generator=g, device="cuda")
    n = min(peaks, vocab)
    at = torch.randint(0, vocab, (rows, n), generator=g, device="cuda")
    return x.scatter_reduce_(1, at, 9 - 1.5 * torch.log1p(torch.arange(n, device="cuda").float()).expand(rows, n), "amax").to(dtype)


def uniforms(rows, seed=1):
    return torch.rand(rows, generator=gen(seed), device="cuda")


ALONE = [{}, dict(temperature=0.7), dict(temperature=3.0), dict(temperature=0.0), dict(top_k=1), dict(top_k=40),
         dict(top_p=0.9), dict(top_p=0.01), dict(min_p=0.05), dict(temperature=0.8, top_k=50, top_p=0.9, min_p=0.02),
         dict(temperature=1.5, top_k=3, top_p=0.999), dict(temperature=1.3, top_p=0.97, min_p=0.001)]


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("given", ALONE, ids=lambda g: "-".join(f"{k}{v}" for k, v in g.items()) or "off")
def test_settings(given, dtype):
    check_sample(logits(7, 4099, dtype=dtype), uniforms(7), **given)


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("vocab", [1, 2, 3, 31, 33, 255, 1024, 8191, 32000, 50001, 131075])
def test_widths(vocab, dtype):
    check_sample(logits(3, vocab, vocab, dtype), uniforms(3, vocab), temperature=[0.7, 1.0, 1.6], top_k=[50, 0, 7000],
                 top_p=[0.9, 0.95, 0.999], min_p=[0.0, 0.01, 0.0])


def test_the_largest_vocabulary():
    check_sample(logits(2, 393216, 5), uniforms(2), temperature=1.1, top_p=0.98)


@pytest.mark.parametrize("rows", [1, 2, 5, 37, 152, 153, 400])
def test_row_counts(rows):
    x = logits(rows, 1500, rows)
    t = [0.5 + 0.25 * (i % 5) for i in range(rows)]
    check_sample(x, uniforms(rows, rows), temperature=t, top_k=[(i * 7) % 60 for i in range(rows)],
                 top_p=[1.0 - 0.1 * (i % 4) for i in range(rows)], min_p=[0.03 * (i % 3) for i in range(rows)])


def test_settings_that_are_off_and_out_of_range():
    n = 14
    check_sample(logits(n, 700), uniforms(n), temperature=[1, 1, 1, 1, 1, 1, -1, math.nan, INF, 1e-35, 1, 1, 1, 1e38],
                 top_k=[0, -5, 700, 701, 2**31 - 1, 0, 0, 0, 0, 0, 0, 0, 0, 0],
                 top_p=[1, 1.5, math.nan, 1, INF, -1, 1, 1, 1, 1, 0.0, 1, 1, 1],
                 min_p=[0, -1, 0, math.nan, 0, 0, 0, 0, 0, 0, 0, 1.0, 1.5, 0])


def test_equal_logits():
    """All equal; two values; equal ones at the border of top-k and of top-p, whose lowest ids stay."""
    x = torch.full((6, 1000), 2.0, device="cuda")
    x[1, 500:] = 1.0
    x[2, ::2] = 1.0
    x[3, 3::7] = 5.0
    x[4] = 0.0
    x[4, 1::2] = -0.0
    check_sample(x, uniforms(6), top_k=[100, 600, 700, 10, 300, 0], top_p=[0.5, 1.0, 0.9, 0.75, 0.5, 0.25])
    check_sample(x, uniforms(6, 3), top_p=[0.25, 0.5, 0.5, 0.125, 1 / 3, 0.999])
    check_sample(x.bfloat16(), uniforms(6, 4), top_k=[1, 999, 501, 142, 143, 144])


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_masked_and_infinite_logits(dtype):
    x = logits(9, 2000, 3, dtype)
    x[0, ::2] = -INF
    x[1] = -INF                            # nothing is left
    x[2, :] = math.nan
    x[3, 5:] = -INF                        # fewer than top_k
    x[4, 100::300] = INF                   # several infinite ones
    x[5, 7] = INF
    x[6, ::3] = math.nan
    x[7] = -INF
    x[7, 1999] = -3.0e38                   # one very small one
    x[8, ::2] = torch.finfo(dtype).min     # masks of the type's lowest value
    check_sample(x, uniforms(9), temperature=0.9, top_k=40, top_p=0.9)
    check_sample(x, uniforms(9, 2))
    check_sample(x, uniforms(9, 3), min_p=0.1, top_p=0.99)
    check_sample(x, uniforms(9, 4), temperature=0.0)


def test_wide_and_narrow_ranges():
    """Differences of thousands, of the last bits of fp32, and of many orders of magnitude."""
    g = gen(9)
    x = torch.randn(8, 3000, generator=g, device="cuda")
    x[0] *= 1e4
    x[1] *= 1e-6
    x[2] = 1000 + 1e-4 * x[2]
    x[3] = x[3] * torch.exp(20 * torch.rand(3000, generator=g, device="cuda") - 10)
    x[4] *= 3e37
    x[5] *= 1e-40
    x[6] = -80 + x[6]
    x[6, 17] = 0.0                         # a peak, and all the rest far below it
    x[7] = torch.linspace(0, 60, 3000, device="cuda")
    for given in ({}, dict(top_p=0.9), dict(top_k=1000, top_p=0.5), dict(temperature=30.0, top_p=0.8), dict(min_p=1e-4)):
        check_sample(x, uniforms(8, 11), **given)


def test_uniforms_at_the_ends():
    x = torch.tensor([[0.0, -INF, 0.0, 0.0, -INF, 0.0, -INF, -INF]], device="cuda").repeat(8, 1)
    u = torch.tensor([0.0, 0.25, 0.5, 0.75, 1 - 2.0 ** -24, 1.0, -1.0, math.nan], device="cuda")
    got = check_sample(x, u)
    assert got.tolist() == [0, 2, 3, 5, 5, 5, 0, 0]


def test_strides_and_neighbours():
    """Rows at odd strides and places; what lies between them is neither read into a result nor written."""
    for dtype in (torch.float32, torch.bfloat16):
        wide = torch.full((5, 3013), 50.0, dtype=dtype, device="cuda")
        wide[:, 3:3003] = logits(5, 3000, 1, dtype)
        check_sample(wide[:, 3:3003], uniforms(5), temperature=0.8, top_k=100, top_p=0.9)
        assert bool((wide[:, :3] == 50).all()) and bool((wide[:, 3003:] == 50).all())
    probs = torch.full((4, 1030), 7.0, device="cuda")
    t = torch.zeros(4, dtype=torch.int32, device="cuda")
    msd.sample(logits(4, 1021), uniforms(4), None, t, probs=probs[:, 5:1026])
    assert bool((probs[:, :5] == 7).all()) and bool((probs[:, 1026:] == 7).all())
    assert torch.allclose(probs[:, 5:1026].sum(1), torch.ones(4, device="cuda"), atol=1e-4)


def test_min_p_between_two_logits_whose_weights_are_the_other_way_round():
    """Weights are taken to 2^-44, so of two logits the lower one's may be the larger by a unit. Where min_p lies between them,
    what is drawn, its probability and what a tree accepts go by the weights alike, through lists (top_k) and without."""
    for top, low in (("0x1.c2f09p+3", "0x1.7ffffep-20"), ("0x1.c646bap+3", "-0x1.800002p-20"), ("0x1.b5f74ep+3", "-0x1.2p-18")):
        top, low = float.fromhex(top), float.fromhex(low)
        high = torch.nextafter(torch.tensor(low), torch.tensor(INF)).item()
        x = torch.tensor([[top, high, low] + [-50.0] * 5], device="cuda")
        p = torch.tensor(math.exp(low - top)).nextafter(torch.tensor(0.0)).item()
        u = torch.tensor([1.0], device="cuda")                       # the last id that is left
        for min_p in (p, math.exp(low - top), torch.tensor(math.exp(low - top)).nextafter(torch.tensor(1.0)).item()):
            for top_k in (0, 3):
                f, _ = settings(1, top_k=top_k, min_p=min_p)
                t, lp, probs = torch.zeros(1, dtype=torch.int32, device="cuda"), torch.zeros(1, device="cuda"), torch.zeros(1, 8, device="cuda")
                msd.sample(x, u, f, t, logp=lp, probs=probs)
                share = probs[0, int(t)].item()
                # half a step of a logarithm of 14 is 2^-21; the probability's own 2^-21; a unit of a weight of 10^7
                assert share > 0 and abs(share - math.exp(lp.item())) <= 2.0 ** -19 * share, (top, min_p, top_k, share, lp.item())
                assert not bool((probs[0, int(t) + 1:] > 0).any())
                # a child with the token that was drawn is accepted where u is 0
                b = msd.Batch(torch.zeros(1, dtype=torch.int32, device="cuda"), torch.tensor([0, 2], dtype=torch.int32, device="cuda"), 2)
                tree = msd.Tree(1, 2)
                tree.tokens.copy_(torch.cat([torch.zeros_like(t), t]))
                tree.parent.copy_(torch.tensor([-1, 0], dtype=torch.int32, device="cuda"))
                path, n, bonus = (torch.zeros(1, c, dtype=torch.int32, device="cuda") for c in (2, 1, 1))
                msd.accept(x.repeat(2, 1), b, tree, torch.zeros(1, 2, 2, device="cuda"), f, path, n.view(1), bonus.view(1))
                assert path.tolist() == [[0, 1]] and n.item() == 1, (top, min_p, top_k)


def test_no_rows():
    msd.sample(torch.empty(0, 100, device="cuda"), torch.empty(0, device="cuda"), None,
               torch.empty(0, dtype=torch.int32, device="cuda"))


def test_every_token_is_drawn_where_its_mass_lies():
    """A grid of uniforms over one row: each token's share of the draws is its mass."""
    x = torch.randn(1, 300, generator=gen(2), device="cuda").repeat(4096, 1)
    u = (torch.arange(4096, device="cuda") + 0.5) / 4096
    got = check_sample(x, u, want_probs=False, temperature=1.0, top_k=100)
    share = torch.softmax(x[0].double().where(x[0] >= x[0].topk(100).values[-1], -INF), 0)
    count = torch.bincount(got.long(), minlength=300)
    assert float((count / 4096 - share).abs().max()) <= 2 / 4096


def test_streams_and_graphs():
    """Two calls at once on two streams, and a captured call replayed on other inputs."""
    a, b = logits(20, 9000, 1), logits(20, 9000, 2)
    u, f, _ = uniforms(20), *settings(20, temperature=0.9, top_p=0.9)
    want = [msd.sample(x, u, f, torch.zeros(20, dtype=torch.int32, device="cuda")).clone() for x in (a, b)]
    torch.cuda.synchronize()
    s = [torch.cuda.Stream(), torch.cuda.Stream()]
    out = [torch.zeros(20, dtype=torch.int32, device="cuda") for _ in s]
    torch.cuda.synchronize()
    for _ in range(10):
        for st, x, t in zip(s, (a, b), out):
            msd.sample(x, u, f, t, stream=st)
    torch.cuda.synchronize()
    assert all(torch.equal(t, w) for t, w in zip(out, want))
    x, t = a.clone(), torch.zeros(20, dtype=torch.int32, device="cuda")
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        msd.sample(x, u, f, t)
    for src, w in zip((a, b, a), (want[0], want[1], want[0])):
        x.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        assert torch.equal(t, w)


def test_the_same_tokens_each_time():
    x, u = logits(64, 32000, 4), uniforms(64)
    f, _ = settings(64, temperature=1.2, top_p=0.98)
    got = []
    for _ in range(4):
        t, lp, p = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.zeros(64, device="cuda"), torch.zeros(64, 32000, device="cuda")
        msd.sample(x, u, f, t, logp=lp, probs=p)
        got.append((t, lp, p))
    for g in got[1:]:
        assert all(torch.equal(a, b) for a, b in zip(g, got[0]))


# -- trees -------------------------------------------------------------------
def trees(counts, nodes, vocab, x, seed=0, width=4):
    """Random trees whose tokens are mostly likely ones of their parents' rows."""
    r = random.Random(seed)
    best = torch.topk(x.float().nan_to_num(-9e9), min(8, x.shape[1])).indices.cpu().tolist()
    toks, pars, at = [], [], 0
    for c in counts:
        t, p, born = [r.randrange(vocab)], [-1], [0] * max(c, 1)
        for j in range(1, c):
            up = r.choice([i for i in range(max(0, j - 10), j) if born[i] < width] or [0])
            p.append(up)
            t.append(r.choice(best[at + up]) if r.random() < 0.8 else r.randrange(vocab))
            born[up] += 1
        toks.append(t[:nodes])
        pars.append(p[:nodes])
        at += c
    return toks, pars


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("given", [{}, dict(temperature=0.6), dict(top_k=5, top_p=0.9), dict(temperature=1.4, min_p=0.1),
                                   dict(temperature=0.0)], ids=str)
def test_trees(given, dtype):
    for seed in range(4):
        counts = [60, 1, 16, 33, 60, 2]
        x = logits(sum(counts), 3001, seed, dtype, peaks=12)
        u = torch.rand(6, 7, 11, generator=gen(seed), device="cuda")
        toks, pars = trees(counts, 60, 3001, x, seed)
        check_accept(x, counts, toks, pars, u, 60, **given)


@pytest.mark.parametrize("given", [{}, dict(top_k=20, top_p=0.9), dict(temperature=0.0)], ids=str)
@pytest.mark.parametrize("vocab,n,dtype", [(900, 40, torch.float32), (32000, 12, torch.float32), (70000, 7, torch.bfloat16), (300, 700, torch.float32)])
def test_more_rows_than_fit(vocab, n, dtype, given):
    """The first nodes ahead of the ones behind accepted children; some sequences without rows, of one, with fewer valid nodes."""
    r = random.Random(n)
    counts = [r.choice([60, 60, 47, 33, 1, 0]) for _ in range(n)] if n < 100 else [1 + i % 2 for i in range(n)]
    counts[0] = 60
    x = logits(sum(counts), vocab, 7, dtype, peaks=6)
    toks, pars = trees(counts, 60, vocab, x, 7, width=3)
    u = torch.rand(n, 7, 5, generator=gen(n), device="cuda") * 0.7                # (long paths too)
    check_accept(x, counts, toks, pars, u, 60, **given)
    check_accept(x, counts, toks, pars, u, 60, n_nodes=[c - c // 3 for c in counts], **given)


def test_trees_with_odd_shapes():
    """Sequences without rows, fewer valid nodes than rows, one child a node at most, no depth, a chain,
    the same token twice among siblings, tokens outside the vocabulary, parents that do not precede."""
    counts = [10, 0, 25, 7, 0, 3]
    x = logits(sum(counts), 500, 1, peaks=4)
    toks, pars = trees(counts, 32, 500, x, 1)
    for shape in ((6, 4, 3), (6, 1, 2), (6, 9, 2), (6, 40, 257)):
        check_accept(x, counts, toks, pars, torch.rand(*shape, generator=gen(3), device="cuda"), 32, top_p=0.95)
        check_accept(x, counts, toks, pars, torch.rand(*shape, generator=gen(4), device="cuda"), 32, n_nodes=[4, 0, 0, 32, 5, 1])
    n = 12
    x = logits(n, 50, 2, peaks=1, spread=0.3)
    top = x.argmax(1).tolist()
    for seed in range(6):
        u = torch.rand(1, 4, 12, generator=gen(seed), device="cuda")
        check_accept(x, [n], [[0] + [top[0]] * 5 + [7, 7, 9, 9, 50, -1]], [[-1] + [0] * 11], u, n)           # siblings alike
        check_accept(x, [n], [[0] + [9, 8, 7, 6, 5, 4, 3, 2, 1, 0, 49]], [[-1] + list(range(11))], u, n)     # a chain
        check_accept(x, [n], [[0] + [top[0]] * 11], [[-1, 5, 0, 3, 12, -7, 2, 7, 1000, 6, 9, 0]], u, n)      # bad parents
    x[0] = -INF
    check_accept(x, [n], [[0] + top[1:]], [[-1] + [0] * 11], u, n)                                          # a row without weight


def test_the_largest_trees():
    x = logits(1024, 64, 5, peaks=3)
    toks, pars = trees([1024], 1024, 64, x, 2, width=300)
    check_accept(x, [1024], toks, pars, torch.rand(1, 65, 257, generator=gen(5), device="cuda"), 1024)
    check_accept(x, [1024], [list(range(64)) * 16], [[-1] + [0] * 1023], torch.rand(1, 3, 257, generator=gen(6), device="cuda"), 1024)


def test_accepted_paths_go_to_the_cache():
    """A paged program's step: 4-bit head, acceptance, and the path kept in the pool."""
    from tests.pages_support import batch, pool
    n, nodes, V, H = 3, 12, 1003, 256
    p = pool([20 + nodes, 33 + nodes, 7 + nodes], seed=1)
    head = msd.Weight4.of(0.2 * torch.randn(V, H, generator=gen(1), device="cuda"), group=64, zeros=True)
    x = torch.randn(n * nodes, H, generator=gen(2), device="cuda")
    lg = head.linear(x, torch.empty(n * nodes, V, device="cuda"))
    toks, pars = trees([nodes] * n, nodes, V, lg, 3)
    u = torch.rand(n, 5, 5, generator=gen(3), device="cuda")
    path, length, _ = check_accept(lg, [nodes] * n, toks, pars, u, nodes, temperature=0.3, top_p=0.9)
    p.compact(batch([0, 1, 2], [nodes] * n), path, length + 1)
    torch.cuda.synchronize()
    assert p.lens.tolist() == [20 + int(length[0]) + 1, 33 + int(length[1]) + 1, 7 + int(length[2]) + 1]


def test_accept_in_a_graph_and_on_a_stream():
    counts = [16, 9]
    xs = [logits(25, 2000, s, peaks=6) for s in (1, 2)]
    toks, pars = trees(counts, 16, 2000, xs[0], 1)
    u = torch.rand(2, 6, 5, generator=gen(1), device="cuda")
    want = [[t.clone() for t in check_accept(x, counts, toks, pars, u, 16)] for x in xs]
    b = msd.Batch(torch.arange(2, dtype=torch.int32, device="cuda"), torch.tensor([0, 16, 25], dtype=torch.int32, device="cuda"), 25)
    tree = msd.Tree(2, 16)
    for i in range(2):
        tree.tokens[i * 16:i * 16 + counts[i]] = torch.tensor(toks[i], dtype=torch.int32, device="cuda")
        tree.parent[i * 16:i * 16 + counts[i]] = torch.tensor(pars[i], dtype=torch.int32, device="cuda")
    x = xs[0].clone()
    out = [torch.zeros(2, 6, dtype=torch.int32, device="cuda")] + [torch.zeros(2, dtype=torch.int32, device="cuda") for _ in range(2)]
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        msd.accept(x, b, tree, u, None, *out)
    for src, w in zip(xs, want):
        x.copy_(src)
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(a, c) for a, c in zip(out, w))
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    msd.accept(x, b, tree, u, None, *out, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(a, c) for a, c in zip(out, want[1]))


def test_accept_beside_another_stream():
    """What the current stream still writes into memory that it has given back does not meet a call on another stream."""
    counts = [60] * 12
    x = logits(720, 2000, 5, peaks=6)
    toks, pars = trees(counts, 60, 2000, x, 5)
    u = torch.rand(12, 7, 5, generator=gen(5), device="cuda") * 0.7
    want = [t.clone() for t in check_accept(x, counts, toks, pars, u, 60)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    b = msd.Batch(torch.arange(12, dtype=torch.int32, device="cuda"), i32([60 * i for i in range(13)]), 720)
    tree = msd.Tree(12, 60)
    tree.tokens.copy_(i32(toks).flatten())
    tree.parent.copy_(i32(pars).flatten())
    out = [torch.zeros_like(t) for t in want]
    s = torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(5):
        used = torch.empty(2 * 720, dtype=torch.int32, device="cuda")
        for _ in range(200):
            used.fill_(-12345)
        del used
        msd.accept(x, b, tree, u, None, *out, stream=s)
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_many_trees_in_a_graph():
    """The launches of more rows than fit, replayed on other logits, links and numbers of nodes; rows past the last sequence's."""
    n, nodes = 14, 60
    counts = [nodes] * n
    xs = [logits(n * nodes + 7, 1500, s, peaks=6) for s in (1, 2, 3)]
    i32 = lambda v: torch.tensor(v, dtype=torch.int32, device="cuda")  # noqa: E731
    u = torch.rand(n, 8, 5, generator=gen(1), device="cuda") * 0.7
    b = msd.Batch(torch.arange(n, dtype=torch.int32, device="cuda"), i32([nodes * i for i in range(n + 1)]), n * nodes + 7)
    tree, f = msd.Tree(n, nodes), settings(n, top_p=0.9)[0]
    x = xs[0].clone()
    out = [torch.zeros(n, 8, dtype=torch.int32, device="cuda")] + [torch.zeros(n, dtype=torch.int32, device="cuda") for _ in range(2)]
    g = torch.cuda.CUDAGraph()
    msd.accept(x, b, tree, u, f, *out)
    torch.cuda.synchronize()
    with torch.cuda.graph(g):
        msd.accept(x, b, tree, u, f, *out)
    for s, src in enumerate(xs):
        live = [nodes - (s * 13 + i) % 50 for i in range(n)]
        toks, pars = trees(counts, nodes, 1500, src[:n * nodes], s, width=3)
        want = check_accept(src[:n * nodes], counts, toks, pars, u, nodes, n_nodes=live, top_p=0.9)
        x.copy_(src)
        tree.tokens.copy_(i32(toks).flatten())
        tree.parent.copy_(i32(pars).flatten())
        tree.n_nodes.copy_(i32(live))
        g.replay()
        torch.cuda.synchronize()
        assert all(torch.equal(p, q) for p, q in zip(out, want))


def test_refusals():
    x, u, t = logits(4, 100), uniforms(4), torch.zeros(4, dtype=torch.int32, device="cuda")
    f3 = msd.Filter(temperature=torch.ones(3, device="cuda"))
    for bad in (lambda: msd.sample(x.half(), u, None, t), lambda: msd.sample(x.t(), u, None, t), lambda: msd.sample(x, u[:3], None, t),
                lambda: msd.sample(x, u.double(), None, t), lambda: msd.sample(x, u, None, t.long()), lambda: msd.sample(x, u, f3, t),
                lambda: msd.sample(x, u, None, t, probs=torch.empty(4, 99, device="cuda")),
                lambda: msd.sample(x, u, None, t, logp=torch.empty(5, device="cuda")), lambda: msd.sample(x[0], u, None, t),
                lambda: msd.Filter(top_k=torch.ones(3, device="cuda")),
                lambda: msd.Filter(temperature=torch.ones(3, device="cuda"), top_p=torch.ones(4, device="cuda"))):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(msd.MsdError):
        msd.sample(torch.empty(1, 393217, device="cuda"), u[:1], None, t[:1])
    b = msd.Batch(torch.arange(2, dtype=torch.int32, device="cuda"), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), 4)
    tree, v = msd.Tree(2, 2), torch.zeros(2, dtype=torch.int32, device="cuda")
    path = torch.zeros(2, 3, dtype=torch.int32, device="cuda")
    uu = torch.rand(2, 3, 4, device="cuda")
    for bad in (lambda: msd.accept(x[:3], b, tree, uu, None, path, v, v), lambda: msd.accept(x, b, msd.Tree(3, 2), uu, None, path, v, v),
                lambda: msd.accept(x, b, tree, uu, None, path[:, :2], v, v), lambda: msd.accept(x, b, tree, uu, f3, path, v, v),
                lambda: msd.accept(x, b, tree, uu[..., None], None, path, v, v), lambda: msd.accept(x, b, tree, uu, None, path, v, v[:1])):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(msd.MsdError):
        msd.accept(x, b, tree, torch.rand(2, 3, 258, device="cuda"), None, path, v, v)


def test_trees_whose_arrays_do_not_fit_are_refused():
    """Arrays of a tree that a program has put in place of the ones that it was made with: host memory, other types, fewer entries."""
    x, b = logits(4, 100), msd.Batch(torch.arange(2, dtype=torch.int32, device="cuda"), torch.tensor([0, 2, 4], dtype=torch.int32, device="cuda"), 4)
    path, v, u = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda"), torch.rand(2, 3, 4, device="cuda")
    for name, change in (("tokens", torch.Tensor.cpu), ("parent", torch.Tensor.cpu), ("n_nodes", torch.Tensor.cpu), ("tokens", torch.Tensor.long),
                         ("parent", torch.Tensor.float), ("tokens", lambda t: t[:3]), ("parent", lambda t: t[:1]), ("n_nodes", lambda t: t[:1]),
                         ("parent", lambda t: t.repeat(2)[::2])):
        tree = msd.Tree(2, 2)
        setattr(tree, name, change(getattr(tree, name)))
        with pytest.raises(ValueError):
            msd.accept(x, b, tree, u, None, path, v, v)
    tree = msd.Tree(2, 2)
    tree.n_nodes = None                    # (as many as rows)
    msd.accept(x, b, tree, u, None, path, v, v.clone())
    torch.cuda.synchronize()
