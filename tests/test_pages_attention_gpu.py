"""Attention over pages (msd_pages_attention) against a plain 64-bit form: grouped heads,
windows with first tokens, trees, chunks, single tokens, odd lengths, hidden values that are
not finite, strides, streams, graphs, long pools, refusals."""
import pytest
import torch

from paper_2505_14260_gb300 import build, msd
from tests.pages_support import attend, batch, bounds, i32, pool, random_tree, starts, tokens, typical, visible

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module", autouse=True)
def _built():
    build.build()


def check(p, b, counts, seqs, q, out, lse, window=0, sinks=0, see=None, depth=None, dtype="bf16", layer=0):
    torch.cuda.synchronize()
    at = 0
    for i, (s, n) in enumerate(zip(seqs, counts)):
        if n == 0:
            continue
        k, v = tokens(p, layer, s)
        ok = visible(k.shape[0] - n, n, window, sinks, None if see is None else see[i], None if depth is None else depth[i])
        ref, rl = attend(q[at:at + n], k, v, ok)
        bo, bl = bounds(q[at:at + n], k, v, ref, torch.where(rl.isfinite(), rl, 0.0), dtype)
        o = out[at:at + n].double()
        fin = ref.isfinite()
        assert torch.equal(fin, o.isfinite()), (i, "which values are finite")
        assert torch.equal(ref.isnan(), o.isnan())
        err = torch.where(fin, (o - ref).abs() - bo, -1.0)
        assert float(err.max() if err.numel() else -1) <= 0, (i, n, float(err.max()))
        rel = float(torch.where(fin, o - ref, 0.0).norm() / torch.where(fin, ref, 0.0).norm().clamp(min=1e-30))
        assert rel <= typical(q[at:at + n], k, dtype), (i, n, rel)
        if lse is not None:
            l = lse[at:at + n].double()
            assert torch.equal(rl == -float("inf"), l == -float("inf"))
            both = rl.isfinite() & l.isfinite()
            assert torch.equal(rl.isfinite(), l.isfinite())
            err = torch.where(both, (l - rl).abs() - bl, -1.0)
            assert float(err.max() if err.numel() else -1) <= 0, (i, "lse", float(err.max()))
        at += n


def run(lens, counts, *, dtype="bf16", heads=4, kv_heads=2, head_dim=64, page=16, window=0, sinks=0, tree=None,
        seed=0, valid=None, stale=float("nan"), scale=1.5):
    p = pool(lens, seed=seed, dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page, stale=stale)
    T, g = sum(counts), torch.Generator(device="cuda").manual_seed(seed + 1)
    q = (scale * torch.randn(T, heads, head_dim, generator=g, device="cuda")).to(p.dtype)
    out = torch.full_like(q, 7.0)
    lse = torch.full((T, heads), 7.0, device="cuda")
    seqs = list(range(len(lens)))
    t = see = depth = None
    if tree:
        t, see, depth = random_tree(len(lens), tree, seed + 2, valid)
    b = batch(seqs, counts)
    p.attention(0, b, q, out, lse=lse, tree=t, window=window, sinks=sinks)
    check(p, b, counts, seqs, q, out, lse, window, sinks, see, depth, dtype)
    return p, b, q, out, lse


WIDTHS = [(4, 4, 64), (4, 2, 64), (8, 1, 128), (14, 2, 128), (6, 2, 64)]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", WIDTHS)
@pytest.mark.parametrize("page", [16, 64, 128])
def test_single_tokens(dtype, heads, kv_heads, head_dim, page):
    lens = [1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 500, 1023]
    run(lens, [1] * len(lens), dtype=dtype, heads=heads, kv_heads=kv_heads, head_dim=head_dim, page=page)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads,head_dim", WIDTHS)
def test_chunks(dtype, heads, kv_heads, head_dim):
    """Prompts alone (len == rows), behind cached tokens, and sequences without rows."""
    run([1, 40, 200, 130, 333, 90, 259], [1, 40, 3, 130, 140, 0, 258], dtype=dtype, heads=heads, kv_heads=kv_heads,
        head_dim=head_dim, page=32)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("window,sinks", [(1, 0), (1, 1), (2, 500), (17, 0), (64, 4), (100, 130), (1000, 3)])
def test_windows(dtype, window, sinks):
    run([300, 1, 129, 700], [140, 1, 129, 5], dtype=dtype, window=window, sinks=sinks, page=16)
    run([300, 1, 129, 2000], [1, 1, 1, 1], dtype=dtype, window=window, sinks=sinks, page=64, heads=8, kv_heads=1)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("nodes", [1, 16, 60, 65, 140])
@pytest.mark.parametrize("window,sinks", [(0, 0), (3, 0), (50, 6)])
def test_trees(dtype, nodes, window, sinks):
    """Trees behind prefixes of every alignment, none, and shorter ones (rows past n_nodes see
    nothing); a sequence with fewer rows than the tree's stride."""
    lens = [nodes, nodes + 1, nodes + 63, nodes + 64, nodes + 300]
    run(lens, [nodes] * 5, dtype=dtype, tree=nodes, window=window, sinks=sinks, valid=[nodes, max(1, nodes - 2), 1, nodes, nodes],
        heads=6, kv_heads=2)
    if nodes > 1:
        run([400, 77], [nodes, nodes // 2], dtype=dtype, tree=nodes, window=window, sinks=sinks, heads=4, kv_heads=4,
            head_dim=128, page=128)


def test_many_rows_of_many_heads():
    """64 query heads to a K/V head, and tiles that end inside a row's heads."""
    run([200, 33], [5, 3], heads=64, kv_heads=1, head_dim=128)
    run([700, 50], [300, 50], heads=10, kv_heads=2, head_dim=128, page=64)
    run([1000], [600], heads=2, kv_heads=2, head_dim=128, page=32, window=200, sinks=10)


def test_many_sequences_and_long_ones():
    lens = [1 + (i * 37) % 200 for i in range(300)]
    run(lens, [1] * 300, heads=2, kv_heads=1, page=16)
    run([1 + (i * 37) % 90 for i in range(700)], [1] * 700, heads=2, kv_heads=2, page=16)       # past one launch's
    run([9 + (i * 5) % 40 for i in range(600)], [7] * 600, tree=7, heads=2, kv_heads=1, valid=[1 + i % 7 for i in range(600)])
    run([1 + (i * 37) % 90 for i in range(600)], [1] * 600, dtype="f32", heads=2, kv_heads=2)
    run([30000, 5, 9000], [1, 1, 2], heads=8, kv_heads=2, head_dim=128, page=64)
    run([20000], [3], dtype="f32", heads=4, kv_heads=4, page=128)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_mask_that_leaves_rows_empty(dtype):
    """A tree whose mask has no bit for a row, and nothing before it."""
    p = pool([20, 4], dtype=dtype)
    t, see, depth = random_tree(2, 4, 3)
    t.mask.view(2, 4)[1, 2] = 0
    t.mask.view(2, 4)[0, 1] = 0                    # row 1 of sequence 0 still sees what is before the tree
    see = see.clone()
    see[1, 2] = False
    see[0, 1] = False
    q = torch.randn(8, 4, 64, device="cuda").to(p.dtype)
    out, lse = torch.full_like(q, 7.0), torch.zeros(8, 4, device="cuda")
    p.attention(0, batch([0, 1], [4, 4]), q, out, lse=lse, tree=t)
    torch.cuda.synchronize()
    assert not out[6].any() and (lse[6] == -float("inf")).all()
    for i, (s, at) in enumerate([(0, 0), (1, 4)]):
        k, v = tokens(p, 0, s)
        L = k.shape[0] - 4
        ok = torch.cat([torch.ones(4, L, dtype=torch.bool, device="cuda"), see[i]], 1)
        ref, rl = attend(q[at:at + 4], k, v, ok)
        bo, _ = bounds(q[at:at + 4], k, v, ref, torch.zeros_like(rl), dtype)
        assert bool(((out[at:at + 4].double() - ref).abs() <= bo).all())


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
@pytest.mark.parametrize("tree", [None, 30])
def test_values_that_are_not_finite_reach_only_the_rows_that_see_them(dtype, value, tree):
    """V entries of some rows (and K of one) are not finite: rows that do not see them give
    what they give without, the others the definition's result."""
    for window, sinks in [(0, 0), (40, 3)]:
        for heads, kv_heads, rows in [(4, 4, 30), (8, 1, 30)] + ([] if tree else [(2, 1, 300)]):
            lens, counts = [rows + 170, rows], [rows, rows]
            p = pool(lens, dtype=dtype, heads=heads, kv_heads=kv_heads, page=16)
            for s, n in enumerate(lens):
                for slot, what, col in [(n - rows + 7, 1, 5), (n - 3, 1, 63), (n - rows // 2, 1, 0)] + \
                                       ([(n - rows - 60, 1, 9)] if n > rows else []):
                    p.kv[0, p.table[s, slot // 16].long(), what, kv_heads - 1, slot % 16, col] = value
            g = torch.Generator(device="cuda").manual_seed(4)
            q = torch.randn(sum(counts), heads, 64, generator=g, device="cuda").to(p.dtype)
            out, lse = torch.empty_like(q), torch.empty(sum(counts), heads, device="cuda")
            t = see = depth = None
            if tree:
                t, see, depth = random_tree(2, tree, 8)
            b = batch([0, 1], counts)
            p.attention(0, b, q, out, lse=lse, tree=t, window=window, sinks=sinks)
            check(p, b, counts, [0, 1], q, out, lse, window, sinks, see, depth, dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_key_that_is_not_a_number(dtype):
    p = pool([100], dtype=dtype)
    p.kv[0, p.table[0, 90 // 16].long(), 0, 1, 90 % 16, 3] = float("nan")       # slot 90, K/V head 1
    q = torch.randn(20, 4, 64, device="cuda").to(p.dtype)
    out, lse = torch.empty_like(q), torch.empty(20, 4, device="cuda")
    p.attention(0, batch([0], [20]), q, out, lse=lse)
    torch.cuda.synchronize()
    bad = out.isnan().any(-1)
    assert not bad[:, :2].any() and not bad[:10].any() and bad[10:, 2:].all()
    assert torch.equal(lse.isnan(), bad)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_large_scores(dtype):
    """Scores of some hundreds: weights of one key, and maxima that move from tile to tile."""
    p = pool([700], dtype=dtype, heads=2, kv_heads=2, page=16)
    k = p.kv[0, :, 0]
    k.mul_(torch.linspace(0, 12, k.shape[0], device="cuda")[:, None, None, None].to(p.dtype))
    q = (6 * torch.randn(300, 2, 64, device="cuda")).to(p.dtype)
    out, lse = torch.empty_like(q), torch.empty(300, 2, device="cuda")
    b = batch([0], [300])
    p.attention(0, b, q, out, lse=lse)
    check(p, b, [300], [0], q, out, lse, dtype=dtype)


def test_strides_layers_and_no_lse():
    """q and out as parts of wider rows, the second of three layers, sequences in any order."""
    p = pool([90, 40, 222], layers=3, heads=4, kv_heads=2, head_dim=128, extra_seqs=2)
    wide = torch.randn(9, 11 * 128, device="cuda").to(p.dtype)
    res = torch.full((9, 7 * 128), 5.0, device="cuda", dtype=p.dtype)
    q, out = wide[:, 256:256 + 512], res[:, 128:128 + 512]
    b = batch([2, 0], [4, 5])
    p.attention(1, b, q, out)
    check(p, b, [4, 5], [2, 0], q.reshape(9, 4, 128), out.reshape(9, 4, 128), None, layer=1)
    assert (res[:, :128] == 5).all() and (res[:, 640:] == 5).all()


def test_streams_and_graphs():
    """On a side stream, ordered by events; recorded once and replayed on other contents and
    lengths; the same inputs give the same bits."""
    p = pool([300, 45], heads=8, kv_heads=2, head_dim=128, extra_pages=30, spare=80)
    q = torch.randn(2, 8, 128, device="cuda").to(p.dtype)
    out, lse, b = torch.empty_like(q), torch.empty(2, 8, device="cuda"), batch([0, 1], [1, 1])
    p.attention(0, b, q, out, lse=lse)
    torch.cuda.synchronize()
    first = out.clone()
    side = torch.cuda.Stream()
    for _ in range(3):
        out.zero_()
        side.wait_stream(torch.cuda.current_stream())
        p.attention(0, b, q, out, lse=lse, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        assert torch.equal(out, first)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.reserve(b)
        p.attention(0, b, q, out, lse=lse)
    p.kv.copy_(torch.randn_like(p.kv))
    for step in range(40):
        q.copy_(torch.randn_like(q))
        graph.replay()
        if step % 13 == 0:
            check(p, b, [1, 1], [0, 1], q, out, lse)
    assert p.lens.tolist() == [340, 85]


def test_a_pool_past_32_bit_offsets():
    """Pages whose elements lie past 2^32 (9 GB of bf16)."""
    page, heads, hd = 128, 8, 128
    n_pages = (1 << 32) // (2 * heads * page * hd) + 40
    p = msd.Pages(dtype="bf16", layers=1, heads=heads, kv_heads=heads, head_dim=hd, page_size=page, n_pages=n_pages,
                  max_seqs=2, max_pages=4)
    p.table[0, :3] = i32([n_pages - 1, 3, n_pages - 7])
    p.lens[0] = 300
    p.restore()
    p.kv[0, [n_pages - 1, 3, n_pages - 7]] = torch.randn(3, 2, heads, page, hd, device="cuda").to(p.dtype)
    for rows in (1, 40):
        q = torch.randn(rows, heads, hd, device="cuda").to(p.dtype)
        out, lse, b = torch.empty_like(q), torch.empty(rows, heads, device="cuda"), batch([0], [rows])
        p.attention(0, b, q, out, lse=lse)
        check(p, b, [rows], [0], q, out, lse)
    del p
    torch.cuda.empty_cache()


def test_refusals():
    p = pool([90, 40])
    q = torch.randn(2, 4, 64, device="cuda").to(p.dtype)
    out, b = torch.empty_like(q), batch([0, 1], [1, 1])
    L, S = msd.lib(), msd._stream(None)
    good = [p.ptr, 0, b.c(), None, 0, 0, 0, q.data_ptr(), 256, out.data_ptr(), 256, None, S]
    assert L.msd_pages_attention(*good) == msd.MSD_OK

    def refused(**kw):
        args = list(good)
        for k, v in kw.items():
            args[int(k[1:])] = v
        return L.msd_pages_attention(*args) == msd.MSD_ERR_INVALID
    assert refused(a1=1) and refused(a1=-1)                       # layers
    assert refused(a2=None) and refused(a7=None) and refused(a9=None)
    assert refused(a5=-1) and refused(a6=-1)
    assert refused(a7=q.data_ptr() + 2) and refused(a8=255) and refused(a8=260) and refused(a10=128)
    t = msd.Tree(2, 1)
    import ctypes
    assert refused(a3=ctypes.byref(t.c()), a4=0) and refused(a3=ctypes.byref(t.c()), a4=1025)
    assert L.msd_pages_attention(None, *good[1:]) == msd.MSD_ERR_INVALID
    with pytest.raises(ValueError):
        p.attention(0, b, q.float(), out)
    with pytest.raises(ValueError):
        p.attention(0, b, q[:1], out)
    with pytest.raises(ValueError):
        p.attention(0, b, q, out, lse=torch.empty(2, 4, device="cuda", dtype=torch.float64))


def test_batches_that_only_the_device_can_refuse():
    """A sequence id out of range, more rows than tokens: reported by the next call, the other
    sequences' rows computed, nothing else written."""
    p = pool([90, 40], extra_seqs=1)
    q = torch.randn(3, 4, 64, device="cuda").to(p.dtype)
    for seqs, counts in [([0, 7], [2, 1]), ([0, -1], [2, 1]), ([0, 2], [2, 1])]:
        out, lse = torch.full_like(q, 7.0), torch.full((3, 4), 7.0, device="cuda")
        b = msd.Batch(i32(seqs), starts(counts), 3)
        p.attention(0, b, q, out, lse=lse)
        torch.cuda.synchronize()
        with pytest.raises(msd.MsdError) as e:
            p.attention(0, b, q, out)
        assert e.value.status == msd.MSD_ERR_DEVICE
        check(p, b, [2], [0], q, out, lse)
        assert (out[2] == 7).all()
